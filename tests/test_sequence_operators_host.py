"""What the operators of a model of word sequences refuse, before any GPU call is made (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2211_10280_amd import binding as B


@pytest.fixture(scope="module")
def mem():
    buf = (C.c_char * 4096)()
    at = (C.addressof(buf) + 255) & ~255
    yield at
    del buf


ROWS = (1 << 31) - 4096


def test_norm(mem):
    L = B.lib()

    def call(x=mem, dtype=B.F32, xs=8, n=4, dim=8, w=mem, b=mem, eps=1e-5, out=mem, od=B.F32, os=8, mean=mem, rstd=mem):
        return L.tensair_norm(x, dtype, xs, n, dim, w, b, eps, out, od, os, mean, rstd, None)

    for bad in (dict(x=None), dict(out=None), dict(dtype=2), dict(od=-1), dict(xs=4), dict(xs=10), dict(os=4), dict(n=-1), dict(n=ROWS), dict(dim=0), dict(dim=6), dict(dim=1028, xs=1028, os=1028),
                dict(x=mem + 8), dict(out=mem + 4), dict(w=mem + 4), dict(b=mem + 8), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(mean=None), dict(rstd=None), dict(mean=mem + 2),
                dict(dtype=B.BF16, x=mem + 4)):
        assert call(**bad) == B.EINVAL, bad
    assert call(n=0, x=None, out=None, mean=None, rstd=None) == B.OK


def test_norm_grad(mem):
    L = B.lib()
    need = B.tensair_norm_workspace_bytes(4, 8)
    assert need > 0
    for n in (1, 1_000, 10 ** 6, 10 ** 9):                      # what n rows need serves fewer
        assert all(B.tensair_norm_workspace_bytes(k, 300) <= B.tensair_norm_workspace_bytes(n, 300) for k in (0, 1, n // 2, n - 1))
    for bad in ((-1, 8), (4, 6), (ROWS, 8)):
        with pytest.raises(B.TensairError):
            B.tensair_norm_workspace_bytes(*bad)

    def call(d=mem, dd=B.F32, ds=8, x=mem, dtype=B.F32, xs=8, n=4, dim=8, w=mem, mean=mem, rstd=mem, add=None, adds=8, dx=mem, dxs=8, dw=mem, db=mem, ws=mem, nbytes=need):
        return L.tensair_norm_grad(d, dd, ds, x, dtype, xs, n, dim, w, mean, rstd, add, adds, dx, dxs, dw, db, ws, nbytes, None)

    assert call(nbytes=need - 1) == B.ECAPACITY and call(n=0, nbytes=0) == B.ECAPACITY
    for bad in (dict(d=None), dict(x=None), dict(dx=None), dict(dd=2), dict(dtype=2), dict(ds=4), dict(xs=6), dict(dxs=4), dict(add=mem, adds=4), dict(add=mem + 4), dict(mean=None), dict(rstd=None),
                dict(rstd=mem + 1), dict(w=mem + 4), dict(dw=mem + 4), dict(db=mem + 8), dict(ws=None), dict(ws=mem + 16), dict(n=-1), dict(dim=3)):
        assert call(**bad) == B.EINVAL, bad
    assert call(n=0, dw=None, db=None, ws=None, nbytes=0, d=None, x=None, dx=None, mean=None, rstd=None) == B.OK


def test_dropout(mem):
    L = B.lib()

    def call(x=mem, dtype=B.F32, xs=8, n=4, dim=8, p=0.1, at=None, r=None, rs=8, out=mem, od=B.F32, os=8):
        return L.tensair_dropout(x, dtype, xs, n, dim, p, 1, 0, 0, at, r, rs, out, od, os, None)

    for bad in (dict(x=None), dict(out=None), dict(dtype=2), dict(od=2), dict(xs=4), dict(os=9), dict(n=-1), dict(n=ROWS), dict(dim=2), dict(p=1.0), dict(p=-0.1), dict(p=float("nan")), dict(at=mem + 4),
                dict(r=mem + 4), dict(r=mem, rs=4), dict(x=mem + 4)):
        assert call(**bad) == B.EINVAL, bad
    assert call(n=0, x=None, out=None) == B.OK


def test_recur(mem):
    L = B.lib()
    need = B.tensair_recur_workspace_bytes(4, 8)
    assert need > 0 and B.tensair_recur_state_rows(0) == B.tensair_recur_state_rows(256) == 1 and B.tensair_recur_state_rows(257) == 2
    for n in (1, 300, 10 ** 5, 10 ** 8):
        assert all(B.tensair_recur_workspace_bytes(k, 300) <= B.tensair_recur_workspace_bytes(n, 300) for k in (0, 1, n // 2, n - 1))
    for bad in ((-1, 8), (4, 6), (ROWS, 8)):
        with pytest.raises(B.TensairError):
            B.tensair_recur_workspace_bytes(*bad)
    with pytest.raises(B.TensairError):
        B.tensair_recur_state_rows(-1)

    def call(x=mem, xs=8, g=mem, gs=8, dtype=B.F32, n=4, dim=8, off=mem, S=1, h0=None, out=mem, os=8, last=None, states=None, ws=mem, nbytes=need, status=None):
        return L.tensair_recur(x, xs, g, gs, dtype, n, dim, off, S, h0, out, os, last, states, ws, nbytes, status, None)

    common = (dict(x=None), dict(g=None), dict(dtype=2), dict(xs=4), dict(gs=6), dict(n=-1), dict(n=ROWS), dict(dim=10), dict(off=None), dict(off=mem + 2), dict(S=-1), dict(S=ROWS), dict(h0=mem + 4),
              dict(ws=None), dict(ws=mem + 8), dict(status=mem + 1), dict(g=mem + 4))
    assert call(nbytes=need - 1) == B.ECAPACITY
    for bad in (*common, dict(out=None), dict(os=4), dict(last=mem + 8), dict(states=mem + 4)):
        assert call(**bad) == B.EINVAL, bad
    assert call(S=0) == B.OK

    def grad(x=mem, xs=8, g=mem, gs=8, dtype=B.F32, n=4, dim=8, off=mem, S=1, h0=None, states=mem, d=mem, ds=8, last=None, dx=mem, dxs=8, dg=mem, dgs=8, dh0=None, ws=mem, nbytes=need, status=None):
        return L.tensair_recur_grad(x, xs, g, gs, dtype, n, dim, off, S, h0, states, d, ds, last, dx, dxs, dg, dgs, dh0, ws, nbytes, status, None)

    assert grad(nbytes=need - 1) == B.ECAPACITY
    for bad in (*common, dict(states=None), dict(states=mem + 4), dict(d=None), dict(ds=4), dict(dx=None), dict(dxs=6), dict(dg=None), dict(dgs=4), dict(last=mem + 4), dict(dh0=mem + 4)):
        assert grad(**bad) == B.EINVAL, bad
    assert grad(S=0) == B.OK

    def step(x=mem, xs=8, g=mem, gs=8, dtype=B.F32, n=4, dim=8, slots=mem, total=4, state=mem, ss=8, out=mem, os=8, status=None):
        return L.tensair_recur_step(x, xs, g, gs, dtype, n, dim, slots, total, state, ss, out, os, status, None)

    for bad in (dict(x=None), dict(g=None), dict(dtype=2), dict(xs=4), dict(gs=4), dict(n=-1), dict(dim=6), dict(slots=mem + 2), dict(slots=None, n=5), dict(n=65537), dict(total=-1), dict(state=None),
                dict(state=mem + 4), dict(ss=6), dict(os=4), dict(out=mem + 4), dict(status=mem + 2)):
        assert step(**bad) == B.EINVAL, bad
    assert step(n=0) == B.OK


def test_sample(mem):
    L = B.lib()
    need = B.tensair_sample_workspace_bytes(4, 8)
    for n, V in ((1, 10), (64, 50_000), (7, 1 << 24), (65_536, 100)):
        assert all(B.tensair_sample_workspace_bytes(k, v) <= B.tensair_sample_workspace_bytes(n, V) for k in (0, 1, n) for v in (1, V // 2 + 1, V - 1))
    for bad in ((-1, 8), (65_537, 8), (4, 0), (4, (1 << 24) + 1)):
        with pytest.raises(B.TensairError):
            B.tensair_sample_workspace_bytes(*bad)

    def call(z=mem, dtype=B.F32, stride=8, n=4, vocab=8, T=None, k=None, p=None, m=None, u=mem, words=mem, prob=None, ws=mem, nbytes=need, status=None):
        return L.tensair_sample(z, dtype, stride, n, vocab, T, k, p, m, u, words, prob, ws, nbytes, status, None)

    assert call(nbytes=need - 1) == B.ECAPACITY
    for bad in (dict(z=None), dict(u=None), dict(words=None), dict(dtype=2), dict(stride=7), dict(n=-1), dict(n=65_537), dict(vocab=0), dict(z=mem + 2), dict(dtype=B.BF16, z=mem + 1), dict(T=mem + 2),
                dict(k=mem + 1), dict(p=mem + 2), dict(m=mem + 2), dict(u=mem + 1), dict(words=mem + 2), dict(prob=mem + 3), dict(status=mem + 2), dict(ws=None), dict(ws=mem + 8)):
        assert call(**bad) == B.EINVAL, bad
    assert call(n=0, z=None, u=None, words=None, ws=None, nbytes=0) == B.OK


def test_tensors_that_are_not_on_a_gpu_are_refused():
    """Their addresses would go to a kernel.  Shapes and types are right; nothing here reaches the library."""
    f, v, w, i = torch.zeros((4, 8)), torch.zeros(4), torch.zeros(8), torch.zeros(5, dtype=torch.int32)
    ws, states = torch.zeros(1 << 16, dtype=torch.uint8), torch.zeros((1, 8))
    for call in (lambda: B.tensair_norm(f, 8, w, w, f.clone(), v, v.clone()), lambda: B.tensair_norm_grad(f, f, 8, w, v, v, f.clone(), w, w, ws), lambda: B.tensair_dropout(f, 8, f.clone(), 0.1, 1),
                 lambda: B.tensair_recur(f, f, 8, i, f.clone(), ws), lambda: B.tensair_recur_grad(f, f, 8, i, states, f, f.clone(), f.clone(), ws),
                 lambda: B.tensair_recur_step(f, f, 8, f.clone()), lambda: B.tensair_sample(f, 8, v, i[:4], ws)):
        with pytest.raises(B.TensairError) as e:
            call()
        assert "GPU" in str(e.value)


@pytest.mark.gpu
def test_each_argument_is_looked_at():
    """On the GPU: every tensor in turn on the host, of another type, of another size."""
    def gpu(x):
        return x.cuda()

    f, v, w = gpu(torch.randn((4, 8))), gpu(torch.rand(4)), gpu(torch.rand(8))
    off, slots, ws = gpu(torch.tensor([0, 4], dtype=torch.int32)), gpu(torch.arange(4, dtype=torch.int32)), gpu(torch.zeros(1 << 20, dtype=torch.uint8))
    h, states, status, at = gpu(torch.randn((1, 8))), gpu(torch.zeros((1, 8))), gpu(torch.zeros(1, dtype=torch.int32)), gpu(torch.ones(1, dtype=torch.int64))
    calls = [(lambda x, w, b, o, m, r: B.tensair_norm(x, 8, w, b, o, m, r), (f, w, w.clone(), f.clone(), v.clone(), v.clone())),
             (lambda d, x, w, m, r, dx, dw, db, ws, a: B.tensair_norm_grad(d, x, 8, w, m, r, dx, dw, db, ws, a), (f, f, w, v, v, f.clone(), w.clone(), w.clone(), ws, f)),
             (lambda x, o, at, r: B.tensair_dropout(x, 8, o, 0.1, 1, 0, at, r), (f, f.clone(), at, f)),
             (lambda x, g, off, o, ws, h, l, s, st: B.tensair_recur(x, g, 8, off, o, ws, h, l, s, st), (f, f, off, f.clone(), ws, h, h.clone(), states, status)),
             (lambda x, g, off, s, d, dx, dg, ws, h, l, dh, st: B.tensair_recur_grad(x, g, 8, off, s, d, dx, dg, ws, h, l, dh, st),
              (f, f, off, states, f, f.clone(), f.clone(), ws, h, h, h.clone(), status)),
             (lambda x, g, s, o, sl, st: B.tensair_recur_step(x, g, 8, s, o, sl, st), (f, f, f.clone(), f.clone(), slots, status)),
             (lambda z, u, wd, ws, T, k, p, m, pr, st: B.tensair_sample(z, 8, u, wd, ws, T, k, p, m, pr, st), (f, v, slots.clone(), ws, v, slots, v, v, v.clone(), status))]
    for call, args in calls:
        call(*args)
        for k, x in enumerate(args):
            wrong = [x.cpu()]
            if x is not ws:
                wrong += [x.double() if x.dtype != torch.int64 else x.int(), x[:0]]
            for bad in wrong:
                with pytest.raises(B.TensairError):
                    call(*args[:k], bad, *args[k + 1:])
    torch.cuda.synchronize()


def test_rows_of_states_are_the_librarys(monkeypatch):
    """The binding checks the states' rows against what the library says, not against a tile size of its own."""
    x, offsets = torch.zeros((300, 8)), torch.zeros(2, dtype=torch.int32)
    assert B.tensair_recur_state_rows(300) == 2
    assert B._recur_inputs(x, x, 8, offsets, torch.zeros((2, 8)))[-1] and B._recur_inputs(x, x, 8, offsets, None)[-1] is None
    monkeypatch.setattr(B, "tensair_recur_state_rows", lambda n: 5)
    assert B._recur_inputs(x, x, 8, offsets, torch.zeros((5, 8)))[-1]
    with pytest.raises(B.TensairError):
        B._recur_inputs(x, x, 8, offsets, torch.zeros((2, 8)))
