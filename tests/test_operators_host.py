"""What the operators of a table that is a model's input and output layer refuse, before any GPU call is made (no GPU needed)."""
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


def test_embed(mem):
    L = B.lib()

    def call(table=mem, dtype=B.F32, vocab=10, dim=8, stride=8, ids=mem, n=4, out=mem, out_dtype=B.F32, out_stride=8, status=None):
        return L.tensair_embed(table, dtype, vocab, dim, stride, ids, n, 1.0, out, out_dtype, out_stride, status, None)

    for bad in (dict(table=None), dict(out=None), dict(ids=None), dict(dtype=2), dict(out_dtype=7), dict(vocab=0), dict(vocab=B.MAX_VOCAB + 1), dict(dim=6),
                dict(dim=0), dict(dim=1028, stride=1028, out_stride=1028), dict(stride=4), dict(stride=10), dict(out_stride=4), dict(n=-1), dict(n=1 << 31),
                dict(table=mem + 4), dict(out=mem + 8), dict(ids=mem + 2), dict(status=mem + 1)):
        assert call(**bad) == B.EINVAL, bad
    assert call(n=0) == B.OK and call(n=0, ids=None, out=None) == B.OK


def test_embed_grad(mem):
    L = B.lib()
    need = B.tensair_embed_workspace_bytes(10, 8, 4)
    assert B.tensair_embed_workspace_bytes(10, 8, 5_000) > need > 0
    for bad in ((0, 8, 4), (10, 6, 4), (10, 8, -1)):
        with pytest.raises(B.TensairError):
            B.tensair_embed_workspace_bytes(*bad)

    def sparse(n=4, cap=4, rows=mem, ids=mem, n_rows=mem, ws=mem, nbytes=need, d=mem, d_dtype=B.F32, d_stride=8, vocab=10, dim=8, tokens=mem):
        g = B.SparseRows(cap, n_rows, ids, rows)
        return L.tensair_embed_grad(tokens, n, d, d_dtype, d_stride, vocab, dim, 1.0, C.byref(g), ws, nbytes, None, None)

    assert sparse(cap=3) == B.ECAPACITY and sparse(nbytes=need - 1) == B.ECAPACITY
    for bad in (dict(rows=None), dict(ids=None), dict(n_rows=None), dict(ws=None), dict(ws=mem + 16), dict(rows=mem + 4), dict(d=None), dict(d_dtype=2),
                dict(d_stride=6), dict(d=mem + 4), dict(tokens=None), dict(vocab=0), dict(dim=2)):
        assert sparse(**bad) == B.EINVAL, bad
    assert L.tensair_embed_grad(mem, 4, mem, B.F32, 8, 10, 8, 1.0, None, mem, need, None, None) == B.EINVAL

    def dense(n=4, grad=mem, dtype=B.F32, stride=8, ws=mem, nbytes=need):
        return L.tensair_embed_grad_dense(mem, n, mem, B.F32, 8, 10, 8, 1.0, grad, dtype, stride, 1, ws, nbytes, None, None)

    assert dense(nbytes=0) == B.ECAPACITY
    for bad in (dict(grad=None), dict(dtype=2), dict(stride=4), dict(grad=mem + 2), dict(ws=None), dict(ws=mem + 8)):
        assert dense(**bad) == B.EINVAL, bad
    assert dense(n=0, ws=None, nbytes=1 << 20) == B.OK            # nothing to add


def test_softmax(mem):
    L = B.lib()
    need = B.tensair_softmax_workspace_bytes(4, 10, 8, torch.float32, True)
    assert need >= B.tensair_softmax_workspace_bytes(4, 10, 8, torch.float32, False) > 0
    # the logits are never kept: what a large vocabulary needs does not grow with tokens times words
    assert B.tensair_softmax_workspace_bytes(16_384, 2_000_000, 512, torch.bfloat16, True) < 6 << 30
    # nor do d_hidden's sums with the ranges of words
    assert B.tensair_softmax_workspace_bytes(262_144, 1_000_000, 300, torch.bfloat16, True) < 4 << 30
    with pytest.raises(B.TensairError):
        B.tensair_softmax_workspace_bytes((1 << 21) + 1, 10, 8, torch.float32, False)
    for bad in ((-1, 10, 8, torch.float32), (4, 0, 8, torch.float32), (4, 10, 6, torch.float32), (4, 10, 8, torch.float8_e4m3fn), (4, 10, 8, torch.float16),
                ((1 << 24) + 1, 10, 8, torch.float32)):
        with pytest.raises(B.TensairError):
            B.tensair_softmax_workspace_bytes(*bad, True)

    def loss(h=mem, hs=8, w=mem, wsd=8, dtype=B.F32, n=4, vocab=10, dim=8, labels=mem, scale=1.0, out=mem, lse=mem, ws=mem, nbytes=need, status=None):
        return L.tensair_softmax_loss(h, hs, w, wsd, dtype, n, vocab, dim, labels, -1, scale, out, lse, ws, nbytes, status, None)

    def grad(lse=mem, d=mem, dh=mem, dhs=8, dw=mem, dws=8, **k):
        a = dict(h=mem, hs=8, w=mem, wsd=8, dtype=B.F32, n=4, vocab=10, dim=8, labels=mem, scale=1.0, ws=mem, nbytes=need, status=None)
        a.update(k)
        return L.tensair_softmax_grad(a["h"], a["hs"], a["w"], a["wsd"], a["dtype"], a["n"], a["vocab"], a["dim"], a["labels"], -1, a["scale"], lse, d, dh, dhs,
                                      dw, dws, a["ws"], a["nbytes"], a["status"], None)

    for call in (loss, grad):
        assert call(nbytes=255) == B.ECAPACITY
        for bad in (dict(h=None), dict(w=None), dict(labels=None), dict(lse=None), dict(ws=None), dict(ws=mem + 64), dict(hs=4), dict(wsd=9), dict(dtype=2),
                    dict(n=-1), dict(n=(1 << 24) + 1), dict(vocab=0), dict(dim=7), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")),
                    dict(h=mem + 4), dict(w=mem + 8), dict(labels=mem + 1), dict(status=mem + 2)):
            assert call(**bad) == B.EINVAL, bad
    assert loss(out=None) == B.EINVAL and loss(n=0) == B.OK
    for bad in (dict(d=None), dict(dh=mem + 4), dict(dws=4), dict(dhs=7)):
        assert grad(**bad) == B.EINVAL, bad
    assert grad(dh=None, dw=None) == B.OK


def test_adamw(mem):
    L = B.lib()

    def tensor(**k):
        t = B.AdamwTensor(mem, mem, mem, mem, mem, mem, None, 100, B.F32, B.F32, 0.0)
        for name, x in k.items():
            setattr(t, name, x)
        return t

    def size(t, state=B.F32, n=1):
        return L.tensair_adamw_workspace_bytes(C.byref(t) if t is not None else None, n, state)

    assert size(tensor()) > 0 and size(tensor(), B.FP8) > 0 and size(tensor(n=0, param=None, grad=None, m=None, v=None)) > 0
    assert size(None) == 0 and size(tensor(), n=0) == 0 and size(tensor(), B.BF16) == 0
    for bad in (dict(n=-1), dict(n=B.MAX_DENSE + 1), dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param_dtype=2), dict(grad_dtype=3),
                dict(weight_decay=-1.0), dict(weight_decay=float("nan")), dict(param=mem + 2), dict(grad=mem + 1), dict(m=mem + 2), dict(param_copy=mem + 1),
                dict(m_scale=mem + 2)):
        assert size(tensor(**bad)) == 0, bad
    assert size(tensor(m_scale=None), B.FP8) == 0 and size(tensor(v=mem + 3), B.FP8) > 0          # a byte needs no alignment
    h = C.c_void_p()
    t = tensor()
    need = size(t)
    assert L.tensair_adamw_init(None, C.byref(t), 1, B.F32, mem, need, None) == B.EINVAL
    assert L.tensair_adamw_init(C.byref(h), C.byref(t), 1, B.F32, mem, need - 1, None) == B.ECAPACITY
    assert L.tensair_adamw_init(C.byref(h), C.byref(t), 1, B.F32, mem + 16, need, None) == B.EINVAL
    assert L.tensair_adamw_init(C.byref(h), C.byref(t), 1, B.F32, None, need, None) == B.EINVAL and h.value is None
    assert L.tensair_adamw_step(None, 0.1, 1, 0.9, 0.999, 1e-8, None, None) == B.EINVAL
    assert L.tensair_adamw_destroy(None) == B.OK


def test_tensors_of_other_shapes_and_types_are_refused_by_the_binding():
    """Nothing here reaches the library."""
    f, i = torch.zeros((4, 8)), torch.zeros(4, dtype=torch.int32)
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for call in (lambda: B.tensair_embed(f, 8, i.long(), f), lambda: B.tensair_embed(f.double(), 8, i, f), lambda: B.tensair_embed(f, 8, i, f[:3]),
                 lambda: B.tensair_embed(f.t(), 4, i, f), lambda: B.tensair_embed(f, 12, i, f), lambda: B.tensair_embed(f, 8, i[::2], f[:2]),
                 lambda: B.tensair_embed_grad(i, f, 8, 4, (i[:1], i, f.bfloat16()), ws), lambda: B.tensair_embed_grad(i, f, 8, 4, (i, i, f), ws),
                 lambda: B.tensair_embed_grad_dense(i, f[:2], 8, f, ws),
                 lambda: B.tensair_softmax_loss(f, f.bfloat16(), 8, i, f[:, 0].contiguous(), f[:, 0].contiguous(), ws),
                 lambda: B.tensair_softmax_loss(f, f, 8, i, f[:, 0], f[:, 0].contiguous(), ws),
                 lambda: B.tensair_softmax_grad(f, f, 8, i, f[:, 0].contiguous(), f[:, 0].contiguous(), f.bfloat16(), None, ws),
                 lambda: B.AdamW([dict(param=f, grad=f, m=f, v=f.bfloat16())]), lambda: B.AdamW([dict(param=f, grad=f[:2], m=f, v=f)]),
                 lambda: B.AdamW([dict(param=f, grad=f, m=f.to(torch.float8_e4m3fn), v=f.to(torch.float8_e4m3fn))]),
                 lambda: B.AdamW([dict(param=f, grad=f, m=f.bfloat16(), v=f.bfloat16())]), lambda: B.AdamW([])):
        with pytest.raises(B.TensairError):
            call()
