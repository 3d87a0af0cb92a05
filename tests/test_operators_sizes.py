"""What the operators of a table as a model's layers say of their workspaces, and what they ask for when they are called."""
import ctypes as C
import random

import pytest
import torch

from paper_2211_10280_amd import binding as B
from paper_2211_10280_amd.softmax_trainer import SoftmaxWorker

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
VOCABS = (1, 1_000, 10_000, 50_000, 262_144, 1_000_000, 2_000_000, 10_000_000)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("D", [4, 64, 128, 300, 512, 1_024])
def test_the_gradient_s_workspace_serves_the_loss(D, dtype):
    for V in VOCABS:
        for n in (1, 8, 9, 64, 65, 128, 129, 300, 1_024, 2_000, 4_096, 10_240, 16_384, 40_960, 100_001, 1 << 21):
            both, loss = (B.tensair_softmax_workspace_bytes(n, V, D, DTYPES[dtype], g) for g in (True, False))
            assert both >= loss, (n, V)


@pytest.fixture(scope="module")
def mem():
    """Host memory that no call gets as far as to touch."""
    buf = (C.c_char * 4096)()
    yield (C.addressof(buf) + 255) & ~255
    del buf


def _softmax_fits(mem, n, V, D, dtype, nbytes, grad):
    """Whether a call takes a workspace of that many bytes.  Its address is one that is refused, but only after its size was looked at."""
    L, code = B.lib(), {"f32": B.F32, "bf16": B.BF16}[dtype]
    if grad:
        rc = L.tensair_softmax_grad(mem, D, mem, D, code, n, V, D, mem, -1, 1.0, mem, mem, mem, D, mem, D, mem + 64, nbytes, None, None)
    else:
        rc = L.tensair_softmax_loss(mem, D, mem, D, code, n, V, D, mem, -1, 1.0, mem, mem, mem + 64, nbytes, None, None)
    assert rc in (B.EINVAL, B.ECAPACITY)
    return rc == B.EINVAL


def test_a_softmax_workspace_serves_fewer_tokens(mem):
    """The last mini-batch of a pass is shorter, and a single token is scored between two steps, in the workspace of a whole mini-batch."""
    assert not _softmax_fits(mem, 4_096, 1_000_000, 300, "bf16", 1 << 20, True)
    rng = random.Random(5)
    cases = [(4_096, 1_000_000, 300, "bf16"), (4_096, 50_000, 128, "f32"), (16_384, 10_000, 512, "bf16"), (40_960, 1_000_000, 300, "f32"), (1 << 21, 1_000, 64, "bf16")]
    for _ in range(120):
        cases.append((int(2 ** rng.uniform(0, 17)), int(2 ** rng.uniform(0, 24)), 4 * int(2 ** rng.uniform(0, 8)), rng.choice(sorted(DTYPES))))
    for n, V, D, dtype in cases:
        fewer = {n, max(1, n - 1), 1, min(n, 8), min(n, 9)} | {rng.randint(1, n) for _ in range(40)} | {max(1, min(n, k + e)) for k in (64, 128, 256, 512, 1_024) for e in (-1, 0, 1)}
        for grad in (False, True):
            nbytes = B.tensair_softmax_workspace_bytes(n, V, D, DTYPES[dtype], grad)
            for k in fewer:
                assert _softmax_fits(mem, k, V, D, dtype, nbytes, False) and (not grad or _softmax_fits(mem, k, V, D, dtype, nbytes, True)), (n, k, V, D, dtype, grad)


def test_a_gradient_s_workspace_serves_fewer_ids(mem):
    L, rng = B.lib(), random.Random(6)
    borders = [2_048 * t + t + e for t in (2, 4, 8, 16, 32, 64, 128) for e in (-2, -1, 0, 1)] + [k + e for k in (4_096, 262_144, 524_288) for e in (-1, 0, 1, 31, 32)]
    for case in range(60):
        n, V, D = int(2 ** rng.uniform(0, 22)), int(2 ** rng.uniform(0, 27)), 4 * int(2 ** rng.uniform(0, 8))
        if case < len(borders):
            n = borders[case]
        nbytes = B.tensair_embed_workspace_bytes(V, D, n)
        for k in {n, max(1, n - 1), 1} | {rng.randint(1, n) for _ in range(30)} | {b for b in borders if b <= n}:
            rc = L.tensair_embed_grad_dense(mem, k, mem, B.F32, D, V, D, 1.0, mem, B.F32, D, 1, mem + 64, nbytes, None, None)
            assert rc == B.EINVAL, (n, k, V, D)          # refused for the workspace's alignment, not for its size


@pytest.mark.gpu
@pytest.mark.parametrize("n,V,D,dtype", [(2_000, 262_144, 512, "f32"), (4_096, 1_000_000, 1_024, "bf16")])
def test_both_calls_in_one_workspace(n, V, D, dtype):
    """Sizes at which the loss lays out more words at a time than the gradient."""
    h, w = (torch.full((k, D), 0.01, dtype=DTYPES[dtype], device="cuda") for k in (n, V))
    labels, d = torch.arange(n, dtype=torch.int32, device="cuda"), torch.ones(n, device="cuda")
    loss, lse, dh, dw = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty_like(h), torch.empty_like(w)
    ws = torch.empty(B.tensair_softmax_workspace_bytes(n, V, D, w.dtype, True), dtype=torch.uint8, device="cuda")
    B.tensair_softmax_loss(h, w, D, labels, loss, lse, ws)
    B.tensair_softmax_grad(h, w, D, labels, lse, d, dh, dw, ws)
    # all logits alike: the loss is the logarithm of the vocabulary, to the few roundings of two numbers of its size
    want = torch.log(torch.tensor(float(V), dtype=torch.float64))
    assert float((loss.double().cpu() - want).abs().max()) <= 16 * 2.0 ** -24 * float(want)
    assert bool(torch.isfinite(dh).all()) and bool(torch.isfinite(dw).all())


@pytest.mark.gpu
def test_a_worker_takes_shorter_mini_batches():
    V, most = 50_000, 4_096
    worker = SoftmaxWorker(V, 128, most, "f32")
    g = torch.Generator(device="cuda").manual_seed(3)
    for n in (most, 3_456, 2_000, 300, 70, 9, 8, 1):
        centers, contexts = (torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32) for _ in range(2))
        loss = worker.step(centers, contexts, torch.full((n,), 1.0 / n, device="cuda"))
        assert loss.shape == (n,) and bool(torch.isfinite(loss).all())
        assert bool(torch.isfinite(worker.score(centers[:3], contexts[:3])).all())
    assert int(worker.status) == 0
    worker.close()
