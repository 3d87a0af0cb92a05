"""What the operators of a table as a model's layers say of their workspaces.  No GPU needed."""
import pytest
import torch

from paper_2211_10280_amd import binding as B

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
VOCABS = (1, 1_000, 10_000, 50_000, 262_144, 1_000_000, 2_000_000, 10_000_000)


@pytest.mark.parametrize("dtype", sorted(DTYPES))
@pytest.mark.parametrize("D", [4, 64, 128, 300, 512, 1_024])
def test_the_gradient_s_workspace_serves_the_loss(D, dtype):
    for V in VOCABS:
        for n in (1, 8, 9, 64, 65, 128, 129, 300, 1_024, 2_000, 4_096, 10_240, 16_384, 40_960, 100_001, 1 << 21):
            both, loss = (B.tensair_softmax_workspace_bytes(n, V, D, DTYPES[dtype], g) for g in (True, False))
            assert both >= loss, (n, V)


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
