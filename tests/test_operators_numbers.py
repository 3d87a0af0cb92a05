"""Numbers at the ends of their range in the operators of a table as a model's layers: very unequal terms, infinities, the largest values.  On the
GPU through the C ABI, against the definitions in 64 bits; tolerances are worked out from the number of roundings (2^-24 each in fp32)."""
import math

import pytest
import torch

from paper_2211_10280_amd import binding as B

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
U16 = 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _loss(h, w, labels, scale=1.0, ignore=-1):
    n, (V, D) = labels.numel(), w.shape
    ws = torch.empty(B.tensair_softmax_workspace_bytes(n, V, D, w.dtype, False), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)
    loss, lse = (torch.full((n,), float("nan"), device="cuda") for _ in range(2))
    B.tensair_softmax_loss(h, w, D, labels, loss, lse, ws, scale, ignore)
    return loss, lse


# ---------------------------------------------------------------- a large word and many small ones
@pytest.mark.parametrize("at", [0, 100_003, 249_999])
@pytest.mark.parametrize("n,D,dtype", [(1, 32, "bf16"), (8, 32, "f32"), (60, 32, "bf16"), (131_072, 32, "bf16"), (131_072, 32, "f32"), (65_536, 328, "bf16")])
def test_small_words_beside_a_large_one(n, D, dtype, at):
    """One word of the vocabulary has a probability near 1, each of the others is below 2^-25 of it, so that a plain fp32 sum that
    holds the large one takes no notice of any: together they are 0.6 %.  Many tokens, so that a sum runs over the whole vocabulary."""
    V, a = 250_000, 17.5
    h = torch.zeros((n, D), dtype=DT[dtype], device="cuda")
    h[:, 3] = 1.0
    w = torch.zeros((V, D), dtype=DT[dtype], device="cuda")
    w[at, 3] = a
    labels = torch.full((n,), at, dtype=torch.int32, device="cuda")
    labels[n // 2:] = (at + 1) % V
    loss, lse = _loss(h, w, labels)
    tail = (V - 1) * math.exp(-a)
    want = a + math.log1p(tail)
    # the terms of a tile of up to 64 words one after the other, a few joins of sums; a logit and the result in units of log 2
    bound = 128 * U32 + 8 * U32 * want
    assert bound < tail / 100
    assert float((lse.double() - want).abs().max()) <= bound
    value = torch.where(labels == at, math.log1p(tail), want).double()
    assert float((loss.double() - value).abs().max()) <= bound
