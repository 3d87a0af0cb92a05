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


@pytest.mark.parametrize("n,V,a", [(1, 4_000_000, 18.0), (1, 64_000_000, 18.0), (8, 64_000_000, 18.0), (9, 4_000_000, 24.0), (60, 64_000_000, 24.0), (100, 4_000_000, 24.0),
                                   (300, 4_000_000, 24.0), (300, 4_000_000, 22.0)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sums_of_many_strips_beside_a_large_word(n, V, a, dtype):
    """Few tokens: the vocabulary is cut into thousands of strips, or walked through by single lanes, and what each has is small beside the strip
    that has the large word."""
    h, w = torch.zeros((n, 8), dtype=DT[dtype], device="cuda"), torch.zeros((V, 8), dtype=DT[dtype], device="cuda")
    h[:, 3] = 1.0
    w[V // 3, 3] = a
    _, lse = _loss(h, w, torch.zeros(n, dtype=torch.int32, device="cuda"))
    want = a + math.log1p((V - 1) * math.exp(-a))
    # 18 to 26 joins that lose at most half a unit each, the result to a few of its own
    assert float((lse.double() - want).abs().max()) <= 32 * U32 + 3 * U32 * want


# ---------------------------------------------------------------- words masked by infinities and the largest numbers
def _grad(h, w, labels, lse, d, scale=1.0, ignore=-1):
    n, (V, D) = labels.numel(), w.shape
    ws = torch.empty(B.tensair_softmax_workspace_bytes(n, V, D, w.dtype, True), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)
    dh, dw = torch.full_like(h, 3.0), torch.full_like(w, 3.0)
    B.tensair_softmax_grad(h, w, D, labels, lse, d, dh, dw, ws, scale, ignore)
    return dh, dw


@pytest.mark.parametrize("how", ["infinite", "lowest", "large hidden"])
@pytest.mark.parametrize("n,D,dtype", [(2, 32, "f32"), (8, 32, "bf16"), (9, 32, "f32"), (30, 64, "f32"), (30, 32, "bf16"), (64, 36, "f32"), (130, 32, "f32"), (130, 32, "bf16"),
                                       (128, 300, "f32"), (300, 332, "bf16"), (600, 128, "f32")])
def test_softmax_words_masked_in_one_column(n, D, dtype, how):
    """The first column holds a mask: minus infinity, the lowest number or a plain one that the hidden rows make as large.  In bits that are not
    those of a bfloat16, so that a product of parts overflows where the number itself is of the other sign or not at all.  The masked words have
    no share in anything, and their gradient is zero whatever tokens lie beside them: those without a loss, those that fill up a tile."""
    from test_operators import _softmax_reference, _gen
    V, scale = 700, -0.7
    g = _gen(n + D)
    h = (torch.randn((n, D), generator=g, device="cuda") * 0.3).to(DT[dtype])
    w = (torch.randn((V, D), generator=g, device="cuda") * 0.3).to(DT[dtype])
    one = 1.0 + torch.rand(n, generator=g, device="cuda")
    masked = torch.arange(0, V, 3, device="cuda")
    rest = torch.ones(V, dtype=torch.bool, device="cuda")
    rest[masked] = False
    w[:, 0] = 0
    if how == "infinite":
        h[:, 0], w[masked, 0] = 1.0, float("inf")              # the scale is negative
    elif how == "lowest":
        h[:, 0], w[masked, 0] = 300.7 * one, torch.finfo(DT[dtype]).max
    else:
        h[:, 0], w[masked, 0] = 1.1e38 * one, 300.7
    place = torch.cumsum(rest, 0) - 1
    labels = rest.nonzero()[:, 0][torch.randint(0, int(rest.sum()), (n,), generator=g, device="cuda")].int()
    labels[::3] = -1
    d = torch.rand(n, generator=g, device="cuda") / n
    loss, lse = _loss(h, w, labels, scale)
    among = torch.where(labels >= 0, place[labels.clamp(min=0).long()], -1).int()
    ref = _softmax_reference(h, w[rest], among, d, scale, dtype)
    assert bool(((lse.double() - ref[0][0]).abs() <= ref[0][1]).all()) and bool(((loss.double() - ref[1][0]).abs() <= ref[1][1]).all())
    dh, dw = _grad(h, w, labels, lse, d, scale)
    assert bool((dw[masked] == 0).all())
    assert bool(((dw[rest].double() - ref[3][0]).abs() <= ref[3][1]).all())
    # (zero times infinity is in the first column's sum where the mask is infinite: what the definition gives)
    at = slice(1 if how == "infinite" else 0, None)
    assert bool(((dh.double() - ref[2][0]).abs() <= ref[2][1])[:, at].all()) and bool((dh[labels < 0] == 0).all())
    # the loss of a masked word is infinite
    labels[n - 1] = 3
    assert float(_loss(h, w, labels, scale)[0][n - 1]) == math.inf


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [5, 60, 200])
def test_numbers_that_are_none_stay_where_they_belong(n, dtype):
    """NaN in a token's row, in its first or its last column: its own loss and its row of the gradient, no other token's.  In a word's row: everything."""
    V, D = 600, 40
    g = torch.Generator(device="cuda").manual_seed(n)
    h, w = ((torch.randn((k, D), generator=g, device="cuda") * 0.3).to(DT[dtype]) for k in (n, V))
    labels, d = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32), torch.rand(n, generator=g, device="cuda")
    loss, lse = _loss(h, w, labels)
    dh, _ = _grad(h, w, labels, lse, d)
    for col in (0, D - 1):
        bad = h.clone()
        bad[n // 2, col] = float("nan")
        others = torch.arange(n, device="cuda") != n // 2
        got, got_lse = _loss(bad, w, labels)
        assert torch.equal(got[others], loss[others]) and bool(got[n // 2].isnan()) and bool(got_lse[n // 2].isnan())
        gh, gw = _grad(bad, w, labels, got_lse, d)
        assert torch.equal(gh[others], dh[others]) and bool(gh[n // 2].isnan().all()) and bool(gw.isnan().all())
        worse = w.clone()
        worse[V // 2, col] = float("nan")
        got, got_lse = _loss(h, worse, labels)
        assert bool(got.isnan().all()) and bool(got_lse.isnan().all())


# ---------------------------------------------------------------- the label's share of a gradient
@pytest.mark.parametrize("weights", ["mean", "each its own"])
@pytest.mark.parametrize("n,V,D,pad", [(9, 300, 36, 0), (26, 2_439, 148, 0), (64, 5_000, 64, 4), (100, 1_000, 64, 0), (128, 257, 324, 0), (300, 5_000, 300, 0), (1_000, 777, 512, 4),
                                       (5_615, 1_530, 120, 0), (2_100, 40_000, 192, 0), (4_096, 20_000, 1_024, 0), (16_383, 3_001, 256, 0), (9_000, 70_000, 64, 0)])
def test_bfloat16_gradients_are_off_by_little_more_than_their_own_rounding(n, V, D, pad, weights):
    """A number that is rounded to bfloat16 is off by up to 2^-9 of it, one below 1 and not below 1/2 by up to 2^-9; errors of their own add up as the root of the sum of
    their squares does.  Beside the outputs' own rounding there is that of dz: of the words that are no labels, and, in the gradient of the table alone, of
    the labels' p - 1, which is off by no more than p.  (What the tokens have in common of d_loss is not rounded at all: were it, the labels' elements
    would be off by as much as the outputs, all of them to the same side.)"""
    g = torch.Generator(device="cuda").manual_seed(n + V)
    h, w = ((torch.randn((k, D + pad), generator=g, device="cuda") * s).bfloat16() for k, s in ((n, 2 / (0.25 * math.sqrt(D))), (V, 0.25)))
    cdf = torch.cumsum(torch.arange(1, V + 1, device="cuda", dtype=torch.float64) ** -1.2, 0)
    labels = torch.searchsorted(cdf, torch.rand(n, generator=g, device="cuda", dtype=torch.float64) * cdf[-1]).clamp(max=V - 1).int()
    labels[::16] = -1
    scale = -1.3 if n % 2 else 0.8
    d = torch.full((n,), 1.0039 / n, device="cuda") if weights == "mean" else torch.rand(n, generator=g, device="cuda") / n
    hd, wd = h[:, :D], w[:, :D]
    ws = torch.empty(B.tensair_softmax_workspace_bytes(n, V, D, w.dtype, True), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)
    loss, lse = (torch.empty(n, device="cuda") for _ in range(2))
    B.tensair_softmax_loss(hd, wd, D, labels, loss, lse, ws, scale)
    ws.fill_(0xFF)
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    B.tensair_softmax_grad(hd, wd, D, labels, lse, d, dh[:, :D], dw[:, :D], ws, scale)
    s = float(torch.tensor(scale, dtype=torch.float32))
    h64, w64, keep = hd.double(), wd.double(), labels >= 0
    at, y = keep.nonzero()[:, 0], labels[keep].long()
    p = torch.softmax(s * (h64 @ w64.t()), 1)
    p_label = p[at, y]
    p *= torch.where(keep, d.double(), 0.0)[:, None]
    rest = p.clone()                                           # dz without the labels' elements
    rest[at, y] = 0
    p[at, y] -= d[at].double()
    # the squares of the labels' errors, in units of 2^-9: of p - 1, or of its product with a factor of a token's own
    own = d[at].double() ** 2 * (torch.clamp(p_label * 512, max=1.0) if weights == "mean" else 1 - p_label) ** 2
    for got, value, spread, label in ((dh, s * (p @ w64), (rest ** 2) @ w64 ** 2, 0.0),
                                      (dw, s * (p.t() @ h64), (rest ** 2).t() @ h64 ** 2, float((own[:, None] * h64[at] ** 2).sum()))):
        off = float((got[:, :D].double() - value).norm())
        bound = 2.0 ** -9 * math.sqrt(float(value.norm()) ** 2 + s * s * (float(spread.sum()) + label))
        assert off <= bound, (off / bound, off / float(value.norm()))
