"""The operators of a table that is a model's input and output layer, on the GPU through the C ABI, against plain 64-bit
implementations of their definitions.  Tolerances are worked out from the number of roundings: a sum of k fp32 terms is off by at most
k * 2^-24 times the sum of their magnitudes, a rounding to bfloat16 (8 significant bits) by 2^-8 of the value."""
import math

import numpy as np
import pytest
import torch

from paper_2211_10280_amd import binding as B

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24          # unit roundoff
U16 = 2.0 ** -8           # of bfloat16
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _matrix(rows, dim, dtype, g, std=1.0, pad=0, fill=float("nan")):
    """Random rows, `pad` more elements in every row that hold `fill`."""
    t = torch.full((max(rows, 1), dim + pad), fill, dtype=DT[dtype], device="cuda")[:rows]
    t[:, :dim] = torch.randn((rows, dim), generator=g, device="cuda") * std
    return t


def _ids(n, V, g, hot=0.0):
    """n words, a share `hot` of them one and the same, the first and the last word of the vocabulary among them."""
    ids = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    if hot:
        ids[torch.rand(n, generator=g, device="cuda") < hot] = V // 2
    if n > 2:
        ids[0], ids[n - 1] = V - 1, 0
    return ids


def _status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------- scaled lookup
@pytest.mark.parametrize("V,D,n,dtype,out,pad", [
    (1, 4, 1, "f32", "f32", 0), (1_000, 32, 64, "f32", "f32", 0), (777, 300, 1_023, "bf16", "f32", 20), (777, 300, 1_023, "f32", "bf16", 4),
    (50_021, 128, 16_385, "bf16", "bf16", 0), (33, 1_024, 5, "f32", "f32", 8), (9, 4, 5_000, "bf16", "f32", 4), (64, 12, 1_025, "f32", "bf16", 0)])
def test_embed(V, D, n, dtype, out, pad):
    g = _gen(V + D)
    table, ids, status = _matrix(V, D, dtype, g, pad=pad), _ids(n, V, g), _status()
    got = torch.full((n, D + pad), 7.0, dtype=DT[out], device="cuda")
    B.tensair_embed(table, D, ids, got, 1.7, status)
    want = (table[:, :D].float()[ids.long()] * torch.tensor(1.7, dtype=torch.float32, device="cuda")).to(DT[out])
    assert torch.equal(got[:, :D], want)                       # one product, one rounding
    assert bool((got[:, D:] == 7.0).all()) and int(status) == 0


def test_embed_ids_out_of_range_and_no_ids():
    g = _gen(1)
    table, status = _matrix(10, 8, "f32", g), _status()
    ids = torch.tensor([3, -1, 10, 9, -2**31, 2**31 - 1], dtype=torch.int32, device="cuda")
    out = torch.ones((6, 8), device="cuda")
    B.tensair_embed(table, 8, ids, out, 1.0, status)
    assert torch.equal(out[[0, 3]], table[[3, 9]]) and bool((out[[1, 2, 4, 5]] == 0).all()) and int(status) == 1
    B.tensair_embed(table, 8, ids, out, 1.0)                   # without a status word
    B.tensair_embed(table, 8, ids[:0], out[:0], 1.0, status)


# ---------------------------------------------------------------- its gradient
def _grad_reference(ids, d, V, scale):
    """(words ascending, sums in 64 bits, their error bound) over ids in range."""
    ok = (ids >= 0) & (ids < V)
    words, place, counts = torch.unique(ids[ok], return_inverse=True, return_counts=True)
    x = d.double()[ok] * float(np.float32(scale))
    sums = torch.zeros((len(words), d.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, place, x)
    mass = torch.zeros_like(sums).index_add_(0, place, x.abs())
    return words, sums, mass * (counts[:, None] + 2) * U32


GRAD_CASES = [
    # V, D, n, dtype, pad, hot
    (1_000, 32, 1, "f32", 0, 0), (1_000, 32, 2, "bf16", 4, 0.9), (1, 4, 70, "f32", 0, 0), (50, 36, 257, "f32", 12, 0.3),
    (50_000, 128, 1_024, "f32", 0, 0.05), (3, 1_024, 4_096, "bf16", 0, 0), (100_003, 300, 4_096, "f32", 4, 0.01),
    (100_003, 300, 4_097, "f32", 0, 0.01), (2, 64, 5_000, "bf16", 0, 0.5), (1_000_000, 300, 20_001, "bf16", 20, 0.2),
    (700, 1_000, 9_001, "f32", 0, 0), (2_000_000, 8, 65_537, "f32", 0, 0.4), (10_000, 256, 100_003, "bf16", 0, 0.34),
    (5, 16, 270_001, "f32", 0, 0.7), (300_000, 20, 300_007, "bf16", 0, 0.1)]


@pytest.mark.parametrize("V,D,n,dtype,pad,hot", GRAD_CASES)
def test_embed_grad(V, D, n, dtype, pad, hot):
    g = _gen(n + D)
    ids, d, status, scale = _ids(n, V, g, hot), _matrix(n, D, dtype, g, pad=pad), _status(), -0.3
    ids[torch.rand(n, generator=g, device="cuda") < 0.02] = -1
    ids[n // 2] = V
    bad = bool(((ids < 0) | (ids >= V)).any())
    words, sums, bound = _grad_reference(ids, d[:, :D], V, scale)
    ws = torch.empty(B.tensair_embed_workspace_bytes(V, D, n), dtype=torch.uint8, device="cuda")
    ws.fill_(0x5A)
    grad = B.RowBuffers(min(V, n) + 3, D)
    grad.row_ids.fill_(-7)
    grad.rows.fill_(7.0)
    B.tensair_embed_grad(ids, d, D, V, grad, ws, scale, status)
    u = int(grad.n_rows)
    assert u == len(words) and torch.equal(grad.row_ids[:u], words) and int(status) == int(bad)
    assert bool(((grad.rows[:u].double() - sums).abs() <= bound).all())
    assert bool((grad.row_ids[u:] == -7).all()) and bool((grad.rows[u:] == 7.0).all())     # nothing is written behind them
    # the same bits again, whatever the workspace held
    again = B.RowBuffers(min(V, n) + 3, D)
    ws.fill_(0xFF)
    B.tensair_embed_grad(ids, d, D, V, again, ws, scale)
    assert torch.equal(again.rows[:u], grad.rows[:u])
    # the whole table's gradient: written and added to, rows as in the message
    if V * D > 40_000_000:
        return
    dense = torch.full((V, D + 8), 5.0, device="cuda")
    B.tensair_embed_grad_dense(ids, d, D, dense, ws, scale)
    want = torch.zeros((V, D), device="cuda")
    want[words.long()] = grad.rows[:u]
    assert torch.equal(dense[:, :D], want) and bool((dense[:, D:] == 5.0).all())
    base = torch.randn((V, D), generator=g, device="cuda")
    dense = base.clone()
    B.tensair_embed_grad_dense(ids, d, D, dense, ws, scale, accumulate=True)
    assert torch.equal(dense, base + want)
    half = base.bfloat16()
    B.tensair_embed_grad_dense(ids, d, D, half, ws, scale, accumulate=True)
    touched = torch.zeros(V, dtype=torch.bool, device="cuda")
    touched[words.long()] = True
    assert torch.equal(half, torch.where(touched[:, None], (base.bfloat16().float() + want).bfloat16(), base.bfloat16()))


@pytest.mark.parametrize("V,D,n,dtype,pad,hot", [(5_000, 8, 600_001, "f32", 0, 0.2), (40_000, 300, 33_000, "f32", 4, 0.1), (20_000, 64, 140_000, "bf16", 0, 0.0),
                                                 (300, 520, 12_000, "bf16", 0, 0.6)])
def test_embed_grad_tiles_of_every_length(V, D, n, dtype, pad, hot):
    test_embed_grad(V, D, n, dtype, pad, hot)


@pytest.mark.parametrize("n", [0, 5, 5_000])
def test_embed_grad_of_nothing(n):
    V, D = 100, 8
    ids = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    d, ws = torch.ones((n, D), device="cuda"), torch.empty(B.tensair_embed_workspace_bytes(V, D, n) + 1, dtype=torch.uint8, device="cuda")
    grad = B.RowBuffers(V, D)
    grad.n_rows.fill_(9)
    B.tensair_embed_grad(ids, d, D, V, grad, ws)
    assert int(grad.n_rows) == 0
    dense = torch.ones((V, D), device="cuda")
    B.tensair_embed_grad_dense(ids, d, D, dense, ws, accumulate=True)
    assert bool((dense == 1).all())
    B.tensair_embed_grad_dense(ids, d, D, dense, ws)
    assert bool((dense == 0).all())


@pytest.mark.parametrize("n", [900, 9_000])
def test_embed_grad_is_the_adjoint_of_embed(n):
    """embed is linear: <d, embed(table + x) - embed(table)> = <gradient, x> for any x."""
    V, D, scale = 500, 48, 2.5
    g = _gen(n)
    ids, d = _ids(n, V, g, 0.2), torch.randn((n, D), generator=g, device="cuda")
    x = torch.randn((V, D), generator=g, device="cuda")
    out = torch.empty((n, D), device="cuda")
    B.tensair_embed(x, D, ids, out, scale)
    ws = torch.empty(B.tensair_embed_workspace_bytes(V, D, n), dtype=torch.uint8, device="cuda")
    grad = torch.empty((V, D), device="cuda")
    B.tensair_embed_grad_dense(ids, d, D, grad, ws, scale)
    left, right = (d.double() * out.double()).sum(), (grad.double() * x.double()).sum()
    mass = (d.double() * out.double()).abs().sum()
    assert abs(float(left - right)) <= float(mass) * n * U32


def test_embed_grad_message_into_the_table_update():
    """The message is what the table update takes: W_in <- W_in - lr * gradient, W_out untouched."""
    V, D, n, lr = 3_000, 64, 700, 0.5
    g = _gen(11)
    w_in, w_out = (torch.randn((V, D), generator=g, device="cuda") for _ in range(2))
    ids, d = _ids(n, V, g, 0.1), torch.randn((n, D), generator=g, device="cuda")
    gb = B.GradBuffers(n, 1, D)
    ws = torch.empty(B.tensair_embed_workspace_bytes(V, D, n), dtype=torch.uint8, device="cuda")
    B.tensair_embed_grad(ids, d, D, V, (gb.n_rows[:1], gb.in_ids, gb.in_rows), ws)
    want = w_in.double().clone()
    words, sums, bound = _grad_reference(ids, d, V, 1.0)
    want[words.long()] -= lr * sums
    before = w_out.clone()
    B.tensair_dasgd_apply_static(w_in, w_out, D, gb, [], lr)
    tol = U32 * 2 * want.abs()
    tol[words.long()] += lr * bound
    assert bool(((w_in.double() - want).abs() <= tol).all()) and torch.equal(w_out, before)


# ---------------------------------------------------------------- softmax loss and its gradient
def _softmax_reference(h, w, labels, d, scale, dtype):
    """Everything in 64 bits, with bounds for what the kernels give: (value, bound) of lse, loss, d_hidden, d_table."""
    h, w, s = h.double(), w.double(), float(np.float32(scale))
    V, D = w.shape
    n = h.shape[0]
    z = s * (h @ w.t())
    keep = labels >= 0
    lse = torch.logsumexp(z, 1)
    y = labels.clamp(min=0).long()
    loss = torch.where(keep, lse - z.gather(1, y[:, None])[:, 0], 0.0)
    # a logit: D products summed in fp32 (of three-part inputs six products each, 2^-23 left out), scaled and turned to powers of two
    ez = abs(s) * (h.abs() @ w.abs().t()).amax(1) * ((6 * D if dtype == "f32" else D) + 8) * U32 + 8 * U32 * z.abs().amax(1)
    e_lse = ez + (V / 32 + 128) * U32 + 8 * U32 * lse.abs()
    p = torch.exp(z - lse[:, None])
    one = torch.zeros_like(p)
    one[torch.arange(n, device="cuda")[keep], y[keep]] = 1
    dd = torch.where(keep, d.double(), 0.0)[:, None]
    dz = dd * (p - one)
    rel = U16 if dtype == "bf16" else 2.0 ** -21                # dz in one part or three
    e_p = dd.abs() * p * (torch.expm1(ez + e_lse) + 16 * U32)[:, None]
    dh, dw = s * (dz @ w), s * (dz.t() @ h)
    out = U16 if dtype == "bf16" else 4 * U32

    def bound(a, b, value, k):
        return abs(s) * ((rel + 6 * k * U32) * (a.abs() @ b.abs())) + out * value.abs() * 1.01 + 1e-38

    hk = torch.where(keep[:, None], h, 0.0)
    return ((lse, e_lse), (loss, ez + e_lse + 8 * U32 * loss.abs()),
            (dh, bound(dz.abs() + e_p / rel, w, dh, V)), (dw, bound((dz.abs() + e_p / rel).t(), hk, dw, n)))


def _softmax(h, w, D, labels, d, scale, ignore=-1, status=None, want=(True, True), stream=None):
    n, V = labels.numel(), w.shape[0]
    ws = torch.empty(B.tensair_softmax_workspace_bytes(n, V, D, w.dtype, True), dtype=torch.uint8, device="cuda")
    ws.fill_(0xFF)                                              # whatever the workspace holds (as numbers: NaN) must not matter
    loss, lse = (torch.full((n,), float("nan"), device="cuda") for _ in range(2))
    B.tensair_softmax_loss(h, w, D, labels, loss, lse, ws, scale, ignore, status, stream)
    dh = torch.full_like(h, 3.0) if want[0] else None
    dw = torch.full_like(w, 3.0) if want[1] else None
    ws.fill_(0xFF)
    B.tensair_softmax_grad(h, w, D, labels, lse, d, dh, dw, ws, scale, ignore, status, stream)
    return loss, lse, dh, dw


SOFTMAX_CASES = [
    # n, V, D, dtype, pad: tokens around the forms' borders, words and rows around the tiles'
    (1, 1, 4, "f32", 0), (1, 1_000, 32, "bf16", 0), (2, 257, 300, "f32", 20), (4, 5_003, 128, "bf16", 4), (5, 255, 1_024, "f32", 0), (8, 3_001, 516, "bf16", 12),
    (9, 256, 8, "f32", 0), (9, 2, 4, "bf16", 0), (64, 1_000, 64, "bf16", 0), (64, 700, 36, "f32", 28), (65, 1_000, 32, "bf16", 0), (127, 513, 100, "f32", 0),
    (128, 10_007, 300, "bf16", 20), (129, 300, 320, "f32", 0), (1_000, 5_003, 300, "bf16", 4), (257, 4_099, 512, "bf16", 0), (300, 2_000, 448, "f32", 0),
    (640, 777, 1_024, "bf16", 0), (200, 513, 1_024, "f32", 4), (2_049, 1_001, 192, "bf16", 0), (5_000, 70, 68, "bf16", 0), (1_030, 1_100, 256, "f32", 0)]


@pytest.mark.parametrize("n,V,D,dtype,pad", SOFTMAX_CASES)
def test_softmax(n, V, D, dtype, pad):
    g = _gen(n + V + D)
    h, w = _matrix(n, D, dtype, g, 2 / (0.25 * math.sqrt(D)), pad), _matrix(V, D, dtype, g, 0.25, pad)
    labels = _ids(n, V, g)
    labels[torch.rand(n, generator=g, device="cuda") < 0.2] = -1
    d = torch.rand(n, generator=g, device="cuda") / n
    scale = -0.7 if n % 2 else 1.3
    ref = _softmax_reference(h[:, :D], w[:, :D], labels, d, scale, dtype)
    loss, lse, dh, dw = _softmax(h, w, D, labels, d, scale)
    for name, got, (value, bound) in zip(("lse", "loss", "d_hidden", "d_table"), (lse, loss, dh[:, :D], dw[:, :D]), ref):
        off = (got.double() - value).abs()
        assert bool((off <= bound).all()), (name, float((off / bound).max()))
    assert bool((loss[labels < 0] == 0).all()) and bool((dh[:, :D][labels < 0] == 0).all())
    assert bool((dh[:, D:] == 3.0).all()) and bool((dw[:, D:] == 3.0).all())           # the padding is left alone
    # a part of the outputs, and the same bits every time
    again = _softmax(h, w, D, labels, d, scale, want=(False, True))
    assert torch.equal(again[0], loss) and torch.equal(again[3][:, :D], dw[:, :D])
    assert torch.equal(_softmax(h, w, D, labels, d, scale, want=(True, False))[2][:, :D], dh[:, :D])


@pytest.mark.parametrize("n,V,D,pad", [(129, 3_000, 40, 24), (256, 33, 64, 0), (257, 1_000, 100, 0), (300, 2_001, 132, 0), (700, 511, 256, 4), (513, 31, 320, 0),
                                       (1_025, 257, 324, 0)])
def test_softmax_with_tokens_in_registers(n, V, D, pad):
    """The form for many tokens with short rows in bfloat16, every number of blocks of columns; one row length beyond it."""
    test_softmax(n, V, D, "bf16", pad)


@pytest.mark.parametrize("n,V,D,dtype", [(4_100, 140_000, 36, "f32"), (9_000, 70_000, 64, "bf16")])
def test_softmax_in_several_ranges_of_words(n, V, D, dtype):
    """dz of all words is more than is kept at a time: d_hidden's sums go on from range to range, the last of which is shorter."""
    test_softmax(n, V, D, dtype, 0)


@pytest.mark.parametrize("n", [3, 40, 200])
def test_softmax_gradient_against_differences(n):
    """Central differences of the loss itself (fp32 inputs), along the gradient of either input.  Along a line a token's logits grow
    at rates a_v; the third derivative of its log of a sum of exponentials is the third central moment of a random one of the a_v,
    which is at most (largest - smallest)^3 / (6 sqrt 3)."""
    V, D, eps = 300, 40, 0.02
    g = _gen(n)
    h, w = _matrix(n, D, "f32", g, 0.3), _matrix(V, D, "f32", g, 0.3)
    labels, d = _ids(n, V, g), torch.full((n,), 1.0, device="cuda")
    loss, _, dh, dw = _softmax(h, w, D, labels, d, 1.0)
    for base, grad, at in ((h, dh, 0), (w, dw, 1)):
        u = grad / grad.norm()
        sides = []
        for sign in (1, -1):
            args = [h, w]
            args[at] = base + sign * eps * u
            sides.append(_softmax(args[0], args[1], D, labels, d, 1.0)[0].double().sum())
        slope, want = float(sides[0] - sides[1]) / (2 * eps), float((grad.double() * u.double()).sum())
        rates = u.double() @ w.double().t() if at == 0 else h.double() @ u.double().t()
        third = float(((rates.amax(1) - rates.amin(1)) ** 3).sum()) / (6 * math.sqrt(3))
        # the points moved to are rounded to fp32 (half a unit of about 1), the losses are off by some units
        tol = eps ** 2 / 6 * third + (float(loss.abs().sum()) * 64 * U32 + U32 * float(grad.abs().sum())) / eps
        assert abs(slope - want) <= tol and abs(want) > 20 * tol


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [3, 50, 200])
def test_softmax_masked_tokens_reach_nothing(n, dtype):
    """NaN and infinities in the rows of tokens without a loss: no sum sees them; labels out of range are such tokens too."""
    V, D = 700, 64
    g = _gen(n)
    h, w, labels = _matrix(n, D, dtype, g, 0.5), _matrix(V, D, dtype, g, 0.5), _ids(n, V, g)
    d = torch.rand(n, generator=g, device="cuda")
    labels[1], labels[n - 1] = -100, V
    clean = h.clone()
    clean[[1, n - 1]] = 0
    status = _status()
    good = _softmax(clean, w, D, torch.where((labels < 0) | (labels >= V), -100, labels), d, 1.0, ignore=-100, status=status)
    assert int(status) == 0
    for bad in (float("nan"), float("inf"), -float("inf"), 3e38):
        h[1], h[n - 1] = bad, bad
        d[1] = float("nan")
        status.zero_()
        loss, lse, dh, dw = _softmax(h, w, D, labels, d, 1.0, ignore=-100, status=status)
        assert int(status) == 1                                                         # V is no label
        assert torch.equal(dw, good[3]) and torch.equal(dh, good[2]) and torch.equal(loss, good[0])
        keep = (labels >= 0) & (labels < V)
        assert torch.equal(lse[keep], good[1][keep])
    # no token at all has a loss
    labels.fill_(-100)
    loss, _, dh, dw = _softmax(h, w, D, labels, d, 1.0, ignore=-100)
    assert bool((loss == 0).all()) and bool((dh == 0).all()) and bool((dw == 0).all())


@pytest.mark.parametrize("n", [2, 30, 130])
def test_softmax_words_masked_by_the_lowest_value(n):
    """Words whose logits lie below everything (minus the largest number): no share in any sum, gradient zero; a label among
    them has an infinite loss.  All other words are as if those were not there."""
    V, D = 600, 32
    g = _gen(n)
    h, w = _matrix(n, D, "bf16", g, 0.3), _matrix(V, D, "bf16", g, 0.3)
    h[:, 0], w[:, 0] = 1.0, 0.0
    masked = torch.arange(0, V, 3, device="cuda")
    w[masked] = 0
    w[masked, 0] = -3.3e38
    labels = torch.full((n,), 1, dtype=torch.int32, device="cuda")
    d = torch.ones(n, device="cuda")
    rest = torch.ones(V, dtype=torch.bool, device="cuda")
    rest[masked] = False
    loss, lse, dh, dw = _softmax(h, w, D, labels, d, 1.0)
    few = torch.zeros_like(labels)                                                      # word 1 is the first of the rest
    ref = _softmax_reference(h, w[rest], few, d, 1.0, "bf16")
    assert bool(((lse.double() - ref[0][0]).abs() <= ref[0][1]).all()) and bool(((loss.double() - ref[1][0]).abs() <= ref[1][1]).all())
    assert bool((dw[masked] == 0).all()) and bool(((dw[rest].double() - ref[3][0]).abs() <= ref[3][1]).all())
    assert bool(((dh[:, 1:].double() - ref[2][0][:, 1:]).abs() <= ref[2][1][:, 1:]).all())
    labels[0] = 0
    assert bool(torch.isinf(_softmax(h, w, D, labels, d, 1.0)[0][0]))


def test_softmax_without_tokens_and_without_outputs():
    w = torch.ones((10, 8), device="cuda")
    h, labels, d = torch.ones((0, 8), device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    loss, lse, dh, dw = _softmax(h, w, 8, labels, d, 1.0)
    assert bool((dw == 0).all())                                                        # a sum over nothing
    _softmax(torch.ones((3, 8), device="cuda"), w, 8, torch.zeros(3, dtype=torch.int32, device="cuda"), torch.ones(3, device="cuda"), 1.0, want=(False, False))


@pytest.mark.parametrize("n,V,D", [(70, 1_100_000, 8), (2, 2_200_000, 1_024)])
def test_softmax_of_a_very_large_vocabulary(n, V, D):
    """More words than are laid out at a time; a table of more than 2^31 elements."""
    g = _gen(V)
    h = _matrix(n, D, "bf16", g, 0.2)
    w = torch.zeros((V, D), dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1, V // 2, V - 257, V - 2, V - 1], device="cuda")
    w[at] = (torch.randn((len(at), D), generator=g, device="cuda") * 0.5).bfloat16()
    labels = at[torch.arange(n, device="cuda") % len(at)].int()
    labels[0] = V - 1
    d = torch.full((n,), 0.5, device="cuda")
    loss, lse, dh, dw = _softmax(h, w, D, labels, d, 1.0)
    z = h.double() @ w[at].double().t()                                                 # all others are 0
    want = torch.log(torch.exp(z).sum(1) + (V - len(at)))
    tol = (V / 32 + 128 + 8 * D) * U32 * (1 + want.abs())
    assert bool(((lse.double() - want).abs() <= tol).all())
    place = torch.full((V,), -1, dtype=torch.long, device="cuda")
    place[at] = torch.arange(len(at), device="cuda")
    y = place[labels.long()]
    picked = z.gather(1, y[:, None])[:, 0]
    assert bool(((loss.double() - (want - picked)).abs() <= 2 * tol).all())
    p = torch.exp(z - want[:, None])
    p[torch.arange(n, device="cuda"), y] -= 1
    gw = 0.5 * p.t() @ h.double()
    mass = 0.5 * p.abs().t() @ h.double().abs()
    assert bool(((dw[at].double() - gw).abs() <= (2 * U16 + 2 * float(tol.max())) * mass + U16 * gw.abs()).all())
    others = 0.5 * torch.exp(-want)[None, :] @ h.double()                               # a word whose row is zero
    probe = torch.tensor([2, V // 3, V - 3], device="cuda")
    massp = 0.5 * torch.exp(-want)[None, :] @ h.double().abs()
    assert bool(((dw[probe].double() - others).abs() <= (2 * U16 + 2 * float(tol.max())) * massp + U16 * others.abs()).all())
    gh = 0.5 * p @ w[at].double()
    assert bool(((dh.double() - gh).abs() <= (2 * U16 + 2 * float(tol.max())) * (0.5 * p.abs() @ w[at].double().abs()) + U16 * gh.abs() + 1e-6).all())


# ---------------------------------------------------------------- AdamW
def _f(x):
    return float(np.float32(x))


def _adamw_reference(t, lr, step, b1, b2, eps, gscale=None):
    """The step as the header writes it, in fp32, operation by operation, each by itself."""
    size, fix = _f(lr / (1 - b1 ** step)), _f(1 / math.sqrt(1 - b2 ** step))
    g, p, n = t["grad"].float(), t["param"].float(), t["param"].numel()
    if gscale is not None:
        g = g * gscale
    eight = t["m"].dtype == torch.float8_e4m3fn
    groups = -(-n // 256)

    def spread(s):
        return s.repeat_interleave(256)[:n]

    if eight:
        m = t["m"].float() * spread(t["m_scale"])
        v = t["v"].float() * spread(t["v_scale"])
        v = v * v
    else:
        m, v = t["m"], t["v"]
    m = m * _f(b1) + g * _f(1 - b1)
    v = v * _f(b2) + (g * g) * _f(1 - b2)
    r = torch.sqrt(v)
    keep = 1 - torch.tensor(t.get("weight_decay", 0.0), device="cuda") * _f(lr)
    p = p * keep - (m * _f(size)) / (r * _f(fix) + _f(eps))
    out = {"param": p.to(t["param"].dtype), "copy": p.bfloat16()}
    if not eight:
        return {**out, "m": m, "v": v}
    pad = groups * 256 - n
    mg = torch.nn.functional.pad(m, (0, pad)).view(-1, 256)
    rg = torch.nn.functional.pad(r, (0, pad)).view(-1, 256)
    ms, rs = mg.abs().amax(1), rg.amax(1)
    tiny = 2.0 ** -100
    mi = torch.where(ms >= tiny, (1 / ms) * 448, 0.0)
    ri = torch.where(rs >= tiny, (1 / rs) * 448, 0.0)
    out["m_scale"] = torch.where(ms >= tiny, ms * _f(1 / 448), 0.0)
    out["v_scale"] = torch.where(rs >= tiny, rs * _f(1 / 448), 0.0)
    out["m"] = (mg * mi[:, None]).to(torch.float8_e4m3fn).view(-1)[:n]
    x = rg * ri[:, None]
    i = torch.arange(groups * 256, device="cuda").view(-1, 256)
    off = (((i * 0x9E3779B1 + step * 0x85EBCA77) & 0xFFFFFFFF) >> 12).int()
    bits = (x.clamp(2.0 ** -6, 448).view(torch.int32) + off) & ~0xFFFFF
    x = torch.where(x > 0, bits.view(torch.float32).clamp(max=448), 0.0)
    out["v"] = x.to(torch.float8_e4m3fn).view(-1)[:n]
    return out


def _adamw_exact(t, lr, step, b1, b2, eps, gscale=None):
    """(value, bound) of the new parameters and fp32 states, in 64 bits: m and v are a few roundings of their terms, the step's size
    has twelve and the parameter one more."""
    g = t["grad"].double() * (float(gscale) if gscale is not None else 1.0)
    p, m, v = t["param"].double(), t["m"].double(), t["v"].double()
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    em = 4 * U32 * (b1 * m.abs() + (1 - b1) * g.abs())
    move = lr / (1 - b1 ** step) * m1 / (torch.sqrt(v1 / (1 - b2 ** step)) + eps)
    e_move = move.abs() * 12 * U32 + lr / (1 - b1 ** step) * em / (torch.sqrt(v1 / (1 - b2 ** step)) + eps)
    p1 = p * (1 - lr * t.get("weight_decay", 0.0)) - move
    out = U16 if t["param"].dtype == torch.bfloat16 else 0.0
    return {"m": (m1, em + 1e-44), "v": (v1, 6 * U32 * v1 + 1e-44), "param": (p1, (out + 2 * U32) * p1.abs() + 3 * U32 * p.abs() + e_move * 1.01)}


def _adamw_tensor(n, dtype, grads, states, g, off=0, copy=False, decay=0.0):
    """A tensor and its states, `off` elements into their buffers."""
    def buf(dt):
        return torch.zeros(n + off + 8, dtype=dt, device="cuda")[off:off + n]
    t = {"param": buf(DT[dtype]), "grad": buf(DT[grads]), "weight_decay": decay}
    t["param"].copy_(torch.randn(n, generator=g, device="cuda"))
    t["grad"].copy_(torch.randn(n, generator=g, device="cuda") * 0.01)
    if copy:
        t["param_copy"] = buf(torch.bfloat16)
    sd = torch.float32 if states == "f32" else torch.float8_e4m3fn
    t["m"], t["v"] = (torch.zeros(n + off + 8, dtype=torch.uint8 if states == "8bit" else sd, device="cuda") for _ in range(2))
    t["m"], t["v"] = (t[k].view(sd)[off:off + n] for k in ("m", "v"))
    if states == "8bit":
        t["m_scale"], t["v_scale"] = (torch.zeros(-(-n // 256), device="cuda") for _ in range(2))
    return t


def _bits(t):
    return t.cpu().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_adamw_many_tensors(states):
    """Sizes around groups and chunks, both types of parameters and gradients in one optimizer, tensors that lie anywhere, one
    without elements: three steps from nothing, bit for bit what the definition gives."""
    g = _gen(5)
    sizes = [1, 3, 255, 256, 257, 1_000, 4_095, 4_096, 4_097, 8_192, 100_003, 0, 12_288]
    tensors = [_adamw_tensor(n, ("f32", "bf16")[k % 2], ("f32", "bf16")[k // 2 % 2], states, g, off=(0, 0, 1, 5)[k % 4], copy=k % 3 == 0, decay=0.1 * (k % 2))
               for k, n in enumerate(sizes)]
    opt = B.AdamW(tensors)
    gscale = torch.tensor([0.37], device="cuda")
    for step in (1, 2, 3):
        scale = gscale if step == 2 else None
        want = [_adamw_reference(t, 3e-3, step, 0.9, 0.999, 1e-8, scale) if t["param"].numel() else None for t in tensors]
        exact = [_adamw_exact(t, 3e-3, step, 0.9, 0.999, 1e-8, scale) for t in tensors] if states == "f32" else []
        opt.step(3e-3, step, grad_scale=scale)
        torch.cuda.synchronize()
        for k, (t, w) in enumerate(zip(tensors, want)):
            if w is None:
                continue
            for name in ("param", "m", "v", "m_scale", "v_scale"):
                if name in t:
                    assert torch.equal(_bits(t[name]), _bits(w[name])), (k, step, name)
            if "param_copy" in t:
                assert torch.equal(_bits(t["param_copy"]), _bits(w["copy"])), (k, step)
            for name, (value, bound) in (exact[k].items() if exact else ()):
                assert bool(((t[name].double() - value).abs() <= bound).all()), (k, step, name)
        for t in tensors:
            if t["grad"].numel():
                t["grad"].copy_(torch.randn(t["grad"].numel(), generator=g, device="cuda") * 10.0 ** -step)
    opt.close()


def test_adamw_around_the_caches():
    """More than the memory-side cache holds: the same step."""
    g = _gen(6)
    for states in ("f32", "8bit"):
        t = _adamw_tensor(30_000_001, "f32", "bf16", states, g)
        opt = B.AdamW([t])
        want = _adamw_reference(t, 1e-3, 1, 0.9, 0.999, 1e-8)
        opt.step(1e-3, 1)
        for name in ("param", "m", "v", "m_scale", "v_scale"):
            if name in t:
                assert torch.equal(_bits(t[name]), _bits(want[name])), (states, name)


@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_adamw_gradients_that_are_zero_or_not_finite(states):
    g = _gen(7)
    t = _adamw_tensor(2_000, "f32", "f32", states, g)
    t["grad"].zero_()
    start = t["param"].clone()
    opt = B.AdamW([t])
    opt.step(1e-2, 1)
    assert torch.equal(t["param"], start) and bool((t["m"].float() == 0).all()) and bool((t["v"].float() == 0).all())
    t["grad"][300] = float("nan")
    t["grad"][700] = float("inf")
    opt.step(1e-2, 2)
    bad = ~torch.isfinite(t["param"])
    assert bad.nonzero()[:, 0].tolist() == [300, 700]                       # the element itself, no other
    if states == "8bit":                                                    # the group's states cannot be told any more: that is seen
        for s in (t["m_scale"], t["v_scale"]):
            assert (~torch.isfinite(s)).nonzero()[:, 0].tolist() == [1, 2]


def test_adamw_8_bit_second_moment_follows_a_slow_average():
    """Gradients that grow threefold in half of every group: the average moves by 0.8 % a step and less, far below half a unit
    of the 3 mantissa bits, and is kept all the same: after 3000 steps within a unit (12.5 %) of the exact one, and
    without bias over the elements (2 %)."""
    n, b2 = 4_096, 0.999
    t = _adamw_tensor(n, "f32", "f32", "8bit", _gen(8))
    level = torch.where(torch.arange(n, device="cuda") % 2 == 0, 1e-3, 3e-3)
    opt = B.AdamW([t])
    v = torch.zeros(n, dtype=torch.float64, device="cuda")
    for step in range(1, 4_001):
        gr = torch.full((n,), 1e-3, device="cuda") if step <= 1_000 else level
        t["grad"].copy_(gr)
        opt.step(0.0, step, 0.9, b2)
        v = b2 * v + (1 - b2) * gr.double() ** 2
    root = t["v"].float().double() * t["v_scale"].double().repeat_interleave(256)[:n]
    ratio = root / v.sqrt()
    assert bool(((ratio - 1).abs() <= 0.125).all())
    for half in (0, 1):
        assert abs(float(ratio[half::2].mean()) - 1) <= 0.02


# ---------------------------------------------------------------- together
def _training_step(x):
    B.tensair_embed(x["w_in"], x["D"], x["centers"], x["h"], x["scale"], x["status"])
    B.tensair_softmax_loss(x["h"], x["w_out"], x["D"], x["contexts"], x["loss"], x["lse"], x["ws"], 1.0, -1, x["status"])
    B.tensair_softmax_grad(x["h"], x["w_out"], x["D"], x["contexts"], x["lse"], x["d_loss"], x["d_h"], x["d_out"], x["ws"], 1.0, -1, x["status"])
    B.tensair_embed_grad_dense(x["centers"], x["d_h"], x["D"], x["d_in"], x["ws"], x["scale"], False, x["status"])
    x["opt"].step(1e-2, 1)


def _training_state(seed, n=300, V=500, D=64):
    g = _gen(seed)
    x = {"D": D, "scale": 8.0, "status": _status(), "w_in": _matrix(V, D, "f32", g, 0.05), "w_out": _matrix(V, D, "f32", g, 0.05)}
    x["centers"], x["contexts"] = _ids(n, V, g, 0.2), _ids(n, V, g, 0.1)
    x["h"], x["d_h"] = (torch.empty((n, D), device="cuda") for _ in range(2))
    x["loss"], x["lse"] = (torch.empty(n, device="cuda") for _ in range(2))
    x["d_loss"] = torch.full((n,), 1.0 / n, device="cuda")
    x["d_in"], x["d_out"] = (torch.empty((V, D), device="cuda") for _ in range(2))
    x["ws"] = torch.empty(max(B.tensair_softmax_workspace_bytes(n, V, D, torch.float32, True), B.tensair_embed_workspace_bytes(V, D, n)),
                          dtype=torch.uint8, device="cuda")
    x["opt"] = B.AdamW([{"param": x[w], "grad": x[gr], "m": torch.zeros((V, D), device="cuda"), "v": torch.zeros((V, D), device="cuda")}
                        for w, gr in (("w_in", "d_in"), ("w_out", "d_out"))])
    return x


@pytest.mark.parametrize("n", [6, 300, 5_000])
def test_a_training_step_as_a_graph(n):
    """One step recorded, replayed five times with other work and waits between: the tables are those of five eager steps, bit for bit."""
    eager, graphed = _training_state(3, n), _training_state(3, n)
    side = torch.cuda.Stream()
    warm = _training_state(3, n)
    with torch.cuda.stream(side):
        _training_step(warm)                                   # first launches load code: not while recording
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        _training_step(graphed)
    for _ in range(5):
        _training_step(eager)
        graph.replay()
        torch.cuda.synchronize()
        torch.ones(1 << 20, device="cuda").sum().item()
        assert torch.equal(graphed["w_in"], eager["w_in"]) and torch.equal(graphed["w_out"], eager["w_out"]) and torch.equal(graphed["loss"], eager["loss"])


def test_calls_on_another_stream():
    """Work queued on a stream of its own follows what that stream did before, and nothing else."""
    a, b = _training_state(4), _training_state(4)
    _training_step(a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fill = b["centers"].clone()
        b["centers"].zero_()
        for _ in range(50):
            torch.mm(torch.ones((512, 512), device="cuda"), torch.ones((512, 512), device="cuda"))
        b["centers"].copy_(fill)
        _training_step(b)
    torch.cuda.synchronize()
    assert torch.equal(a["w_in"], b["w_in"]) and torch.equal(a["w_out"], b["w_out"]) and int(a["status"]) == 0
