"""Drawing words where the weights themselves decide: words far below the most probable one, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from test_sequence_operators import U32, _draw, _draw_reference, _gen

pytestmark = pytest.mark.gpu


def _check(z, V, u, T=None, k=None, p=None, m=None):
    """Words and probabilities of every row; what is not given is not given to the call either.  Weights and sums are in 64 bits: one rounding to fp32, whose smallest number is 2^-149."""
    n = len(u)
    given = {key: np.asarray(v) for key, v in (("temperature", T), ("top_k", k), ("top_p", p), ("min_p", m)) if v is not None}
    words, prob, st = _draw(z, V, u=u, **given)
    host, f = z[:, :V].float().cpu().numpy(), lambda x, i, none: none if x is None else float(np.float32(x[i]))      # noqa: E731
    for i in range(n):
        v, q = _draw_reference(host[i], f(T, i, 1.0), 0 if k is None else int(k[i]), f(p, i, 1.0), f(m, i, 0.0), float(np.float32(u[i])))
        assert int(words[i]) == v, (i, V, {key: x[i] for key, x in given.items()}, u[i], int(words[i]), v)
        assert abs(float(prob[i]) - q) <= 2 * U32 * q + 2.0 ** -150, (i, float(prob[i]), q)
    assert int(st) == 0


@pytest.mark.parametrize("V", [6_000, 8_193, 20_000, 100_003])
@pytest.mark.parametrize("k", [0, 50, 300])
@pytest.mark.parametrize("p", [1.0, 0.999])
def test_words_of_tiny_weight(V, k, p):
    """At a temperature of 0.05 words among the first 50 have weights of e^-40 and less: min_p parts them, and where none is given the first and the last word that is left have them.
    Rows of lists of few and of hundreds of words, of one launch and of several."""
    n = 12
    z = torch.randn((n, V), generator=_gen(V + k), device="cuda") * 4
    z[4:8, V // 3:] = -60.0                                    # the last third of the words, far below, has the last word that is left, if k leaves one
    least = np.array([0.0, 1e-20, 1e-12, 1e-28] * 3)
    for u in (np.zeros(n), np.full(n, 0.5), np.full(n, 0.999)):
        _check(z, V, u, np.full(n, 0.05), np.full(n, k), np.full(n, p), least)


def test_a_word_is_drawn_where_min_p_leaves_none_of_a_part():
    """The last words of the list are all below min_p: the last word that is left is before them."""
    V, k = 20_000, 300
    z = -100 - 100 * torch.rand((1, V), generator=_gen(1), device="cuda")
    z[0, 10], z[0, 11] = 0.0, -0.5
    z[0, V - 250:] = -2.5                                      # e^-50 at this temperature
    for least in (0.0, 1e-21, 1e-22):
        for u in (0.0, 1.0):
            _check(z, V, [u], [0.05], [k], [1.0], [least])
    words, prob, _ = _draw(z, V, temperature=[0.05], top_k=[k], min_p=[1e-21], u=[1.0])
    assert int(words) == 11 and float(prob) > 0


@pytest.mark.parametrize("V", [6_000, 8_193, 20_000, 100_003, 1_100_000])
@pytest.mark.parametrize("k,p", [(0, 1.0), (300, 1.0), (50, 1.0), (0, 0.9999)])
def test_u_of_one_is_the_last_word(V, k, p):
    """Whatever its weight is beside the sum, which no running sum of 64 bits may show."""
    n = 12
    z = torch.randn((n, V), generator=_gen(V + k + 1), device="cuda") * 4
    z[4:8, :V // 3] -= 10                                      # the likely words last, or first
    z[8:, V // 3:] -= 10
    _check(z, V, np.array([1.0, 1.5, float("inf")] * 4), np.array([0.05, 0.1, 0.05, 1.0] * 3), np.full(n, k), np.full(n, p), np.array([0.0, 1e-28, 1e-20] * 4))


@pytest.mark.parametrize("V", [6_000, 8_193, 20_000, 100_003])
@pytest.mark.parametrize("k,p", [(0, 1.0), (300, 1.0), (50, 1.0), (600, 0.999999)])
def test_tiny_u(V, k, p):
    """A u far below the last place of 32 bits falls among words of tiny weights that come before the likely ones."""
    n = 12
    z = torch.randn((n, V), generator=_gen(V + k + 2), device="cuda") * 4
    z[:, 3 * V // 4:] += 8                                     # the likely words last
    _check(z, V, 10.0 ** -np.arange(8, 44, 3), np.array([0.05, 0.1, 0.2] * 4), np.full(n, k), np.full(n, p), np.array([0.0, 1e-30] * 6))


@pytest.mark.parametrize("V", [6_000, 20_000])
def test_u_does_not_matter_where_the_first_word_is_taken(V):
    """Two words of the largest logit: the first of them, by temperature, top-k or top-p, whatever u is."""
    z = torch.randn((6, V), generator=_gen(V), device="cuda")
    z[:, 17] = z[:, V - 9] = 8.0
    for u in (0.0, 0.7, 1.0, 2.0):
        words, prob, _ = _draw(z, V, temperature=[0.0, 0.0, 1.0, 1.0, 1.0, 1.0], top_k=[0, 9, 1, 1, 0, 5], top_p=[1.0, 0.5, 1.0, 0.5, 0.0, 0.0], u=np.full(6, u))
        assert words.tolist() == [17] * 6 and prob.tolist() == [1.0] * 6


def _last_left(row, p):
    """The first and the last place that the last word left by top-p may have, of a row in falling order: sums in extended precision, moved by what the operator may round.  A weight is off
    by at most (0.7 |log2 w| + 4) units of 2^-53, which the tails here, below 1e-3 of the sum, make small; sums and products of 64 bits are off by 8 of them with room."""
    z = row.double().cpu().numpy()
    # the tail by itself: 2^23 equal words of 2^-43 added to 1 in 64 bits of mantissa may be off by 2^-64 each, which is 4 of them; added to each other by 2^-84, 2^-61 in all
    run = 1 + np.concatenate([[np.longdouble(0)], np.cumsum(np.exp((z[1:] - z[0]).astype(np.longdouble)))])
    off = (8 + 1e-3 * (0.7 * 50 + 4)) * 2.0 ** -53 * run[-1]
    want = np.longdouble(np.float32(p)) * run[-1]
    lo, hi = (int(np.searchsorted(run, x, side="left")) for x in (want - off, want + off))
    assert 0 < lo <= hi <= lo + 1 and hi < len(z) - 1          # the places tell
    return lo, hi


@pytest.mark.parametrize("V,p,first,fall,rows", [(128_000, 0.99999, 20.0, 4.0, (1, 64)), (1_000_000, 0.9999, 20.0, 4.0, (1, 25, 256)), (1_048_577, 0.9999, 20.0, 4.0, (1, 130)),
                                                 (4_000_000, 0.999998, 25.0, 5.0, (1, 64)), (16_777_216, 0.999999, 29.0, 2.0, (1, 16))])
def test_border_in_a_long_tail(V, p, first, fall, rows):
    """One likely word and a tail in falling order, in which top-p ends: with u of 1 the word that is drawn is the last one that is left.  A row gives the same word alone and among others."""
    row = -first - fall * torch.arange(V, device="cuda", dtype=torch.float64) / V
    row[0] = 0.0
    row = row.float()
    lo, hi = _last_left(row, p)
    got = set()
    for n in rows:
        words, _, st = _draw(row.expand(n, V).contiguous(), V, top_p=np.full(n, p), u=np.ones(n))
        got |= set(words.tolist())
        assert int(st) == 0
    assert len(got) == 1 and lo <= min(got) <= hi, (got, lo, hi)


@pytest.mark.parametrize("V,p,n", [(300_000, 0.999997, 1), (300_000, 0.999997, 30), (16_777_216, 0.999999, 16)])
def test_border_among_a_tail_of_equal_words(V, p, n):
    """The same where all words but one have one logit, so that roundings of their weights are the same ones."""
    row = torch.full((V,), -25.25 if V < 1 << 20 else -29.75, device="cuda").bfloat16()
    row[0] = 0.0
    lo, hi = _last_left(row, p)
    words, _, st = _draw(row.expand(n, V).contiguous(), V, top_p=np.full(n, p), u=np.ones(n))
    assert set(words.tolist()) <= {lo, hi} and len(set(words.tolist())) == 1 and int(st) == 0, (words.tolist(), lo, hi)


@pytest.mark.parametrize("V,n", [(20_000, 8), (100_003, 6)])
def test_border_behind_top_k(V, n):
    """top-p beside top-k, both in a tail of words of 1e-9 and less."""
    row = -20 - 4 * torch.arange(V, device="cuda", dtype=torch.float64) / V
    row[0] = 0.0
    row = row.float()
    for k in (200, 3_000, 17_000):
        run = np.cumsum(np.exp(row[:k].double().cpu().numpy().astype(np.longdouble)))
        p = float(np.float32((run[k // 2] / run[-1])))
        assert float(run[0] / run[-1]) < p < 1
        lo, hi = _last_left(row[:k], p)
        words, _, _ = _draw(row.expand(n, V).contiguous(), V, top_k=np.full(n, k), top_p=np.full(n, p), u=np.ones(n))
        assert set(words.tolist()) <= {lo, hi}, (k, words.tolist(), lo, hi)


@pytest.mark.parametrize("V,dtype", [(1, "f32"), (6_000, "f32"), (8_193, "bf16"), (20_000, "f32"), (100_003, "bf16"), (1_100_000, "f32")])
@pytest.mark.parametrize("given", ["", "T", "m", "k", "p", "Tm", "kp", "Tkpm"])
def test_filters_that_are_not_given(V, dtype, given):
    """Every filter's address may be NULL: no vector but u, each by itself, and some together; rows with masked words and with infinite ones."""
    n, r = 9 if V < 50_000 else 5, np.random.RandomState(V)
    z = torch.randn((n, V), generator=_gen(V + 7), device="cuda") * 3
    if V > 1:
        z[1, ::2] = -float("inf")
        z[2, V // 2:] = torch.finfo(torch.float32).min
        z[3, 5] = z[3, V - 3] = float("inf")
        z[4, ::3] = float("nan")
    z = z.to(torch.float32 if dtype == "f32" else torch.bfloat16)
    some = {"T": r.choice([0.0, 0.3, 1.0, 2.0], n), "m": r.choice([0.0, 0.01, 0.5], n), "k": r.choice([0, 1, 40, 900], n), "p": r.choice([0.3, 0.9, 1.0], n)}
    for u in (np.ones(n), np.zeros(n), r.rand(n), r.rand(n) * 0.01)[:4 if V < 50_000 else 3]:
        _check(z, V, u, **{x: some[x] for x in given})
