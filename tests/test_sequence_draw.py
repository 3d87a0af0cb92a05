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
