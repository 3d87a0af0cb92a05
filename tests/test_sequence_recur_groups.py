"""The recurrence where its state is handed on between groups of tiles: long sequences, narrow and wide layers, both types, sequence borders beside the groups' borders."""
import numpy as np
import pytest
import torch

from paper_2211_10280_amd import binding as B
from test_sequence_operators import DT, U32, UNIT, _bytes, _gen, _near, _status

pytestmark = pytest.mark.gpu

TILE = 256


def _scan(a, b, reset):
    """h[t] = a[t] h[t - 1] + b[t] in 64 bits by doubling; a does not count where reset."""
    a, b = torch.where(reset[:, None], 0.0, a), b.clone()
    step = 1
    while step < len(a):
        b[step:] = a[step:] * b[:-step] + b[step:]
        a[step:] = a[step:] * a[:-step]
        step *= 2
    return b


def _inputs(n, D, dtype, seed):
    """Gates from 3 to 7: a state is remembered for 20 to 1 000 tokens, over tiles' borders, and groups' ones."""
    g = _gen(seed)
    x, d = (torch.randn((n, D), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    gate = (3 + 4 * torch.rand((n, D), generator=g, device="cuda")).to(DT[dtype])
    return g, x, gate, d


TILES = 131
# groups of 32 tiles, 64 where a layer has few channels, counted from the first tile and, for the gradient, from the last; borders at them, a token before and behind
BORDERS = sorted([32 * TILE, 64 * TILE, 96 * TILE] + [(TILES - k) * TILE for k in (32, 64, 96)])


@pytest.mark.parametrize("D,dtype", [(40, "f32"), (40, "bf16"), (132, "f32"), (132, "bf16"), (260, "bf16")])
@pytest.mark.parametrize("cut", [None, 0, 1, -1])
def test_recur_over_groups(D, dtype, cut):
    """One sequence of 131 tiles, or sequences that begin at, behind and before borders of groups, forward and back, against 64 bits."""
    n = (TILES - 1) * TILE + 77
    g, x, gate, d = _inputs(n, D, dtype, D + (cut or 0))
    off = np.array([0] + ([] if cut is None else [b + cut for b in BORDERS]) + [n], np.int32)
    S = len(off) - 1
    h0, d_last = (torch.randn((S, D), generator=g, device="cuda") for _ in range(2))
    offsets, status = torch.from_numpy(off).cuda(), _status()
    out, dx, dg = (torch.empty((n, D), dtype=DT[dtype], device="cuda") for _ in range(3))
    last, dh0, states = torch.empty((S, D), device="cuda"), torch.empty((S, D), device="cuda"), torch.empty((B.tensair_recur_state_rows(n), D), device="cuda")
    ws = _bytes(B.tensair_recur_workspace_bytes(n, D))
    B.tensair_recur(x, gate, D, offsets, out, ws, h0, last, states, status)
    B.tensair_recur_grad(x, gate, D, offsets, states, d, dx, dg, ws, h0, d_last, dh0, status)

    head, tail = (torch.zeros(n, dtype=torch.bool, device="cuda") for _ in range(2))
    head[torch.from_numpy(off[:-1]).long()], tail[torch.from_numpy(off[1:] - 1).long()] = True, True
    x, gate, d = x.double(), gate.double(), d.double()
    a, b = torch.sigmoid(gate), torch.sigmoid(-gate)
    push = b * x
    push[head] += a[head] * h0.double()
    h = _scan(a, push, head)
    before = torch.roll(h, 1, 0)
    before[head] = h0.double()
    come = d.clone()
    come[tail] += d_last.double()
    nxt = torch.roll(a, -1, 0)
    lam = _scan(nxt.flip(0), come.flip(0), tail.flip(0)).flip(0)
    # A token rounds a by 2 units and b's e^-gate by (1.5 * 7 + 4) more, product and sum by one each; an error of h or l is remembered for at most 1 / (1 - a) tokens, 1 100 for gates of 7, and
    # h is then as large as what made it.  So h is off by at most (2 + 15 + 2) 1 100 units of the largest |h|, as a share of it b times as much where a is small; twice that for the maps.
    # Errors of single tokens are of either sign: their sum is taken as 6 times the root of their number.
    near = 2 * 19 * 6 * 1_100 ** 0.5 * U32
    eh, el = near * h.abs().amax(), near * lam.abs().amax()
    _near(out, h, eh + UNIT[dtype] * (h.abs() + eh), "out")
    _near(last, h[tail], torch.full_like(h[tail], float(eh)), "h_last")
    rx, rg = b * lam, lam * (before - x) * a * b
    ex = b * el + 20 * U32 * rx.abs()
    eg = a * b * (el * (before - x).abs() + lam.abs() * eh) + 40 * U32 * rg.abs()
    _near(dx, rx, ex + UNIT[dtype] * (rx.abs() + ex), "d_x")
    _near(dg, rg, eg + UNIT[dtype] * (rg.abs() + eg), "d_gate")
    want = (a * lam)[head]
    _near(dh0, want, torch.full_like(want, float(el)), "d_h0")
    assert int(status) == 0
