"""Steps of the optimizer that are recorded into a graph."""
import ctypes as C

import pytest
import torch

from paper_2211_10280_amd import binding as B


def _state(seed, states):
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for n, dtype in ((70_001, torch.float32), (300, torch.bfloat16)):
        t = {"param": torch.randn(n, generator=g, device="cuda").to(dtype), "grad": (torch.randn(n, generator=g, device="cuda") * 1e-2).to(dtype), "weight_decay": 0.1}
        if states == "8bit":
            t["m"], t["v"] = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
            t["m_scale"], t["v_scale"] = (torch.zeros(-(-n // 256), device="cuda") for _ in range(2))
        else:
            t["m"], t["v"] = (torch.zeros(n, device="cuda") for _ in range(2))
        out.append(t)
    return out


def _same(a, b):
    return all(torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)) for x, y in zip(a, b) for k in x if k != "weight_decay")


@pytest.mark.gpu
@pytest.mark.parametrize("states", ["f32", "8bit"])
def test_replays_of_a_recorded_step_are_the_steps_that_follow(states):
    """One step recorded, its number counted up in the graph, its size changed between replays: bit for bit what as many eager steps give."""
    eager, graphed, warm = (_state(1, states) for _ in range(3))
    a, b, w = B.AdamW(eager), B.AdamW(graphed), B.AdamW(warm)
    step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.full((1,), 1e-2, dtype=torch.float64, device="cuda")
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        w.step(lr, step + 1)                                   # first launches load code: not while recording
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step.add_(1)
        b.step(lr, step)
    for k in range(1, 8):
        rate = 1e-2 / k
        lr.fill_(rate)
        a.step(rate, k)
        graph.replay()
        torch.cuda.synchronize()
        torch.ones(1 << 20, device="cuda").sum().item()
        assert int(step) == k and _same(eager, graphed), k
        for x, y in zip(eager, graphed):
            x["grad"].mul_(-0.7)
            y["grad"].mul_(-0.7)
    # far on, and a step below 1, which is taken as the first
    for k, same in ((100_003, 100_003), (2 ** 33 + 5, 2 ** 33 + 5), (0, 1)):
        step.fill_(k - 1)
        lr.fill_(3e-3)
        graph.replay()
        a.step(3e-3, same)
        torch.cuda.synchronize()
        assert _same(eager, graphed), k
    for opt in (a, b, w):
        opt.close()


@pytest.mark.gpu
def test_a_slow_average_moves_in_replays():
    """8-bit second moments under gradients three times as large in half of every group: after 3 000 replays they are within a unit (12.5 %) of
    the exact average (a step repeated with the same offsets would leave most of them standing)."""
    n, b2 = 4_096, 0.999
    t = {"param": torch.zeros(n, device="cuda"), "grad": torch.full((n,), 1e-3, device="cuda"), "m_scale": torch.zeros(16, device="cuda"),
         "v_scale": torch.zeros(16, device="cuda"), **{k: torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for k in "mv"}}
    opt = B.AdamW([t])
    step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")
    opt.step(lr, step + 1)
    for k in ("m", "v"):
        t[k].view(torch.uint8).zero_()
        t[k + "_scale"].zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        opt.step(lr, step, 0.9, b2)
    v = torch.zeros(n, dtype=torch.float64, device="cuda")
    for k in range(1, 4_001):
        if k == 1_001:
            t["grad"][1::2] = 3e-3
        graph.replay()
        v = b2 * v + (1 - b2) * t["grad"].double() ** 2
    torch.cuda.synchronize()
    ratio = t["v"].float().double() * t["v_scale"].double().repeat_interleave(256) / v.sqrt()
    assert bool(((ratio - 1).abs() <= 0.125).all())
    opt.close()


def test_refusals():
    L = B.lib()
    buf = (C.c_char * 4096)()
    mem = (C.addressof(buf) + 255) & ~255
    assert L.tensair_adamw_step_at(None, mem, mem, 0.9, 0.999, 1e-8, None, None) == B.EINVAL
    t = torch.zeros(1)
    for lr, step in ((t.double(), t.long()), (0.1, t.long())):
        with pytest.raises((B.TensairError, AttributeError)):
            B.tensair_adamw_step_at(None, lr, step)


@pytest.mark.gpu
def test_refusals_of_a_handle():
    opt = B.AdamW(_state(2, "f32"))
    lr, step = torch.zeros(2, dtype=torch.float64, device="cuda"), torch.ones(2, dtype=torch.int64, device="cuda")

    def call(lr=lr.data_ptr(), step=step.data_ptr(), b1=0.9, b2=0.999, eps=1e-8, scale=None):
        return B.lib().tensair_adamw_step_at(opt.h, lr, step, b1, b2, eps, scale, torch.cuda.current_stream().cuda_stream)

    for bad in (dict(lr=None), dict(step=None), dict(lr=lr.data_ptr() + 4), dict(step=step.data_ptr() + 4), dict(b1=1.0), dict(b2=-0.1), dict(eps=0.0), dict(scale=2)):
        assert call(**bad) == B.EINVAL, bad
    for bad in ((lr.float(), step), (lr, step.int()), (lr, step.cpu()), (lr.cpu(), step), (lr[:0], step)):
        with pytest.raises(B.TensairError):
            opt.step(*bad)
    assert call() == B.OK
    torch.cuda.synchronize()
    opt.close()
