"""The operators of a model of word sequences recorded into graphs, on other streams, and with workspaces that others use."""
import pytest
import torch

from paper_2211_10280_amd import binding as B

pytestmark = pytest.mark.gpu


class Layer:
    """Buffers of a step through all operators that goes through every launch they have: n tokens of D, S sequences, a vocabulary of V, drawn rows R."""

    def __init__(self, seed, dtype, workspace=None, n=9_000, D=72, S=5, V=20_000, R=3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.n, self.D, self.V = n, D, V
        dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]

        def rows(h, w, kind=dt):
            return torch.randn((h, w), generator=g, device="cuda").to(kind)

        self.x, self.both, self.d, self.h0, self.logits = rows(n, D), rows(n, 2 * D), rows(n, D), rows(S, D, torch.float32), rows(R, V)
        self.weight, self.bias, self.u = torch.rand(D, generator=g, device="cuda"), torch.rand(D, generator=g, device="cuda"), torch.rand(R, generator=g, device="cuda")
        self.state, self.slots = rows(S, D, torch.float32), torch.tensor([3, 0, 3], dtype=torch.int32, device="cuda")
        self.offsets = torch.linspace(0, n, S + 1, device="cuda").round().to(torch.int32)
        self.top_k, self.top_p = torch.tensor([0, 30, 0], dtype=torch.int32, device="cuda"), torch.tensor([0.9, 0.9, 1.0], device="cuda")
        self.step = torch.zeros(1, dtype=torch.int64, device="cuda")
        need = self.need()
        self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda") if workspace is None else workspace
        f = lambda *s: torch.zeros(s, device="cuda")      # noqa: E731
        self.out = {"y": torch.zeros_like(self.x), "mean": f(n), "rstd": f(n), "drop": torch.zeros_like(self.x), "h": torch.zeros_like(self.x), "last": f(S, D),
                    "states": f(B.tensair_recur_state_rows(n), D), "d_both": torch.zeros_like(self.both), "d_h0": f(S, D), "d_x": torch.zeros_like(self.x), "d_w": f(D), "d_b": f(D),
                    "words": torch.zeros(R, dtype=torch.int32, device="cuda"), "prob": f(R), "one": torch.zeros_like(self.x[:3]), "state": self.state}

    def need(self):
        return max(B.tensair_recur_workspace_bytes(self.n, self.D), B.tensair_norm_workspace_bytes(self.n, self.D), B.tensair_sample_workspace_bytes(3, self.V))

    def run(self):
        o, D, ws = self.out, self.D, self.workspace
        self.step.add_(1)
        B.tensair_norm(self.x, D, self.weight, self.bias, o["y"], o["mean"], o["rstd"])
        B.tensair_dropout(o["y"], D, o["drop"], 0.3, 7, 2, self.step, self.x)
        B.tensair_recur(o["drop"], self.both[:, D:], D, self.offsets, o["h"], ws, self.h0, o["last"], o["states"])
        B.tensair_recur_grad(o["drop"], self.both[:, D:], D, self.offsets, o["states"], self.d, o["d_both"][:, :D], o["d_both"][:, D:], ws, self.h0, o["last"], o["d_h0"])
        B.tensair_norm_grad(o["d_both"][:, :D].contiguous(), self.x, D, self.weight, o["mean"], o["rstd"], o["d_x"], o["d_w"], o["d_b"], ws, self.d)
        B.tensair_sample(self.logits, self.V, self.u, o["words"], ws, None, self.top_k, self.top_p, None, o["prob"])
        B.tensair_recur_step(self.x[:3], self.both[:3, D:], D, o["state"], o["one"], self.slots)

    def change(self, k):
        self.x.mul_(-0.9 if k % 2 else 1.1)
        self.logits.copy_(self.logits.roll(k + 1, 1))
        self.u.mul_(0.7)

    def same(self, other):
        return [k for k in self.out if not torch.equal(self.out[k].view(torch.uint8), other.out[k].view(torch.uint8))]


def _noise():
    torch.ones(1 << 20, device="cuda").sum().item()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_replays_are_the_eager_calls(dtype):
    """Recorded once, replayed with other inputs and the step counted up in the graph: bit for bit what the calls give, eager work and other contents of the workspace in between."""
    eager, graphed, warm = (Layer(1, dtype) for _ in range(3))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        warm.run()                                             # first launches load code: not while recording
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        graphed.run()
    for k in range(5):
        graphed.workspace.fill_(255 if k % 2 else 77)
        eager.run()
        graph.replay()
        torch.cuda.synchronize()
        assert eager.same(graphed) == [], k
        assert int(graphed.step) == k + 1
        _noise()
        eager.change(k)
        graphed.change(k)


def test_two_graphs_share_a_workspace():
    """On one stream, replayed in turn and out of turn."""
    a, b = Layer(2, "f32"), Layer(3, "bf16")
    c, d = Layer(2, "f32"), Layer(3, "bf16")
    shared = torch.empty(max(a.need(), b.need()), dtype=torch.uint8, device="cuda")
    c.workspace = d.workspace = shared
    side = torch.cuda.Stream()
    graphs = []
    for layer, first in ((c, Layer(4, "f32")), (d, Layer(4, "bf16"))):
        with torch.cuda.stream(side):
            first.run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            layer.run()
        graphs.append(graph)
    for order in ((0, 1), (1, 0), (0, 1, 1, 0)):
        for k in order:
            graphs[k].replay()
            (a, b)[k].run()
        torch.cuda.synchronize()
        assert a.same(c) == [] and b.same(d) == []
        _noise()


def test_two_streams_at_once():
    """Calls on two streams, each with a workspace of its own, while both are busy: the bits of calls one after the other."""
    alone = [Layer(5, "bf16"), Layer(6, "f32")]
    for layer in alone:
        for _ in range(4):
            layer.run()
    torch.cuda.synchronize()
    both = [Layer(5, "bf16"), Layer(6, "f32")]
    streams = [torch.cuda.Stream() for _ in both]
    torch.cuda.synchronize()
    for _ in range(4):
        for layer, s in zip(both, streams):
            with torch.cuda.stream(s):
                layer.run()
    torch.cuda.synchronize()
    for x, y in zip(alone, both):
        assert x.same(y) == []


def test_stream_argument():
    """The calls' own stream argument, beside the current stream."""
    a, b = Layer(7, "f32", n=700), Layer(7, "f32", n=700)
    a.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    o, D, ws = b.out, b.D, b.workspace
    b.step.add_(1)
    torch.cuda.synchronize()
    B.tensair_norm(b.x, D, b.weight, b.bias, o["y"], o["mean"], o["rstd"], stream=s)
    B.tensair_dropout(o["y"], D, o["drop"], 0.3, 7, 2, b.step, b.x, stream=s)
    B.tensair_recur(o["drop"], b.both[:, D:], D, b.offsets, o["h"], ws, b.h0, o["last"], o["states"], stream=s)
    B.tensair_recur_grad(o["drop"], b.both[:, D:], D, b.offsets, o["states"], b.d, o["d_both"][:, :D], o["d_both"][:, D:], ws, b.h0, o["last"], o["d_h0"], stream=s)
    s.synchronize()
    d = o["d_both"][:, :D].contiguous()
    torch.cuda.synchronize()
    B.tensair_norm_grad(d, b.x, D, b.weight, o["mean"], o["rstd"], o["d_x"], o["d_w"], o["d_b"], ws, b.d, stream=s)
    B.tensair_sample(b.logits, b.V, b.u, o["words"], ws, None, b.top_k, b.top_p, None, o["prob"], stream=s)
    B.tensair_recur_step(b.x[:3], b.both[:3, D:], D, o["state"], o["one"], b.slots, stream=s)
    torch.cuda.synchronize()
    assert a.same(b) == []


def test_the_same_call_gives_the_same_bits():
    """70 000 tokens, where the tiles' workgroups meet in another order every time."""
    first = Layer(8, "bf16", n=70_000, D=260, S=2)
    first.run()
    torch.cuda.synchronize()
    keep = {k: v.clone() for k, v in first.out.items()}
    for _ in range(6):
        first.step.zero_()
        first.run()
        torch.cuda.synchronize()
        assert [k for k in keep if k not in ("state", "one") and not torch.equal(keep[k].view(torch.uint8), first.out[k].view(torch.uint8))] == []
