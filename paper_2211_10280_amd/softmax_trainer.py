"""A skip-gram model trained against the whole vocabulary, with AdamW.

Where :mod:`trainer` follows the paper (negative sampling, Eq. 1), this sequences the operators for a table that is
a model's input and output layer: the vectors of the center words (``tensair_embed``), the exact softmax over all
words with the context word as the label (``tensair_softmax_loss``, ``tensair_softmax_grad``), the gradient of the
center words' table by sorted words (``tensair_embed_grad_dense``), one optimizer step over both tables
(``tensair_adamw_step``).  The optimizer holds the tables in float32; with ``dtype="bf16"`` the products read bfloat16
copies that the optimizer step writes beside them.

    python -m paper_2211_10280_amd.softmax_trainer --steps 50 --states 8bit

Everything numerical happens inside the library; this file only sequences calls and keeps buffers.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B

IGNORE = -1      # the label of a pair that is none (a window cut off by the stream's ends)


class SoftmaxWorker:
    def __init__(self, vocab, dim, max_pairs, dtype="bf16", states="f32", seed=0, lr=1e-2, weight_decay=0.0, device="cuda"):
        """max_pairs: most (center, context) pairs of a step.  states: what the optimizer's moments are kept in, "f32" or "8bit"."""
        self.vocab, self.dim, self.max_pairs, self.lr, self.step_no = vocab, dim, max_pairs, lr, 0
        self.scale = dim ** 0.5                      # vectors of a length that does not depend on dim
        dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        g = torch.Generator(device=device).manual_seed(seed)
        self.w_in, self.w_out = (torch.randn((vocab, dim), generator=g, device=device) / dim for _ in range(2))
        copies = [w.to(dt) if dt != torch.float32 else None for w in (self.w_in, self.w_out)]
        self.in_rows, self.out_rows = (c if c is not None else w for c, w in zip(copies, (self.w_in, self.w_out)))
        self.d_in = torch.zeros((vocab, dim), dtype=dt, device=device)
        self.d_out = torch.zeros_like(self.d_in)
        tensors = []
        for w, d, copy in zip((self.w_in, self.w_out), (self.d_in, self.d_out), copies):
            t = {"param": w.view(-1), "grad": d.view(-1), "weight_decay": weight_decay}
            if states == "8bit":
                groups = -(-w.numel() // 256)
                t["m"], t["v"] = (torch.zeros(w.numel(), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn) for _ in range(2))
                t["m_scale"], t["v_scale"] = (torch.zeros(groups, device=device) for _ in range(2))
            else:
                t["m"], t["v"] = (torch.zeros(w.numel(), device=device) for _ in range(2))
            if copy is not None:
                t["param_copy"] = copy.view(-1)
            tensors.append(t)
        self.optimizer = B.AdamW(tensors)
        self.h = torch.empty((max_pairs, dim), dtype=dt, device=device)
        self.d_h = torch.empty_like(self.h)
        self.loss, self.lse = (torch.empty(max_pairs, device=device) for _ in range(2))
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        nbytes = max(B.tensair_softmax_workspace_bytes(max_pairs, vocab, dim, dt, True), B.tensair_embed_workspace_bytes(vocab, dim, max_pairs))
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)

    def step(self, centers, contexts, d_loss):
        """One step on int32 [n] center words and context words (IGNORE: no pair); d_loss: float32 [n], 1 / pairs for their mean.
        Returns the losses of the pairs, before the step."""
        n, D = centers.numel(), self.dim
        h, d_h, loss, lse = self.h[:n], self.d_h[:n], self.loss[:n], self.lse[:n]
        B.tensair_embed(self.in_rows, D, centers, h, self.scale, self.status)
        B.tensair_softmax_loss(h, self.out_rows, D, contexts, loss, lse, self.workspace, 1.0, IGNORE, self.status)
        B.tensair_softmax_grad(h, self.out_rows, D, contexts, lse, d_loss, d_h, self.d_out, self.workspace, 1.0, IGNORE, self.status)
        B.tensair_embed_grad_dense(centers, d_h, D, self.d_in, self.workspace, self.scale, False, self.status)
        self.step_no += 1
        self.optimizer.step(self.lr, self.step_no)
        return loss

    def score(self, center, context):
        """Minus log probability of a context word beside a center word, for few pairs: what a server answers."""
        n = center.numel()
        h = torch.empty((n, self.dim), dtype=self.h.dtype, device=self.h.device)
        loss, lse = torch.empty((2, n), device=self.h.device)
        B.tensair_embed(self.in_rows, self.dim, center, h, self.scale, self.status)
        B.tensair_softmax_loss(h, self.out_rows, self.dim, context, loss, lse, self.workspace, 1.0, IGNORE, self.status)
        return loss

    def close(self):
        self.optimizer.close()


def window_pairs(tokens, begin, n_centers, window):
    """(centers, contexts, 1 / pairs for every pair) of a run of center positions in a device int32 stream; contexts beyond its ends
    are IGNORE, so that every run of a length has as many pairs."""
    pos = torch.arange(begin, begin + n_centers, device=tokens.device)
    off = torch.cat([torch.arange(-window, 0, device=tokens.device), torch.arange(1, window + 1, device=tokens.device)])
    at = pos[:, None] + off
    inside = (at >= 0) & (at < tokens.numel())
    contexts = torch.where(inside, tokens[at.clamp(0, tokens.numel() - 1)], IGNORE).view(-1)
    centers = tokens[pos][:, None].expand(-1, 2 * window).reshape(-1)
    return centers, contexts, (1.0 / inside.sum()).expand(contexts.numel()).float().contiguous()


def main(argv=None):
    import workload as W

    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--config", type=int, default=2, choices=sorted(W.CONFIGS), help="workload whose vocabulary, row length, window and mini-batch are taken")
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--dtype", default="bf16", choices=("f32", "bf16"))
    ap.add_argument("--states", default="f32", choices=("f32", "8bit"))
    ap.add_argument("--lr", type=float, default=1e-2)
    a = ap.parse_args(argv)
    cfg = W.CONFIGS[a.config]
    cfg = cfg.scaled(tokens=min(cfg.tokens, a.steps * cfg.batch + 1))
    tokens = torch.from_numpy(W.make_stream(cfg)[0]).cuda()
    worker = SoftmaxWorker(cfg.vocab, cfg.dim, 2 * cfg.window * cfg.batch, a.dtype, a.states, cfg.seed, a.lr)
    for t in range(a.steps):
        begin, n, _ = W.batch_slice(cfg, t)
        centers, contexts, d_loss = window_pairs(tokens, begin, n, cfg.window)
        loss = worker.step(centers, contexts, d_loss)
        if t % 10 == 0 or t + 1 == a.steps:
            print(f"step {t}: mean loss {float((loss * d_loss).sum()):.4f}", flush=True)
    assert int(worker.status) == 0
    worker.close()


if __name__ == "__main__":
    main()
