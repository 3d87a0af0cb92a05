"""A model of word sequences: the next word from all words before it, trained with AdamW and asked for words.

Where :mod:`softmax_trainer` scores a word beside one other word, this puts layers between a table's two ends: looked-up
vectors (``tensair_embed``) with dropout (``tensair_dropout``), then blocks of layer norm (``tensair_norm``), a product that gives inputs and
gates, a gated linear recurrence over the mini-batch's ragged sequences (``tensair_recur``), dropout and the residual path; a last norm, and the exact
softmax over all words (``tensair_softmax_loss``).  Gradients go the same way back, and one ``tensair_adamw_step`` updates everything.  A step may be given the
sequences' states before it, cut off for the gradient, and leaves those behind it, so that a caller whose sequences go on from step to step can carry them; the command below
begins every sequence with zeros, since its mini-batches are runs of one stream.  ``generate`` is the server's side: a word at a time (``tensair_recur_step``), drawn from the
logits (``tensair_sample``).

    python -m paper_2211_10280_amd.sequence_trainer --steps 50 --layers 2

The products (a block's, and the logits of ``generate``) are torch's; everything else numerical happens inside the library; this file only
sequences calls and keeps buffers.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B

IGNORE = -1      # the label of a word that has none, as the stream's last one


class SequenceWorker:
    def __init__(self, vocab, dim, max_tokens, max_sequences, layers=1, dtype="bf16", dropout=0.1, seed=0, lr=1e-3, weight_decay=0.01, device="cuda"):
        """max_tokens, max_sequences: most words and sequences of a step."""
        self.vocab, self.dim, self.layers, self.p, self.seed, self.lr, self.step_no = vocab, dim, layers, dropout, seed, lr, 0
        self.scale = dim ** 0.5
        self.dtype = dt = {"f32": torch.float32, "bf16": torch.bfloat16}[dtype]
        self.device = device
        g = torch.Generator(device=device).manual_seed(seed)

        def param(value, decay):
            p = {"param": value, "grad": torch.zeros_like(value), "m": torch.zeros_like(value), "v": torch.zeros_like(value), "weight_decay": decay}
            if dt != torch.float32 and value.dim() > 1:       # the products read bfloat16 copies, which the optimizer step writes
                p["grad"] = p["grad"].to(dt)
                p["param_copy"] = value.to(dt)
            self.params.append(p)
            return p

        def norm():
            return param(torch.ones(dim, device=device), 0.0), param(torch.zeros(dim, device=device), 0.0)

        self.params = []
        self.w_in, self.w_out = (param(torch.randn((vocab, dim), generator=g, device=device) / dim, weight_decay) for _ in range(2))
        self.blocks = []
        for _ in range(layers):
            w = torch.randn((dim, 2 * dim), generator=g, device=device) * dim ** -0.5     # columns: inputs, then gates
            self.blocks.append((*norm(), param(w, weight_decay), param(torch.full((dim,), 1.0, device=device), 0.0)))
        self.last = norm()
        self.optimizer = B.AdamW([{k: v.view(-1) if isinstance(v, torch.Tensor) else v for k, v in p.items()} for p in self.params])

        def rows(n, width, kind):
            return torch.empty((n, width), dtype=kind, device=device)

        n = max_tokens
        # the residual path is fp32, what goes through the products is of the model's type
        self.x = [rows(n, dim, torch.float32) for _ in range(layers + 1)]
        self.norms = [(rows(n, dim, dt), torch.empty(n, device=device), torch.empty(n, device=device)) for _ in range(layers + 1)]
        self.both = [rows(n, 2 * dim, dt) for _ in range(layers)]
        self.h = rows(n, dim, dt)
        self.states = [rows(B.tensair_recur_state_rows(n), dim, torch.float32) for _ in range(layers)]
        self.carried = [torch.zeros((max_sequences, dim), device=device) for _ in range(layers)]       # states at the sequences' ends
        self.carry_in = [torch.zeros((max_sequences, dim), device=device) for _ in range(layers)]
        self.d_x, self.d_h, self.d_both, self.d_norm = rows(n, dim, torch.float32), rows(n, dim, dt), rows(n, 2 * dim, dt), rows(n, dim, dt)
        self.loss, self.lse = (torch.empty(n, device=device) for _ in range(2))
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        nbytes = max(B.tensair_softmax_workspace_bytes(n, vocab, dim, dt, True), B.tensair_embed_workspace_bytes(vocab, dim, n),
                     B.tensair_recur_workspace_bytes(n, dim), B.tensair_norm_workspace_bytes(n, dim))
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)

    @staticmethod
    def _read(p):
        """What the products and lookups read of a parameter."""
        return p.get("param_copy", p["param"])

    def forward(self, words, offsets, states=None, train=True):
        """Rows that the logits are products of, for int32 [n] words in sequences that begin at int32 offsets; states: for every layer fp32 [sequences, dim],
        the sequences' states before (None: zeros).  The states behind them are in self.carried."""
        n, D, S = words.numel(), self.dim, offsets.numel() - 1
        p = self.p if train else 0.0
        x = self.x[0][:n]
        B.tensair_embed(self._read(self.w_in), D, words, x, self.scale, self.status)
        if p:
            B.tensair_dropout(x, D, x, p, self.seed, 0, self.step_no)
        for k, (weight, bias, w, gate_bias) in enumerate(self.blocks):
            y, mean, rstd = (t[:n] for t in self.norms[k])
            B.tensair_norm(x, D, weight["param"], bias["param"], y, mean, rstd)
            both = self.both[k][:n]
            torch.mm(y, self._read(w), out=both)
            both[:, D:] += gate_bias["param"].to(self.dtype)
            if states is None:
                h0 = None
            else:
                h0 = self.carry_in[k][:S]
                h0.copy_(states[k])
            B.tensair_recur(both[:, :D], both[:, D:], D, offsets, self.h[:n], self.workspace, h0, self.carried[k][:S], self.states[k][:B.tensair_recur_state_rows(n)],
                            self.status)
            nxt = self.x[k + 1][:n]
            B.tensair_dropout(self.h[:n], D, nxt, p, self.seed, k + 1, self.step_no, x)
            x = nxt
        y, mean, rstd = (t[:n] for t in self.norms[self.layers])
        B.tensair_norm(x, D, self.last[0]["param"], self.last[1]["param"], y, mean, rstd)
        return y

    def step(self, words, offsets, labels, d_loss, states=None):
        """One training step: labels int32 [n] (IGNORE: none), d_loss float32 [n], 1 / labels for their mean.  Returns the losses before the step."""
        loss = self.gradients(words, offsets, labels, d_loss, states)
        self.step_no += 1
        self.optimizer.step(self.lr, self.step_no)
        return loss

    def gradients(self, words, offsets, labels, d_loss, states=None):
        """The losses; the gradients of all parameters are left in their buffers."""
        n, D, S = words.numel(), self.dim, offsets.numel() - 1
        y = self.forward(words, offsets, states)
        loss, lse, table = self.loss[:n], self.lse[:n], self._read(self.w_out)
        B.tensair_softmax_loss(y, table, D, labels, loss, lse, self.workspace, 1.0, IGNORE, self.status)
        d_norm, d_x, d_h, d_both = self.d_norm[:n], self.d_x[:n], self.d_h[:n], self.d_both[:n]
        B.tensair_softmax_grad(y, table, D, labels, lse, d_loss, d_norm, self.w_out["grad"], self.workspace, 1.0, IGNORE, self.status)
        _, mean, rstd = (t[:n] for t in self.norms[self.layers])
        B.tensair_norm_grad(d_norm, self.x[self.layers][:n], D, self.last[0]["param"], mean, rstd, d_x, self.last[0]["grad"], self.last[1]["grad"], self.workspace)
        for k in range(self.layers - 1, -1, -1):
            weight, bias, w, gate_bias = self.blocks[k]
            B.tensair_dropout(d_x, D, d_h, self.p, self.seed, k + 1, self.step_no)
            both = self.both[k][:n]
            h0 = self.carry_in[k][:S] if states is not None else None
            B.tensair_recur_grad(both[:, :D], both[:, D:], D, offsets, self.states[k][:B.tensair_recur_state_rows(n)], d_h, d_both[:, :D], d_both[:, D:], self.workspace, h0,
                                 status=self.status)
            y, mean, rstd = (t[:n] for t in self.norms[k])
            torch.mm(y.t(), d_both, out=w["grad"])
            torch.sum(d_both[:, D:], 0, dtype=torch.float32, out=gate_bias["grad"])
            torch.mm(d_both, self._read(w).t(), out=d_norm)
            # the residual path's gradient is added to, in place
            B.tensair_norm_grad(d_norm, self.x[k][:n], D, weight["param"], mean, rstd, d_x, weight["grad"], bias["grad"], self.workspace, d_x)
        if self.p:
            B.tensair_dropout(d_x, D, d_x, self.p, self.seed, 0, self.step_no)
        B.tensair_embed_grad_dense(words, d_x, D, self.w_in["grad"], self.workspace, self.scale, False, self.status)
        return loss

    def generate(self, words, u, states=None, temperature=None, top_k=None, top_p=None, min_p=None):
        """Continues n sequences by as many words as u (float32 [words, n]) has rows: words int32 [n], the last word of each, states for every layer fp32 [n, dim], those
        before it, updated (None: zeros).  Returns int32 [words, n] and the words' probabilities; filters as of tensair_sample, for every sequence."""
        n, D = words.numel(), self.dim
        if states is None:
            states = [torch.zeros((n, D), device=self.device) for _ in range(self.layers)]
        out = torch.empty((u.shape[0], n), dtype=torch.int32, device=self.device)
        prob = torch.empty((u.shape[0], n), device=self.device)
        x, nxt = torch.empty((n, D), device=self.device), torch.empty((n, D), device=self.device)
        y, both, h = (torch.empty((n, w), dtype=self.dtype, device=self.device) for w in (D, 2 * D, D))
        logits = torch.empty((n, self.vocab), dtype=self.dtype, device=self.device)
        workspace = torch.empty(B.tensair_sample_workspace_bytes(n, self.vocab), dtype=torch.uint8, device=self.device)
        for t in range(u.shape[0]):
            B.tensair_embed(self._read(self.w_in), D, words, x, self.scale, self.status)
            for k, (weight, bias, w, gate_bias) in enumerate(self.blocks):
                B.tensair_norm(x, D, weight["param"], bias["param"], y)
                torch.mm(y, self._read(w), out=both)
                both[:, D:] += gate_bias["param"].to(self.dtype)
                B.tensair_recur_step(both[:, :D], both[:, D:], D, states[k], h, None, self.status)
                B.tensair_dropout(h, D, nxt, 0.0, 0, 0, 0, x)
                x, nxt = nxt, x
            B.tensair_norm(x, D, self.last[0]["param"], self.last[1]["param"], y)
            torch.mm(y, self._read(self.w_out).t(), out=logits)
            B.tensair_sample(logits, self.vocab, u[t], out[t], workspace, temperature, top_k, top_p, min_p, prob[t], self.status)
            words = out[t]
        return out, prob

    def close(self):
        self.optimizer.close()


def next_word_batch(tokens, begin, n, sequences):
    """(words, offsets, labels, 1 / labels for every word) of a run of positions of a device int32 stream cut into sequences of nearly equal length; a word's label is the next
    one, the last word of a sequence has the next one too, unless it is the stream's last."""
    words = tokens[begin:begin + n]
    offsets = torch.linspace(0, n, sequences + 1, dtype=torch.float64, device=tokens.device).round().to(torch.int32)
    labels = torch.full_like(words, IGNORE)
    more = min(n, tokens.numel() - begin - 1)
    labels[:more] = tokens[begin + 1:begin + 1 + more]
    return words, offsets, labels, torch.full((n,), 1.0 / max(more, 1), device=tokens.device)


def main(argv=None):
    import workload as W

    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--config", type=int, default=2, choices=sorted(W.CONFIGS), help="workload whose vocabulary, row length and mini-batch are taken")
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--layers", type=int, default=1)
    ap.add_argument("--sequences", type=int, default=8, help="sequences of a mini-batch")
    ap.add_argument("--dtype", default="bf16", choices=("f32", "bf16"))
    ap.add_argument("--dropout", type=float, default=0.1)
    ap.add_argument("--lr", type=float, default=1e-3)
    ap.add_argument("--words", type=int, default=20, help="words drawn at the end")
    a = ap.parse_args(argv)
    cfg = W.CONFIGS[a.config]
    cfg = cfg.scaled(tokens=min(cfg.tokens, a.steps * cfg.batch + 1))
    tokens = torch.from_numpy(W.make_stream(cfg)[0]).cuda()
    worker = SequenceWorker(cfg.vocab, cfg.dim, cfg.batch, a.sequences, a.layers, a.dtype, a.dropout, cfg.seed, a.lr)
    for t in range(a.steps):
        begin, n, _ = W.batch_slice(cfg, t)
        words, offsets, labels, d_loss = next_word_batch(tokens, begin, n, min(a.sequences, n))
        loss = worker.step(words, offsets, labels, d_loss)
        if t % 10 == 0 or t + 1 == a.steps:
            print(f"step {t}: mean loss {float((loss * d_loss).sum()):.4f}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(cfg.seed)
    out, prob = worker.generate(tokens[:4], torch.rand((a.words, 4), generator=g, device="cuda"), top_p=torch.full((4,), 0.95, device="cuda"))
    for i in range(4):
        print(f"after word {int(tokens[i])}:", *out[:, i].tolist())
    assert int(worker.status) == 0
    worker.close()


if __name__ == "__main__":
    main()
