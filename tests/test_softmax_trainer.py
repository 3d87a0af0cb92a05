"""A model trained against the whole vocabulary: the operators one after the other, as a program uses them."""
import math

import pytest
import torch

from paper_2211_10280_amd.softmax_trainer import IGNORE, SoftmaxWorker, window_pairs


def test_window_pairs_against_a_loop():
    tokens = torch.tensor([5, 7, 5, 2, 9], dtype=torch.int32)
    for begin, n, w in ((0, 5, 2), (1, 3, 1), (4, 1, 6)):
        want = [(int(tokens[p]), int(tokens[p + o]) if 0 <= p + o < 5 else IGNORE) for p in range(begin, begin + n) for o in [*range(-w, 0), *range(1, w + 1)]]
        centers, contexts, d_loss = window_pairs(tokens, begin, n, w)
        assert list(zip(centers.tolist(), contexts.tolist())) == want
        pairs = sum(c != IGNORE for _, c in want)
        assert centers.dtype == contexts.dtype == torch.int32 and d_loss.shape == contexts.shape and bool((d_loss == torch.tensor(1 / pairs)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,states", [("f32", "f32"), ("bf16", "f32"), ("bf16", "8bit"), ("f32", "8bit")])
def test_training_finds_the_words_that_go_together(dtype, states):
    """A stream in which every word is followed by one of two, so that its neighbours are four words alike: the loss begins at
    log(vocabulary) and comes near log 4; the losses are those of the tables in 64 bits; scoring single pairs agrees."""
    V, D, w = 64, 32, 1
    g = torch.Generator(device="cuda").manual_seed(1)
    steps = torch.randint(1, 3, (4_000,), generator=g, device="cuda")
    tokens = (torch.cumsum(steps, 0) % V).to(torch.int32)
    worker = SoftmaxWorker(V, D, 2 * w * 400, dtype, states, seed=2, lr=2e-2)
    means = []
    for t in range(150):
        centers, contexts, d_loss = window_pairs(tokens, t % 10 * 400, 400, w)
        if t in (0, 149):
            z = ((worker.in_rows.double() * worker.scale)[centers.long()].to(worker.h.dtype).double() @ worker.out_rows.double().t())
            keep = contexts >= 0
            want = torch.where(keep, torch.logsumexp(z, 1) - z.gather(1, contexts.clamp(min=0).long()[:, None])[:, 0], 0.0)
        loss = worker.step(centers, contexts, d_loss).clone()
        if t in (0, 149):
            # a vector's product with its scale may round to either neighbour in the type of the vectors
            tol = (2.0 ** -7 if dtype == "bf16" else 1e-5) * (1 + z.abs().amax(1))
            assert bool(((loss.double() - want).abs() <= tol).all())
        means.append(float((loss * d_loss).sum()))
    assert abs(means[0] - math.log(V)) < 0.1 and means[-1] < math.log(4) + 0.15 and int(worker.status) == 0
    if dtype == "bf16":
        assert torch.equal(worker.in_rows, worker.w_in.bfloat16()) and torch.equal(worker.out_rows, worker.w_out.bfloat16())
    one = worker.score(tokens[:3], tokens[1:4])
    z = ((worker.in_rows.double() * worker.scale)[tokens[:3].long()].to(worker.h.dtype).double() @ worker.out_rows.double().t())
    want = torch.logsumexp(z, 1) - z.gather(1, tokens[1:4].long()[:, None])[:, 0]
    assert bool(((one.double() - want).abs() <= (2.0 ** -7 if dtype == "bf16" else 1e-5) * (1 + z.abs().amax(1))).all())
    worker.close()
