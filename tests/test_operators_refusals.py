"""What calls of the operators of a table as a model's layers leave alone when they are refused."""

import pytest
import torch

from paper_2211_10280_amd import binding as B


@pytest.mark.gpu
@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("n", [5, 5_000])
def test_a_refused_gradient_leaves_the_table_alone(n, accumulate):
    """No workspace, one that is not aligned, one that is too small: the gradient of the whole table is what it was."""
    V, D = 100, 8
    ids, d = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.ones((n, D), device="cuda")
    grad = torch.full((V, D), 7.0, device="cuda")
    need = B.tensair_embed_workspace_bytes(V, D, n)
    ws = torch.empty(need + 256, dtype=torch.uint8, device="cuda")

    def call(at, nbytes):
        return B.lib().tensair_embed_grad_dense(ids.data_ptr(), n, d.data_ptr(), B.F32, D, V, D, 1.0, grad.data_ptr(), B.F32, D, accumulate, at, nbytes, None,
                                                torch.cuda.current_stream().cuda_stream)

    for at, nbytes, want in ((None, need, B.EINVAL), (ws.data_ptr() + 16, need, B.EINVAL), (ws.data_ptr(), 0, B.ECAPACITY)):
        assert call(at, nbytes) == want
        torch.cuda.synchronize()
        assert bool((grad == 7.0).all())
    assert call(ws.data_ptr(), need) == B.OK
    torch.cuda.synchronize()
    assert bool((grad[0] == n + 7 * accumulate).all()) and bool((grad[1:] == 7 * accumulate).all())
