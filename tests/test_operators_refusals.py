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


def test_tensors_that_are_not_on_a_gpu_are_refused():
    """Their addresses would go to a kernel.  Shapes and types are right; nothing here reaches the library."""
    f, i, v = torch.zeros((4, 8)), torch.zeros(4, dtype=torch.int32), torch.zeros(4)
    ws = torch.zeros(1 << 20, dtype=torch.uint8)
    f8 = f.to(torch.float8_e4m3fn)
    for call in (lambda: B.tensair_embed(f, 8, i, f.clone()), lambda: B.tensair_embed_grad(i, f, 8, 4, B.RowBuffers(4, 8, "cpu"), ws),
                 lambda: B.tensair_embed_grad_dense(i, f, 8, f.clone(), ws), lambda: B.tensair_softmax_loss(f, f, 8, i, v, v.clone(), ws),
                 lambda: B.tensair_softmax_grad(f, f, 8, i, v, v, f.clone(), None, ws), lambda: B.AdamW([dict(param=f, grad=f, m=f, v=f)]),
                 lambda: B.AdamW([dict(param=f, grad=f, m=f8, v=f8, m_scale=v[:1], v_scale=v[:1])]),
                 lambda: B.tensair_adamw_step(None, 0.1, 1, grad_scale=v[:1])):
        with pytest.raises(B.TensairError) as e:
            call()
        assert "GPU" in str(e.value)


@pytest.mark.gpu
def test_one_tensor_that_is_not_on_the_gpu_is_refused():
    """Each argument in turn; a status word and a scale of other types; a workspace whose bytes do not follow one another."""
    def gpu(x):
        return x.cuda()

    f, i, v = gpu(torch.zeros((4, 8))), gpu(torch.zeros(4, dtype=torch.int32)), gpu(torch.zeros(4))
    ws, status = gpu(torch.zeros(1 << 20, dtype=torch.uint8)), gpu(torch.zeros(1, dtype=torch.int32))
    rows = tuple(B.RowBuffers(4, 8))
    calls = [(lambda t, i, o, s: B.tensair_embed(t, 8, i, o, 1.0, s), (f, i, f.clone(), status)),
             (lambda i, d, n, r, g, w, s: B.tensair_embed_grad(i, d, 8, 4, (n, r, g), w, 1.0, s), (i, f, *rows, ws, status)),
             (lambda i, d, g, w, s: B.tensair_embed_grad_dense(i, d, 8, g, w, 1.0, False, s), (i, f, f.clone(), ws, status)),
             (lambda h, t, y, lo, ls, w, s: B.tensair_softmax_loss(h, t, 8, y, lo, ls, w, status=s), (f, f, i, v, v.clone(), ws, status)),
             (lambda h, t, y, ls, d, dh, dt, w, s: B.tensair_softmax_grad(h, t, 8, y, ls, d, dh, dt, w, status=s), (f, f, i, v, v, f.clone(), f.clone(), ws, status))]
    for call, args in calls:
        call(*args)
        for k in range(len(args)):
            with pytest.raises(B.TensairError):
                call(*args[:k], args[k].cpu(), *args[k + 1:])
        for bad in (status.long(), status[:0], status.float()):
            with pytest.raises(B.TensairError):
                call(*args[:-1], bad)
        if args[-2] is ws:
            with pytest.raises(B.TensairError):
                call(*args[:-2], ws[:1].expand(1 << 20), status)
    tensor = dict(param=f.clone(), grad=f.clone(), m=f.clone(), v=f.clone(), param_copy=f.bfloat16())
    opt = B.AdamW([tensor])
    opt.step(0.1, 1, grad_scale=v[:1])
    for bad in (v[:1].cpu(), v[:1].double(), v[:0]):
        with pytest.raises(B.TensairError):
            opt.step(0.1, 2, grad_scale=bad)
    for name in tensor:
        with pytest.raises(B.TensairError):
            B.AdamW([{**tensor, name: tensor[name].cpu()}])
    torch.cuda.synchronize()
