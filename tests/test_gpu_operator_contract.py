"""What the training operators promise beside their numbers: which calls give the same bits."""
import pytest
import torch

import paper_2609_18178_amd as pk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _weight(n, k, seed=9):
    return pk.fp8_quantize((torch.randn(n, k, generator=_gen(seed)) * 0.02).to(DEV), square=True)


# rows quantised on the way and in the workspace; squares of every size, halves, parts of K, cut along a side
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 17000, 520), (1, 33000, 4096), (5, 16400, 129), (16, 17000, 520),
                                   (16, 70001, 1000), (9, 40, 4096), (16, 17000, 4096), (17, 17000, 520), (33, 48, 640),
                                   (300, 1100, 9000), (513, 2999, 640), (517, 520, 1003), (1100, 260, 385),
                                   (4201, 4099, 4100)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_linear_is_quantize_and_product_bit_for_bit(m, n, k, dtype):
    print("linear", m, n, k, dtype, flush=True)
    w = _weight(n, k)
    x = torch.randn(m, k, generator=_gen(m)).to(dtype).to(DEV)
    for out in (torch.float32, torch.bfloat16):
        assert torch.equal(pk.fp8_linear(x, w, dtype=out), pk.fp8_matmul(pk.fp8_quantize(x), w, dtype=out)), out


@pytest.mark.parametrize("m,n,k", [(1, 300, 129), (12, 700, 20000), (300, 9000, 1100), (1100, 600, 513)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_backward_is_quantize_and_products_bit_for_bit(m, n, k, dtype):
    print("backward", m, n, k, dtype, flush=True)
    wt = pk.fp8_quantize((torch.randn(n, k, generator=_gen(2)) * 0.05).to(DEV), "columns", square=True)
    xt = pk.fp8_quantize(torch.randn(m, k, generator=_gen(1)).to(DEV), "columns")
    dy = (torch.randn(m, n, generator=_gen(3)) * 1e-3).to(dtype).to(DEV)
    dx, dw = pk.fp8_linear_backward(dy, wt, xt)
    along_rows, along_columns = pk.fp8_quantize(dy, "both")
    assert torch.equal(dx, pk.fp8_matmul(along_rows, wt, dtype=dtype))
    assert torch.equal(dw, pk.fp8_matmul(along_columns, xt, dtype=torch.float32))


def test_more_columns_than_squares_of_16_in_a_launch():
    """A launch has at most 2^32 work-items: beyond 134 million columns few rows are in larger squares, either way."""
    print("columns", flush=True)
    n, k = (1 << 27) + 130, 100
    assert pk._lib().pact_fp8_linear_workspace_bytes(1, (1 << 27) - 16, k) == 0 < pk._lib().pact_fp8_linear_workspace_bytes(1, n, k)
    part = _weight(300, k)
    data = torch.zeros(n, 128, dtype=torch.uint8, device=DEV)
    scale = torch.zeros(n, 4, dtype=torch.uint8, device=DEV)
    data[-300:], scale[-300:] = part.data, part.scale
    w = pk.Fp8Matrix(data, scale, k)
    x = torch.randn(1, k, generator=_gen(4)).to(DEV)
    got = pk.fp8_linear(x, w)
    assert torch.equal(got, pk.fp8_matmul(pk.fp8_quantize(x), w))
    assert not got[:, :-300].any() and torch.equal(got[:, -300:], pk.fp8_linear(x, part))


@pytest.mark.parametrize("kept", [0, 1])
def test_either_of_a_pair_is_kept_without_the_other_s_memory(kept):
    x = torch.zeros(2048, 4096, dtype=torch.bfloat16, device=DEV)
    before = torch.cuda.memory_allocated()
    held = pk.fp8_quantize(x, "both")[kept]
    one = held.data.numel() + held.scale.numel()
    assert one <= torch.cuda.memory_allocated() - before <= one + 4096
    del held
    assert torch.cuda.memory_allocated() == before


def test_input_and_output_as_slices_of_one_matrix():
    w = _weight(70, 203)
    for rows in (3, 200):
        x = torch.randn(rows, 203, generator=_gen(rows)).to(DEV)
        room = torch.full((rows, 300), 5.0, device=DEV)
        room[:, 11:214] = x
        pk.fp8_linear(room[:, 11:214], w, out=room[:, 214:284])
        assert torch.equal(room[:, 214:284], pk.fp8_linear(x, w, dtype=torch.float32)) and torch.equal(room[:, 11:214], x)
        assert (room[:, :11] == 5).all() and (room[:, 284:] == 5).all()
    logits = torch.randn(40, 1003, generator=_gen(5)).bfloat16().to(DEV)
    top, index = torch.topk(logits.float(), 8, 1)
    room = torch.zeros(40, 2006, dtype=torch.bfloat16, device=DEV)
    room[:, 1003:] = logits
    # (the order of a row's sums follows where it starts in its 16 bytes: the same slice of another matrix)
    loss, grad = pk.distill_step(room.clone()[:, 1003:], top, index, 2.0)
    assert torch.equal(pk.distill_step(room[:, 1003:], top, index, 2.0, grad=room[:, :1003])[0], loss)
    assert torch.equal(room[:, :1003], grad) and torch.equal(room[:, 1003:], logits)
    with pytest.raises(pk.PactError):
        pk.distill_step(room[:, 1003:], top, index, 2.0, grad=room[:, 1:1004])


def test_autograd_sees_what_is_written_in_place_and_results_have_no_graph():
    x = torch.randn(20, 130, generator=_gen(1)).to(DEV).requires_grad_()
    w = _weight(60, 130)
    top, index = torch.randn(20, 4, device=DEV), torch.zeros(20, 4, dtype=torch.int32, device=DEV)
    wt, xt = pk.fp8_quantize(torch.zeros(60, 130, device=DEV), "columns"), pk.fp8_quantize(x, "columns")
    y = pk.fp8_linear(x, w, dtype=torch.float32)
    assert not y.requires_grad and not pk.distill_step(x, top, index)[1].requires_grad

    def written(t):
        """An output of exp, which its backward pass reads, and the tensor that a call writes (of the same memory)."""
        z = torch.exp(t.requires_grad_())
        return z, z.detach()

    dy, lse = torch.zeros(20, 60, device=DEV), torch.zeros(20, device=DEV)
    for like, call in ((y, lambda out: pk.fp8_linear(x, w, out=out)),
                       (y, lambda out: pk.fp8_matmul(pk.fp8_quantize(x), w, out=out)),
                       (torch.zeros(60, 130, device=DEV), lambda out: pk.fp8_linear_backward(dy, wt, xt, grad_weight=out)),
                       (x.detach(), lambda out: pk.distill_step(out, top, index, grad=out)),
                       (x.detach(), lambda out: pk.distill_grad(x, top, index, lse, grad=out))):
        z, out = written(like.clone())
        z.sum().backward()                  # (without a call nothing is wrong)
        z, out = written(like.clone())
        call(out)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            z.sum().backward()
    held = pk.fp8_quantize(x)
    for m in (held, pk.Fp8Matrix(held.data.clone(), held.scale.clone(), 130)):
        before = m.data._version, m.scale._version
        pk.fp8_quantize(x, out=m)
        assert m.data._version > before[0] and m.scale._version > before[1]
    with torch.inference_mode():            # (tensors that keep no count)
        pk.fp8_linear(x, w, out=torch.empty(20, 60, device=DEV))


def test_refusals_name_the_argument():
    x = torch.zeros(6, 130, device=DEV)
    top, index = x[:, :4].contiguous(), torch.zeros(6, 4, device=DEV, dtype=torch.int32)
    xt = pk.fp8_quantize(x, "columns")
    wt = pk.fp8_quantize(torch.zeros(9, 130, device=DEV), "columns")
    with pytest.raises(TypeError, match="grad_weight"):
        pk.fp8_linear_backward(x[:, :9].contiguous(), wt, xt, grad_weight=[0.0])
    for bad in (None, "1", top):
        with pytest.raises(TypeError, match="temperature"):
            pk.distill_loss(x, top, index, temperature=bad)
    for bad in (1e39, -1e39, float("inf")):
        with pytest.raises(pk.PactError):
            pk.distill_step(x, top, index, temperature=bad)
