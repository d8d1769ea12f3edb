"""The training operators past the sizes where they take other kernels: quantised matrices that go past the caches, long rows
of logits in place."""
import pytest
import torch

import paper_2609_18178_amd as pk

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _randn(*shape, seed=0):
    return torch.randn(*shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(seed))


@pytest.mark.parametrize("along", ["rows", "columns", "both"])
@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_quantisation_is_that_of_its_strips(dtype, square, along):
    """From 16 million elements on results go past the caches: the bytes of strips of whole squares, each below that."""
    rows, cols = 4099, 4101
    print("large", dtype, square, along, flush=True)
    room = torch.zeros(rows, cols + 9, dtype=dtype, device=DEV)
    x = room[:, 5:5 + cols]
    x.copy_(_randn(rows, cols) * torch.exp(_randn(rows, 1, seed=1) * 4))
    x[7, 4100], x[4098, 0], x[130, 131] = float("inf"), float("nan"), 0.0
    got = pk.fp8_quantize(x, along, square=square)
    by_rows, by_cols = {"rows": (got, None), "columns": (None, got), "both": got if along == "both" else None}[along]
    assert x.numel() >= 16 << 20
    for at in range(0, rows, 1024):
        part = x[at:at + 1024]
        assert part.numel() < 16 << 20
        a, b = pk.fp8_quantize(part, "both", square=square)
        if by_rows is not None:
            assert torch.equal(by_rows.data[at:at + 1024], a.data) and torch.equal(by_rows.scale[at:at + 1024], a.scale)
        if by_cols is not None:
            wide, blocks = b.data.shape[1], -(-part.shape[0] // 128)
            assert torch.equal(by_cols.data[:, at:at + wide], b.data)
            assert torch.equal(by_cols.scale[:, at // 128:at // 128 + blocks], b.scale[:, :blocks])
    if by_cols is not None:
        assert by_cols.scale.shape[1] == 36 and not by_cols.scale[:, 33:].any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_backward_of_a_large_gradient(dtype):
    """A gradient of 16 million elements: its halves, quantised below that, give the same rows of dx; and dw is the product of
    what the large quantisation holds."""
    m, n, k = 4099, 4101, 70
    dy = (_randn(m, n) * 1e-3).to(dtype)
    wt = pk.fp8_quantize(_randn(n, k, seed=1) * 0.05, "columns", square=True)
    xt = pk.fp8_quantize(_randn(m, k, seed=2), "columns")
    dx, dw = pk.fp8_linear_backward(dy, wt, xt)
    rows, columns = pk.fp8_quantize(dy, "both")
    assert torch.equal(dx, pk.fp8_matmul(rows, wt, dtype=dtype))
    assert torch.equal(dw, pk.fp8_matmul(columns, xt, dtype=torch.float32))
    for part in (slice(0, 2048), slice(2048, m)):
        assert torch.equal(pk.fp8_quantize(dy[part]).data, rows.data[part])


# rows that are held in registers; that are read twice (bf16 from 32776 entries, the loss and the gradient of binary32 from
# 16388, both together from 65540); the odd ones start anywhere in their 16 bytes
@pytest.mark.parametrize("vocab", [5003, 32768, 70001, 139300])
@pytest.mark.parametrize("top", [16, 64, 100])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_distillation_in_place_over_long_rows(vocab, top, dtype):
    print("in place", vocab, top, dtype, flush=True)
    logits = (_randn(6, vocab, seed=vocab) * 2.5).to(dtype)
    value, index = torch.topk(logits.float() + _randn(6, vocab, seed=3), top, 1)
    index[1, 3] = index[1, 7]           # listed twice
    index[2] = -1                       # nothing listed
    weight = torch.tensor([1.0, 0.5, 1.0, 0.0, 2.0, 1.0], device=DEV)
    keys = dict(temperature=1.5, row_weight=weight)
    loss, grad = pk.distill_step(logits, value, index, **keys)
    lse = pk.distill_loss(logits, value, index, **keys)[1]
    alone = pk.distill_grad(logits, value, index, lse, **keys)
    z = logits.clone()
    got = pk.distill_step(z, value, index, grad=z, **keys)
    assert got[1] is z and torch.equal(z, grad) and torch.equal(got[0], loss)
    z = logits.clone()
    assert torch.equal(pk.distill_grad(z, value, index, lse, grad=z, **keys), alone)
    # a log-sum-exp too large to go by: the row is read for it, and then overwritten
    far = lse + 1000.0
    shifted = logits.float() + 1500.0
    z = shifted.clone()
    assert torch.equal(pk.distill_grad(z, value, index, far, grad=z, **keys),
                       pk.distill_grad(shifted, value, index, far, **keys))
