"""How many bits the products keep, in the 2-norm: what tells the kernels whose sums are binary32 from the 8-bit instruction,
which holds the sum of a block of 128 in fewer bits and is 1.3e-5 off at any K."""
import pytest
import torch

import paper_2609_18178_amd as pk
from tests import operator_refs as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KS = [128, 1000, 4096, 14336]


def _values(m):
    """What a matrix stands for, in 64 bits on the GPU."""
    q = torch.from_numpy(ref.E4M3).to(DEV)[m.data.long()]
    s = torch.exp2(m.scale.double() - 127)[:, :q.shape[1] // 128].repeat_interleave(128, 1)
    return (q * s)[:, :m.cols].contiguous()


def _off(got, a, b):
    want = _values(a) @ _values(b).t().contiguous()
    return float((got.double() - want).norm() / want.norm())


def _parts(m, n, k):
    gen = torch.Generator(device=DEV).manual_seed(m + n + k)
    a = torch.randn(m, k, device=DEV, generator=gen)
    b = torch.randn(n, k, device=DEV, generator=gen) * 0.02
    return a, pk.fp8_quantize(a), pk.fp8_quantize(b, square=True)


# Sums of normally distributed products grow as the root of how many there are; each of N additions rounds the sum so far
# by 2^-24 of it at most, which is below sqrt(N / 6) 2^-24 of the result in the 2-norm. The instruction adds 32 products
# at least before it rounds: N = 448 at K = 14336, 5e-7.
BINARY32 = 1e-6


# squares of 16 (few rows too), 32 and 64, those of 64 in eight waves or four, of 128 one a CU (K = 14336: in parts of it),
# of 128, of 256, and cut along a side
@pytest.mark.parametrize("m,n", [(5, 300), (64, 300), (300, 700), (700, 1400), (900, 2000), (1500, 2000), (300, 1100), (2500, 4096),
                                 (3900, 3800), (4201, 4099)])
@pytest.mark.parametrize("k", KS)
def test_binary32_results_have_binary32_sums(m, n, k):
    print("binary32", m, n, k, flush=True)
    x, a, b = _parts(m, n, k)
    got = pk.fp8_matmul(a, b, dtype=torch.float32)
    assert _off(got, a, b) <= BINARY32
    into = torch.full_like(got, 0.0)
    pk.fp8_matmul(a, b, out=into, accumulate=True)
    assert torch.equal(into, got)
    assert _off(pk.fp8_linear(x, b, dtype=torch.float32), a, b) <= BINARY32


@pytest.mark.parametrize("m,n,k", [(7, 300, 500), (300, 700, 1100), (4096, 900, 1300)])
def test_weight_gradients_have_binary32_sums(m, n, k):
    gen = torch.Generator(device=DEV).manual_seed(m)
    dy = torch.randn(m, n, device=DEV, generator=gen).bfloat16()
    x = torch.randn(m, k, device=DEV, generator=gen)
    wt = pk.fp8_quantize(torch.randn(n, k, device=DEV, generator=gen), "columns", square=True)
    xt = pk.fp8_quantize(x, "columns")
    dx, dw = pk.fp8_linear_backward(dy, wt, xt)
    rows, columns = pk.fp8_quantize(dy, "both")
    assert _off(dw, columns, xt) <= BINARY32
    # rounded to bf16: 2^-9 of an element at most
    assert _off(dx, rows, wt) <= 2.0 ** -9
    # a gradient in binary32 has the other one in binary32 too
    assert _off(pk.fp8_linear_backward(dy.float(), wt, xt)[0], rows, wt) <= BINARY32
