"""The training operators where numbers are at the ends of their types."""
import math

import numpy as np
import pytest
import torch

import paper_2609_18178_amd as pk
from tests import operator_refs as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS32 = 2.0 ** -23


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _teacher_softmax(t, temperature):
    """p and log p of a row of listed logits in 64 bits, relative to the largest."""
    t = (t.double() - t.double().max()) / temperature
    log_p = t - torch.logsumexp(t, 0)
    return torch.exp(log_p), log_p


@pytest.mark.parametrize("top", [7, 64, 100])
@pytest.mark.parametrize("temperature", [0.25, 0.5, 1.0, 3.0])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_teacher_logits_at_the_ends_of_their_type(top, temperature, dtype):
    """Teacher logits that are masked with the type's lowest number, all or some, or are as large as the type allows:
    what counts is their difference, also where logit / temperature has no finite number.  A probability is off by three
    roundings (the quotient, 2^x, the division by the sum) and the sum by one for each of its levels; the loss by that times
    the logarithms beside it, of which the largest here is below 64."""
    print("teacher", top, temperature, dtype, flush=True)
    info = torch.finfo(dtype)
    rows, vocab = 6, 501
    z = torch.randn(rows, vocab, generator=_gen(1)) * 2
    t = torch.randn(rows, top, generator=_gen(2)).to(dtype)
    t[0] = info.min                     # all masked: uniform
    t[1, 1:] = info.min                 # all but one
    t[2] = info.max                     # uniform
    t[3, ::2] = info.max                # half of them, and the others have nothing
    t[4, :3] = info.min
    index = torch.stack([torch.randperm(vocab, generator=_gen(10 + r))[:top] for r in range(rows)]).to(torch.int32)
    args = (z.to(DEV), t.to(DEV), index.to(DEV))
    loss, lse = pk.distill_loss(*args, temperature=temperature)
    alone = pk.distill_grad(*args, lse, temperature=temperature).cpu().double()
    loss2, grad = pk.distill_step(*args, temperature=temperature)
    log_q = torch.log_softmax(z.double() / temperature, 1)
    assert float(log_q.abs().max()) < 64
    near = 64 * EPS32
    for r in range(rows):
        p, log_p = _teacher_softmax(t[r], temperature)
        at = index[r].long()
        want = float(torch.where(p > 0, p * (log_p - log_q[r, at]), 0.0).sum())
        for got in (loss, loss2):
            assert abs(float(got[r]) - want) <= near * 64, (r, float(got[r]), want)
        q = torch.exp(log_q[r])
        want_grad = q.clone()
        want_grad[at] -= p
        want_grad /= temperature
        size = q
        size[at] += p
        for got in (alone, grad.cpu().double()):
            assert bool(((got[r] - want_grad).abs() <= 2 * near * size / temperature + 1e-37).all()), r
