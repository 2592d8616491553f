"""The choice of a token where the weights that occur lie further apart than the buckets that masses are added up in: logits of one step apart, at temperatures where a step is some buckets, so that
hardly a bucket around min-p's least weight holds a token.  Against the oracle in 64 bits, tolerances as in test_gpu_sample.py; and vocabularies beyond those there."""
import numpy as np
import pytest
import torch

from test_gpu_sample import check, spread

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = [0.0, 0.3, 0.51, 0.7, 0.9, 0.97, 0.99, 0.999, 1.0 - 2.0 ** -24, 0.45, 0.6, 0.8]
LEAST = [0.91, 0.5, 0.91, 0.1, 0.95, 0.7, 0.91, 0.5, 0.3, 0.01, 0.999, 0.2]


def steps(V, dtype, top, step, R=12):
    """Rows of top - n * step, n from 0 to 60, small ones as likely as all others together; the first is the largest."""
    gen = torch.Generator(device=DEV).manual_seed(V)
    n = torch.where(torch.rand(R, V, device=DEV, generator=gen) < 0.5, 3, 60)
    n = (torch.rand(R, V, device=DEV, generator=gen) * (n + 1)).floor()
    n[:, 0] = 0
    x = (top - n.double() * step).to(dtype)
    assert (x.double() == top - n.double() * step).all()
    return x


@pytest.mark.parametrize("kw", [dict(top_p=[0.999] * 12), dict(top_p=[0.9, 0.99, 0.5, 0.95] * 3), dict(), dict(top_k=[900, 3000, 400, 1500] * 3), dict(top_k=[3000] * 12, top_p=[0.99] * 12),
                                dict(top_k=[40] * 12, top_p=[0.9] * 12)], ids=str)
@pytest.mark.parametrize("V", [4, 61, 2000, 50001])
@pytest.mark.parametrize("dtype,top,step,temperature", [(torch.float32, 1e6, 0.0625, 1.0), (torch.float32, 10.0, 2.0 ** -20, 1e-6), (torch.float32, -3.0, 2.0 ** -22, 3e-6),
                                                        (torch.bfloat16, 20.0, 0.125, 1.0), (torch.bfloat16, 300.0, 2.0, 7.0), (torch.float32, 5.0, 0.75, 0.9), (torch.float32, 2.0, 2.0 ** -10, 1.0)])
def test_steps_of_some_buckets(dtype, top, step, temperature, V, kw):
    check(steps(V, dtype, top, step), U, temperature=[temperature] * 12, min_p=LEAST, **kw)


def test_no_token_in_the_buckets_around_the_least_weight():
    """Weights 1, 0.94, 0.88, 0.83 and a least one of 0.91: two tokens are kept, and only these are drawn."""
    x = torch.tensor([[1e6, 1e6 - 0.0625, 1e6 - 0.125, 1e6 - 0.1875]] * 5, device=DEV)
    assert check(x, [0.99, 0.9, 0.6, 0.5, 0.1], min_p=[0.91] * 5, top_p=[0.999] * 5) == [1, 1, 1, 0, 0]
    x = torch.full((3, 1), 10.0, device=DEV)
    for _ in range(5):
        x = torch.cat([x, torch.nextafter(x[:, -1:], torch.zeros_like(x[:, :1]))], 1)
    assert check(x, [0.99, 0.7, 0.2], temperature=[1e-6] * 3, min_p=[0.5] * 3, top_p=[0.999] * 3) == [0, 0, 0]


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [151936, 262147])
def test_large_vocabularies(V, dtype):
    x, u = spread(8, V, dtype, seed=V)
    check(x, u)
    check(x, u, top_p=[0.9, 0.99] * 4, min_p=[1e-4, 0.01] * 4)
    check(x, u, top_k=[50, 5000] * 4, top_p=[0.95] * 8, temperature=[0.0, 0.7, 1.0, 2.0] * 2)
