"""Attention over 8-bit codes for rows that see a few tokens, where the rounding of single weights shows: tolerances as in test_gpu_coded_attention.py (with bf16 queries every weight is off by 2^-8 of
itself, so the numerator by 2^-8 of the weighted mean of |v|, while the sum of weights is not rounded, and the result rounds once more)."""
import numpy as np
import pytest
import torch

from test_gpu_coded_attention import ALL, case, check

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("types", ALL)
@pytest.mark.parametrize("n,block", [(2, 16), (3, 32), (20, 16), (70, 16)])
def test_rows_of_few_tokens(n, block, types):
    """200 sequences, scales of all sizes, values of one sign, and in half of the elements 0 but for the last token."""
    keys = [n] * 200
    q, kv, chunk, facts, table = case([1] * 200, keys, 16, 2, 16, types, 32, block, seed=n)
    vc = kv.both[1].view(torch.uint8)
    vc &= 0x7F
    if "e4m3" in types:
        vc.masked_fill_(vc == 0x7F, 0x30)
    for s in range(200):
        for t in range(n - 1):
            vc[int(table[s][t // 32]), :, t % 32, ::2] = 0
    check(q, kv, chunk, facts, table, keys, 32, block)
    check(q, kv, chunk, facts, table, keys, 32, block, softcap=4.0)


@pytest.mark.parametrize("types", ALL)
def test_heads_of_80_in_two_sequences(types):
    """With bf16 queries over int8 a row here was off by 1.06 of the bound when weights were summed up as they are rounded."""
    q, kv, chunk, facts, table = case([7, 65], [22, 66], 24, 3, 80, types, 32, 32, seed=131)
    check(q, kv, chunk, facts, table, [22, 66], 32, 32)
