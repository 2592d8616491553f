"""Attention over 8-bit codes whose value scales are about as large as fp32 has them, while code times scale is finite: against the oracle in 64 bits, tolerances as in test_gpu_coded_attention.py."""
import numpy as np
import pytest
import torch

from test_gpu_coded_attention import ALL, U, case, check, dense, pkg

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
LARGE = [2.0 ** 100, 2.0 ** 120, 1.5 * 2.0 ** 126, 1.5 * 2.0 ** 127]


def small_codes(c, seed):
    """Codes of numbers up to 1 in place of those that are there."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    if c.dtype == torch.int8:
        new = torch.randint(-1, 2, c.shape, device=DEV, generator=gen).to(torch.int8).view(torch.uint8)
    else:
        new = (torch.randint(0, 0x39, c.shape, device=DEV, generator=gen) + 128 * torch.randint(0, 2, c.shape, device=DEV, generator=gen)).to(torch.uint8)
    c.view(torch.uint8).copy_(new)


@pytest.mark.parametrize("types", ALL)
@pytest.mark.parametrize("mods", [dict(), dict(softcap=6.0, slopes=True, window=150)], ids=str)
@pytest.mark.parametrize("rows,keys,H,D", [([1], [1], 4, 64), ([2], [300], 4, 64), ([70, 3], [300, 40], 4, 128), ([1], [4000], 8, 128), ([5, 1], [2000, 700], 8, 80)])
def test_value_scales_up_to_the_largest_number(rows, keys, H, D, mods, types):
    q, kv, chunk, facts, table = case(rows, keys, H, 2, D, types, 32, 16, seed=7)
    vc, ks, vs = kv.both[1:]
    small_codes(vc, 1)
    for large in LARGE:
        vs.fill_(large)                                           # all of them: sums of weights times scales
        check(q, kv, chunk, facts, table, keys, 32, 16, **mods)
        vs.copy_(torch.where(torch.rand(vs.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(5)) < 0.3, large, 1e-3))
        check(q, kv, chunk, facts, table, keys, 32, 16, **mods)
    pages = torch.tensor(table[0][:-(-keys[0] // 32)].tolist(), device=DEV)
    ks[pages] *= torch.linspace(0.05, 1.5, len(pages), device=DEV)[:, None, None]   # scores that grow from block to block: the running maximum moves, or lags behind
    check(q, kv, chunk, facts, table, keys, 32, 16, **mods)


@pytest.mark.parametrize("types", ALL)
@pytest.mark.parametrize("rows", [[20], [80]])
def test_a_large_scale_stays_with_the_rows_that_see_it(rows, types):
    keys = [100]
    q, kv, chunk, facts, table = case(rows, keys, 4, 2, 64, types, 32, 16, seed=4)
    clean = pkg().chunk_attention(q, kv, chunk)
    n, page = rows[0], int(table[0][3])                           # tokens 96 to 99, the first block of the last page
    small_codes(kv.both[1][page, 1:2, :16], 2)
    for large in LARGE:
        kv.both[3][page, 1, 0] = large
        got = pkg().chunk_attention(q, kv, chunk)
        assert torch.equal(got[:n - 4], clean[:n - 4]) and torch.equal(got[:, :2], clean[:, :2])
        check(q, kv, chunk, facts, table, keys, 32, 16)


@pytest.mark.parametrize("types", ALL)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("mods", [dict(), dict(softcap=3.0, window=300)], ids=str)
def test_more_than_8192_columns(mods, D, types):
    n, H, page, block = 1037, 8, 64, 16
    q, kv, chunk, facts, table = case([n], [n], H, 1, D, types, page, block)
    small_codes(kv.both[1], 3)
    vs = kv.both[3]
    for share in (1.0, 0.2):
        vs.copy_(torch.where(torch.rand(vs.shape, device=DEV, generator=torch.Generator(device=DEV).manual_seed(5)) < share, LARGE[-1], 0.5))
        got = pkg().chunk_attention(q, kv, chunk, **mods)
        want, mean, big = dense(q, kv, table, n, page, block, **mods)
        count = torch.minimum(torch.arange(1, n + 1, device=DEV), torch.tensor(mods.get("window") or n, device=DEV))[:, None, None].double()
        tol = (2 * (64 * U * big + 5 * U * (big + mods.get("softcap", 0.0))) + (count / 8 + 33) * U) * mean + 1e-30
        if q.dtype == torch.bfloat16:
            tol = tol + 2.0 ** -8 * 1.001 * (mean + want.abs())
        err = ((got.double() - want).abs() / tol).nan_to_num(float("inf")).max()
        assert err <= 1.0, float(err)
