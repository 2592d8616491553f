"""Append to a cache of 8-bit codes along draft trees whose nodes reach beyond the sequence's tokens: codes and scales at or behind key_len stay as they are, against the oracle in 64 bits."""
import numpy as np
import pytest

from test_gpu_coded_append import run, tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cache", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("keys", [[110, 45], [101, 31], [100, 30], [126, 33], [90, 45], [112, 0]], ids=str)
def test_nodes_behind_the_last_token(keys, dtype, cache):
    """Trees of 26 and 15 nodes behind 100 and 30 tokens, of which fewer are held: nodes that are not are not stored, and do not count for a block's scale."""
    rng = np.random.default_rng(6)
    masks = tree(26, rng) + tree(15, rng)
    for block in (16, 32):
        run([26, 15], keys, 4, 2, 64, dtype, cache, 32, block, masks=masks, base=[100, 30], max_keys=200)
