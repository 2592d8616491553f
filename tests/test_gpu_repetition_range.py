"""Repetition penalties at the ends of fp32.  A quotient is within 2^-23 of itself (a reciprocal, its product, and what the quotient leaves put right), or a subnormal step off; a product 2^-24."""
import numpy as np
import pytest
import torch

from oracle import operators as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("vocab", [40, 4100])
def test_any_repetition(vocab):
    import paper_2401_15077_amd as p
    reps = np.float32([1e-45, 1e-40, 2.9e-39, 1.1e-38, 1.17549435e-38, 2e-38, 1e-3, 0.7, 1.0, 3.0, 1e20, 1.7e38, 3.4e38, np.inf, 0.0, -2.0, np.nan])
    S = len(reps)
    x = np.float32([0.0, 1e-3, 0.5, 3.25, 17.0, -1e-3, -2.5, -17.0, 1e-30, -1e-30, 2.5e-38, 1e-41])
    x = np.tile(np.resize(x, vocab), (S, 1))
    tokens = np.tile(np.arange(vocab), (S, 1))
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)
    rules = p.LogitRules(i32(tokens), i32([vocab] * S), n_prompt=i32([vocab] * S), repetition=torch.tensor(reps, device=DEV))
    got = p.apply_logit_rules(torch.tensor(x, device=DEV), rules).double().cpu().numpy()
    counted = np.where(reps > 0, np.maximum(reps, np.float32(2.0 ** -126)), np.float32(1.0))
    with np.errstate(all="ignore"):
        want = np.where(x > 0, x.astype(np.float64) / counted[:, None], x.astype(np.float64) * counted[:, None])
        want = np.where(np.abs(want) > float(np.finfo(np.float32).max), np.sign(want) * np.inf, want)
    finite = np.isfinite(want)
    np.testing.assert_array_equal(got[~finite], want[~finite])
    assert (np.abs(got - want)[finite] <= 2.0 ** -23 * np.abs(want)[finite] + 2.0 ** -148).all()
    y, _ = ref.logit_rules(x[6:14], np.arange(9), tokens=tokens[6:14], n_tokens=[vocab] * 8, n_prompt=[vocab] * 8, repetition=reps[6:14])
    with np.errstate(all="ignore"):
        np.testing.assert_allclose(want[6:11], y[:5], rtol=1e-12)   # (the oracle's own reading, where fp32 holds it)
