"""Angles of the append to 8-bit codes: keys whose rotated elements lie as close to the border between two codes as fp32 keys can be chosen to.  The pair turns by a radian a position, the block's
scale is 1, and a key x at position p becomes x cos(p) and x sin(p) in front of rounding.  In 64 bits that is known to 2^-51 of itself (cosine and product to 2^-53 each); what is nearer to a border
than 2^-46 is left out, and the kernel's own roundings (turn 2^-62 a position below 2^12, angle and series some 2^-52) are below that."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def near_borders(turned, n_codes=126):
    """For every cosine (or sine) the fp32 number whose product with it comes closest to a half, beyond 2^-46 of itself, and the product."""
    half = np.arange(n_codes) + 0.5
    x = (half / turned[:, None]).astype(np.float32)
    x = np.stack([x, np.nextafter(x, np.float32(0)), np.nextafter(x, np.float32(np.inf) * np.sign(x))])
    product = x.astype(np.float64) * turned[None, :, None]
    far = np.abs(product / half - 1.0)
    far = np.where((far < 2.0 ** -46) | (np.abs(x) > 126.0), np.inf, far)
    flat = far.transpose(1, 0, 2).reshape(len(turned), -1)
    best = flat.argmin(1)
    pick = lambda a: a.transpose(1, 0, 2).reshape(len(turned), -1)[np.arange(len(turned)), best]
    return pick(x), pick(product), flat[np.arange(len(turned)), best]


@pytest.mark.parametrize("which", ["cosine", "sine"])
def test_next_to_the_borders(which):
    import paper_2401_15077_amd as p
    at = np.arange(1, 4097)
    turned = (np.cos if which == "cosine" else np.sin)(at.astype(np.float64))
    at, turned = at[np.abs(turned) > 0.02], turned[np.abs(turned) > 0.02]
    at, turned = at[:len(at) // 16 * 16], turned[:len(at) // 16 * 16]
    x, product, far = near_borders(turned)
    assert np.median(far) < 2.0 ** -30 and (far < 2.0 ** -38).sum() > 20
    R, D = len(at), 16
    k = torch.zeros(R, 1, D, device=DEV)
    k[:, 0, 0] = torch.tensor(x, device=DEV)                      # (x, 0) -> (x cos, x sin)
    k[:, 0, 2] = 127.0                                            # behind the turned pair: the block's largest, so its scale is 1
    kc, vc = (torch.zeros(R // 16, 1, 16, D, dtype=torch.int8, device=DEV) for _ in range(2))
    ks, vs = (torch.zeros(R // 16, 1, 1, device=DEV) for _ in range(2))
    i32 = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)
    kv = p.PagedKV8(kc, vc, i32([list(range(R // 16))]), ks, vs)
    p.rope(p.rope_plan(D, rot_dim=2), None, k, chunk=p.Chunk(i32([0, R]), i32([R]), R, R, R), kv=kv, positions=i32(at))
    assert (ks == 1.0).all()
    got = kc.view(R, D)[:, 0 if which == "cosine" else 1].cpu().numpy().astype(np.float64)
    wrong = got != np.rint(product)
    assert not wrong.any(), (wrong.sum(), at[wrong][:5], product[wrong][:5], got[wrong][:5])
