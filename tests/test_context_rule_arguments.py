"""What Eagle.set_logit_rules refuses before the library sees it (no GPU needed: the context is a stand-in, addresses are never followed)."""
from types import SimpleNamespace

import pytest
import torch

import paper_2401_15077_amd as pkg


class Library:
    """Takes the rules and remembers them."""

    def eagle_set_logit_rules(self, handle, rules):
        self.rules = rules._obj if rules is not None else None
        return 0


def context(vocab=50, max_batch=2, nodes=3):
    return SimpleNamespace(torch=torch, device=torch.device("cpu"), max_batch=max_batch, M=nodes, shape=SimpleNamespace(vocab=vocab), lib=Library(), h=None, _chk=lambda rc: None)


ROWS = torch.zeros(6, dtype=torch.int32)


@pytest.mark.parametrize("allowed", [torch.zeros(1, 2, dtype=torch.int32).expand(4, 2), torch.zeros(9, dtype=torch.int32).as_strided((4, 2), (1, 1)),
                                     torch.zeros(4, 1, dtype=torch.int32), torch.zeros(4, 2), torch.zeros(4, 4, dtype=torch.int32)[:, ::2]],
                         ids=["one mask expanded", "rows a word apart", "too few words", "floats", "words apart"])
def test_masks_that_would_be_read_behind_their_end(allowed):
    with pytest.raises(ValueError, match="allowed"):
        pkg.Eagle.set_logit_rules(context(), allowed=allowed, allowed_row=ROWS)


@pytest.mark.parametrize("allowed,stride", [(torch.zeros(4, 2, dtype=torch.int32), 2), (torch.zeros(4, 5, dtype=torch.int32)[:, :2], 5), (torch.zeros(1, 2, dtype=torch.int32), 2),
                                            (torch.zeros(1, 2, dtype=torch.int32).expand(1, 2), 2)])
def test_masks_that_lie_within_their_tensor(allowed, stride):
    c = context()
    pkg.Eagle.set_logit_rules(c, allowed=allowed, allowed_row=ROWS)
    r = c.lib.rules
    assert (r.n_masks, r.mask_stride, r.allowed) == (allowed.shape[0], stride, allowed.data_ptr())
    last = (r.n_masks - 1) * r.mask_stride + 2                    # words from the first mask to the end of the last
    assert allowed.storage_offset() + last <= allowed.untyped_storage().nbytes() // 4
