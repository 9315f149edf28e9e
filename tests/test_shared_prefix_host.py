"""Host side of the shared-prefix layer and of the rotary binding (no GPU): what they refuse before anything is
launched."""
import pytest
import torch

import paper_2402_18096_gb300 as pkg
from paper_2402_18096_gb300.layer import SharedPrefixLayer


def test_key_lengths_are_refused():
    """Requests of several lengths: the own caches hold the same number of tokens for every request, so padding would be
    kept and attended. Refused before anything is turned."""
    B, Hq, Hkv, P, T = 2, 4, 2, 8, 6
    shape = pkg.shape_for_context(B, Hq, Hkv, 2, 32, T, 0.5, 1)
    prefix = tuple(torch.ones(1, h, P, 128, dtype=torch.bfloat16) for h in (Hq, Hkv, Hkv))
    own = tuple(torch.ones(B, h, T, 128, dtype=torch.bfloat16) for h in (Hq, Hkv, Hkv))
    with pytest.raises(ValueError, match="key_len"):
        SharedPrefixLayer.from_prompts(shape, pkg.RotaryTable(device="cpu"), prefix, own, torch.empty_like(prefix[0]),
                                       torch.empty_like(own[0]),
                                       key_len=torch.tensor([P + T, P + 2], dtype=torch.int32))
    assert all(bool((x == 1).all()) for x in prefix + own)
