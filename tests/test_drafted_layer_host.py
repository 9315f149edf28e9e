"""Host side of the layer for drafted tokens (no GPU): what it refuses before anything is launched."""
import pytest
import torch

import paper_2402_18096_gb300 as pkg
from paper_2402_18096_gb300 import layer as layers


def make(nodes=3, steps=2, **kw):
    shape = pkg.Shape(1, 4, 2, kw.pop("bits", 2), 32, 16, 64, **kw)
    ints = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    return layers.DraftedLayer(pkg.LayerCache(shape, device="cpu"), None, nodes, steps, ints(1), ints(1), ints(1, 2), ints(1))


@pytest.mark.parametrize("kw", [dict(hi_bits=8), dict(k_channel_group=64), dict(nodes=129), dict(nodes=0), dict(steps=0),
                                dict(steps=200)])
def test_caches_and_sizes_that_the_kernels_do_not_take_are_refused_at_once(kw):
    with pytest.raises(pkg.MikvError) as e:
        make(**kw)
    assert e.value.status == "MIKV_ERR_UNSUPPORTED"


@pytest.mark.parametrize("kw", [dict(), dict(bits=0), dict(nodes=128, steps=128)])
def test_others_are_taken(kw):
    assert make(**kw).drafted is None


@pytest.mark.parametrize("pairs", [[(0,)], [(0, 1, 2), (3,)], [(), (0, 1, 2, 3)]])
def test_pairs_of_other_lengths_are_refused(pairs):
    c = pkg.LayerCache(pkg.Shape(4, 4, 2, 2, 32, 16, 64), device="cpu")
    with pytest.raises(ValueError, match="from, to"):
        pkg.mikv_copy_requests(c, c, pairs)
