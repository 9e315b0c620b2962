"""Refusals of the 4-bit cache's entry points that need no GPU: a cache of other sizes
than those given, and a scale that f32 cannot hold in base 2."""
import pytest

import paper_2608_01563_amd as mg
from paper_2608_01563_amd import _kv4
from test_kv4_cpu import GOOD, attn, lib  # noqa: F401


@pytest.mark.parametrize("other", [(2, 3, 65, 64), (2, 4, 64, 64), (3, 3, 64, 64),
                                   (2, 3, 64, 128), (2, 3, 64, 32), (1, 3, 64, 64)])
def test_a_cache_of_other_sizes_is_refused(lib, other):  # noqa: F811
    """Larger ones too: another layout would be read from them."""
    import torch
    sizes = (2, 3, 64, 64)
    _kv4._need_room(torch.empty(mg.mg_kv4_cache_bytes(*sizes), dtype=torch.uint8), *sizes)
    with pytest.raises(ValueError, match="bytes"):
        _kv4._need_room(torch.empty(mg.mg_kv4_cache_bytes(*other), dtype=torch.uint8), *sizes)


@pytest.mark.parametrize("scale,refused", [(2.3e38, "device"), (2.4e38, "scale"),
                                           (-3.3e38, "scale")])
def test_a_scale_beyond_f32_in_base_2_is_refused(lib, scale, refused):  # noqa: F811
    """scale log2 e has to be finite.  (In range, the pointers, which are nobody's, are
    what is refused.)"""
    assert attn(lib, GOOD[:4] + [0] + GOOD[5:], scale=scale) == 1
    assert refused in mg.mg_last_error_detail()
