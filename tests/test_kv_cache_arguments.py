"""Configurations that KVCache refuses before it allocates anything: no GPU needed."""
import os

import pytest

import paper_2312_11514_amd as lif
from paper_2312_11514_amd import binding


@pytest.mark.parametrize("change", [dict(head_dim=0), dict(head_dim=-8), dict(head_dim=60), dict(heads=0), dict(dtype="f64"), dict(scale=0.0),
                                    dict(scale=float("nan")), dict(pages=0), dict(max_seqs=1025), dict(rotary_dim=32)])
def test_refused_with_the_error_of_the_library(change):
    if not os.path.exists(binding.LIB_PATH):
        from paper_2312_11514_amd.build import build_library
        build_library()
    good = dict(layers=1, heads=4, kv_heads=2, head_dim=64, page_tokens=16, pages=4, max_seqs=2, max_pages=2)
    with pytest.raises(lif.LifError):
        lif.KVCache(**dict(good, **change))
