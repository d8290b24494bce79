"""Which strides of the pages ltri_paged_create takes (host only)."""
import ctypes

import pytest

from paper_2412_04757_b200 import binding, build

AXES = ["layer", "page", "head", "token"]
COUNTS = dict(layer="n_layers", page="n_pages", head="n_kv_heads", token="page_tokens")


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def takes(lib, **kw):
    p = dict(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=128, type=0, cache_type=0, page_tokens=16, max_rows=4, n_pages=10,
             layer_stride=10 * 4096, page_stride=4096, head_stride=2048, token_stride=128, softmax_scale=0.0, weight_decay=1.0)
    p.update(kw)
    return lib.ltri_paged_workspace_bytes(ctypes.byref(binding.LtriPagedParams(**p))) > 0


@pytest.mark.parametrize("axis", AXES)
@pytest.mark.parametrize("stride", [0, 1, 7, -4096, 1 << 62, -(1 << 63)])
def test_the_stride_of_an_axis_of_one_entry_is_not_looked_at(lib, axis, stride):
    assert takes(lib, **{COUNTS[axis]: 1, axis + "_stride": stride})
    assert not takes(lib, **{axis + "_stride": stride})
