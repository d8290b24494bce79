"""Host-only checks of 4-bit pages: the C entry points' refusals, and the format's definition."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2412_04757_b200 import binding, build
from tests import paged_int4_reference as i4
from tests.test_paged_abi import params


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def int4(**kw):
    return params(**{**dict(cache_type=binding.TYPE_INT4), **kw})


def create(lib, p, scales=4096):
    h = ctypes.c_void_p(1)
    rc = lib.ltri_paged_create_int4(ctypes.byref(p), scales, None, ctypes.byref(h))
    assert not h.value
    return rc


def test_4_bit_pages_are_created_with_their_scales_only(lib):
    assert lib.ltri_paged_workspace_bytes(ctypes.byref(int4())) > 0
    h = ctypes.c_void_p(1)
    assert lib.ltri_paged_create(ctypes.byref(int4()), None, ctypes.byref(h)) == binding.LTRI_EINVAL and not h.value
    for p, scales in ((int4(), None), (int4(), 4096 + 8), (params(), 4096), (params(cache_type=2), 4096), (int4(k_scale=4096), 4096),
                      (int4(k_pages=None), 4096), (int4(v_pages=4100), 4096), (int4(workspace=None), 4096), (int4(weights=4096), 4096)):
        assert create(lib, p, scales) == binding.LTRI_EINVAL
    assert create(lib, int4(workspace_bytes=0)) == binding.LTRI_ECAPACITY
    assert lib.ltri_paged_create_int4(ctypes.byref(int4()), 4096, None, None) == binding.LTRI_EINVAL
    assert lib.ltri_paged_create_int4(None, 4096, None, ctypes.byref(h)) == binding.LTRI_EINVAL


@pytest.mark.parametrize("kw", [dict(token_stride=144), dict(page_stride=4096 + 16), dict(head_stride=2048 + 8), dict(token_stride=96),
                                dict(layer_stride=10 * 4096 + 16), dict(head_dim=96), dict(type=4, cache_type=4)])
def test_strides_are_multiples_of_16_bytes(lib, kw):
    assert lib.ltri_paged_workspace_bytes(ctypes.byref(int4(**kw))) == 0 and create(lib, int4(**kw)) == binding.LTRI_EINVAL
    assert lib.ltri_paged_workspace_bytes(ctypes.byref(int4(token_stride=160, head_stride=2560, page_stride=5120))) > 0


def test_null_handles_are_refused(lib):
    assert lib.ltri_paged_read(None, 0, None, 1, 1, None, 1, None, None, 1, None, None, 0, None) == binding.LTRI_EINVAL


def test_definition_of_the_format():
    grid = i4.scales64()[:0xC0]
    assert (grid.diff() > 0).all() and float(grid[1]) == 2.0 ** -17 and float(grid[-1]) == 480.0
    halves = (torch.arange(0xC0, dtype=torch.int16) << 7).view(torch.float16).double()
    assert torch.equal(grid, halves)
    assert float((torch.tensor([i4.NAN], dtype=torch.int16) << 7).view(torch.float16)) != 0 and math.isnan(
        float((torch.tensor([i4.NAN], dtype=torch.int16) << 7).view(torch.float16)))
    x = torch.zeros(6, 64)
    x[0, :3] = torch.tensor([7.0, 0.5, -1.5])    # midpoints to the even number
    x[1, 32] = 7 * 1.0625                        # of two scales to the even one, 1
    x[2, 0] = 1e30                               # the largest scale, and clamped
    x[3, 5] = math.nan
    x[4, 1] = 7 * 2.0 ** -18                     # half the smallest scale: 0
    x[5, 1] = -7 * 1.01 * 2.0 ** -18             # a little more: the smallest one
    code, scale, value = i4.quantise(x)
    assert value[0, :3].tolist() == [7.0, 0.0, -2.0] and scale[1].tolist() == [0, 0x78] and value[1, 32] == 7.0
    assert value[2, 0] == 7 * 480.0 and scale[3].tolist() == [i4.NAN, 0] and value[3, :32].isnan().all()
    assert scale[4].tolist() == [0, 0] and scale[5].tolist() == [1, 0] and value[5, 1] == -4 * 2.0 ** -17
    y = torch.randn(50, 128, dtype=torch.float64)
    code, scale, value = i4.quantise(y)
    assert torch.equal(i4.values(code, scale), value)
    s = i4.scales64()[scale.long()].repeat_interleave(32, -1)
    assert ((value - y).abs() <= s / 2 * (1 + 1e-9)).all()  # (the nearest scale is at most 1/17 below the block's seventh)


def test_null_handles_of_attend_are_refused(lib):
    bad = binding.LTRI_EINVAL
    assert lib.ltri_paged_attend(None, 0, None, 1, 1, None, 1, None, 1, None, 0, None, None, None, 0, None) == bad
    assert lib.ltri_paged_attend_workspace_bytes(None, 8) == 0


def test_every_tile_of_4_bit_rows_is_dealt_once_and_in_order(tmp_path):
    here, out = os.path.dirname(os.path.abspath(__file__)), str(tmp_path / "deal")
    subprocess.check_call(["g++", "-O1", "-std=c++20", "-pthread", os.path.join(here, "paged_deal_even_host.cpp"), "-o", out])
    r = subprocess.run([out], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
