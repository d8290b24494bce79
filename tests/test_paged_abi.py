"""Host-only checks of the paged cache's C entry points and of its 64-bit definition."""
import ctypes

import pytest
import torch

from paper_2412_04757_b200 import binding, build
from tests import paged_reference as ref


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def params(**kw):
    base = dict(n_layers=2, n_q_heads=8, n_kv_heads=2, head_dim=128, type=0, cache_type=0, page_tokens=16, max_rows=4,
                n_pages=10, layer_stride=10 * 4096, page_stride=4096, head_stride=2048, token_stride=128, softmax_scale=0.0,
                weight_decay=1.0, k_pages=4096, v_pages=8192, workspace=4096, workspace_bytes=1 << 40)
    base.update(kw)
    return binding.LtriPagedParams(**base)


def test_struct_size_matches_header():
    assert ctypes.sizeof(binding.LtriPagedParams) == 8 * 4 + 5 * 8 + 2 * 4 + 8 * 8


@pytest.mark.parametrize("kw", [
    dict(n_layers=0), dict(n_q_heads=7), dict(n_q_heads=0), dict(n_kv_heads=0), dict(n_q_heads=130), dict(head_dim=96),
    dict(head_dim=512), dict(type=2), dict(type=-1), dict(cache_type=1), dict(cache_type=3), dict(page_tokens=0),
    dict(page_tokens=65537), dict(max_rows=0), dict(max_rows=65536), dict(n_pages=0), dict(n_pages=1 << 31),
    dict(n_pages=(1 << 31) - 1, page_tokens=65536), dict(n_pages=(1 << 31) - 1, page_stride=1 << 40),
    dict(n_layers=65535, n_pages=1 << 30, page_tokens=512, n_kv_heads=64, n_q_heads=64), dict(token_stride=132), dict(token_stride=64), dict(page_stride=-4096),
    dict(layer_stride=0), dict(head_stride=2044), dict(softmax_scale=-1.0), dict(softmax_scale=float("nan")),
    dict(softmax_scale=float("inf")), dict(weight_decay=1.5), dict(weight_decay=-0.1), dict(weight_decay=float("nan")),
])
def test_bad_parameters_are_rejected_on_the_host(lib, kw):
    p = params(**kw)
    assert lib.ltri_paged_workspace_bytes(ctypes.byref(p)) == 0
    h = ctypes.c_void_p(1)
    assert lib.ltri_paged_create(ctypes.byref(p), None, ctypes.byref(h)) == binding.LTRI_EINVAL and not h.value


@pytest.mark.parametrize("kw,code", [
    (dict(k_pages=None), "EINVAL"), (dict(v_pages=4096 + 8), "EINVAL"), (dict(workspace=None), "EINVAL"),
    (dict(workspace=4096 + 16), "EINVAL"), (dict(workspace_bytes=0), "ECAPACITY"), (dict(weights=4096), "EINVAL"),
    (dict(positions=4096), "EINVAL"), (dict(weights=4098, positions=4096), "EINVAL"), (dict(k_scale=4096), "EINVAL"),
    (dict(cache_type=2), "EINVAL"), (dict(cache_type=2, k_scale=4096), "EINVAL"),
])
def test_create_refuses_what_it_is_not_given(lib, kw, code):
    h = ctypes.c_void_p()
    assert lib.ltri_paged_create(ctypes.byref(params(**kw)), None, ctypes.byref(h)) == getattr(binding, "LTRI_" + code)
    assert not h.value


def test_null_handles_are_refused(lib):
    assert lib.ltri_paged_create(ctypes.byref(params()), None, None) == binding.LTRI_EINVAL
    assert lib.ltri_paged_destroy(None) == binding.LTRI_EINVAL
    assert lib.ltri_paged_sync_status(None, None) == binding.LTRI_EINVAL
    assert lib.ltri_paged_launch_count(None) == 0 and lib.ltri_paged_last_cuda_error(None) == 0
    bad = binding.LTRI_EINVAL
    assert lib.ltri_paged_decode(None, 0, None, 1, 1, None, 1, None, 0, None, None, 0, None, None, None, None) == bad
    assert lib.ltri_paged_append(None, 0, None, 1, 1, None, 1, None, 1, None, None, 0, None, None, None) == bad
    assert lib.ltri_paged_evict(None, 0, 1, None, 1, 1, None, None, 1, 1, 0, 0, None) == bad


def test_axes_of_one_entry_need_no_stride_and_weights_need_room(lib):
    one = params(n_layers=1, layer_stride=0, n_kv_heads=1, head_stride=0)
    a = lib.ltri_paged_workspace_bytes(ctypes.byref(one))
    assert a > 0
    assert lib.ltri_paged_workspace_bytes(ctypes.byref(params(weights=4096, positions=4096))) > a


def test_the_binding_runs_on_cuda_tensors_only():
    k = torch.zeros(1, 2, 1, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.LtriPaged(k, k.clone(), 1)


def test_definition_of_an_eviction():
    inf, nan = float("inf"), float("nan")
    # two protected at the ends, then by weight, ties to the lower slot; the highest kept slots fill the lowest holes
    assert ref.evict_unit([0, 5, 1, 5, 5, 0], [0, 1, 2, 3, 4, 5], 4, 1, 1) == ([5], [2])
    assert ref.evict_unit([nan, -inf, inf, nan], [3, 2, 1, 0], 2, 0, 0) == ([2], [1])
    assert ref.evict_unit([0.0, -0.0, 0.0], [7, 8, 9], 2, 0, 0) == ([], [])
    assert ref.evict_unit([0.1, 0.2, 0.3], [5, 6, 4], 1, 0, 1) == ([1], [0])


def test_definition_of_the_8_bit_rows():
    x = torch.linspace(-9, 9, 4001)[:, None, None]
    got = ref.quantise(x, torch.tensor([0.02]))
    want = (x / torch.tensor(0.02)).clamp(-448, 448).to(torch.float8_e4m3fn).double()
    assert torch.equal(got, want)


def test_page_of_a_slot_by_multiplication():
    # the kernels' slot / page_tokens: one product and a shift, for slots below 2^31
    for page in [1, 2, 3, 5, 7, 16, 31, 100, 641, 4095, 4097, 65535, 65536]:
        shift = 31 + (page - 1).bit_length()
        mul = (1 << shift) // page + 1
        assert mul < 1 << 32
        top = (1 << 31) - 1
        for slot in {0, 1, page - 1, page, page + 1, top, top - 1, top // page * page, top // page * page - 1, 123456789}:
            if 0 <= slot <= top:
                assert slot * mul >> shift == slot // page, (page, slot)
