"""Paged caches, what needs no GPU: refused configurations, NULL arguments, and that the eviction order's definition is total."""
import ctypes as C

import pytest
import torch

from paper_2503_01330_b200 import binding
from paper_2503_01330_b200.build import build_library

GOOD = dict(n_layers=2, n_pages=100, page_size=16, n_q_heads=8, n_kv_heads=2, head_dim=128, max_batch=4, max_pages=32)


@pytest.fixture(scope="module")
def lib():
    build_library()
    return binding.lib()


@pytest.mark.parametrize("change,fragment", [
    ({}, None),
    ({"page_size": 64, "head_dim": 64, "dtype": binding.WKV_F32, "scores": 1}, None),
    ({"n_layers": 0}, "n_layers"),
    ({"n_pages": 0}, "n_pages"),
    ({"page_size": 0}, "page_size"),
    ({"page_size": 24}, "page_size"),
    ({"page_size": 128}, "page_size"),
    ({"n_q_heads": 7}, "multiple"),
    ({"n_q_heads": 6}, "1, 2, 4 or 8"),
    ({"n_q_heads": 32}, "1, 2, 4 or 8"),
    ({"n_q_heads": 2048, "n_kv_heads": 2048}, "1024"),
    ({"n_kv_heads": 0}, "n_kv_heads"),
    ({"head_dim": 96}, "head_dim"),
    ({"max_batch": 0}, "max_batch"),
    ({"max_batch": 1025}, "max_batch"),
    ({"max_pages": 0}, "max_pages"),
    ({"max_pages": (1 << 20) + 1}, "max_pages"),
    ({"n_pages": (1 << 30) - 1}, "2^31"),
    ({"dtype": 2}, "dtype"),
    ({"scale": -1.0}, "scale"),
    ({"scale": float("inf")}, "scale"),
    ({"scale": float("nan")}, "scale"),
    ({"scores": 2}, "scores"),
    ({"k_pool": 4096}, "k_pool"),
    ({"k_pool": 4096, "v_pool": 4104}, "aligned"),
])
def test_config_validation(lib, change, fragment):
    cfg = binding.make_paged_config(**{**GOOD, **change})
    msg = binding.wkv_paged_config_error(cfg)
    if fragment is None:
        assert msg is None
    else:
        assert msg is not None and fragment in msg
        h = C.c_void_p()
        assert lib.wkv_paged_create(C.byref(cfg), C.byref(h)) == binding.WKV_ERR_INVALID and not h.value


def test_null_arguments(lib):
    h = C.c_void_p()
    assert lib.wkv_paged_create(None, None) == binding.WKV_ERR_INVALID
    assert lib.wkv_paged_create(None, C.byref(h)) == binding.WKV_ERR_INVALID
    N = None
    assert lib.wkv_paged_decode(N, 0, 1, N, 0, N, N, 0, N, 1, N, 0, 0, N, 0, N, N) == binding.WKV_ERR_INVALID
    assert lib.wkv_paged_prefill(N, 0, 1, N, 0, N, N, 0, N, 1, N, 1, N, 0, 0, N, 0, N, N) == binding.WKV_ERR_INVALID
    assert lib.wkv_paged_evict(N, 0, 1, N, 1, N, 1, N, N, 1, 0, 0, N, 0, N, 0, N) == binding.WKV_ERR_INVALID
    assert lib.wkv_paged_set_stream(N, N) == binding.WKV_ERR_INVALID
    assert lib.wkv_paged_status(N) == binding.WKV_ERR_INVALID
    assert lib.wkv_paged_pools(N, C.byref(h), C.byref(h)) == binding.WKV_ERR_INVALID
    lib.wkv_paged_destroy(N)
    assert lib.wkv_paged_launch_count(N) == 0 and lib.wkv_paged_device_bytes(N) == 0
    assert lib.wkv_paged_last_error(N) == b""


@pytest.mark.skipif(torch.cuda.is_available(), reason="checks the no-GPU failure mode")
def test_create_without_gpu_fails_loudly(lib):
    cfg = binding.make_paged_config(**GOOD)
    h = C.c_void_p()
    assert lib.wkv_paged_create(C.byref(cfg), C.byref(h)) == binding.WKV_ERR_CUDA and not h.value
    with pytest.raises(Exception):
        binding.PagedCache(1, 8, 16, 4, 2, 64, 2, 4)
