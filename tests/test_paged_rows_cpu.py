"""Appending, 4-bit rows and page selection, what needs no GPU: refused configurations and arguments, and the format's definition."""
import ctypes as C

import os
import re

import numpy as np
import pytest
import torch

import paged_rows_util as util
from paper_2503_01330_b200 import binding
from paper_2503_01330_b200.build import build_library
from test_paged_calls_cpu import Recorder
from test_paged_cpu import GOOD

NULL = None


@pytest.fixture(scope="module")
def lib():
    build_library()
    return binding.lib()


@pytest.mark.parametrize("change,fragment", [
    ({"dtype": binding.WKV_KV4}, None),
    ({"dtype": binding.WKV_KV4, "head_dim": 64, "page_size": 64}, None),
    ({"dtype": binding.WKV_KV4, "scores": 1}, "4 bits"),
    ({"dtype": 3}, "dtype"),
    ({"dtype": 5}, "dtype"),
])
def test_config(lib, change, fragment):
    msg = binding.wkv_paged_config_error(binding.make_paged_config(**{**GOOD, **change}))
    assert msg is None if fragment is None else fragment in msg


def test_merged_cache_takes_no_4_bit_rows(lib):
    assert "dtype" in binding.wkv_config_error(binding.make_config(1, 1, 4, 4, 64, 128, 16, dtype=binding.WKV_KV4))


def test_null_handles(lib):
    N = NULL
    assert lib.wkv_paged_append(N, 0, 1, N, 0, N, N, 0, N, 1, N, 1, N, N, 0, 0, 0, N, N, 0, N, N) == binding.WKV_ERR_INVALID
    assert lib.wkv_paged_select(N, 0, 1, N, 0, N, 1, N, N, N, 1, 1, 0, N, 1, N) == binding.WKV_ERR_INVALID
    assert lib.wkv_paged_decode_pages(N, 0, 1, N, 0, N, 1, N, N, 1, N, N) == binding.WKV_ERR_INVALID
    assert lib.wkv_paged_expand(N, 0, 1, N, 1, N, N, 0, N, 1) == binding.WKV_ERR_INVALID


@pytest.fixture
def cache(monkeypatch):
    """A handle of 4 query heads on 2 kv heads of 64, 2 layers of 10 pages of 16, on CPU tensors; the C calls are recorded."""
    rec = Recorder()
    monkeypatch.setattr(binding, "lib", lambda: rec)
    c = binding.PagedCache.__new__(binding.PagedCache)
    c.device, c._index, c.dtype, c.tdtype = torch.device("cpu"), -1, binding.WKV_BF16, torch.bfloat16
    c.n_q_heads, c.n_kv_heads, c.head_dim, c.page_size, c.shape = 4, 2, 64, 16, (2, 10, 2, 16, 64)
    c._bufs, c._h, c._lib = {}, C.c_void_p(1), rec
    yield c
    c._h = None


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def good_append(**change):
    T = 6
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)
    a = dict(q=bf(T, 4, 64), k=bf(T, 2, 64), v=bf(T, 2, 64), block_table=i32(3, 5), seq_lens=i32(3), q_start=i32(4), rope=torch.zeros(100, 32),
             positions=i32(T), q_out=bf(T, 4, 64), page_bounds=torch.zeros(2, 10, 2, 2, 64, dtype=torch.int8), page_scale=torch.zeros(2, 10, 2))
    a.update(change)
    return a


@pytest.mark.parametrize("change", [
    dict(q=None), dict(q_out=None), dict(k=None), dict(v=None), dict(q=None, q_out=None, k=None, v=None),
    dict(q=torch.zeros(6, 4, 64)), dict(q=torch.zeros(6, 2, 64, dtype=torch.bfloat16)), dict(k=torch.zeros(5, 2, 64, dtype=torch.bfloat16)),
    dict(q_out=torch.zeros(1, 4, 64, dtype=torch.bfloat16).expand(6, 4, 64)), dict(seq_lens=i32(4)), dict(q_start=i32(3)),
    dict(q_start=torch.zeros(4)), dict(rope=torch.zeros(100)), dict(rope=torch.zeros(100, 32, dtype=torch.float64)),
    dict(rope=torch.zeros(32, 100).T), dict(positions=i32(5)), dict(page_bounds=None), dict(page_scale=None),
    dict(page_bounds=torch.zeros(2, 10, 2, 2, 64, dtype=torch.uint8)), dict(page_scale=torch.zeros(2, 10)),
    dict(page_bounds=torch.zeros(2, 9, 2, 2, 64, dtype=torch.int8)), dict(block_table=torch.zeros(3, 5, dtype=torch.int64)),
])
def test_append_refuses(cache, change):
    with pytest.raises(binding.WkvError) as e:
        cache.wkv_paged_append(0, **good_append(**change))
    assert e.value.code == binding.WKV_ERR_INVALID and not cache._lib.calls


def test_append_hands_on(cache):
    a = good_append()
    cache.wkv_paged_append(1, paired=True, **a)
    name, c = cache._lib.calls[-1]
    assert name == "wkv_paged_append" and c[1:3] == (1, 3) and c[3] == a["q"].data_ptr() and c[9] == 6 and c[11] == 5
    assert c[4] == 256 and c[7] == 128 and c[19] == 256 and c[20] == a["page_bounds"].data_ptr()
    assert c[13:17] == (a["rope"].data_ptr(), 100, 32, 1) and c[17] == a["positions"].data_ptr()
    wide = torch.zeros(3, 10, 64, dtype=torch.bfloat16)
    cache.wkv_paged_append(0, wide[:, :4], wide[:, 4:6], wide[:, 6:8], i32(3, 5), i32(3), q_out=wide[:, :4])
    c = cache._lib.calls[-1][1]
    assert c[4] == c[7] == c[19] == 640 and c[8] is None and c[13] is None and c[17] is None and c[20] is None and c[21] is None
    cache.wkv_paged_append(0, None, wide[:, 4:6], wide[:, 6:8], i32(3, 5), i32(3))
    c = cache._lib.calls[-1][1]
    assert c[3] is None and c[18] is None


def good_select(**change):
    a = dict(q=torch.zeros(3, 4, 64, dtype=torch.bfloat16), block_table=i32(3, 5), seq_lens=i32(3),
             page_bounds=torch.zeros(2, 10, 2, 2, 64, dtype=torch.int8), page_scale=torch.zeros(2, 10, 2),
             page_scores=torch.zeros(3, 2, 5), pages=i32(3, 2, 4))
    a.update(change)
    return a


@pytest.mark.parametrize("change", [
    dict(q=torch.zeros(3, 4, 64)), dict(q=torch.zeros(1, 4, 64, dtype=torch.bfloat16).expand(3, 4, 64)), dict(block_table=i32(2, 5)),
    dict(page_scores=torch.zeros(3, 4, 5)), dict(page_scores=torch.zeros(3, 2, 5, dtype=torch.float64)), dict(pages=i32(3, 4, 4)),
    dict(pages=torch.zeros(3, 2, 4, dtype=torch.int64)), dict(page_bounds=torch.zeros(10, 2, 2, 64, dtype=torch.int8)),
])
def test_select_refuses(cache, change):
    with pytest.raises(binding.WkvError):
        cache.wkv_paged_select(0, **good_select(**change))
    assert not cache._lib.calls


def test_select_and_decode_pages_hand_on(cache):
    a = good_select()
    cache.wkv_paged_select(1, recent=2, sink=1, **a)
    c = cache._lib.calls[-1][1]
    assert c[1:3] == (1, 3) and c[6] == 5 and c[10:13] == (4, 2, 1) and c[13] == a["page_scores"].data_ptr() and c[14] == 5
    out = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    cache.wkv_paged_decode_pages(1, a["q"], a["block_table"], a["seq_lens"], a["pages"], out)
    c = cache._lib.calls[-1][1]
    assert c[8] == a["pages"].data_ptr() and c[9] == 4 and c[10] == out.data_ptr() and c[11] is None
    for bad in (dict(pages=i32(3, 2, 4)[:, :, ::2]), dict(pages=i32(2, 2, 4))):
        with pytest.raises(binding.WkvError):
            cache.wkv_paged_decode_pages(0, a["q"], a["block_table"], a["seq_lens"], bad["pages"], out)


def test_expand_refuses(cache):
    for bad in (dict(dst=object()), dict(seq_lens=i32(2)), dict(dst_table=i32(2, 5)), dict(block_table=torch.zeros(3, 5))):
        a = dict(block_table=i32(3, 5), seq_lens=i32(3), dst=cache, dst_layer=0, dst_table=i32(3, 5))
        a.update(bad)
        with pytest.raises(binding.WkvError):
            cache.wkv_paged_expand(0, **a)
    assert not cache._lib.calls


def test_expand_keeps_pools_for_its_stream(cache):
    """A destination of another stream may be dropped right after the call."""
    class Pool:
        def __init__(self):
            self.streams = []

        def record_stream(self, s):
            self.streams.append(s)
    cache._stream = "a"
    dst = binding.PagedCache.__new__(binding.PagedCache)
    dst._h = None
    for theirs, want in (("a", []), ("b", ["a"])):
        dst._stream, dst.k_pool, dst.v_pool = theirs, Pool(), Pool()
        cache.wkv_paged_expand(0, i32(3, 5), i32(3), dst, 0, i32(3, 5))
        assert dst.k_pool.streams == want and dst.v_pool.streams == want


# ---------------------------------------------------------------- the kernels' source

CSRC = os.path.join(os.path.dirname(os.path.abspath(binding.__file__)), "csrc")
HOST = ("wkv_paged_host.cuh", "wkv_paged_rows.cu", "wkv_paged_pages.cu", "wkv_paged_kv4.cu")


def source(name):
    return open(os.path.join(CSRC, name)).read()


def test_nothing_runs_on_the_default_stream():
    for name in HOST:
        assert not re.search(r"cudaMem(set|cpy)\(", source(name)) and "<<<" not in source(name), name


def test_waits_that_give_up_are_heeded_and_kernels_wait_for_the_one_before():
    for line in source("wkv_paged_decode_kv4.cuh").splitlines():
        for call in re.finditer(r"\b(mbar_wait|wait)\(&?[a-z]", line):
            assert re.search(r"if \(|= |return |&& |\|\| ", line[:call.start()]), line
    for name, kernels in (("wkv_paged_rows.cuh", 2), ("wkv_paged_choose.cuh", 1), ("wkv_paged_decode_kv4.cuh", 1)):
        bodies = re.split(r"\b__global__\b", source(name))[1:]
        assert len(bodies) == kernels
        for body in bodies:
            assert body.index("griddep_launch();") < body.index("griddep_wait();"), name


def test_rings_have_an_even_number_of_stages():
    """Two teams take turns on the stages: with an odd number they would share one, and a barrier's parity would not tell their phases apart."""
    text = source("wkv_paged_decode_kv4.cuh")
    assert re.search(r"kStages = .*/ 2 \* 2;", text) and "kKv4Warps == 2 * kKv4TileWarps" in text


# ---------------------------------------------------------------- the format

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["k", "v"])
def test_every_code_has_a_place_of_its_own(d, kind):
    byte, shift = util.places(kind, d, 16)
    assert len({(int(b), int(s)) for b, s in zip(byte.ravel(), shift.ravel())}) == 16 * d
    assert byte.min() == 0 and byte.max() == 16 * d // 2 - 1
    for i in range(16):                                  # a row's codes stay in its d / 2 bytes
        assert (byte[i] // (d // 2) == i).all()


def test_values_are_bf16_and_fp16_numbers_within_a_step():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((4000, 64)) * 2.0 ** rng.integers(-30, 18, (4000, 1))).astype(np.float32)
    x[::5] = np.abs(x[::5])
    n, s, byte, z = util.quantise(x)
    v = util.dequantise(n, s, z)
    t = torch.from_numpy(v)
    assert torch.equal(t, t.float().bfloat16().double()) and (v.astype(np.float16).astype(np.float64) == v).all()
    assert (s == (byte.astype(np.uint16) << 7).view(np.float16)).all() and byte.min() >= 1 and byte.max() <= 0xd8
    # s = 4096 is the largest scale: 15 steps of it reach over a group only if hi - lo <= 15 * 4096, hi and lo as the format takes them
    g = x.reshape(4000, 2, 32)
    span = np.maximum(g.max(-1), 0).astype(np.float64) - np.minimum(g.min(-1), 0)
    fits = np.repeat(span <= 4096 * 15, 32, -1)
    assert (np.abs(v - x)[fits] <= np.repeat(s, 32, -1)[fits] * (1 + 2.0 ** -20)).all()


def test_bounds_hold_their_keys():
    rng = np.random.default_rng(1)
    k = rng.standard_normal((16, 64)).astype(np.float32)
    b, s = util.page_bounds(k)
    assert (b[0] * s * (1 + 2.0 ** -22) >= k.max(0) - 1e-6).all() and (b[1] * s * (1 + 2.0 ** -22) <= k.min(0) + 1e-6).all()
    q = rng.standard_normal((4, 64)).astype(np.float32)
    code = util.query_codes(q)
    step = max(np.maximum(q, 0).sum(0).max(), -np.minimum(q, 0).sum(0).min()) / 127
    bound = float((b.astype(np.int64) * code).sum()) * float(s) * step
    assert bound >= float((q @ k.T).sum(0).max()) - 64 * step * np.abs(k).max()      # half a step a channel, both parts
