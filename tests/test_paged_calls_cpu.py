"""The binding's checks of a paged call's arguments, without a GPU: a cache on CPU tensors whose C calls are recorded."""
import ctypes as C
import os
import re

import pytest
import torch

from paper_2503_01330_b200 import binding
from paper_2503_01330_b200.build import CSRC


class Recorder:
    """Stands in for the C library: notes every call and accepts it."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        if name.startswith("wkv_"):
            return lambda *a: self.calls.append((name, a)) or 0
        raise AttributeError(name)


@pytest.fixture
def cache(monkeypatch):
    rec = Recorder()
    monkeypatch.setattr(binding, "lib", lambda: rec)
    c = binding.PagedCache.__new__(binding.PagedCache)
    c.device, c._index, c.dtype, c.tdtype = torch.device("cpu"), -1, binding.WKV_BF16, torch.bfloat16
    c.n_q_heads, c.n_kv_heads, c.head_dim, c.page_size = 4, 2, 64, 16
    c._bufs, c._h, c._lib = {}, C.c_void_p(1), rec
    yield c
    c._h = None


def call(cache, q, k, v, prefill):
    n = q.shape[0]
    i32 = lambda *shape: torch.zeros(*shape, dtype=torch.int32)
    out = torch.empty(n, 4, 64, dtype=torch.bfloat16)
    if prefill:
        cache.wkv_paged_prefill(0, q, k, v, i32(n + 1), i32(n, 5), i32(n), out)
    else:
        cache.wkv_paged_decode(0, q, k, v, i32(n, 5), i32(n), out)
    return cache._lib.calls[-1][1]


@pytest.mark.parametrize("prefill", [False, True])
@pytest.mark.parametrize("which", ["q", "k", "v", "kv"])
def test_rows_broadcast_over_the_batch_are_refused(cache, prefill, which):
    """x.expand(n, heads, d) has row stride 0, which the C call reads as packed rows: n - 1 rows behind the tensor's only one."""
    rows = {x: torch.zeros(3, h, 64, dtype=torch.bfloat16) for x, h in (("q", 4), ("k", 2), ("v", 2))}
    for x in which:
        rows[x] = rows[x][:1].expand_as(rows[x])
    with pytest.raises(binding.WkvError) as e:
        call(cache, **rows, prefill=prefill)
    assert e.value.code == binding.WKV_ERR_INVALID and not cache._lib.calls


@pytest.mark.parametrize("prefill", [False, True])
def test_row_strides_that_are_handed_on(cache, prefill):
    wide = torch.zeros(3, 10, 64, dtype=torch.bfloat16)
    a = call(cache, wide[:, :4], wide[:, 4:6], wide[:, 6:8], prefill)
    assert a[4] == 640 and a[7] == 640
    one = wide[:1].expand(1, 10, 64)                       # a single row: its stride says nothing
    a = call(cache, one[:, :4], one[:, 4:6], one[:, 6:8], prefill)
    assert a[4] == 4 * 64 and a[7] == 2 * 64


class Block:
    """A device tensor as far as its allocator's stream records go."""

    def __init__(self):
        self.streams = []

    def record_stream(self, stream):
        self.streams.append(stream)


class Stream:
    def __init__(self, handle, device=None):
        self.cuda_stream, self.device = handle, device


@pytest.mark.parametrize("raw", [False, True])
def test_all_memory_is_kept_for_a_changed_stream(cache, monkeypatch, raw):
    """Workspaces and pools that are freed while the new stream still uses them wait for it, a raw handle's stream too."""
    monkeypatch.setattr(binding.torch.cuda, "Stream", Stream)
    monkeypatch.setattr(binding.torch.cuda, "ExternalStream", type("ExternalStream", (Stream,), {}))
    monkeypatch.setattr(binding.torch.cuda, "default_stream", lambda device: Stream(0, device))
    cache._bufs, cache.k_pool, cache.v_pool = {1: Block(), 2: Block()}, Block(), Block()
    for handle in (4096, 0):
        cache.wkv_set_stream(handle if raw else Stream(handle))
        name, args = cache._lib.calls[-1]
        assert name == "wkv_paged_set_stream" and (args[1].value or 0) == handle
        for block in (*cache._bufs.values(), cache.k_pool, cache.v_pool):
            assert block.streams[-1].cuda_stream == handle
    cache.wkv_set_stream(None)                              # the default stream
    assert (cache._lib.calls[-1][1][1].value or 0) == 0 and cache.k_pool.streams[-1].cuda_stream == 0


def test_selftest_refuses_null():
    from paper_2503_01330_b200.build import build_library
    build_library()
    assert binding.lib().wkv_paged_selftest_wait_timeout(None) == binding.WKV_ERR_INVALID


# What only a race or a hang on the GPU would show is checked in the source.

def test_dependent_kernels_start_behind_the_tmem_allocation():
    """A kernel that may start early and takes TMEM first would keep it until the one that it waits for has ended."""
    kernels = open(os.path.join(CSRC, "wkv_paged_prefill.cuh")).read().split("__global__")[1:]
    with_tmem = [k for k in kernels if "tmem_take(" in k]
    assert len(with_tmem) == 2
    for k in with_tmem:
        assert k.count("griddep_launch();") == 1 and k.index("griddep_launch();") > k.index("tmem_take(")


def test_nothing_runs_on_the_default_stream():
    """Calls on the default stream are not ordered with the handle's where that one does not wait for it."""
    text = open(os.path.join(CSRC, "wkv_paged_api.cu")).read()
    assert not re.search(r"cudaMem(set|cpy)\(", text) and "<<<" not in text


def test_waits_that_give_up_are_heeded():
    """No paged kernel ignores what a wait says: its result is tested where it stands (mbar_wait's in the decode kernel's vote)."""
    for name in ("wkv_paged_prefill.cuh", "wkv_paged_decode.cuh", "wkv_paged_f32.cuh"):
        for line in open(os.path.join(CSRC, name)):
            for call in re.finditer(r"\b(warp_wait|thread_wait|mbar_wait|wait)\(&?[a-z]", line):
                assert re.search(r"if \(|= |return |&& |\|\| ", line[:call.start()]), line
