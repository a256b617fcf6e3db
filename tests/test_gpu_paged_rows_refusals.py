"""What appending, 4-bit caches and page selection refuse on the host; nothing is launched."""
import ctypes as C

import pytest
import torch

from paged_rows_util import Pool, angle_table
from paper_2503_01330_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def bf16():
    P = Pool([20, 20, 20], kind="bf16", layers=2, seed=1)
    return P, P.cache()


def refused(c, text, name, *a):
    before = c.wkv_launch_count()
    rc = getattr(binding.lib(), name)(c._h, *a)
    assert rc == binding.WKV_ERR_INVALID and text in binding.lib().wkv_paged_last_error(c._h).decode()
    assert c.wkv_launch_count() == before and c.wkv_status() == 0


def test_append(bf16):
    P, c = bf16
    buf = torch.zeros(3, 8, 128, dtype=torch.bfloat16, device="cuda")
    table, n = P.dev()
    rope = angle_table(40, 128).cuda()
    gb = torch.zeros(2, P.n_pages, 2, 2, 128, dtype=torch.int8, device="cuda")
    gs = torch.zeros(2, P.n_pages, 2, device="cuda")
    p, t, l = buf.data_ptr(), table.data_ptr(), n.data_ptr()
    good = dict(layer=0, batch=3, q=p, q_stride=1024, k=p, v=p, kv_stride=1024, q_start=None, total=3, table=t, width=P.width, lens=l, rope=rope.data_ptr(),
                rows=40, dim=128, paired=0, pos=None, q_out=p, q_out_stride=1024, gb=gb.data_ptr(), gs=gs.data_ptr())
    for text, change in (("layer", dict(layer=2)), ("layer", dict(layer=-1)), ("batch", dict(batch=4)), ("batch", dict(batch=-1)),
                         ("rows must", dict(total=-1)), ("one token per sequence", dict(total=2)), ("table_width", dict(width=0)),
                         ("table_width", dict(width=P.width + 1)), ("k and v", dict(k=None)), ("q and q_out", dict(q=None)),
                         ("q and q_out", dict(q_out=None)), ("block_table", dict(table=None)), ("seq_lens", dict(lens=None)),
                         ("smaller", dict(q_stride=256)), ("smaller", dict(kv_stride=128)), ("smaller", dict(q_out_stride=8)),
                         ("aligned", dict(q=p + 2)), ("aligned", dict(v=p + 8)), ("aligned", dict(q_out=p + 4)), ("aligned", dict(q_stride=1025)),
                         ("aligned", dict(kv_stride=1026)), ("in place", dict(q_out_stride=2048)), ("rope must", dict(rope=rope.data_ptr() + 4)),
                         ("rope_rows", dict(rows=0)), ("rope_dim", dict(dim=0)), ("rope_dim", dict(dim=24)), ("rope_dim", dict(dim=144)),
                         ("rope_paired", dict(paired=2)), ("page_bounds", dict(gb=None)), ("page_bounds", dict(gs=None)),
                         ("page_bounds", dict(gb=gb.data_ptr() + 8)), ("page bounds need", dict(k=None, v=None)),
                         ("2^24", dict(q_start=l, total=(1 << 24) + 1))):
        refused(c, text, "wkv_paged_append", *{**good, **change}.values())
    assert binding.lib().wkv_paged_append(c._h, *{**good, "batch": 0, "total": 0}.values()) == 0


def test_select_and_decode_pages(bf16):
    P, c = bf16
    table, n = P.dev()
    q = torch.zeros(3, 4, 128, dtype=torch.bfloat16, device="cuda")
    gb = torch.zeros(2, P.n_pages, 2, 2, 128, dtype=torch.int8, device="cuda")
    gs = torch.zeros(2, P.n_pages, 2, device="cuda")
    ps, pages = torch.zeros(3, 2, P.width, device="cuda"), torch.zeros(3, 2, 2, dtype=torch.int32, device="cuda")
    good = dict(layer=0, batch=3, q=q.data_ptr(), qs=0, table=table.data_ptr(), width=P.width, lens=n.data_ptr(), gb=gb.data_ptr(), gs=gs.data_ptr(),
                n_select=2, recent=1, sink=1, ps=ps.data_ptr(), stride=P.width, pages=pages.data_ptr())
    for text, change in (("layer", dict(layer=2)), ("batch", dict(batch=9)), ("q, ", dict(q=None)), ("aligned", dict(q=q.data_ptr() + 2)),
                         ("smaller", dict(qs=8)), ("n_select", dict(n_select=0)), ("n_select", dict(n_select=(1 << 20) + 1)), ("recent", dict(recent=0)),
                         ("recent", dict(sink=-1)), ("recent", dict(recent=2)), ("page_score_stride", dict(stride=P.width - 1)),
                         ("page_bounds", dict(gb=None)), ("page_scale", dict(gs=None)), ("page_scores", dict(ps=None)), ("pages", dict(pages=None)),
                         ("aligned", dict(gb=gb.data_ptr() + 1)), ("table_width", dict(width=0)), ("seq_lens", dict(lens=None))):
        refused(c, text, "wkv_paged_select", *{**good, **change}.values())
    out = torch.zeros_like(q)
    good = dict(layer=0, batch=3, q=q.data_ptr(), qs=0, table=table.data_ptr(), width=P.width, lens=n.data_ptr(), pages=pages.data_ptr(), n_select=2,
                out=out.data_ptr(), lse=None)
    for text, change in (("layer", dict(layer=-1)), ("out", dict(out=None)), ("pages", dict(pages=None)), ("n_select", dict(n_select=0)),
                         ("n_select", dict(n_select=(1 << 20) + 1)), ("aligned", dict(out=out.data_ptr() + 8))):
        refused(c, text, "wkv_paged_decode_pages", *{**good, **change}.values())


def test_4_bit_handles(bf16):
    P, c = bf16
    K = Pool([20, 20, 20], seed=2)
    k4 = K.cache()
    table, n = K.dev()
    t, l = table.data_ptr(), n.data_ptr()
    q = torch.zeros(3, 4, 128, dtype=torch.bfloat16, device="cuda")
    refused(k4, "wkv_paged_expand", "wkv_paged_prefill", 0, 3, q.data_ptr(), 0, None, None, 0, l, 3, t, K.width, l, 0, 0, None, 0, q.data_ptr(), None)
    refused(k4, "scores", "wkv_paged_evict", 0, 3, t, K.width, t, K.width, l, l, 4, 1, 0, None, 99, None, 0, None)
    refused(k4, "scores", "wkv_paged_decode", 0, 3, q.data_ptr(), 0, None, None, 0, t, K.width, l, 0, 0, q.data_ptr(), 99, q.data_ptr(), None)
    good = dict(layer=0, batch=3, table=t, width=K.width, lens=l, dst=c._h, dst_layer=1, dst_table=t, dst_width=K.width)
    other = Pool([20], kind="f32", seed=3).cache()
    heads = Pool([20], kind="bf16", hq=1, hk=1, seed=4).cache()
    narrow = Pool([20], kind="bf16", d=64, seed=5).cache()
    for text, change in (("dst must not", dict(dst=None)), ("dst must hold", dict(dst=other._h)), ("dst must hold", dict(dst=heads._h)),
                         ("dst must hold", dict(dst=narrow._h)), ("dst must hold", dict(dst=k4._h)), ("dst_layer", dict(dst_layer=2)),
                         ("layer", dict(layer=1)), ("dst_width", dict(dst_width=0)), ("dst_table", dict(dst_table=None)),
                         ("seq_lens", dict(lens=None)), ("batch", dict(batch=4))):
        refused(k4, text, "wkv_paged_expand", *{**good, **change}.values())
    refused(c, "4 bits", "wkv_paged_expand", *good.values())
    with pytest.raises(binding.WkvError):
        binding.PagedCache(1, 4, 16, 4, 2, 128, 1, 4, dtype=binding.WKV_KV4, k_pool=torch.zeros(1, 4, 2, 16, 128, device="cuda"),
                           v_pool=torch.zeros(1, 4, 2, 16, 128, device="cuda"))


def test_pools_of_the_librarys_own():
    c = binding.PagedCache(2, 6, 32, 4, 2, 64, 2, 3, dtype=binding.WKV_KV4)
    assert c.k_pool.dtype == torch.uint8 and tuple(c.k_pool.shape) == (2, 6, 2, 32 * 36)
    L = binding.lib()
    cfg = binding.make_paged_config(1, 6, 16, 4, 2, 128, 2, 3, dtype=binding.WKV_KV4)
    h = C.c_void_p()
    assert L.wkv_paged_create(C.byref(cfg), C.byref(h)) == 0
    assert L.wkv_paged_device_bytes(h) >= 2 * 6 * 2 * 16 * 72 and L.wkv_paged_status(h) == 0
    L.wkv_paged_destroy(h)
