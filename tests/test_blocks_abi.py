"""Argument errors of the block-sparse and page-map calls, found on the host before anything touches a device: the calls
get a block of zeros for a context, which an accepted call could not use."""
import ctypes as C

import pytest

from paper_2410_05076_b200 import binding

INV, UNS = binding.ERR_INVALID, binding.ERR_UNSUPPORTED
CTX = C.cast(C.create_string_buffer(1 << 16), C.c_void_p)
P = 1 << 20                                               # an aligned address that is never dereferenced


def kv(**over):
    s = binding.tidal_kv_t()
    s.batch, s.num_q_heads, s.num_kv_heads, s.head_dim = 2, 8, 2, 128
    s.kv_layout, s.k, s.v = binding.KV_PAGED, P, P
    s.stride_pos, s.stride_head, s.stride_page = 256, 4096, 8192
    s.page_table, s.page_size, s.max_pages_per_seq, s.num_pages = P, 16, 64, 100
    s.ctx_lens, s.max_ctx_len = P, 1024
    for k, v in over.items():
        setattr(s, k, v)
    return s


def contiguous(**over):
    return kv(kv_layout=binding.KV_CONTIG, stride_b=2 * 1024 * 256, stride_head=1024 * 256, stride_page=0, **over)


def call(name, defaults, over):
    args = dict(defaults)
    args.update(over)
    args = [C.byref(v) if isinstance(v, binding.tidal_kv_t) else v for v in args.values()]
    return getattr(binding.load(), name)(*args, None)


MAP = dict(ctx=CTX, batch=4, old=P, new=P, table=P, width=8, pages=32, free=P, num_free=P, num_free_out=P, cap=64, slots=P, pos=None, off=None)
WRITE = dict(ctx=CTX, kv=kv(), T=4, k=P, v=P, ks=256, vs=256, slots=P)
BOUNDS = dict(ctx=CTX, kv=kv(), start=None, max_new=0, bounds=P, blocks=100)
SELECT = dict(ctx=CTX, kv=kv(), q=P, bounds=P, blocks=100, m=4, gran=0, first=0, last=0, idx=P, count=P)
ATTN = dict(ctx=CTX, kv=kv(), q=P, idx=P, count=None, m=4, hi=8, out=P)


@pytest.mark.parametrize("name,defaults,over,status", [
    ("tidal_page_map", MAP, dict(ctx=None), INV), ("tidal_page_map", MAP, dict(old=None), INV), ("tidal_page_map", MAP, dict(new=None), INV),
    ("tidal_page_map", MAP, dict(table=None), INV), ("tidal_page_map", MAP, dict(free=None), INV), ("tidal_page_map", MAP, dict(num_free=None), INV),
    ("tidal_page_map", MAP, dict(num_free_out=None), INV), ("tidal_page_map", MAP, dict(slots=None), INV), ("tidal_page_map", MAP, dict(batch=0), INV),
    ("tidal_page_map", MAP, dict(batch=4097), UNS), ("tidal_page_map", MAP, dict(width=0), INV), ("tidal_page_map", MAP, dict(width=16385), UNS),
    ("tidal_page_map", MAP, dict(pages=0), INV), ("tidal_page_map", MAP, dict(cap=-1), INV),
    ("tidal_kv_write", WRITE, dict(ctx=None), INV), ("tidal_kv_write", WRITE, dict(T=-1), INV), ("tidal_kv_write", WRITE, dict(k=None), INV),
    ("tidal_kv_write", WRITE, dict(v=P + 8), INV), ("tidal_kv_write", WRITE, dict(slots=None), INV), ("tidal_kv_write", WRITE, dict(ks=252), INV),
    ("tidal_kv_write", WRITE, dict(vs=-8), INV), ("tidal_kv_write", WRITE, dict(kv=kv(head_dim=64)), UNS),
    ("tidal_kv_write", WRITE, dict(kv=kv(num_kv_heads=1, num_q_heads=1, batch=1), T=0), binding.OK),
    ("tidal_block_bounds", BOUNDS, dict(ctx=None), INV), ("tidal_block_bounds", BOUNDS, dict(bounds=None), INV),
    ("tidal_block_bounds", BOUNDS, dict(bounds=P + 8), INV), ("tidal_block_bounds", BOUNDS, dict(blocks=99), INV),
    ("tidal_block_bounds", BOUNDS, dict(max_new=-1), INV), ("tidal_block_bounds", BOUNDS, dict(kv=contiguous(), blocks=63), INV),
    ("tidal_block_bounds", BOUNDS, dict(kv=kv(page_size=32)), UNS),
    ("tidal_block_select", SELECT, dict(ctx=None), INV), ("tidal_block_select", SELECT, dict(q=None), INV), ("tidal_block_select", SELECT, dict(q=P + 4), INV),
    ("tidal_block_select", SELECT, dict(bounds=None), INV), ("tidal_block_select", SELECT, dict(blocks=99), INV), ("tidal_block_select", SELECT, dict(m=0), INV),
    ("tidal_block_select", SELECT, dict(m=16385), INV), ("tidal_block_select", SELECT, dict(gran=3), INV), ("tidal_block_select", SELECT, dict(first=-1), INV),
    ("tidal_block_select", SELECT, dict(last=-1), INV), ("tidal_block_select", SELECT, dict(idx=None), INV), ("tidal_block_select", SELECT, dict(kv=contiguous(), blocks=63), INV),
    ("tidal_block_attn", ATTN, dict(ctx=None), INV), ("tidal_block_attn", ATTN, dict(q=None), INV), ("tidal_block_attn", ATTN, dict(q=P + 8), INV),
    ("tidal_block_attn", ATTN, dict(idx=None), INV), ("tidal_block_attn", ATTN, dict(m=0), INV), ("tidal_block_attn", ATTN, dict(hi=4), INV),
    ("tidal_block_attn", ATTN, dict(out=None), INV), ("tidal_block_attn", ATTN, dict(kv=kv(sm_scale=-1.0)), INV),
    ("tidal_block_attn", ATTN, dict(kv=kv(num_q_heads=18, num_kv_heads=2), hi=18), UNS),
])
def test_refused_on_the_host(name, defaults, over, status):
    assert call(name, defaults, over) == status


def test_page_error_has_a_text():
    assert "page" in binding.strerror(binding.ERR_PAGES)
