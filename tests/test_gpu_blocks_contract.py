"""What the header and the design notes promise of the block-sparse and page calls beyond their results on usual input: signs
of zeros, memory that is held, the status word, far pages, the precision of the softmax weights."""
import math

import pytest
import torch

from paper_2410_05076_b200 import binding, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D, BLK = 128, 16


@pytest.fixture()
def td():
    t = binding.Tidal(0)
    yield t
    t.close()


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def hnd(k, v, hq, fp8=False, scales=None, sm_scale=0.0):
    """One sequence, [Hkv, n, 128] keys and values side by side."""
    hkv, n = k.shape[:2]
    buf = torch.stack((k, v), 2).to(torch.float8_e4m3fn if fp8 else torch.bfloat16)[None].contiguous()
    more = dict(k_scale=scales[0], v_scale=scales[1]) if scales else {}
    return synth.LayerKV(k=buf[..., 0, :], v=buf[..., 1, :], batch=1, num_q_heads=hq, num_kv_heads=hkv, head_dim=D, ctx_lens=i32([n]),
                         max_ctx_len=n, stride_b=hkv * n * 2 * D, stride_pos=2 * D, stride_head=n * 2 * D, sm_scale=sm_scale,
                         kv_dtype=int(fp8), keep=[buf], **more)


def one_page(batch, hq, hkv, ctx):
    """`batch` sequences of one token each that share a page, in a cache for up to `ctx` positions."""
    pool = torch.zeros(1, hkv, BLK, 2, D, dtype=torch.bfloat16, device=DEV)
    lay = synth.LayerKV(k=pool[..., 0, :], v=pool[..., 1, :], batch=batch, num_q_heads=hq, num_kv_heads=hkv, head_dim=D,
                        ctx_lens=torch.ones(batch, dtype=torch.int32, device=DEV), max_ctx_len=ctx, stride_pos=2 * D,
                        stride_head=BLK * 2 * D, stride_page=hkv * BLK * 2 * D, keep=[pool], max_pages_per_seq=ctx // BLK,
                        page_table=torch.zeros(batch, ctx // BLK, dtype=torch.int32, device=DEV))
    lay.num_pages = 1
    return lay


def free_bytes():
    torch.cuda.synchronize()
    return torch.cuda.mem_get_info(0)[0]


# ---- writing tokens ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("scale", [1.0, 0.037, 2.0 ** 70])
def test_quantised_zeros_keep_their_sign(td, scale):
    """IEEE: -0 / s = -0 for a positive s, whose nearest code is 0x80; and quotients that round to zero keep theirs."""
    sc = torch.full((1,), scale, device=DEV)
    zero = torch.zeros(1, BLK, D, device=DEV)
    lay = hnd(zero, zero, 1, True, (sc, sc))
    x = torch.zeros(1, 1, D)
    x[0, 0, ::2] = -0.0
    x[0, 0, 4:12] = torch.tensor([-1e-30, 1e-30, -1e-38, 1e-38, -9.2e-41, 9.2e-41, -1.0, 1.0])
    x = x.to(torch.bfloat16).to(DEV)
    td.kv_write(lay, x, x, torch.tensor([3], device=DEV))
    want = (x.float().cpu() / sc.cpu()).to(torch.float8_e4m3fn).view(torch.uint8)[0, 0]
    assert int(want[0]) == 0x80 and int(want[1]) == 0
    for got in (lay.k, lay.v):
        assert torch.equal(got[0, 0, 3].contiguous().view(torch.uint8).cpu(), want)


@pytest.mark.parametrize("scale", [1.0, 0.037, 3.3e-5, 1234.5, 2.0 ** -60, 2.0 ** 60, 2.0 ** -61, 1.3 * 2.0 ** 60, 2.0 ** -126])
def test_every_bf16_number_gets_the_code_of_its_quotient(td, scale):
    """All 65536 of them, zeros of both signs, subnormal numbers, infinities and not-a-numbers included."""
    x = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(512, 1, D)
    sc = torch.full((1,), scale, device=DEV)
    zero = torch.zeros(1, 512, D, device=DEV)
    lay = hnd(zero, zero, 1, True, (sc, sc))
    td.kv_write(lay, x.to(DEV), x.to(DEV), torch.arange(512, device=DEV))
    quotient = x[:, 0].float() / sc.cpu()
    want = quotient.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    nan = quotient.isnan()
    for got in (lay.k, lay.v):
        got = got[0, 0].contiguous().view(torch.uint8).cpu()
        assert ((got[nan] & 0x7F) == 0x7F).all() and torch.equal(got[~nan], want[~nan])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("above", [True, False])
def test_writes_into_pages_four_gigabytes_long(td, fp8, above):
    """Page strides next to 2^32 bytes, where the offset arithmetic changes from 32 to 64 bits."""
    hkv, size = 2, 1 if fp8 else 2
    stride = 2 ** 32 // size - (0 if above else 16 // size)
    dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
    used = hkv * BLK * 2 * D
    buf = torch.empty(2 * stride + used, dtype=dt, device=DEV)
    pool = buf.as_strided((3, hkv, BLK, 2, D), (stride, BLK * 2 * D, 2 * D, D, 1))
    for p in range(3):
        pool[p].view(torch.uint8).fill_(0x11)
    ones = torch.ones(hkv, device=DEV)
    lay = synth.LayerKV(k=pool[..., 0, :], v=pool[..., 1, :], batch=1, num_q_heads=hkv, num_kv_heads=hkv, head_dim=D, ctx_lens=i32([48]),
                        max_ctx_len=48, stride_pos=2 * D, stride_head=BLK * 2 * D, stride_page=stride, page_table=i32([[0, 1, 2]]),
                        max_pages_per_seq=3, keep=[buf], kv_dtype=int(fp8), **(dict(k_scale=ones, v_scale=ones) if fp8 else {}))
    lay.num_pages = 3
    k, v = (torch.randn(5, hkv, D, generator=gen(i), device=DEV).to(torch.bfloat16) for i in range(2))
    slots = [2 * BLK + 15, BLK, 0, 2 * BLK, BLK + 7]
    td.kv_write(lay, k, v, torch.tensor(slots, device=DEV))
    assert td.device_status() == binding.OK
    want = torch.full((3, hkv, BLK, 2, D), 0, dtype=dt, device=DEV)
    want.view(torch.uint8).fill_(0x11)
    for t, s in enumerate(slots):
        for i, rows in enumerate((k, v)):
            want[s // BLK, :, s % BLK, i] = rows[t].float().clamp(-448, 448).to(dt)
    for p in range(3):
        assert torch.equal(pool[p].contiguous().view(torch.uint8), want[p].view(torch.uint8)), p


# ---- key bounds ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("max_new", [0, 1])
@pytest.mark.parametrize("fp8", [False, True])
def test_bounds_follow_sequences_that_become_shorter(td, fp8, max_new):
    """Tokens taken back (100 -> 97) no longer count in the last block's bounds, although it starts before the old length."""
    old, new = [100, 100, 64, 40, 33, 16, 5, 5], [97, 20, 48, 41, 32, 0, 5, 1]
    hkv, width = 3, 7
    keys = torch.randn(len(old) * width, hkv, BLK, 2, D, generator=gen(1), device=DEV).to(torch.float8_e4m3fn if fp8 else torch.bfloat16)
    lens = i32(old)
    lay = synth.LayerKV(k=keys[..., 0, :], v=keys[..., 1, :], batch=len(old), num_q_heads=hkv, num_kv_heads=hkv, head_dim=D, ctx_lens=lens,
                        max_ctx_len=112, stride_pos=2 * D, stride_head=BLK * 2 * D, stride_page=hkv * BLK * 2 * D, kv_dtype=int(fp8),
                        page_table=torch.randperm(len(old) * width, generator=gen(2), device=DEV).to(torch.int32).view(len(old), width),
                        max_pages_per_seq=width, keep=[keys])
    bounds = td.block_bounds(lay)
    start = lens.clone()
    lens.copy_(i32(new))
    td.block_bounds(lay, bounds, start_lens=start, max_new=max_new)
    fresh = td.block_bounds(lay)
    for b, n in enumerate(new):
        page = lay.page_table[b, : -(-n // BLK)].long()
        assert torch.equal(bounds[page], fresh[page]), (b, n)
        rows = keys[page][..., 0, :].float().transpose(1, 2).flatten(0, 1)[:n]                      # [n, Hkv, 128]
        if n:
            last = rows[(n - 1) // BLK * BLK:]
            assert torch.equal(bounds[page[-1]].float(), torch.stack((last.amin(0), last.amax(0)), 1))
    assert td.device_status() == binding.OK


# ---- the status word -----------------------------------------------------------------------------------------------

def test_two_kinds_of_trouble_are_both_reported(td):
    zero = torch.zeros(1, BLK, D, device=DEV)
    lay = hnd(zero, zero, 1)
    rows = torch.ones(1, 1, D, dtype=torch.bfloat16, device=DEV)
    td.kv_write(lay, rows, rows, torch.tensor([BLK], device=DEV))                    # behind the cache
    td.page_map(i32([0]), i32([17]), i32([[0, 0]]), i32([0]), i32([1]), torch.zeros(17, dtype=torch.int64, device=DEV))      # two pages, one free
    assert sorted([td.device_status(), td.device_status()]) == sorted([binding.ERR_PAGES, binding.ERR_INDEX])
    assert td.device_status() == binding.OK


def used_by(fn):
    """Device memory that a call takes for good (code that it loads apart: it has run before)."""
    before = free_bytes()
    fn()
    return before - free_bytes()


# ---- memory --------------------------------------------------------------------------------------------------------

def test_reserve_holds_nothing_for_selections_that_need_no_scratch():
    """Up to 16384 positions tidal_block_select uses none: a reservation takes what the token selection takes."""
    lay = one_page(1024, 32, 4, 16384)
    q = torch.zeros(1024, 32, D, dtype=torch.bfloat16, device=DEV)
    out = torch.zeros(1024, 32, D, device=DEV)
    idx, cnt = torch.zeros(1024, 32, 4, dtype=torch.int32, device=DEV), torch.zeros(1024, dtype=torch.int32, device=DEV)
    torch.cuda.empty_cache()
    a, b, c = binding.Tidal(0), binding.Tidal(0), binding.Tidal(0)
    c.select_attn(lay, q, 4, out=out, idx=idx, idx_count=cnt)
    c.close()
    try:
        called = used_by(lambda: a.select_attn(lay, q, 4, out=out, idx=idx, idx_count=cnt))
        reserved = used_by(lambda: b.reserve(lay, 4))
        assert reserved <= called + 2 ** 25, (reserved, called)         # (the scratch of 1024 blocks in 32768 rows: 128 MB)
    finally:
        a.close(); b.close()


def long_select(t, batch, hq):
    lay = one_page(batch, hq, hq // 8, 262144)
    q = torch.zeros(batch, hq, D, dtype=torch.bfloat16, device=DEV)
    bounds = torch.zeros(binding.block_bounds_shape(lay), dtype=torch.bfloat16, device=DEV)
    idx, cnt = torch.zeros(batch, hq, 1, dtype=torch.int32, device=DEV), torch.zeros(batch, dtype=torch.int32, device=DEV)
    return lambda: t.block_select(lay, bounds, q, 1, idx=idx, idx_count=cnt)


def test_outgrown_scratch_that_no_graph_names_is_given_back(td):
    small, large = long_select(td, 64, 64), long_select(td, 192, 64)    # 16384 blocks: 256 MB and 768 MB of scores
    small()
    before = free_bytes()
    large()
    grown = before - free_bytes()
    assert grown <= 2 ** 29 + 2 ** 25, grown                            # 512 MB more
    small(); large()
    assert td.device_status() == binding.OK


def fill(leave):
    """Takes all of the device's memory but `leave` bytes."""
    torch.cuda.empty_cache()
    return torch.empty(free_bytes() - leave, dtype=torch.uint8, device=DEV)


def test_scratch_grows_to_what_is_needed_where_twice_does_not_fit(td):
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    small, large = long_select(td, 128, 64), long_select(td, 160, 64)   # 512 MB and 640 MB
    small()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            small()                                                     # (a graph names the first buffer: it stays)
    most = fill(900 << 20)
    try:
        large()
        assert td.device_status() == binding.OK
    finally:
        del most
        torch.cuda.empty_cache()
    graph.replay()
    assert td.device_status() == binding.OK
    del graph


def test_a_reservation_for_token_selection_does_not_fail_for_block_scratch():
    """Memory for all of the token calls, but not for 256 MB of block scores besides."""
    lay = one_page(64, 64, 8, 262144)
    a, b = binding.Tidal(0), binding.Tidal(0)
    try:
        q = torch.zeros(64, 64, D, dtype=torch.bfloat16, device=DEV)
        out = torch.zeros(64, 64, D, device=DEV)
        idx, cnt = torch.zeros(64, 64, 4, dtype=torch.int32, device=DEV), torch.zeros(64, dtype=torch.int32, device=DEV)
        b.select_attn(lay, q, 4, out=out, idx=idx, idx_count=cnt)
        b.close()
        b = binding.Tidal(0)
        torch.cuda.empty_cache()
        called = used_by(lambda: a.select_attn(lay, q, 4, out=out, idx=idx, idx_count=cnt))
        a.close()
        most = fill(called + (160 << 20))
        try:
            b.reserve(lay, 4)
        finally:
            del most
            torch.cuda.empty_cache()
        b.select_attn(lay, q, 4, out=out, idx=idx, idx_count=cnt)
        assert b.device_status() == binding.OK
    finally:
        a.close(); b.close()


# ---- the softmax weights -------------------------------------------------------------------------------------------

@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_every_weight_enters_with_22_bits(td, fp8, G):
    """Weights laid bare: a query with one channel, so that a logit is one exact product; values with a one in the position's own
    channel, so that output channel j is weight j over their sum. Divided by the sum of the outputs, the common denominator is gone.

    Relative error of a weight, in units of 2^-24, with |t| <= 2 the logits to base 2: scale times log2 e (2 roundings) and t (one),
    3 * 2 ln 2 = 4.2; t minus the maximum, 4 ln 2 = 2.8; over an 8-bit cache 14 is added to that: two roundings of at most 16 ln 2 =
    11.1 each more; 2^x 4 (2^-22); the split 4; the factor between warps 4 and its argument 2.8; two products and the quotient 3. Together
    25, or 47 over an 8-bit cache; dividing by the sum doubles it. A weight of 16 bits is off by up to 256 such units."""
    n = 8 * BLK
    g = gen(G)
    logit = torch.rand(n, generator=g, device=DEV) * 4 - 2
    k = torch.zeros(1, n, D, device=DEV)
    k[0, :, 7] = logit
    v = torch.eye(n, D, device=DEV)[None]
    ones = torch.ones(1, device=DEV)
    scale = 0.7 / 1.4426950408889634
    lay = hnd(k, v, G, fp8, (ones, ones), sm_scale=scale)
    q = torch.zeros(1, G, D, dtype=torch.bfloat16, device=DEV)
    q[0, :, 7] = (1.0 - 0.125 * torch.arange(G, device=DEV)).to(torch.bfloat16)                  # exact
    out = td.block_attn(lay, q, torch.arange(8, dtype=torch.int32, device=DEV).expand(1, 1, 8).contiguous())[0].double()
    kept = lay.k[0, 0].float().double()[:, 7]
    t = q[0, :, 7].double()[:, None] * kept * float(torch.tensor(scale, dtype=torch.float32))
    assert float(t.abs().max()) * 1.4426950408889634 <= 2
    want = torch.softmax(t, -1)
    off = ((out / out.sum(-1, keepdim=True)) / want - 1).abs().max()
    assert off <= 2 * (47 if fp8 else 25) * 2.0 ** -24, float(off) * 2 ** 24


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("m", [16, 128, 256])
@pytest.mark.parametrize("hq,hkv,hi", [(8, 2, 8), (32, 8, 8), (32, 8, 1)])
def test_error_of_long_lists_in_norm(td, fp8, m, hq, hkv, hi):
    """The error of whole rows against 64 bits, in the 2-norm. Roundings are independent and add as squares: 2^x 2^-22 at most and half of that
    on average, a logit's and its argument's roundings as much, the two products' sums 2^-23 each: near 2^-21.5, and 2^-20 is asked for.
    Weights in 16 bits (about 2^-18.5) or a matrix instruction's accumulator carried through a list (one part in 10^6) are above it."""
    n = 2 * m * BLK
    g = gen(m + hi)
    k, v = (torch.randn(hkv, n, D, generator=g, device=DEV) for _ in range(2))
    scales = (torch.full((hkv,), 0.05, device=DEV), torch.full((hkv,), 0.03, device=DEV))
    lay = hnd(k / 0.05 if fp8 else k, v / 0.03 if fp8 else v, hq, fp8, scales if fp8 else None)
    q = torch.randn(1, hq, D, generator=g, device=DEV).to(torch.bfloat16)
    idx = torch.stack([torch.randperm(2 * m, generator=g, device=DEV)[:m].sort().values for _ in range(hi)])[None].to(torch.int32)
    out = td.block_attn(lay, q, idx).double()[0]
    kk, vv = (x[0].float().double() * (s.double()[:, None, None] if fp8 else 1.0) for x, s in zip((lay.k, lay.v), scales))
    for h in range(hq):
        pos = (idx[0, h * hi // hq].long()[:, None] * BLK + torch.arange(BLK, device=DEV)).flatten()
        gh = h // (hq // hkv)
        want = torch.softmax(kk[gh, pos] @ q[0, h].double() / math.sqrt(D), 0) @ vv[gh, pos]
        off = float((out[h] - want).norm() / want.norm())
        assert off <= 2.0 ** -20, (h, off)
