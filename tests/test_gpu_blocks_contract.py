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


# ---- writing tokens ------------------------------------------------------------------------------------------------

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
