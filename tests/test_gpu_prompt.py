"""A prompt's way through the cache: rotary positions and norms, chunk attention, attention weights per cached position, eviction;
against plain definitions in 64 bits."""
import copy
import math

import pytest
import torch

from paper_2410_05076_b200 import binding
from tests import util
from tests.test_gpu_blocks import BLK, D, DEV, gen, make, pages

pytestmark = pytest.mark.gpu
HALF, INTER = binding.ROPE_HALF, binding.ROPE_INTERLEAVED


@pytest.fixture(scope="module")
def td():
    t = binding.Tidal(0)
    yield t
    assert t.device_status() == binding.OK
    t.close()


@pytest.fixture(scope="module")
def td16():
    t = binding.Tidal(0)
    t.set_output_bf16(True)
    yield t
    assert t.device_status() == binding.OK
    t.close()


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def randn(seed, *shape):
    return torch.randn(*shape, generator=gen(seed), device=DEV).to(torch.bfloat16)


# ---- norms and rotary positions ------------------------------------------------------------------------------------

def ref_rope(x, pos, freq, scale, layout, weight, eps):
    """In 64 bits; angles from integer positions and exact frequencies."""
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    n = 2 * len(freq)
    # p f mod 2 pi in two pieces of p, so that a double's 53 bits do for positions up to 2^31
    f = torch.tensor(freq, dtype=torch.float64, device=DEV)
    p = pos.double()[:, None]
    angle = torch.remainder(torch.floor(p / 65536) * torch.remainder(65536 * f, 2 * math.pi), 2 * math.pi) + torch.remainder(p, 65536) * f
    c, s = torch.cos(angle)[:, None] * scale, torch.sin(angle)[:, None] * scale
    out = x.clone()
    a, b = (x[..., : n // 2], x[..., n // 2: n]) if layout == HALF else (x[..., :n:2], x[..., 1:n:2])
    ra, rb = a * c - b * s, b * c + a * s
    if layout == HALF:
        out[..., : n // 2], out[..., n // 2: n] = ra, rb
    else:
        out[..., :n:2], out[..., 1:n:2] = ra, rb
    return out


def rope_bound(ref, far):
    """fp32: the turn is off by 2^-32 + p 2^-65 and rounded to fp32 (2^-25), cosine and sine by 2^-23 (1 ulp and the factor), a product
    chain of five roundings and the norm's (sum of 128 squares in 8 + 4 additions, rsqrt within 2^-22): 2^-20 of the largest element of a
    row in all, doubled for the pair; then a rounding to bf16, 2^-8 of the value. The reference's own angle is good to
    p 2^-52 (its frequencies are doubles, so are the library's)."""
    return (2.0 ** -19 + far * 2.0 ** -50) * ref.abs().amax(-1, keepdim=True) + 2.0 ** -8 * ref.abs() + 2.0 ** -120


def rope_inputs(T, hq, hkv, far, seed=0):
    qkv = randn(seed, T, hq + 2 * hkv, D)
    pos = torch.randint(0, far, (T,), generator=gen(seed + 1), device=DEV).to(torch.int32)
    if T > 1:
        pos[0], pos[-1] = 0, far - 1
    return qkv[:, :hq], qkv[:, hq: hq + hkv], qkv[:, hq + hkv:], pos


def frequencies(n, base=10000.0):
    return [base ** (-2 * i / n) for i in range(n // 2)]


@pytest.mark.parametrize("layout", [HALF, INTER])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("T,hq,hkv,rotary,far", [(1, 1, 1, 128, 2 ** 31 - 1), (3, 7, 1, 16, 100), (64, 32, 8, 128, 262144), (17, 15, 5, 96, 2 ** 24 + 5),
                                                 (1000, 8, 2, 64, 131072), (7000, 4, 4, 112, 7000)])
def test_rope(td, layout, norm, T, hq, hkv, rotary, far):
    q, k, _, pos = rope_inputs(T, hq, hkv, far, seed=T)
    qw, kw = (1 + 0.3 * randn(1, D), 1 - 0.3 * randn(2, D)) if norm else (None, None)
    plan = binding.rope_plan(rotary, layout=layout)
    qo, ko = util.Guarded((T, hq, D), torch.bfloat16, DEV), util.Guarded((T, hkv, D), torch.bfloat16, DEV)
    got = td.rope(plan, q, k, pos, qw, kw, 1e-5, qo.t, ko.t)
    assert got[0] is qo.t and got[1] is ko.t
    for x, y, w in ((q, qo, qw), (k, ko, kw)):
        ref = ref_rope(x, pos, frequencies(rotary), 1.0, layout, w, 1e-5)
        assert ((y.t.double() - ref).abs() <= rope_bound(ref, far)).all(), float(((y.t.double() - ref).abs() - rope_bound(ref, far)).max())
        y.check("rope")
    if not norm:
        assert torch.equal(qo.t[..., rotary:], q[..., rotary:])          # channels that do not turn are copied
    # one weight only, one tensor only
    only = td.rope(plan, q, None, pos, qw, None, 1e-5)
    assert only[1] is None and torch.equal(only[0], qo.t)
    assert torch.equal(td.rope(plan, None, k, pos, None, kw, 1e-5)[1], ko.t)
    # in place, in the projection's output
    td.rope(plan, q, k, pos, qw, kw, 1e-5, q, k)
    assert torch.equal(q, qo.t) and torch.equal(k, ko.t)
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("scaling,factor,low,high,trained", [(binding.ROPE_PLAIN, 1, 1, 4, 1), (binding.ROPE_LINEAR, 4, 1, 4, 1), (binding.ROPE_BASE, 8, 1, 4, 1),
                                                             (binding.ROPE_BANDS, 8, 1, 4, 8192), (binding.ROPE_RAMP, 16, 1, 32, 4096)])
def test_rope_scalings_on_the_device(td, scaling, factor, low, high, trained):
    q, k, _, pos = rope_inputs(50, 4, 2, 131072)
    plan = binding.rope_plan(128, base=500000.0, scaling=scaling, factor=factor, low=low, high=high, trained_len=trained)
    freq = [int(plan.step[i]) * 2.0 ** -64 * 2 * math.pi for i in range(64)]
    qo, _ = td.rope(plan, q, k, pos)
    ref = ref_rope(q, pos, freq, plan.scale, HALF, None, 0)
    assert ((qo.double() - ref).abs() <= rope_bound(ref, 131072)).all()


def test_rope_leaves_padding_and_keeps_odd_values_apart(td):
    """Negative positions are left unwritten; an infinity meets the other channel of its pair and no other."""
    q, k, _, pos = rope_inputs(40, 3, 1, 1000)
    pos[::3] = -1
    pos[1] = -2 ** 31
    q[2, 0, 100] = math.inf
    q[4, 1, 3] = math.nan
    for layout in (HALF, INTER):
        plan = binding.rope_plan(64, layout=layout)
        qo, ko = torch.full((40, 3, D), 7.0, dtype=torch.bfloat16, device=DEV), torch.full((40, 1, D), 7.0, dtype=torch.bfloat16, device=DEV)
        td.rope(plan, q, k, pos, q_out=qo, k_out=ko)
        assert (qo[pos < 0] == 7).all() and (ko[pos < 0] == 7).all() and (ko[pos >= 0] != 7).any()
        assert qo[2, 0, 100] == math.inf and int((~torch.isfinite(qo[2])).sum()) == 1       # a channel that does not turn
        assert int((~torch.isfinite(qo[4])).sum()) == 2


def ref_code(x):
    """The E4M3 value nearest to x (64 bits) is within half a step: 2^-4 of the value, 2^-10 near zero."""
    return 2.0 ** -4 * x.abs() + 2.0 ** -10


@pytest.mark.parametrize("layout", ["paged", "hnd", "nhd"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T,hq,hkv,rotary,norm", [(1, 4, 1, 128, True), (37, 10, 5, 64, False), (300, 32, 8, 128, True)])
def test_rope_write(td, layout, fp8, T, hq, hkv, rotary, norm):
    rows = pages(T + 5) * BLK
    lay = make([rows], hq, hkv, layout, fp8, seed=5)
    q, k, v, pos = rope_inputs(T, hq, hkv, 131072, seed=T)
    qw, kw = (1 + 0.3 * randn(1, D), 1 - 0.3 * randn(2, D)) if norm else (None, None)
    at = torch.randperm(rows, generator=gen(9), device=DEV)[:T]
    slots = lay.page_table[0, at // BLK].long() * BLK + at % BLK if layout == "paged" else at
    slots, pos = slots.clone(), pos.clone()
    if T > 3:
        slots[1], pos[2] = -1, -1                         # no row in the cache; no token
    before = [x.clone().view(torch.uint8) for x in lay.keep]
    plan = binding.rope_plan(rotary, base=500000.0, layout=HALF)
    qo = torch.full((T, hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    assert td.rope_write(lay, plan, q, k, v, pos, slots, qw, kw, 1e-6, qo) is qo
    same, _ = td.rope(plan, q, None, pos, qw, None, 1e-6, torch.full_like(qo, 7.0))
    assert torch.equal(qo, same)
    written = (slots >= 0) & (pos >= 0)
    ref = ref_rope(k, pos, frequencies(rotary, 500000.0), 1.0, HALF, kw, 1e-6)

    def row(x, i):
        a = int(at[i])
        return x[int(lay.page_table[0, a // BLK]), :, a % BLK] if layout == "paged" else x[0, :, a] if layout == "hnd" else x[0, a]

    for i in range(T):
        if not written[i]:
            continue
        kk, vv = row(lay.k, i).float().double(), row(lay.v, i)
        if fp8:
            x = ref[i] / lay.k_scale.double()[:, None]
            bound = ref_code(x) + 1.1 * (2.0 ** -19 + 2.0 ** -33) * x.abs().amax(-1, keepdim=True)
            assert ((kk - x.clamp(-448, 448)).abs() <= bound).all()
            want = (v[i].float() / lay.v_scale[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
            assert torch.equal(vv.view(torch.uint8), want.view(torch.uint8))
        else:
            assert ((kk - ref[i]).abs() <= rope_bound(ref[i], 131072)).all()
            assert torch.equal(vv, v[i])
    # everything else is as it was
    gone = [x.clone() for x in before]
    for x, b in zip(lay.keep, gone):
        now, old = x.view(torch.uint8).view(b.shape), b
        changed = (now != old).nonzero()
        assert changed.shape[0] <= int(written.sum()) * hkv * D * 2 * (1 if fp8 else 2)
    assert td.device_status() == binding.OK
    # without queries the cache gets the same
    after = [x.clone().view(torch.uint8) for x in lay.keep]
    assert td.rope_write(lay, plan, None, k, v, pos, slots, None, kw, 1e-6) is None
    assert all(torch.equal(x.view(torch.uint8), a) for x, a in zip(lay.keep, after))


@pytest.mark.parametrize("layout", ["paged", "hnd", "nhd"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("turn", [HALF, INTER])
@pytest.mark.parametrize("T,hq,hkv,rotary,norm", [(1, 2, 1, 16, False), (9, 6, 3, 96, True), (200, 8, 2, 128, True), (64, 5, 5, 48, False), (2600, 4, 4, 64, True)])
def test_rope_write_changes_its_rows_and_no_other_byte(td, layout, fp8, turn, T, hq, hkv, rotary, norm):
    """Both layouts of the channels into every cache, rows with places all over it; bounds as in test_rope_write."""
    rows = pages(T + 20) * BLK
    lay = make([rows], hq, hkv, layout, fp8, seed=T)
    q, k, v, pos = rope_inputs(T, hq, hkv, 262144, seed=T + 1)
    qw, kw = (1 + 0.3 * randn(1, D), 1 - 0.3 * randn(2, D)) if norm else (None, None)
    at = torch.randperm(rows, generator=gen(9), device=DEV)[:T]
    slots = lay.page_table[0, at // BLK].long() * BLK + at % BLK if layout == "paged" else at
    slots, pos = slots.clone(), pos.clone()
    if T > 3:
        slots[2::7], pos[3::5] = -1, -1
    written = ((slots >= 0) & (pos >= 0)).nonzero()[:, 0]

    def place(x):
        a = at[written]
        x = x.view(torch.uint8 if fp8 else torch.int16)
        return (x, (lay.page_table[0, a // BLK].long(), slice(None), a % BLK)) if layout == "paged" else (x[0].transpose(0, 1) if layout == "hnd" else x[0], (a,))

    before = [x.clone() for x in lay.keep]
    (kx, ki), (vx, vi) = place(lay.k), place(lay.v)
    old = kx[ki].clone(), vx[vi].clone()
    plan = binding.rope_plan(rotary, base=500000.0, layout=turn)
    qo = td.rope_write(lay, plan, q, k, v, pos, slots, qw, kw, 1e-6, torch.full((T, hq, D), 7.0, dtype=torch.bfloat16, device=DEV))
    there = pos >= 0
    ref = ref_rope(q, pos, frequencies(rotary, 500000.0), 1.0, turn, qw, 1e-6)
    assert ((qo.double() - ref).abs() <= rope_bound(ref, 262144))[there].all() and (qo[~there] == 7).all()
    ref = ref_rope(k, pos, frequencies(rotary, 500000.0), 1.0, turn, kw, 1e-6)[written]
    if fp8:
        x = ref / lay.k_scale.double()[:, None]
        got = kx[ki].view(torch.float8_e4m3fn).double()
        bound = ref_code(x) + 1.1 * (2.0 ** -19 + 2.0 ** -32) * x.abs().amax(-1, keepdim=True)
        assert ((got - x.clamp(-448, 448)).abs() <= bound).all()
        want = (v[written].float() / lay.v_scale[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
        assert torch.equal(vx[vi], want.view(torch.uint8))
    else:
        assert ((kx[ki].view(torch.bfloat16).double() - ref).abs() <= rope_bound(ref, 262144)).all()
        assert torch.equal(vx[vi], v[written].contiguous().view(torch.int16))
    kx[ki], vx[vi] = old
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(lay.keep, before))
    assert td.device_status() == binding.OK


def test_rope_write_equals_rope_and_kv_write(td):
    """16 bits: the same rows as in two calls; slots outside the cache are skipped and reported."""
    one, two = make([64], 8, 2, seed=1), make([64], 8, 2, seed=1)
    q, k, v, pos = rope_inputs(30, 8, 2, 5000)
    slots = one.page_table[0, torch.arange(30, device=DEV) // BLK].long() * BLK + torch.arange(30, device=DEV) % BLK
    plan = binding.rope_plan(128)
    td.rope_write(one, plan, q, k, v, pos, slots)
    _, turned = td.rope(plan, None, k, pos)
    td.kv_write(two, turned, v, slots)
    a, b = one.keep[0].view(torch.int16), two.keep[0].view(torch.int16)
    assert torch.equal(a, b)
    slots[3], slots[4] = one.num_pages * BLK, -2
    td.rope_write(one, plan, q, k, v, pos, slots)
    assert torch.equal(one.keep[0].view(torch.int16), a)
    assert td.device_status() == binding.ERR_INDEX and td.device_status() == binding.OK


@pytest.mark.parametrize("scale", [2.0 ** -70, 2.0 ** 70, 0.01])
def test_rope_write_saturates(td, scale):
    lay = make([16], 1, 1, "hnd", True)
    lay.k_scale.fill_(scale)
    k = torch.full((1, 1, D), 3.0, dtype=torch.bfloat16, device=DEV)
    k[0, 0, 1] = math.nan
    td.rope_write(lay, binding.rope_plan(16), None, k, k, i32([0]), torch.tensor([2], device=DEV))
    want = min(3.0 / scale, 448.0)
    got = lay.k[0, 0, 2].float()
    assert torch.isnan(got[1]) and got[0] == torch.tensor(want).to(torch.float8_e4m3fn).float() and got[100] == got[0]


# ---- chunk attention ---------------------------------------------------------------------------------------------------

def chunk_inputs(lay, new, seed=0, extra=0):
    T = sum(new)
    q = randn(500 + seed, T + extra, lay.num_q_heads + 2 * lay.num_kv_heads, D)[:, : lay.num_q_heads]
    return q, i32([sum(new[:i]) for i in range(len(new) + 1)])


def ref_chunk(lay, q, new, causal=True, window=0, skip=()):
    """(out, lse, weights, bounds of the three): softmax over what each row sees, in 64 bits. Bounds: a logit's 8 matrix instructions add exact
    products with at most 2^-22 of the sum of their magnitudes each (2^-19), the exponent's argument is rounded twice (2^-23 of |t|
    log2 e), exponentials are within 2^-21, the sum of n weights (in chains of at most n / 2, of tiles) within 2^-17: together e. Weights enter
    the second product as bf16, off by 2^-8 each (fp16: 2^-11, and the running maximum may stand 2^8 below, so that
    weights below 2^-14 of it are off by 2^-25; the query in fp16 by 2^-25 per channel). An error r of all weights moves the mean by r max|v|."""
    B, hq, hkv = lay.batch, lay.num_q_heads, lay.num_kv_heads
    G, scale, fp8 = hq // hkv, lay.sm_scale or 1 / math.sqrt(D), bool(lay.kv_dtype)
    T = sum(new)
    out, lse = torch.zeros(T, hq, D, dtype=torch.float64, device=DEV), torch.full((T, hq), -math.inf, dtype=torch.float64, device=DEV)
    w = torch.zeros(B, hkv, lay.max_ctx_len, dtype=torch.float64, device=DEV)
    tol_o, tol_l, tol_w = torch.zeros(T, hq, 1, dtype=torch.float64, device=DEV), torch.zeros_like(lse), torch.zeros_like(w)
    at = 0
    for b, n in enumerate(new):
        k, v = lay.dense[b]
        N = k.shape[1]
        if n == 0:
            continue
        pos = N - n + torch.arange(n, device=DEV)
        j = torch.arange(N, device=DEV)
        seen = torch.ones(n, N, dtype=torch.bool, device=DEV)
        if causal:
            seen &= j[None] <= pos[:, None]
        if window:
            seen &= j[None] > pos[:, None] - window
        for pg in skip:
            seen &= (j // BLK != pg)[None]
        for h in range(hq):
            g = h // G
            qq = q[at: at + n, h].double()
            t = (qq @ k[g].t()) * scale
            mag = (qq.abs() @ k[g].abs().t()).amax(-1) * scale
            e = 2.0 ** -19 * mag + 2.0 ** -22 * t.abs().amax(-1) + 2.0 ** -17
            if fp8:
                e = e + 2.0 ** -25 * k[g].abs().sum(-1).max() * scale
            t = t.masked_fill(~seen, -math.inf)
            some = seen.any(-1)
            rows = slice(at, at + n)
            l = torch.logsumexp(t, -1)
            lse[rows, h] = torch.where(some, l, -math.inf)
            p = torch.where(some[:, None], torch.softmax(t, -1), 0.0).nan_to_num(0.0)
            vv = v[g].nan_to_num(0.0)
            out[rows, h] = p @ vv
            big = v[g][:, :].abs().amax() if N else 0.0
            tol_o[rows, h, 0] = (2 * e + 2.0 ** (-11 if fp8 else -8) + (N * 2.0 ** -25 if fp8 else 0)) * big
            tol_l[rows, h] = e + 2.0 ** -21 * l.abs().nan_to_num(0, 0, 0)
            w[b, g, :N] += p.sum(0)
            tol_w[b, g, :N] += (p * (2 * e + 2.0 ** -20 + 2.0 ** -21 * l.abs().nan_to_num(0, 0, 0))[:, None]).sum(0) + 2.0 ** -100
        at += n
    return out, lse, w, tol_o, tol_l, tol_w


def check_chunk(td, lay, new, causal=True, window=0, max_new=None, seed=0, bf16=False, skip=()):
    q, off = chunk_inputs(lay, new, seed, extra=3)
    T = sum(new)
    og = util.Guarded((T + 3, lay.num_q_heads, D), torch.bfloat16 if bf16 else torch.float32, DEV, fill=9.0)
    lg = util.Guarded((T + 3, lay.num_q_heads), torch.float32, DEV, fill=9.0)
    got = td.chunk_attn(lay, q, off, max_new=max(new) if max_new is None else max_new, causal=causal, window=window, out=og.t, lse=lg.t)
    assert got is og.t
    out, lse, w, tol_o, tol_l, tol_w = ref_chunk(lay, q, new, causal, window, skip)
    og.check("out"); lg.check("lse")
    assert (og.t[T:] == 9).all() and (lg.t[T:] == 9).all()              # rows behind the last sequence
    blind = torch.isinf(lse)
    assert torch.equal(torch.isinf(lg.t[:T]), blind) and (lg.t[:T][blind] < 0).all() and (og.t[:T][blind] == 0).all()
    err = (og.t[:T].double() - out).abs()
    tol = tol_o + (2.0 ** -8 * (out.abs() + tol_o) if bf16 else 0)
    assert torch.isfinite(og.t[:T].float()).all()
    assert (err <= tol).all(), f"out: {float((err - tol).max()):.3e} over, max {float(err.max()):.3e} of {float(out.abs().max()):.3e}"
    el = (lg.t[:T].double() - lse).abs()[~blind]
    assert (el <= tol_l[~blind]).all(), f"lse: max {float(el.max()):.3e}"
    return q, off, lg.t[:T + 3], w, tol_w


CHUNKS = [
    # lengths, new tokens, query heads, KV heads
    ([1], [1], 1, 1), ([128], [128], 4, 1), ([129], [1], 8, 1), ([700], [33], 8, 2), ([300, 5, 1, 0, 257], [300, 2, 1, 0, 100], 6, 2),
    ([1000, 17, 640], [0, 17, 1], 10, 2), ([2000], [400], 7, 1), ([50, 50], [50, 0], 16, 2), ([130, 260, 520], [64, 65, 200], 3, 3),
    ([4103], [7], 8, 2), ([1500] * 6, [1] * 6, 32, 8),
]


@pytest.mark.parametrize("layout", ["paged", "hnd", "nhd"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,new,hq,hkv", CHUNKS)
def test_chunk_attention(td, layout, fp8, lens, new, hq, hkv):
    lay = make(lens, hq, hkv, layout, fp8, seed=len(lens) + hq)
    check_chunk(td, lay, new, max_new=0)
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("causal,window", [(True, 1), (True, 40), (True, 129), (True, 100000), (False, 0), (False, 70)])
@pytest.mark.parametrize("lens,new,hq,hkv", [([700, 90, 3], [300, 90, 1], 8, 2), ([1900, 40], [1, 1], 4, 1)])
def test_chunk_attention_masks(td, fp8, causal, window, lens, new, hq, hkv):
    lay = make(lens, hq, hkv, "paged", fp8, seed=window)
    check_chunk(td, lay, new, causal, window)


def test_chunk_attention_options(td, td16):
    """bf16 outputs, an explicit scale, a bound on the lengths beyond the longest, tokens beyond max_new left out, no log-sum-exp."""
    lay = make([300, 77], 12, 4, "paged", seed=4, max_len=1000, sm_scale=0.31)
    q, off, lse, _, _ = check_chunk(td, lay, [140, 77])
    check_chunk(td16, lay, [140, 77], bf16=True)
    one, two = td.chunk_attn(lay, q, off), td.chunk_attn(lay, q, off, lse=torch.empty(220, 12, device=DEV))
    assert torch.equal(one[:217], two[:217])
    td.chunk_attn(lay, q, off, max_new=1)                 # (no more than left out)
    one = q[:1].clone()
    assert torch.equal(td.chunk_attn(make([5], 12, 4, "hnd"), one, i32([0, 1])), td.chunk_attn(make([5], 12, 4, "hnd"), q[:1], i32([0, 1])))


def test_chunk_rows_that_see_nothing(td):
    """More new tokens than the cache counts: the first of them stand before position 0."""
    lay = make([10, 0], 4, 2, "hnd", seed=1)
    q = randn(3, 20, 4, D)
    lse = torch.zeros(20, 4, device=DEV)
    out = td.chunk_attn(lay, q, i32([0, 15, 20]), lse=lse)
    dead = torch.tensor([True] * 5 + [False] * 10 + [True] * 5, device=DEV)
    assert (out[dead] == 0).all() and (lse[dead] == -math.inf).all() and torch.isfinite(lse[~dead]).all()
    ref = ref_chunk(lay, q[5:15].contiguous(), [10, 0])
    assert ((out[5:15].double() - ref[0]).abs() <= ref[3]).all()


@pytest.mark.parametrize("window", [262143, 262144, 2 ** 31 - 1])
def test_windows_beyond_every_context(td, window):
    """Rows before position 0 among them: nothing wraps."""
    lay = make([10, 700], 4, 2, "hnd", seed=1)
    q = randn(3, 320, 4, D)
    off, lse = i32([0, 20, 320]), torch.zeros(320, 4, device=DEV)
    want, w = td.chunk_attn(lay, q, off, lse=lse), torch.zeros(2, 2, 700, device=DEV)
    assert torch.equal(td.chunk_attn(lay, q, off, window=window), want)
    td.chunk_weights(lay, q, off, lse, w)
    assert torch.equal(td.chunk_weights(lay, q, off, lse, torch.zeros_like(w), window=window), w)
    one = td.chunk_attn(lay, q[:2], i32([0, 1, 2]), max_new=1, window=window)
    assert float((one - td.chunk_attn(lay, q[:2], i32([0, 1, 2]), max_new=1)).abs().max()) <= 2.0 ** -8 * 6


def test_chunk_offsets_out_of_order_are_cut_and_reported(td):
    lay = make([40, 40, 40], 2, 1, "paged")
    q = randn(3, 30, 2, D)
    for off in ([0, 20, 10, 30], [0, 10, 20, 31], [-5, 10, 20, 30]):
        td.chunk_attn(lay, q, i32(off))
        assert td.device_status() == binding.ERR_INDEX
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("heads", [1, 2])
@pytest.mark.parametrize("off", [[0, 20, 10, 30], [0, 10, 20, 31], [-5, 10, 20, 30], [0, 40, 40, 40], [0, 0, 31, 30]])
def test_weights_of_offsets_out_of_order_are_cut_and_reported(td, heads, off):
    lay = make([40, 0, 40], 4, 2, "paged")
    q, lse = randn(3, 30, 4, D), torch.zeros(30, 4, device=DEV)
    got = td.chunk_weights(lay, q, i32(off), lse, torch.zeros(3, heads, 40, device=DEV))
    assert td.device_status() == binding.ERR_INDEX and td.device_status() == binding.OK
    assert torch.isfinite(got).all()
    td.chunk_weights(lay, q, i32([0, 10, 20, 30]), lse, got)
    assert td.device_status() == binding.OK


def test_weights_report_the_offsets_of_the_last_of_many_sequences(td):
    lay = make([1] * 700, 1, 1, "hnd")
    q, lse = randn(3, 700, 1, D), torch.zeros(700, 1, device=DEV)
    off = torch.arange(701, dtype=torch.int32, device=DEV)
    w = torch.zeros(700, 1, 1, device=DEV)
    td.chunk_weights(lay, q, off, lse, w)
    assert td.device_status() == binding.OK
    off[700] = 698
    td.chunk_weights(lay, q, off, lse, w)
    assert td.device_status() == binding.ERR_INDEX


@pytest.mark.parametrize("fp8", [False, True])
def test_chunk_bad_pages_are_skipped_and_reported(td, fp8):
    lay = make([400], 4, 2, "paged", fp8, seed=2)
    table = lay.page_table.clone()
    lay.page_table[0, 3], lay.page_table[0, 20] = -1, lay.num_pages
    q, off, lse, w, tol = check_chunk(td, lay, [30], skip=(3, 20))
    assert td.device_status() == binding.ERR_INDEX
    got = td.chunk_weights(lay, q, off, lse, torch.full((1, 2, 400), 5.0, device=DEV), decay=0.0)
    assert ((got.double() - w).abs() <= tol).all() and (got[..., 48:64] == 0).all()
    assert td.device_status() == binding.ERR_INDEX
    lay.page_table.copy_(table)
    td.chunk_attn(lay, q, off)
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hq,hkv,new", [(20, 20, 3), (32, 16, 200), (8, 1, 40)])
@pytest.mark.parametrize("max_new", [0, 1])
def test_weights_of_all_heads_together_next_to_bad_pages(td, fp8, hq, hkv, new, max_new):
    """Every tile has other bad pages, and the tiles of many heads lie between one of a warpgroup's and its next."""
    new = 1 if max_new else new
    lay = make([6000], hq, hkv, "paged", fp8, seed=3)
    bad = [pg for pg in range(375) if (pg * pg + pg // 8) % 7 == 3]
    lay.page_table[0, bad] = lay.num_pages
    q, off, lse, w, tol = check_chunk(td, lay, [new], skip=bad, max_new=0)
    for heads, want, bound in ((hkv, w, tol), (1, w.sum(1, keepdim=True), tol.sum(1, keepdim=True) + 2.0 ** -20 * w.sum(1, keepdim=True))):
        for _ in range(3):
            got = td.chunk_weights(lay, q, off, lse, torch.full((1, heads, 6000), 5.0, device=DEV), decay=0.0, max_new=max_new)
            assert ((got.double() - want).abs() <= bound).all()
            blind = torch.isin(torch.arange(6000, device=DEV) // BLK, torch.tensor(bad, device=DEV))
            assert (got[..., blind] == 0).all() and (got[..., : 6000 - new][..., ~blind[: 6000 - new]] > 0).all()
    assert td.device_status() == binding.ERR_INDEX


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,new,window,last", [([3000], [50], 200, 0), ([3000, 700, 90], [300, 1, 0], 33, 0), ([5000], [1], 1000, 0), ([900], [250], 17, 20), ([130], [1], 2, 0)])
def test_pages_that_no_window_reaches_are_nobodys(td, fp8, causal, lens, new, window, last):
    """Pages before the first new token's window, and those of a sequence without new tokens, may be gone; the first that is seen may not."""
    lay = make(lens, 8, 2, "paged", fp8, seed=6)
    q, off = chunk_inputs(lay, new)
    lse = [torch.zeros(q.shape[:2], device=DEV) for _ in range(2)]
    old = torch.rand(len(lens), 2, max(lens), generator=gen(1), device=DEV)
    first = [max(n - t - window + 1, 0) // BLK for n, t in zip(lens, new)]
    outs = []
    for i in range(2):
        outs.append((td.chunk_attn(lay, q, off, causal=causal, window=window, lse=lse[i]), lse[i],
                     td.chunk_weights(lay, q, off, lse[i], old.clone(), decay=0.5, causal=causal, window=window, last=last)))
        assert td.device_status() == binding.OK
        for b, t in enumerate(new):
            lay.page_table[b, : first[b] if t else pages(lens[b])] = -1
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    lay.page_table[0, first[0]] = lay.num_pages
    td.chunk_attn(lay, q, off, causal=causal, window=window)
    assert td.device_status() == binding.ERR_INDEX
    if not last:
        td.chunk_weights(lay, q, off, lse[0], old.clone(), causal=causal, window=window)
        assert td.device_status() == binding.ERR_INDEX


def test_chunk_attention_over_infinite_and_missing_numbers(td):
    """A logit that is not a number, or a value, spoils the rows that see it."""
    lay = make([260], 2, 1, "hnd", seed=7)
    q, off = chunk_inputs(lay, [100])
    lay.k[0, 0, 200, 3] = math.nan
    lse = torch.empty(100, 2, device=DEV)
    out = td.chunk_attn(lay, q, off, lse=lse)
    assert torch.isnan(out[40:]).all() and torch.isnan(lse[40:]).all() and torch.isfinite(out[:40]).all() and torch.isfinite(lse[:40]).all()


@pytest.mark.parametrize("bad,fp8", [(math.nan, False), (math.inf, False), (-math.inf, False), (math.nan, True)])     # (codes hold no infinities)
@pytest.mark.parametrize("lens,new,at,window", [([260], [100], 200, 0), ([1000], [300], 750, 0), ([5000], [20], 4985, 0), ([600], [200], 450, 64)])
def test_a_value_spoils_only_the_rows_that_see_it(td, bad, fp8, lens, new, at, window):
    lay = make(lens, 4, 2, "hnd", fp8, seed=7)
    q, off = chunk_inputs(lay, new)
    want = td.chunk_attn(lay, q, off, window=window)
    if fp8:
        lay.v.view(torch.uint8)[0, 1, at, 5] = 0x7F
    else:
        lay.v[0, 1, at, 5] = bad
    got = td.chunk_attn(lay, q, off, window=window)
    pos = lens[0] - new[0] + torch.arange(new[0], device=DEV)
    seen = (pos >= at) & ((pos < at + window) if window else True)
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[:, 2:, 5] = seen[:, None]
    close = (got - want).abs() <= 2.0 ** -6 * want.abs().amax()          # (another way of adding up: weights in fp32)
    assert (close | hit).all()
    assert (torch.isnan(got[hit]) if math.isnan(bad) else got[hit] == bad).all()


def spoil_values(lay, spots):
    """Values that are not finite at (sequence, KV head, position, channel): the cache's, and the plain copy's."""
    for b, g, pos, c, bad in spots:
        at = (lay.page_table[b, pos // BLK], g, pos % BLK) if lay.paged else (b, g, pos) if lay.stride_head > lay.stride_pos else (b, pos, g)
        if lay.kv_dtype:
            lay.v.view(torch.uint8)[at][c] = 0x7F
        else:
            lay.v[at][c] = bad
        lay.dense[b][1][g, pos, c] = math.nan if lay.kv_dtype else bad


def check_spoiled(td, lay, new, causal, window, bf16=False):
    """Against 64 bits: numbers where a row sees finite values only, and what infinities and not-a-numbers add up to where it does not."""
    q, off = chunk_inputs(lay, new)
    lse = torch.zeros(q.shape[:2], device=DEV)
    got = td.chunk_attn(lay, q, off, causal=causal, window=window, lse=lse).double()
    finite = copy.copy(lay)
    finite.dense = [(k, torch.where(torch.isfinite(v), v, 0.0)) for k, v in lay.dense]
    out, ref_lse, _, tol, tol_l, _ = ref_chunk(finite, q, new, causal, window)
    tol = tol + (2.0 ** -8 * (out.abs() + tol) if bf16 else 0)
    G, at = lay.num_q_heads // lay.num_kv_heads, 0
    for b, n in enumerate(new):
        N = lay.dense[b][0].shape[1]
        pos, j = N - n + torch.arange(n, device=DEV), torch.arange(N, device=DEV)
        seen = torch.ones(n, N, dtype=torch.bool, device=DEV)
        seen &= (j[None] <= pos[:, None]) | (not causal)
        seen &= (j[None] > pos[:, None] - window) | (not window)
        for g in range(lay.num_kv_heads):
            v = lay.dense[b][1][g]
            up, down, none = ((seen.double() @ x.double() > 0)[:, None].expand(n, G, D) for x in (v == math.inf, v == -math.inf, torch.isnan(v)))
            o = got[at: at + n, g * G: (g + 1) * G]
            none, hit = none | (up & down), none | up | down
            assert torch.equal(torch.isnan(o), none) and (o[up & ~none] == math.inf).all() and (o[down & ~none] == -math.inf).all()
            err = (o - out[at: at + n, g * G: (g + 1) * G]).abs()
            assert ((err <= tol[at: at + n, g * G: (g + 1) * G]) | hit).all() and (~hit).any()
        at += n
    assert ((lse.double() - ref_lse).abs() <= tol_l).all()


@pytest.mark.parametrize("layout", ["paged", "hnd", "nhd"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 70), (True, 300), (False, 130)])
@pytest.mark.parametrize("lens,new,hq,hkv", [([700], [500], 8, 2), ([300, 2000], [300, 30], 6, 2), ([900], [250], 3, 3), ([6000], [5], 8, 1), ([400, 260], [64, 130], 16, 2)])
def test_values_that_are_not_finite(td, td16, layout, fp8, causal, window, lens, new, hq, hkv):
    """Several of them: in tiles that all rows see, some or none, in both streams' tiles, on either side of a page's and of a tile's end, in one position and in many."""
    r = torch.Generator().manual_seed(len(lens) + hq + window)
    pick = lambda n: int(torch.randint(0, n, (1,), generator=r))  # noqa: E731
    lay = make(lens, hq, hkv, layout, fp8, seed=hq)
    spots = []
    for b, n in enumerate(lens):
        first = n - new[b]
        for i in range(8):
            pos = [n - 1, first, min(first + 1, n - 1), pick(n), pick(n), first + pick(new[b]), first + pick(new[b]), max(first - 1, 0)][i]
            for c in range(1 + pick(3)):
                spots.append((b, pick(hkv), pos, 8 * i + 64 * (c == 1) + pick(4), [math.nan, math.inf, -math.inf][pick(3)]))
    spoil_values(lay, spots)
    check_spoiled(td, lay, new, causal, window)
    check_spoiled(td16, lay, new, causal, window, bf16=True)
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("max_new", [0, 1])
@pytest.mark.parametrize("at,high", [(100, 2900), (2900, 100), (40, 60), (100, 200)])
def test_an_infinity_far_below_the_largest_logit_is_not_lost(td, at, high, max_new):
    """A weight of e^-300 times an infinity is an infinity, and in 32 bits not a number; whichever parts of the context the two positions lie in."""
    lay = make([3000, 3000], 1, 1, "hnd", seed=3)
    q, off = chunk_inputs(lay, [1, 1])
    want = td.chunk_attn(lay, q, off, max_new=max_new)
    lay.k[0, 0, high] = (q[0, 0].float() * (300 * math.sqrt(D) / float((q[0, 0].double() ** 2).sum()))).to(torch.bfloat16)
    lay.v[0, 0, at, 5] = math.inf
    got = td.chunk_attn(lay, q, off, max_new=max_new)
    assert not math.isfinite(float(got[0, 0, 5])) and torch.isfinite(got[0, 0, :5]).all() and torch.isfinite(got[0, 0, 6:]).all()
    assert float((got[1] - want[1]).abs().max()) <= 2.0 ** -8 * float(lay.dense[1][1].abs().max())


@pytest.mark.parametrize("fp8", [False, True])
def test_one_odd_value_does_not_hold_up_a_call(td, fp8):
    """60000 positions, one not-a-number among the new tokens' values: about as long as without it."""
    lay = make([60000], 8, 2, "paged", fp8, seed=1)
    q, off = chunk_inputs(lay, [400])

    def once():
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        td.chunk_attn(lay, q, off)
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b)

    once()
    plain = min(once() for _ in range(5))
    spoil_values(lay, [(0, 1, 59700, 7, math.inf)])
    assert min(once() for _ in range(3)) <= 3 * plain + 0.5


@pytest.mark.parametrize("layout", ["paged", "hnd", "nhd"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,new,hq,hkv", [([40000], [1], 8, 1), ([20000], [1], 32, 8), ([9000, 1, 5000, 300, 6000], [1, 1, 0, 1, 1], 6, 2), ([700] * 70, [1] * 69 + [0], 4, 2),
                                             ([6000, 30000], [0, 1], 5, 1)])
def test_single_tokens_of_long_caches(td, layout, fp8, causal, lens, new, hq, hkv):
    """The form that streams the cache: one token a sequence, or none, with max_new = 1."""
    lay = make(lens, hq, hkv, layout, fp8, seed=len(lens) + hq)
    assert lay.max_ctx_len * len(lens) * hkv >= 32768
    for _ in range(2):                                    # (the counters are as they were)
        q, off, lse, w, tol = check_chunk(td, lay, new, causal, max_new=1)
    got = td.chunk_weights(lay, q, off, lse, torch.zeros(len(lens), hkv, lay.max_ctx_len, device=DEV), max_new=1, causal=causal)
    assert ((got.double() - w).abs() <= tol).all()
    assert td.device_status() == binding.OK


def close_bound(lay, q, new):
    """(out in 64 bits, bound per element, two results that are wrong). A weight is off by its logit's and exponential's error (2 e, see ref_chunk) and by its
    rounding to bf16, 2^-8 (over an 8-bit cache to fp16, 2^-11, or 2^-25 in all where it is small): so much of sum p |v| in its channel. The product's
    sums are rounded once per 16 positions, each by at most 2^-22 of that."""
    hq, G, fp8, scale, T = lay.num_q_heads, lay.num_q_heads // lay.num_kv_heads, bool(lay.kv_dtype), lay.sm_scale, sum(new)
    out, tol, wrong = torch.zeros(T, hq, D, dtype=torch.float64, device=DEV), torch.zeros(T, hq, D, dtype=torch.float64, device=DEV), []
    swapped, half = torch.zeros_like(out), torch.zeros_like(out)
    at = 0
    for b, n in enumerate(new):
        k, v = lay.dense[b]
        N = k.shape[1]
        for h in range(hq if n else 0):
            kk, vv, qq = k[h // G], v[h // G], q[at: at + n, h].double()
            t = qq @ kk.t() * scale
            e = 2.0 ** -19 * (qq.abs() @ kk.abs().t()).amax(-1) * scale + 2.0 ** -22 * t.abs().amax(-1) + 2.0 ** -17 + (2.0 ** -25 * kk.abs().sum(-1).max() * scale if fp8 else 0)
            p = torch.softmax(t, -1)
            out[at: at + n, h] = p @ vv
            tol[at: at + n, h] = (2 * e + 2.0 ** (-11 if fp8 else -8) + N * 2.0 ** -26)[:, None] * (p @ vv.abs()) + (2.0 ** -25 * vv.abs().sum(0) if fp8 else 0) + 2.0 ** -60
            swapped[at: at + n, h] = p @ vv.roll(16, 0)                 # the next page's values
            half[at: at + n, h] = torch.softmax(t[:, : (N + 1) // 2], -1) @ vv[: (N + 1) // 2]
        at += n
    return out, tol, (torch.zeros_like(out), swapped, half)


@pytest.mark.parametrize("layout", ["paged", "hnd", "nhd"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("scale", [0.088, 0.25])
@pytest.mark.parametrize("lens,hq,hkv", [([40000], 8, 1), ([20000], 32, 8), ([9000, 20000, 33000], 6, 2), ([1500] * 40, 4, 2)])
def test_single_tokens_of_long_caches_closely(td, layout, fp8, scale, lens, hq, hkv):
    """Bounds that results without the values, with other positions' values, or of half the positions miss."""
    lay = make(lens, hq, hkv, layout, fp8, seed=len(lens) + hq, sm_scale=scale)
    new = [1] * len(lens)
    q, off = chunk_inputs(lay, new)
    out, tol, wrong = close_bound(lay, q, new)
    for w in wrong:
        assert float(((w - out).abs() > tol).double().mean()) > 0.5
    for max_new in (1, 0):
        got = td.chunk_attn(lay, q, off, max_new=max_new)
        assert ((got.double() - out).abs() <= tol).all(), (max_new, float(((got.double() - out).abs() / tol).max()))
    if not fp8:
        got = td.full_attn(lay, q.contiguous())           # the decode step's
        assert ((got.double() - out).abs() <= tol).all()
    assert td.device_status() == binding.OK


def test_single_tokens_where_there_are_more(td):
    """max_new = 1 and two tokens: the first of them is worked out, with the positions that it sees."""
    lay = make([30000, 9000], 4, 2, "paged", seed=5)
    q = randn(6, 3, 4, D)
    got = td.chunk_attn(lay, q, i32([0, 2, 3]), max_new=1)
    want = td.chunk_attn(lay, q, i32([0, 2, 3]))
    big = max(float(v.abs().max()) for _, v in lay.dense)
    assert float((got - want)[[0, 2]].abs().max()) <= 2 * 2.0 ** -8 * big
    lay.ctx_lens.copy_(i32([1, 0]))
    lse = torch.zeros(3, 4, device=DEV)
    got = td.chunk_attn(lay, q, i32([0, 2, 3]), max_new=1, lse=lse)
    assert (got[[0, 2]] == 0).all() and (lse[[0, 2]] == -math.inf).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,new", [([0, 5000], [0, 1]), ([0], [1]), ([0, 0, 700, 0] * 8, [1, 0, 1, 0] * 8), ([40, 20000], [0, 1])])
def test_single_tokens_beside_idle_places(td, fp8, lens, new):
    """Sequences without a token, or without a cached position, whose page tables hold nothing: their pages are nobody's business."""
    lay = make(lens, 8, 2, "paged", fp8, seed=4)
    idle = [b for b, (n, t) in enumerate(zip(lens, new)) if n == 0 or t == 0]
    lay.page_table[idle] = -1
    q, off = chunk_inputs(lay, new)
    there = [t if n else 0 for n, t in zip(lens, new)]
    full = torch.tensor([bool(n) for n, t in zip(lens, new) if t], device=DEV)       # of the tokens, in order
    ref, ref_lse, _, tol, tol_l, _ = ref_chunk(lay, q[full], there)
    for max_new in (1, 0):
        lse = torch.zeros(q.shape[:2], device=DEV)
        got = td.chunk_attn(lay, q, off, max_new=max_new, lse=lse)
        assert td.device_status() == binding.OK
        assert (got[~full] == 0).all() and (lse[~full] == -math.inf).all()
        assert ((got[full].double() - ref).abs() <= tol).all() and ((lse[full].double() - ref_lse).abs() <= tol_l).all()


def test_single_tokens_next_to_numbers_that_are_none(td):
    lay = make([40000], 4, 2, "hnd", seed=7)
    q, off = chunk_inputs(lay, [1])
    want = td.chunk_attn(lay, q, off, max_new=1)
    lay.k[0, 1, 20000, 3] = math.nan
    lse = torch.zeros(1, 4, device=DEV)
    got = td.chunk_attn(lay, q, off, max_new=1, lse=lse)
    assert torch.isnan(got[:, 2:]).all() and torch.isnan(lse[:, 2:]).all() and torch.isfinite(lse[:, :2]).all()
    assert float((got - want)[:, :2].abs().max()) <= 2.0 ** -8 * float(lay.dense[0][1].abs().max())
    off[0] = 5
    td.chunk_attn(lay, q, off, max_new=1)
    assert td.device_status() == binding.ERR_INDEX


def test_chunk_of_one_equals_the_decode_step(td):
    lay = make([900, 31, 4000], 16, 4, "paged", seed=3)
    q = randn(8, 3, 16, D)
    a, b = td.chunk_attn(lay, q, i32([0, 1, 2, 3]), max_new=1), td.full_attn(lay, q)
    big = max(float(v.abs().max()) for _, v in lay.dense)
    assert float((a - b).abs().max()) <= 2 * 2.0 ** -8 * big            # weights rounded to bf16 in both


@pytest.mark.parametrize("fp8", [False, True])
def test_chunk_attention_beyond_32_bits(td, fp8):
    """Pages more than 4 GB apart."""
    hkv, stride = 2, 1 << 16
    pages_ = (5 << 30) // (stride * (1 if fp8 else 2)) + 8
    pool = torch.zeros(pages_ * stride, dtype=torch.uint8 if fp8 else torch.bfloat16, device=DEV)
    pool = pool.view(torch.float8_e4m3fn) if fp8 else pool
    small = make([70], 4, hkv, "paged", fp8, seed=1)
    far = torch.tensor([pages_ - 1 - i for i in range(5)], device=DEV)
    view = pool.view(pages_, stride)[:, : hkv * BLK * 2 * D]
    (view.view(torch.uint8) if fp8 else view)[far] = (small.keep[0].view(torch.uint8) if fp8 else small.keep[0])[small.page_table[0, :5].long()].reshape(5, -1)
    lay = copy.copy(small)
    lay.k, lay.v = view[:, :D], view[:, D:2 * D]
    lay.stride_page, lay.num_pages = stride, pages_
    lay.page_table = far[None].to(torch.int32).contiguous()
    lay.max_pages_per_seq, lay.max_ctx_len = 5, 70
    q, off = chunk_inputs(lay, [33])
    lse, lse2 = torch.empty(33, 4, device=DEV), torch.empty(33, 4, device=DEV)
    assert torch.equal(td.chunk_attn(lay, q, off, lse=lse), td.chunk_attn(small, q, off, lse=lse2)) and torch.equal(lse, lse2)
    w, w2 = torch.zeros(1, hkv, 70, device=DEV), torch.zeros(1, hkv, 70, device=DEV)
    assert torch.equal(td.chunk_weights(lay, q, off, lse, w), td.chunk_weights(small, q, off, lse, w2))
    td.kv_gather(lay, i32([[[3, 69]]]), i32([2]))
    td.kv_gather(small, i32([[[3, 69]]]), i32([2]))
    a = view[far[0]].view(torch.uint8)
    assert torch.equal(a, small.keep[0][small.page_table[0, 0].long()].reshape(-1).view(torch.uint8))


# ---- attention weights ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("layout", ["paged", "hnd", "nhd"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,new,hq,hkv", CHUNKS)
def test_chunk_weights(td, layout, fp8, lens, new, hq, hkv):
    lay = make(lens, hq, hkv, layout, fp8, seed=len(lens) + hq)
    q, off, lse, w, tol = check_chunk(td, lay, new)
    stride = lay.max_ctx_len + 5
    old = torch.rand(lay.batch, hkv, stride, generator=gen(3), device=DEV)
    n = torch.tensor(lens, device=DEV)[:, None, None]
    first = n - torch.tensor(new, device=DEV)[:, None, None]
    j = torch.arange(stride, device=DEV)
    for decay, max_new in ((0.0, 0), (1.0, max(new)), (0.75, 0)):
        g = util.Guarded(old.shape, torch.float32, DEV)
        g.t.copy_(old if decay else torch.full_like(old, math.nan))
        assert td.chunk_weights(lay, q, off, lse, g.t, decay=decay, max_new=max_new) is g.t
        want = torch.where(j < first, decay * old.double(), 0.0)
        want[..., : lay.max_ctx_len] += w
        bound = torch.zeros_like(want)
        bound[..., : lay.max_ctx_len] = tol
        there = j < n
        err = (g.t.double() - want).abs()[there.expand_as(want)]
        assert (err <= (bound + 2.0 ** -23 * want)[there.expand_as(want)]).all(), float(err.max())
        rest = g.t[(~there).expand_as(want)]
        assert torch.isnan(rest).all() if not decay else torch.equal(rest, old[(~there).expand_as(want)])
        g.check("weights")
    # all heads together; the same sums every time
    one = td.chunk_weights(lay, q, off, lse, torch.zeros(lay.batch, 1, stride, device=DEV))
    bound = (tol.sum(1) + 2.0 ** -20 * w.sum(1))
    assert ((one[:, 0, : lay.max_ctx_len].double() - w.sum(1)).abs() <= bound).all()
    assert torch.equal(one, td.chunk_weights(lay, q, off, lse, torch.zeros(lay.batch, 1, stride, device=DEV)))
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("causal,window,last", [(True, 0, 16), (True, 50, 0), (False, 0, 0), (False, 33, 100), (True, 200, 7), (True, 0, 1000)])
def test_chunk_weights_masks(td, fp8, causal, window, last):
    lens, new = [900, 300, 20, 64], [200, 300, 1, 0]
    lay = make(lens, 6, 2, "paged", fp8, seed=9)
    q, off, lse, _, _ = check_chunk(td, lay, new, causal, window)
    got = td.chunk_weights(lay, q, off, lse, torch.zeros(4, 2, 900, device=DEV), causal=causal, window=window, last=last, max_new=300)
    lse = lse.double()
    at = 0
    for b, n in enumerate(new):
        k = lay.dense[b][0]
        N = lens[b]
        pos, j = N - n + torch.arange(n, device=DEV), torch.arange(N, device=DEV)
        seen = torch.ones(n, N, dtype=torch.bool, device=DEV)
        if causal:
            seen &= j[None] <= pos[:, None]
        if window:
            seen &= j[None] > pos[:, None] - window
        if last:
            seen &= (torch.arange(n, device=DEV) >= n - last)[:, None]
        for g in range(2):
            want = torch.zeros(N, dtype=torch.float64, device=DEV)
            for h in range(3 * g, 3 * g + 3):
                t = q[at: at + n, h].double() @ k[g].t() / math.sqrt(D)
                want += torch.where(seen, torch.exp(t - lse[at: at + n, h, None]), 0.0).sum(0)
            assert ((got[b, g, :N].double() - want).abs() <= 2.0 ** -12 * want + 1e-30).all()
        at += n


# ---- eviction --------------------------------------------------------------------------------------------------------------

def ref_evict(w, lens, m, first, last):
    B, H, _ = w.shape
    kept, cnt = torch.full((B, H, m), -1, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
    for b in range(B):
        n = lens[b]
        cnt[b] = c = min(m, n)
        for h in range(H):
            x = w[b, h, :n].double().cpu()
            x = torch.where(torch.isnan(x), -math.inf, x)
            rank = torch.where(torch.isnan(w[b, h, :n].cpu()), 0, 1)     # not-a-numbers below -infinity
            j = torch.arange(n)
            rank = torch.where((j < first) | (j >= n - last), 2, rank)
            x = torch.where(rank == 2, 0.0, x) + 0.0
            order = torch.sort(x, descending=True, stable=True).indices
            order = order[torch.sort(rank[order], descending=True, stable=True).indices]
            kept[b, h, :c] = order[:c].sort().values
    return kept, cnt


def weight_cache(lens, hq, hkv, layout="hnd", **kw):
    return make(lens, hq, hkv, layout, **kw)


@pytest.mark.parametrize("kind", ["random", "ties", "zeros", "odd", "steps", "sorted"])
@pytest.mark.parametrize("lens,heads,m,first,last", [([1], 1, 1, 0, 0), ([40, 0, 17, 16], 2, 16, 1, 2), ([5000, 300, 4097], 3, 4096, 4, 32), ([20000], 2, 777, 0, 0),
                                                     ([3000] * 40, 1, 1500, 10, 100), ([70000], 1, 4096, 4, 64), ([100, 60], 1, 30, 20, 20), ([2000], 1, 5, 50, 50)])
def test_evict_select(td, kind, lens, heads, m, first, last):
    lay = make(lens, 4 * heads, heads, "paged", spoil=False)
    stride = max(lens) + 3
    w = torch.rand(len(lens), heads, stride, generator=gen(m), device=DEV) ** 8
    if kind == "ties":
        w = torch.floor(w * 20) / 20
    elif kind == "zeros":
        w = torch.where(torch.rand(w.shape, generator=gen(1), device=DEV) < 0.9, torch.zeros_like(w), w)
        w[..., 1::2] *= -1.0                              # both zeros, and negative weights
    elif kind == "odd":
        w[..., ::5], w[..., 1::7], w[..., 2::11] = math.nan, math.inf, -math.inf
    elif kind == "steps":
        w = torch.arange(stride, device=DEV).float().expand_as(w) // 100
    elif kind == "sorted":
        w = w.sort(-1).values
    w = w.contiguous()
    kept, cnt = util.Guarded((len(lens), heads, m), torch.int32, DEV), util.Guarded((len(lens),), torch.int32, DEV)
    got = td.evict_select(lay, w, m, first, last, kept.t, cnt.t)
    assert got[0] is kept.t and got[1] is cnt.t
    want = ref_evict(w, lens, m, first, last)
    assert torch.equal(cnt.t.cpu(), want[1])
    assert torch.equal(kept.t.cpu(), want[0]), (kept.t.cpu() != want[0]).nonzero()[:5]
    kept.check("kept"); cnt.check("new_lens")


def test_evict_select_of_the_longest_context(td):
    lay = make([262144], 1, 1, "paged", spoil=False)
    w = torch.rand(1, 1, 262144, generator=gen(4), device=DEV)
    for m in (1, 100000, 262143, 262144):
        kept, cnt = td.evict_select(lay, w, m)
        want = torch.sort(w[0, 0], descending=True, stable=True).indices[:m].sort().values
        assert int(cnt) == m and torch.equal(kept[0, 0].long(), want)


def gathered(lay, kept, cnt, heads):
    """Rows after a gather, per sequence: (keys, values) codes of the first cnt positions."""
    out = []
    for b in range(lay.batch):
        c = int(cnt[b])
        rows = []
        for g in range(lay.num_kv_heads):
            idx = kept[b, g if heads > 1 else 0, :c].long()
            rows.append((lay.codes[b][0][g, idx], lay.codes[b][1][g, idx]))
        out.append((torch.stack([r[0] for r in rows]), torch.stack([r[1] for r in rows])))
    return out


def read_rows(lay, b, c):
    pos = torch.arange(c, device=DEV)
    if lay.paged:
        pg = lay.page_table[b, pos // BLK].long()
        return [x.view(torch.uint8)[pg, :, pos % BLK].transpose(0, 1).contiguous().view(x.dtype).float().double() if lay.kv_dtype else x[pg, :, pos % BLK].transpose(0, 1).double()
                for x in (lay.k, lay.v)]
    if lay.stride_head > lay.stride_pos:
        return [x[b, :, :c].float().double() for x in (lay.k, lay.v)]
    return [x[b, :c].transpose(0, 1).float().double() for x in (lay.k, lay.v)]


@pytest.mark.parametrize("layout", ["paged", "hnd", "nhd"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("lens,hkv,heads,m", [([1], 1, 1, 1), ([40, 0, 17], 2, 2, 16), ([5000, 2300], 3, 3, 2100), ([700, 700], 4, 1, 333), ([3000], 8, 1, 2999)])
def test_kv_gather(td, layout, fp8, inplace, lens, hkv, heads, m):
    lay = make(lens, hkv, hkv, layout, fp8, seed=m)
    stride = max(max(lens), 1) + 1
    w = torch.rand(len(lens), heads, stride, generator=gen(2), device=DEV)
    w0 = w.clone()
    kept, cnt = td.evict_select(lay, w, m)
    want = gathered(lay, kept, cnt, heads)
    into = None if inplace else make([min(n, m) for n in lens], hkv, hkv, {"paged": "hnd", "hnd": "nhd", "nhd": "paged"}[layout], fp8, seed=1, max_len=max(min(max(lens), m), 1))
    keep = [x.clone() for x in lay.keep]
    out = None if inplace else torch.full((len(lens), heads, m + 2), 5.0, device=DEV)
    td.kv_gather(lay, kept, cnt, into=into, weights=w, weights_out=out)
    for b, n in enumerate(lens):
        c = int(cnt[b])
        got = read_rows(lay if inplace else into, b, c)
        assert torch.equal(got[0], want[b][0]) and torch.equal(got[1], want[b][1]), b
        for h in range(heads):
            assert torch.equal((w if inplace else out)[b, h, :c], w0[b, h, kept[b, h, :c].long()])
            if inplace:
                assert torch.equal(w[b, h, c:], w0[b, h, c:])
            else:
                assert (out[b, h, c:] == 5).all()
    if not inplace:
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(keep, lay.keep)) and torch.equal(w, w0)
    # without weights the rows are the same
    again = make(lens, hkv, hkv, layout, fp8, seed=m)
    td.kv_gather(again, kept, cnt, into=into)
    assert not inplace or all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(again.keep, lay.keep))
    assert td.device_status() == binding.OK


def test_kv_gather_reports_positions_and_pages_outside(td):
    lay, into = make([50], 1, 1, "paged"), make([50], 1, 1, "hnd", seed=5)
    before = into.keep[0].clone()
    td.kv_gather(lay, i32([[[3, 50, -1, 7, -9]]]), i32([5]), into=into)
    assert td.device_status() == binding.ERR_INDEX
    got = into.k[0, 0, :5]
    assert torch.equal(got[0], lay.codes[0][0][0, 3].to(torch.bfloat16)) and torch.equal(got[3], lay.codes[0][0][0, 7].to(torch.bfloat16))
    assert torch.equal(got[[1, 2, 4]], before[0, 0, [1, 2, 4], 0])
    lay.page_table[0, 2] = -3
    td.kv_gather(lay, i32([[[1, 40]]]), i32([2]), into=into)
    assert td.device_status() == binding.ERR_INDEX
    td.kv_gather(lay, i32([[[1, 40]]]), i32([2]))
    assert td.device_status() == binding.ERR_INDEX
    td.kv_gather(lay, i32([[[1, 20]]]), i32([-4]))        # counts below nothing move nothing
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads", [1, 2])
@pytest.mark.parametrize("layout,room", [("hnd", 30), ("paged", 40), ("nhd", 1)])
def test_kv_gather_reports_rows_that_find_no_room(td, fp8, heads, layout, room):
    """Lists longer than the receiving cache: what fits is moved, the rest is reported; -1 entries there are nothing."""
    lay = make([100, 100], 2, 2, "paged", fp8, seed=2)
    into = make([room, room], 2, 2, layout, fp8, seed=5, max_len=room)
    kept = torch.arange(0, 100, 2, dtype=torch.int32, device=DEV).expand(2, heads, 50).contiguous()
    td.kv_gather(lay, kept, i32([room, 0]), into=into)
    assert td.device_status() == binding.OK
    want = [read_rows(into, b, room) for b in range(2)]
    out = torch.full((2, heads, 50), 5.0, device=DEV)
    again = make([room, room], 2, 2, layout, fp8, seed=5, max_len=room)
    td.kv_gather(lay, kept, i32([50, 0]), into=again, weights=torch.ones(2, heads, 100, device=DEV), weights_out=out)
    assert td.device_status() == binding.ERR_INDEX and td.device_status() == binding.OK
    for b in range(2):
        assert all(torch.equal(x, y) for x, y in zip(read_rows(again, b, room), want[b]))
    assert (out[0, :, :room] == 1).all() and (out[0, :, room:] == 5).all() and (out[1] == 5).all()
    assert torch.equal(again.keep[0].view(torch.uint8), into.keep[0].view(torch.uint8))
    kept[:, :, room:] = -1
    td.kv_gather(lay, kept, i32([50, 50]), into=again)
    assert td.device_status() == binding.OK


def test_kv_gather_in_place_reports_lists_longer_than_their_sequence(td):
    lay = make([20, 40], 2, 2, "paged", seed=2)
    kept = torch.full((2, 2, 40), -1, dtype=torch.int32, device=DEV)
    kept[:, :, :10] = torch.arange(5, 15, device=DEV)
    td.kv_gather(lay, kept, i32([40, 40]))
    assert td.device_status() == binding.OK
    before = lay.keep[0].clone()
    kept[:] = torch.arange(40, device=DEV)
    td.kv_gather(lay, kept, i32([40, 40]))
    assert td.device_status() == binding.ERR_INDEX and td.device_status() == binding.OK
    assert torch.equal(lay.keep[0].view(torch.int16), before.view(torch.int16))       # (NaN behind the sequences)


def test_gather_takes_the_token_selection_lists(td):
    """A cache cut down to the positions that a selection layer keeps per KV head attends as the sparse layer does."""
    lay = make([3000], 8, 2, "hnd", seed=11)
    q = randn(4, 1, 8, D)
    _, idx, cnt = td.select_attn(lay, q, 256, binding.SEL_PER_KVHEAD)
    want = td.sparse_attn(lay, q, idx, cnt)
    td.kv_gather(lay, idx, cnt)
    lay.ctx_lens = cnt
    got = td.full_attn(lay, q)
    big = float(lay.dense[0][1].abs().max())
    assert float((got - want).abs().max()) <= 2 * 2.0 ** -8 * big


# ---- together, as a server uses them ---------------------------------------------------------------------------------------

class Prompts:
    """Sequences fed chunk by chunk into a paged cache: page maps, rotated and normed rows written, attention, weights, eviction."""

    def __init__(self, td, batch, hq, hkv, fp8, pages_, width, cap, budget):
        self.td, self.B, self.hq, self.hkv, self.budget = td, batch, hq, hkv, budget
        self.lay = make([1] * batch, hq, hkv, "paged", fp8, seed=1, max_len=width * BLK)
        dt = self.lay.keep[0].dtype
        pool = torch.zeros(pages_, hkv, BLK, 2, D, dtype=torch.uint8 if fp8 else dt, device=DEV)
        pool = pool.view(dt)
        self.lay.keep, self.lay.k, self.lay.v = [pool], pool[..., 0, :], pool[..., 1, :]
        self.lay.page_table = torch.full((batch, width), -1, dtype=torch.int32, device=DEV)
        self.lay.max_pages_per_seq, self.lay.num_pages = width, pages_
        self.old, self.new = i32([0] * batch), i32([0] * batch)
        self.lay.ctx_lens = self.new
        self.free, self.n_free = torch.randperm(pages_, generator=gen(3), device=DEV).to(torch.int32), i32([pages_])
        self.slots, self.pos = torch.zeros(cap, dtype=torch.int64, device=DEV), torch.zeros(cap, dtype=torch.int32, device=DEV)
        self.off = torch.zeros(batch + 1, dtype=torch.int32, device=DEV)
        self.qkv = torch.zeros(cap, hq + 2 * hkv, D, dtype=torch.bfloat16, device=DEV)
        self.q = torch.zeros(cap, hq, D, dtype=torch.bfloat16, device=DEV)
        self.out, self.lse = torch.zeros(cap, hq, D, device=DEV), torch.zeros(cap, hq, device=DEV)
        self.w = torch.zeros(batch, hkv, width * BLK, device=DEV)
        self.kept, self.left = torch.zeros(batch, hkv, budget, dtype=torch.int32, device=DEV), i32([0] * batch)
        self.qw, self.kw = 1 + 0.2 * randn(1, D), 1 + 0.2 * randn(2, D)
        self.plan = binding.rope_plan(128, base=500000.0)
        self.none = torch.zeros(0, dtype=torch.int64, device=DEV)

    def chunk(self):
        """What a step enqueues: nothing here waits for the device."""
        t, hq, hkv = self.td, self.hq, self.hkv
        t.page_map(self.old, self.new, self.lay.page_table, self.free, self.n_free, self.slots, positions=self.pos, token_offsets=self.off)
        t.rope_write(self.lay, self.plan, self.qkv[:, :hq], self.qkv[:, hq: hq + hkv], self.qkv[:, hq + hkv:], self.pos, self.slots, self.qw, self.kw, q_out=self.q)
        t.chunk_attn(self.lay, self.q, self.off, out=self.out, lse=self.lse)
        t.chunk_weights(self.lay, self.q, self.off, self.lse, self.w)

    def evict(self):
        t = self.td
        t.evict_select(self.lay, self.w, self.budget, 2, 8, self.kept, self.left)
        t.kv_gather(self.lay, self.kept, self.left, weights=self.w)
        t.page_map(self.new, self.left, self.lay.page_table, self.free, self.n_free, self.none)
        self.new.copy_(self.left)

    def rows(self, b, n):
        k, v = read_rows(self.lay, b, n)
        if self.lay.kv_dtype:
            k, v = k * self.lay.k_scale.double()[:, None, None], v * self.lay.v_scale.double()[:, None, None]
        return k, v


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("captured", [False, True])
def test_prompts_in_chunks_with_eviction(fp8, captured):
    td = binding.Tidal(0)
    s = Prompts(td, 3, 8, 2, fp8, pages_=60, width=24, cap=500, budget=64)
    graphs = {}

    def run(name, f):
        if not captured:
            return f()
        if name not in graphs:                            # the context's first calls are captured, the same graphs replayed from then on
            graphs[name] = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graphs[name]):
                f()
        graphs[name].replay()

    lens, weights = [0, 0, 0], [torch.zeros(2, 0, dtype=torch.float64, device=DEV) for _ in range(3)]
    for i, add in enumerate([[200, 1, 0], [100, 64, 7], [1, 1, 1], [50, 0, 300], [1, 1, 1]]):
        s.old.copy_(i32(lens))
        lens = [a + b for a, b in zip(lens, add)]
        s.new.copy_(i32(lens))
        s.qkv.copy_(randn(70 + i, *s.qkv.shape))
        run("chunk", s.chunk)
        torch.cuda.synchronize()
        at = 0
        for b, n in enumerate(add):                       # rotated queries against what the cache holds now
            N = lens[b]
            s.lay.dense = None
            one = copy.copy(s.lay)
            one.batch, one.max_ctx_len = 1, max(N, 1)
            one.dense = [s.rows(b, N)]
            pos = torch.arange(N - n, N, device=DEV)
            q = s.q[at: at + n]
            freq = frequencies(128, 500000.0)
            turned = ref_rope(s.qkv[at: at + n, :8], pos, freq, 1.0, HALF, s.qw, 1e-6)
            assert ((q.double() - turned).abs() <= rope_bound(turned, 512)).all() if n else True
            out, lse, w, tol_o, tol_l, tol_w = ref_chunk(one, q, [n])
            assert ((s.out[at: at + n].double() - out).abs() <= tol_o).all() and ((s.lse[at: at + n].double() - lse).abs() <= tol_l).all()
            old = torch.cat((weights[b], torch.zeros(2, n, dtype=torch.float64, device=DEV)), 1)
            weights[b] = old + (w[0, :, :N] if n else 0)
            got = s.w[b, :, :N].double()
            assert ((got - weights[b]).abs() <= 2.0 ** -9 * weights[b] + 1e-20).all()
            weights[b] = got
            at += n
        if i in (1, 3):
            before = [s.rows(b, lens[b]) for b in range(3)]
            n_free = int(s.n_free)
            run("evict", s.evict)
            torch.cuda.synchronize()
            kept, cnt = ref_evict(torch.stack([torch.nn.functional.pad(x.float(), (0, 400 - x.shape[1])) for x in weights]), lens, 64, 2, 8)
            assert torch.equal(s.kept.cpu(), kept) and s.left.tolist() == cnt.tolist()
            for b in range(3):
                c = int(cnt[b])
                k, v = s.rows(b, c)
                idx = kept[b, :, :c].long().to(DEV)
                for g in range(2):
                    assert torch.equal(k[g], before[b][0][g, idx[g]]) and torch.equal(v[g], before[b][1][g, idx[g]])
                weights[b] = torch.stack([weights[b][g, idx[g]] for g in range(2)])
                assert torch.equal(s.w[b, :, :c].double(), weights[b])
            assert int(s.n_free) == n_free + sum(pages(n) - pages(int(c)) for n, c in zip(lens, cnt))
            lens = cnt.tolist()
    assert td.device_status() == binding.OK
    graphs.clear()
    td.close()


def test_two_contexts_on_two_streams():
    a, b = binding.Tidal(0), binding.Tidal(0)
    lay = make([5000, 1234], 8, 2, "paged", seed=13)
    ins = [chunk_inputs(lay, new, i) for i, new in enumerate(([70, 300], [1, 1]))]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for _ in range(20):
        for t, st, (q, off) in zip((a, b), streams, ins):
            with torch.cuda.stream(st):
                lse = torch.zeros(q.shape[:2], device=DEV)
                out = t.chunk_attn(lay, q, off, max_new=300 if t is a else 1, lse=lse)
                outs.append((out, lse, t.chunk_weights(lay, q, off, lse, torch.zeros(2, 2, 5000, device=DEV))))
    torch.cuda.synchronize()
    for i, o in enumerate(outs):                          # the same bits every time; single tokens' parts come in any order
        for x, y in zip(o, outs[i % 2]):
            assert torch.equal(x, y) if i % 2 == 0 else float((x - y).abs().max()) <= 1e-2 * float(y.abs().max())
    for (q, off), new, i in zip(ins, ([70, 300], [1, 1]), range(2)):
        ref = ref_chunk(lay, q, new)
        assert ((outs[i][0].double() - ref[0]).abs() <= ref[3]).all()
    a.close(); b.close()


def test_many_sequences(td):
    n = 300
    lens = [(7 * i) % 90 + 1 for i in range(n)]
    new = [0 if i % 5 == 0 else 1 if i % 3 else min(lens[i], 40) for i in range(n)]
    lay = make(lens, 4, 1, "paged", seed=2)
    q, off, lse, w, tol = check_chunk(td, lay, new, max_new=0)
    got = td.chunk_weights(lay, q, off, lse, torch.zeros(n, 1, 91, device=DEV))
    assert ((got[..., :90].double() - w).abs() <= tol).all()


@pytest.mark.parametrize("seed", range(12))
def test_random_chunks(td, seed):
    r = torch.Generator().manual_seed(seed)
    pick = lambda lo, hi: int(torch.randint(lo, hi + 1, (1,), generator=r))  # noqa: E731
    hkv, g, b = pick(1, 4), pick(1, 8), pick(1, 5)
    lens = [pick(0, 1500) if pick(0, 4) else 0 for _ in range(b)]
    new = [min(n, pick(0, 300) if pick(0, 2) else 1) for n in lens]
    lay = make(lens, hkv * g, hkv, ["paged", "hnd", "nhd"][pick(0, 2)], bool(pick(0, 1)), seed=seed, max_len=max(max(lens), 1) + pick(0, 50))
    if sum(new) == 0:
        new[0] = min(1, lens[0])
    causal, window = bool(pick(0, 3)), pick(0, 1) * pick(1, 700)
    q, off, lse, w, tol = check_chunk(td, lay, new, causal, window, max_new=pick(0, 1) * max(max(new), 1), seed=seed)
    got = td.chunk_weights(lay, q, off, lse, torch.zeros(b, hkv, lay.max_ctx_len, device=DEV), causal=causal, window=window)
    assert ((got.double() - w).abs() <= tol).all()
    assert td.device_status() == binding.OK


def test_the_binding_refuses_tensors_it_cannot_take(td):
    lay = make([100], 4, 2, "hnd")
    q, off = chunk_inputs(lay, [10])
    plan, pos = binding.rope_plan(128), i32(list(range(10)))
    w, lse = torch.zeros(1, 2, 100, device=DEV), torch.zeros(10, 4, device=DEV)
    bad = [(lambda: td.chunk_attn(lay, q.float(), off), "q"), (lambda: td.chunk_attn(lay, q[:, :3], off), "q"), (lambda: td.chunk_attn(lay, q, off[:1]), "q_offsets"),
           (lambda: td.chunk_attn(lay, q, off.long()), "q_offsets"), (lambda: td.chunk_attn(lay, q, off, out=torch.zeros(10, 4, D, dtype=torch.bfloat16, device=DEV)), "out"),
           (lambda: td.chunk_attn(lay, q, off, lse=lse[:9]), "lse"), (lambda: td.chunk_attn(lay, q.cpu(), off), "q"), (lambda: td.chunk_attn(lay, q.transpose(0, 1), off), "q"),
           (lambda: td.chunk_weights(lay, q, off, lse, w[0]), "weights"), (lambda: td.chunk_weights(lay, q, off, lse, w.double()), "weights"),
           (lambda: td.rope(plan, q, None, pos[:9]), "positions"), (lambda: td.rope(plan, q, None, pos, q_out=q[:5]), "q_out"), (lambda: td.rope(plan, q[..., :64], None, pos), "q"),
           (lambda: td.rope(plan, q, q[:5], pos), "k"), (lambda: td.rope_write(lay, plan, q, q, q, pos, torch.zeros(10, dtype=torch.int64, device=DEV)), "k_new"),
           (lambda: td.evict_select(lay, w, 4, kept=torch.zeros(1, 2, 5, dtype=torch.int32, device=DEV)), "kept"),
           (lambda: td.kv_gather(lay, torch.zeros(2, 2, 5, dtype=torch.int32, device=DEV), i32([1])), "kept"),
           (lambda: td.kv_gather(lay, torch.zeros(1, 2, 5, dtype=torch.int32, device=DEV), i32([1]), weights=w[:, :1].contiguous()), "weights")]
    for f, name in bad:
        with pytest.raises(ValueError, match=name):
            f()
    for f in (lambda: td.chunk_weights(lay, q, off, lse, torch.zeros(1, 3, 100, device=DEV)), lambda: td.chunk_attn(lay, q, off, window=-1),
              lambda: td.evict_select(lay, w[..., :50].contiguous(), 4), lambda: td.evict_select(lay, w, 0), lambda: td.rope(plan, q, None, pos, eps=-1.0)):
        with pytest.raises(binding.TidalError) as e:
            f()
        assert e.value.status == binding.ERR_INVALID
    closed = binding.Tidal(0)
    closed.close()
    with pytest.raises(binding.TidalError):
        closed.chunk_attn(lay, q, off)
    empty = td.chunk_attn(lay, q[:0], i32([0, 0]))
    assert empty.shape == (0, 4, D)
    td.rope(plan, q[:0], None, pos[:0])
