"""Argument errors of the prompt calls, found on the host before anything touches a device, and the frequencies of rotary positions:
the calls get a block of zeros for a context, which an accepted call could not use."""
import ctypes as C
import math

import pytest

from paper_2410_05076_b200 import binding
from tests.test_blocks_abi import CTX, INV, P, UNS, contiguous, kv

HALF, INTER = binding.ROPE_HALF, binding.ROPE_INTERLEAVED


def plan(**over):
    p = binding.tidal_rope_t()
    p.rotary_dim, p.layout, p.scale = 128, HALF, 1.0
    for k, v in over.items():
        setattr(p, k, v)
    return p


def call(name, defaults, over):
    args = dict(defaults)
    args.update(over)
    args = [C.byref(v) if isinstance(v, C.Structure) else v for v in args.values()]
    return getattr(binding.load(), name)(*args, None)


Q, K = 8 * 128, 2 * 128
ROPE = dict(ctx=CTX, rope=plan(), T=4, hq=8, hkv=2, q=P, qs=Q, k=P, ks=K, pos=P, qw=None, kw=None, eps=1e-6, qo=P, qos=Q, ko=P, kos=K)
WRITE = dict(ctx=CTX, rope=plan(), kv=kv(), T=4, q=P, qs=Q, k=P, ks=K, v=P, vs=K, pos=P, slots=P, qw=None, kw=None, eps=1e-6, qo=P, qos=Q)
CHUNK = dict(ctx=CTX, kv=kv(), T=4, q=P, qs=Q, off=P, max_new=0, causal=1, window=0, out=P, lse=None)
WEIGHTS = dict(ctx=CTX, kv=kv(), T=4, q=P, qs=Q, off=P, max_new=0, causal=1, window=0, last=0, lse=P, decay=1.0, w=P, stride=1024, heads=2)
SELECT = dict(ctx=CTX, kv=kv(), w=P, stride=1024, heads=2, m=4, first=0, last=0, kept=P, lens=2 * P)
GATHER = dict(ctx=CTX, kv=kv(), into=None, kept=P, counts=P, m=4, heads=2, w=None, stride=0, wo=None, stride_out=0)


@pytest.mark.parametrize("over,status", [
    (dict(ctx=None), INV), (dict(rope=None), INV), (dict(rope=plan(rotary_dim=0)), INV), (dict(rope=plan(rotary_dim=130)), INV), (dict(rope=plan(rotary_dim=24)), INV),
    (dict(rope=plan(layout=2)), INV), (dict(T=-1), INV), (dict(hq=-1), INV), (dict(hq=0), INV), (dict(hq=0, hkv=0, q=None, k=None, qo=None, ko=None), INV),
    (dict(q=None), INV), (dict(q=P + 8), INV), (dict(qs=Q + 4), INV), (dict(qs=Q - 8), INV), (dict(ks=K - 8), INV), (dict(k=None), INV), (dict(pos=None), INV),
    (dict(qw=P + 2), INV), (dict(kw=P + 8), INV), (dict(eps=-1.0), INV), (dict(eps=math.nan), INV), (dict(eps=math.inf), INV), (dict(qo=None), INV), (dict(ko=P + 4), INV),
    (dict(qos=0), INV), (dict(kos=8), INV), (dict(qos=Q + 8), INV), (dict(hq=70000, qs=70000 * 128, qos=70000 * 128), UNS), (dict(T=0, q=None, pos=None), binding.OK),
])
def test_rope_refusals(over, status):
    assert call("tidal_rope", ROPE, over) == status


@pytest.mark.parametrize("over,status", [
    (dict(ctx=None), INV), (dict(rope=None), INV), (dict(kv=kv(head_dim=64)), UNS), (dict(T=-1), INV), (dict(k=None), INV), (dict(v=None), INV), (dict(slots=None), INV),
    (dict(pos=None), INV), (dict(q=None), INV), (dict(qo=None), INV), (dict(k=P + 8), INV), (dict(vs=K - 8), INV), (dict(ks=K + 1), INV), (dict(qos=Q + 8), INV),
    (dict(eps=-1.0), INV), (dict(T=0, k=None), binding.OK),
])
def test_rope_write_refusals(over, status):
    assert call("tidal_rope_write", WRITE, over) == status


@pytest.mark.parametrize("over,status", [
    (dict(ctx=None), INV), (dict(T=-1), INV), (dict(q=None), INV), (dict(q=P + 8), INV), (dict(qs=Q + 4), INV), (dict(qs=Q - 8), INV), (dict(off=None), INV),
    (dict(max_new=-1), INV), (dict(window=-1), INV), (dict(out=None), INV), (dict(out=P + 8), INV), (dict(lse=P + 2), INV), (dict(kv=kv(page_size=32)), UNS),
    (dict(kv=kv(num_q_heads=18)), UNS), (dict(kv=kv(sm_scale=-1.0)), INV), (dict(kv=kv(stride_page=1 << 40)), UNS), (dict(kv=contiguous(stride_pos=1 << 39)), UNS),
    (dict(kv=kv(stride_pos=64)), INV), (dict(qs=1 << 39), UNS), (dict(T=0, q=None), binding.OK),
])
def test_chunk_attn_refusals(over, status):
    assert call("tidal_chunk_attn", CHUNK, over) == status


@pytest.mark.parametrize("over,status", [
    (dict(ctx=None), INV), (dict(T=-1), INV), (dict(q=None), INV), (dict(off=None), INV), (dict(lse=None), INV), (dict(lse=P + 1), INV), (dict(w=None), INV),
    (dict(w=P + 2), INV), (dict(stride=1023), INV), (dict(heads=8), INV), (dict(heads=0), INV), (dict(last=-1), INV), (dict(decay=math.nan), INV), (dict(decay=math.inf), INV),
    (dict(window=-3), INV), (dict(T=0, q=None, lse=None), binding.OK),
])
def test_chunk_weights_refusals(over, status):
    assert call("tidal_chunk_weights", WEIGHTS, over) == status


@pytest.mark.parametrize("over,status", [
    (dict(ctx=None), INV), (dict(w=None), INV), (dict(stride=1000), INV), (dict(heads=8), INV), (dict(m=0), INV), (dict(m=262145), INV), (dict(first=-1), INV),
    (dict(last=-1), INV), (dict(kept=None), INV), (dict(lens=None), INV), (dict(lens=P), INV), (dict(kv=kv(max_ctx_len=0)), INV),
])
def test_evict_select_refusals(over, status):
    assert call("tidal_evict_select", SELECT, over) == status


@pytest.mark.parametrize("over,status", [
    (dict(ctx=None), INV), (dict(kept=None), INV), (dict(counts=None), INV), (dict(m=0), INV), (dict(heads=8), INV), (dict(into=kv(batch=3)), INV),
    (dict(into=kv(num_kv_heads=4)), INV), (dict(into=kv(kv_dtype=1)), INV), (dict(w=P, stride=1024), INV), (dict(w=P, stride=1000, wo=P, stride_out=1024), INV),
    (dict(w=P, stride=1024, wo=P, stride_out=2048), INV), (dict(into=kv(), w=P, stride=1024, wo=P, stride_out=1024), INV),
    (dict(w=P, stride=1024, wo=2 * P, stride_out=3), INV), (dict(w=P + 2, stride=1024, wo=2 * P, stride_out=8), INV), (dict(m=262145), INV),
])
def test_kv_gather_refusals(over, status):
    assert call("tidal_kv_gather", GATHER, over) == status


def test_rope_plans_refuse():
    for over, status in ((dict(rotary_dim=0), INV), (dict(rotary_dim=20), UNS), (dict(rotary_dim=144), UNS), (dict(base=1.0), INV), (dict(base=math.nan), INV),
                         (dict(layout=2), INV), (dict(scaling=5), INV), (dict(scaling=1, factor=0.5), INV), (dict(scaling=3, factor=2.0, low=0.0), INV),
                         (dict(scaling=4, factor=2.0, low=4.0, high=2.0), INV), (dict(scaling=3, factor=2.0, trained_len=0.0), INV),
                         (dict(inv_freq=[math.inf] * 64), INV), (dict(inv_freq=[1.0] * 64, cos_scale=math.nan), INV)):
        with pytest.raises(binding.TidalError) as e:
            binding.rope_plan(**over)
        assert e.value.status == status, over
    with pytest.raises(ValueError, match="64 frequencies"):
        binding.rope_plan(128, inv_freq=[1.0])


def turns(p):
    return [p.step[i] * 2.0 ** -64 * 2 * math.pi for i in range(p.rotary_dim // 2)]


@pytest.mark.parametrize("n,base", [(128, 10000.0), (64, 500000.0), (16, 1e6), (96, 12345.6)])
def test_rope_frequencies(n, base):
    f = [base ** (-2 * i / n) for i in range(n // 2)]
    near = lambda got, want: all(abs(a - b) <= 1e-15 + 1e-14 * b for a, b in zip(got, want))  # noqa: E731
    assert near(turns(binding.rope_plan(n, base)), f)
    assert near(turns(binding.rope_plan(n, base, scaling=binding.ROPE_LINEAR, factor=4.0)), [x / 4 for x in f])
    wide = base * 8.0 ** (n / (n - 2))
    assert near(turns(binding.rope_plan(n, base, scaling=binding.ROPE_BASE, factor=8.0)), [wide ** (-2 * i / n) for i in range(n // 2)])
    # stretched by wavelength: three ranges
    L, factor, low, high = 8192.0, 8.0, 1.0, 4.0
    want = []
    for x in f:
        wavelength = 2 * math.pi / x
        if wavelength < L / high:
            want.append(x)
        elif wavelength > L / low:
            want.append(x / factor)
        else:
            s = (L / wavelength - low) / (high - low)
            want.append((1 - s) * x / factor + s * x)
    p = binding.rope_plan(n, base, scaling=binding.ROPE_BANDS, factor=factor, low=low, high=high, trained_len=L)
    assert near(turns(p), want) and p.scale == 1.0
    # a ramp over the channels
    at = lambda t: n * math.log(4096 / (t * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
    lo, hi = max(math.floor(at(32)), 0), min(math.ceil(at(1)), n - 1)
    ramp = [min(max((i - lo) / max(hi - lo, 1e-3), 0), 1) for i in range(n // 2)]
    p = binding.rope_plan(n, base, INTER, binding.ROPE_RAMP, 16.0, 1.0, 32.0, 4096.0)
    assert near(turns(p), [x / 16 * r + x * (1 - r) for x, r in zip(f, ramp)])
    assert p.layout == INTER and abs(p.scale - (0.1 * math.log(16) + 1)) <= 2.0 ** -23
    assert near(turns(binding.rope_plan(n, inv_freq=f, cos_scale=0.5)), f) and binding.rope_plan(n, inv_freq=f, cos_scale=0.5).scale == 0.5


def test_rope_steps_hold_far_positions():
    """A turn's fraction in 64 bits: the product with position 2^31 - 1 is off by less than 2^-32 of a turn."""
    from fractions import Fraction
    two_pi = Fraction(62831853071795864769252867665590057683943387987502, 10 ** 49)
    p = binding.rope_plan(128, inv_freq=[0.1 ** (i / 9) for i in range(64)])
    for i in range(64):
        exact = Fraction(0.1 ** (i / 9)) / two_pi
        off = (Fraction(int(p.step[i]), 2 ** 64) - exact) * (2 ** 31 - 1)
        assert abs(off - round(off)) < Fraction(1, 2 ** 32)


def test_a_closed_context_and_wrong_tensors_are_refused():
    td = binding.Tidal.__new__(binding.Tidal)
    td.lib, td.ctx, td.device, td.out_dtype = binding.load(), C.c_void_p(), 0, None
    with pytest.raises(ValueError, match="slots"):
        td.rope_write(kv(), plan(), None, None, None, None, None)
    with pytest.raises(ValueError, match="plan"):
        td.rope(kv(), None, None, None)
    with pytest.raises(ValueError, match="q, k"):
        td.rope(plan(), None, None, None)
    with pytest.raises(ValueError, match="kept"):
        td.kv_gather(kv(), None, None)
