"""Block-sparse decode attention and the paged cache's page maps and writes, against plain definitions in 64 bits."""
import math

import pytest
import torch

from paper_2410_05076_b200 import binding, synth
from tests import util

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D, BLK = 128, 16
GRANS = [binding.SEL_PER_QHEAD, binding.SEL_PER_KVHEAD, binding.SEL_SHARED]


@pytest.fixture(scope="module")
def td():
    t = binding.Tidal(0)
    yield t
    assert t.device_status() == binding.OK
    t.close()


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def pages(n):
    return -(-n // BLK)


def make(lens, hq, hkv, layout="paged", fp8=False, seed=0, spoil=True, max_len=None, sm_scale=0.0):
    """A cache with those lengths. Everything that is not a cached position holds NaN (spoil)."""
    g = gen(seed)
    B, N = len(lens), max_len or max(max(lens), 1)
    nb = pages(N)
    dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
    nan = 0x7F if fp8 else float("nan")

    def noise(*shape):
        x = torch.randn(*shape, generator=g, device=DEV)
        x[..., 5] += 3.0                                  # a channel off centre
        return (x * (16.0 if fp8 else 1.0)).clamp(-448, 448).to(dt)

    def blank(*shape):
        t = torch.zeros(*shape, dtype=dt, device=DEV)
        if spoil:
            (t.view(torch.uint8) if fp8 else t).fill_(nan)
        return t

    common = dict(batch=B, num_q_heads=hq, num_kv_heads=hkv, head_dim=D, ctx_lens=torch.tensor(lens, dtype=torch.int32, device=DEV),
                  max_ctx_len=N, sm_scale=sm_scale, kv_dtype=int(fp8))
    if fp8:
        common["k_scale"] = 0.03 + 0.05 * torch.rand(hkv, generator=g, device=DEV)
        common["v_scale"] = 0.03 + 0.05 * torch.rand(hkv, generator=g, device=DEV)
    raw = (lambda t: t.view(torch.uint8)) if fp8 else (lambda t: t)
    ks, vs = [noise(hkv, n, D) for n in lens], [noise(hkv, n, D) for n in lens]
    if layout == "paged":
        total = sum(map(pages, lens)) + 4
        pool = blank(total, hkv, BLK, 2, D)
        table = torch.full((B, nb + 1), -7, dtype=torch.int32, device=DEV)   # entries behind a sequence are no pages
        perm = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
        at = 0
        for b, n in enumerate(lens):
            table[b, : pages(n)] = perm[at: at + pages(n)]
            at += pages(n)
            pos = torch.arange(n, device=DEV)
            for i, rows in ((0, ks[b]), (1, vs[b])):
                raw(pool)[table[b, pos // BLK].long(), :, pos % BLK, i] = raw(rows).transpose(0, 1)
        lay = synth.LayerKV(k=pool[..., 0, :], v=pool[..., 1, :], stride_pos=2 * D, stride_head=BLK * 2 * D,
                            stride_page=hkv * BLK * 2 * D, page_table=table, max_pages_per_seq=nb + 1, keep=[pool], **common)
        lay.num_pages = total
    elif layout == "hnd":
        buf = blank(B, hkv, N, 2, D)
        for b, n in enumerate(lens):
            raw(buf)[b, :, :n, 0], raw(buf)[b, :, :n, 1] = raw(ks[b]), raw(vs[b])
        lay = synth.LayerKV(k=buf[..., 0, :], v=buf[..., 1, :], stride_b=hkv * N * 2 * D, stride_pos=2 * D, stride_head=N * 2 * D,
                            keep=[buf], **common)
    else:                                                 # separate K and V, heads inside positions
        kb, vb = blank(B, N, hkv, D), blank(B, N, hkv, D)
        for b, n in enumerate(lens):
            raw(kb)[b, :n], raw(vb)[b, :n] = raw(ks[b]).transpose(0, 1), raw(vs[b]).transpose(0, 1)
        lay = synth.LayerKV(k=kb, v=vb, stride_b=N * hkv * D, stride_pos=hkv * D, stride_head=D, keep=[kb, vb], **common)
    lay.codes = [(k.float().double(), v.float().double()) for k, v in zip(ks, vs)]       # without the scales
    one = torch.ones(hkv, device=DEV)
    sk, sv = (x.double()[:, None, None] for x in ((lay.k_scale, lay.v_scale) if fp8 else (one, one)))
    lay.dense = [(k * sk, v * sv) for k, v in lay.codes]
    return lay


def query(lay, seed):
    return torch.randn(lay.batch, lay.num_q_heads, D, generator=gen(900 + seed), device=DEV).to(torch.bfloat16)


# ---- definitions in 64 bits ----------------------------------------------------------------------------------------

def ref_bounds(lay, b):
    """[Hkv, blocks, 2, 128] of sequence b."""
    keys = lay.codes[b][0]
    return torch.stack([torch.stack((r.amin(1), r.amax(1)), 1) for r in keys.split(BLK, 1)], 1) if keys.shape[1] else None


def bounds_at(lay, bounds, b, blk):
    return bounds[int(lay.page_table[b, blk])] if lay.paged else bounds[b, :, blk]


def index_heads(lay, gran):
    return {0: lay.num_q_heads, 1: lay.num_kv_heads, 2: 1}[gran]


def ref_select(lay, q, m, gran, first, last):
    hi, hq, G = index_heads(lay, gran), lay.num_q_heads, lay.num_q_heads // lay.num_kv_heads
    idx = torch.full((lay.batch, hi, m), -1, dtype=torch.int32)
    cnt = torch.zeros(lay.batch, dtype=torch.int32)
    for b in range(lay.batch):
        bd = ref_bounds(lay, b)
        if bd is None:
            continue
        n = bd.shape[1]
        s = torch.zeros(hi, n, dtype=torch.float64, device=DEV)
        for h in range(hq):
            g = h // G
            one = torch.maximum(q[b, h].double() * bd[g, :, 0], q[b, h].double() * bd[g, :, 1]).sum(-1)
            s[h * hi // hq] += one * (lay.k_scale[g].double() if lay.kv_dtype and gran == 2 else 1.0)
        blk = torch.arange(n, device=DEV)
        s[:, (blk < first) | (blk >= n - last)] = math.inf
        c = min(m, n)
        idx[b, :, :c] = torch.sort(s, dim=-1, descending=True, stable=True).indices[:, :c].sort(-1).values.cpu()
        cnt[b] = c
    return idx, cnt


def ref_attn(lay, q, idx, cnt=None):
    """(out, tolerance) in 64 bits. Tolerance: the 16 matrix instructions of a logit add exact products with at most 2^-22 of the
    sum of their magnitudes each, 2^-18 together; the exponent's argument is rounded to fp32 (2^-24 of |t| log2 e, twice) and
    ex2.approx gives 2^-22; a weight enters the second product with 2^-22 (two fp16, each off by at most 2^-11, or three bf16, 2^-8 each) and its up to
    n / 16 instructions add 2^-22 each. An error r of the weights moves a weighted mean of v by at most 2 r max|v|."""
    B, hi = idx.shape[:2]
    hq, G = lay.num_q_heads, lay.num_q_heads // lay.num_kv_heads
    scale = lay.sm_scale or 1 / math.sqrt(D)
    out = torch.zeros(B, hq, D, dtype=torch.float64, device=DEV)
    tol = torch.zeros(B, hq, 1, dtype=torch.float64, device=DEV)
    for b in range(B):
        k, v = lay.dense[b]
        n = k.shape[1]
        for h in range(hq):
            row = idx[b, h * hi // hq].long().to(DEV)
            if cnt is not None:
                row = row[: max(int(cnt[b]), 0)]
            row = row[(row >= 0) & (row * BLK < n)]
            pos = (row[:, None] * BLK + torch.arange(BLK, device=DEV)).flatten()
            pos = pos[pos < n]
            if pos.numel() == 0:
                continue
            kk, vv, qq = k[h // G, pos], v[h // G, pos], q[b, h].double()
            t = (kk @ qq) * scale
            out[b, h] = torch.softmax(t, 0) @ vv
            r = 2.0 ** -18 * float((kk.abs() @ qq.abs()).max()) * scale + 2.0 ** -22 * float(t.abs().max()) + 2.0 ** -22 + 2.0 ** -22 * (2 + row.numel())
            tol[b, h] = 2 * r * float(vv.abs().max())
    return out, tol


def close(got, ref, tol, what, bf16=False):
    err = (got.double() - ref).abs()
    if bf16:
        tol = tol + 2.0 ** -8 * (ref.abs() + tol)         # a rounding to bf16: half a step, eps / 2 = 2^-8 of the value
    assert torch.isfinite(got.float()).all(), f"{what}: not finite"
    assert (err <= tol).all(), f"{what}: {float((err - tol).max()):.3e} over the bound, max error {float(err.max()):.3e}"


# ---- key bounds ----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("layout", ["paged", "hnd", "nhd"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,hkv", [([1], 1), ([16, 0, 17, 300], 3), ([15, 31, 32, 1000, 5], 8)])
def test_bounds(td, layout, fp8, lens, hkv):
    lay = make(lens, 2 * hkv, hkv, layout, fp8, seed=len(lens))
    guard = util.Guarded(binding.block_bounds_shape(lay), torch.bfloat16, DEV, fill=123.0)
    out = td.block_bounds(lay, guard.t)
    assert out is guard.t
    seen = torch.zeros(out.shape[:1] if lay.paged else (lay.batch, out.shape[2]), dtype=torch.bool)
    for b in range(lay.batch):
        ref = ref_bounds(lay, b)
        for i in range(pages(lens[b])):
            assert torch.equal(bounds_at(lay, out, b, i).double(), ref[:, i]), (b, i)
            seen[int(lay.page_table[b, i]) if lay.paged else (b, i)] = True
    rest = out[~seen.to(DEV)] if lay.paged else out.transpose(1, 2)[~seen.to(DEV)]
    assert (rest == 123.0).all()                          # blocks that no sequence has are left alone
    guard.check("bounds")
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("layout", ["paged", "hnd"])
@pytest.mark.parametrize("old,new", [([0, 3, 16, 31, 32, 40], [1, 4, 17, 32, 33, 40]), ([0, 15, 16, 17, 100, 64], [50, 66, 16, 67, 151, 115])])
def test_bounds_after_an_append_touch_only_the_new_blocks(td, layout, old, new):
    lay = make(new, 4, 2, layout, seed=3)
    out = torch.full(binding.block_bounds_shape(lay), 55.0, dtype=torch.bfloat16, device=DEV)
    start = torch.tensor(old, dtype=torch.int32, device=DEV)
    more = max(n - o for o, n in zip(old, new))
    for max_new in (more, 0):                             # a bound on the new tokens, or none
        out.fill_(55.0)
        td.block_bounds(lay, out, start_lens=start, max_new=max_new)
        for b in range(len(new)):
            ref = ref_bounds(lay, b)
            for i in range(pages(new[b])):
                got = bounds_at(lay, out, b, i).double()
                if i >= old[b] // BLK:
                    assert torch.equal(got, ref[:, i]), (b, i)
                else:
                    assert (got == 55.0).all(), (b, i)


def test_bounds_carry_nan_and_infinities_of_cached_keys(td):
    lay = make([40], 2, 1, "hnd", seed=4)
    lay.k[0, 0, 3, 7] = float("nan")
    lay.k[0, 0, 20, 9] = float("inf")
    lay.k[0, 0, 21, 9] = float("-inf")
    out = td.block_bounds(lay)
    assert out[0, 0, 0, :, 7].isnan().all() and not out[0, 0, 0, :, :7].isnan().any()
    assert out[0, 0, 1, 0, 9] == -math.inf and out[0, 0, 1, 1, 9] == math.inf


# ---- selection -----------------------------------------------------------------------------------------------------

SELECT = [
    # lens, hq, hkv, m, first, last
    ([1], 2, 1, 1, 0, 0),
    ([5], 4, 4, 3, 1, 1),
    ([256], 8, 2, 4, 0, 1),
    ([0, 17, 700, 16], 8, 2, 7, 1, 2),
    ([4096], 8, 2, 16, 0, 0),
    ([999, 2047, 33], 15, 3, 31, 3, 0),
    ([1500], 8, 1, 90, 0, 3),
    ([3000, 64], 8, 8, 5, 7, 7),                          # more kept blocks than m
    ([20000], 4, 1, 100, 0, 1),
    ([90000, 17, 0, 33333], 8, 2, 70, 2, 1),
    ([16400, 16385, 70001], 12, 3, 1025, 0, 0),
    ([170000], 2, 2, 33, 1, 1),
]


@pytest.mark.parametrize("layout,fp8", [("paged", False), ("hnd", True)])
@pytest.mark.parametrize("gran", GRANS)
@pytest.mark.parametrize("lens,hq,hkv,m,first,last", SELECT)
def test_select_gives_the_set_of_the_scores_in_64_bits(td, layout, fp8, gran, lens, hq, hkv, m, first, last):
    lay = make(lens, hq, hkv, layout, fp8, seed=m)
    q = query(lay, m)
    bounds = td.block_bounds(lay)
    hi = index_heads(lay, gran)
    gi, gc = util.Guarded((len(lens), hi, m), torch.int32, DEV, fill=77), util.Guarded((len(lens),), torch.int32, DEV, fill=77)
    idx, cnt = td.block_select(lay, bounds, q, m, gran, keep_first=first, keep_last=last, idx=gi.t, idx_count=gc.t)
    ref, ref_cnt = ref_select(lay, q, m, gran, first, last)
    assert torch.equal(cnt.cpu(), ref_cnt)
    assert torch.equal(idx.cpu(), ref)
    gi.check("idx"); gc.check("idx_count")
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("kind", ["equal", "zero", "few_values", "one_outlier", "near_ties", "nan"])
@pytest.mark.parametrize("ctx", [3000, 50000, 80000, 200000])
def test_select_with_ties_and_ranges_that_collapse(td, kind, ctx):
    """Rows whose border falls among many equal or almost equal scores: the histogram's bin holds most of the row."""
    lay = make([ctx], 4, 2, "hnd", seed=9)
    n = pages(ctx)
    q = query(lay, 5)
    bounds = torch.zeros(1, 2, n, 2, D, dtype=torch.bfloat16, device=DEV)
    g = gen(11)
    if kind == "equal":
        bounds[:] = torch.randn(1, 2, 1, 2, D, generator=g, device=DEV).sort(-2).values.to(torch.bfloat16)
    elif kind == "few_values":
        bounds[:] = torch.randn(1, 2, 5, 2, D, generator=g, device=DEV).sort(-2).values.to(torch.bfloat16)[:, :, torch.randint(0, 5, (n,), generator=g, device=DEV)]
    elif kind == "one_outlier":
        bounds[:] = torch.randn(1, 2, n, 2, D, generator=g, device=DEV).sort(-2).values.to(torch.bfloat16)
        bounds[:, :, n // 2] *= 1e4
    elif kind == "near_ties":                             # equal but for one small channel
        bounds[:] = torch.randn(1, 2, 1, 2, D, generator=g, device=DEV).sort(-2).values.to(torch.bfloat16)
        bounds[..., 1, 17] = (1.0 + torch.randint(0, 60, (1, 2, n), generator=g, device=DEV) / 128.0).to(torch.bfloat16) * 2.0 ** -20
        bounds[..., 0, 17] = 0.0
    elif kind == "nan":
        bounds[:] = torch.randn(1, 2, n, 2, D, generator=g, device=DEV).sort(-2).values.to(torch.bfloat16)
        bounds[:, :, 5, 0, 3] = float("nan")
    s = torch.maximum(q.double().view(1, 2, 2, 1, D) * bounds[:, :, None, :, 0].double(),
                      q.double().view(1, 2, 2, 1, D) * bounds[:, :, None, :, 1].double()).sum(-1)      # [1, Hkv, G, n]
    for gran, score in ((0, s.reshape(1, 4, n)), (1, s.sum(2)), (2, s.sum((1, 2))[:, None])):
        for m in (1, 37, n // 2, n - 1):
            idx, _ = td.block_select(lay, bounds, q, m, gran)
            if kind == "nan":                             # an unspecified set, but a well-formed one
                got = idx.cpu()
                assert (got[..., 1:] > got[..., :-1]).all() and (got >= 0).all() and (got < n).all()
            else:
                ref = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :m].sort(-1).values
                assert torch.equal(idx.long(), ref), (gran, m)


@pytest.mark.parametrize("gran", GRANS)
@pytest.mark.parametrize("batch,hq,hkv,lo,hi,m", [
    (45, 32, 32, 0, 85, 3), (40, 16, 2, 900, 3000, 20), (24, 32, 4, 2000, 6000, 40), (40, 8, 1, 16, 1024, 9),
    (3, 64, 8, 17, 573, 4), (2, 32, 32, 1000, 3000, 33), (1, 40, 5, 16000, 16000, 300), (2, 30, 30, 1025, 4111, 60)])
def test_select_of_many_items_and_many_heads(td, gran, batch, hq, hkv, lo, hi, m):
    """A warp per row, a cluster per item, the KV heads of a shared set spread over warps."""
    lens = [hi - (hi - lo) * i // max(batch - 1, 1) for i in range(batch)]
    lay = make(lens, hq, hkv, "paged" if batch % 2 else "hnd", False, seed=batch)
    q = query(lay, m)
    gi = util.Guarded((batch, index_heads(lay, gran), m), torch.int32, DEV, fill=77)
    idx, cnt = td.block_select(lay, td.block_bounds(lay), q, m, gran, keep_first=1, keep_last=1, idx=gi.t)
    ref, ref_cnt = ref_select(lay, q, m, gran, 1, 1)
    assert torch.equal(cnt.cpu(), ref_cnt)
    assert torch.equal(idx.cpu(), ref)
    gi.check("idx")
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("kind", ["equal", "zero", "few_values", "near_ties", "nan"])
@pytest.mark.parametrize("batch,hq,hkv,ctx", [(1, 8, 2, 1000), (3, 4, 1, 130), (24, 16, 2, 3000), (24, 16, 2, 6000), (1, 24, 12, 1000)])
def test_select_with_ties_in_rows_ranked_by_a_warp(td, kind, batch, hq, hkv, ctx):
    lay = make([ctx] * batch, hq, hkv, "hnd", seed=9)
    n, G = pages(ctx), hq // hkv
    q, g = query(lay, 5), gen(12)
    rand = lambda *shape: torch.randn(*shape, 2, D, generator=g, device=DEV).sort(-2).values.to(torch.bfloat16)  # noqa: E731
    if kind == "zero":
        bounds = torch.zeros(batch, hkv, n, 2, D, dtype=torch.bfloat16, device=DEV)
    elif kind == "few_values":
        bounds = rand(batch, hkv, 3)[:, :, torch.randint(0, 3, (n,), generator=g, device=DEV)].contiguous()
    elif kind == "nan":
        bounds = rand(batch, hkv, n)
        bounds[:, :, 5, 0, 3] = float("nan")
    else:
        bounds = rand(batch, hkv, 1).expand(batch, hkv, n, 2, D).contiguous()
        if kind == "near_ties":                           # equal but for one small channel
            bounds[..., 1, 17] = (1.0 + torch.randint(0, 60, (batch, hkv, n), generator=g, device=DEV) / 128.0).to(torch.bfloat16) * 2.0 ** -20
            bounds[..., 0, 17] = 0.0
    s = torch.maximum(q.double().view(batch, hkv, G, 1, D) * bounds[:, :, None, :, 0].double(),
                      q.double().view(batch, hkv, G, 1, D) * bounds[:, :, None, :, 1].double()).sum(-1)      # [B, Hkv, G, n]
    for gran, score in ((0, s.reshape(batch, hq, n)), (1, s.sum(2)), (2, s.sum((1, 2))[:, None])):
        for m in (1, n // 2, n - 1):
            idx, _ = td.block_select(lay, bounds, q, m, gran)
            if kind == "nan":                             # an unspecified set, but a well-formed one
                got = idx.cpu()
                assert (got[..., 1:] > got[..., :-1]).all() and (got >= 0).all() and (got < n).all()
            else:
                ref = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :m].sort(-1).values
                assert torch.equal(idx.long(), ref), (gran, m)


@pytest.mark.parametrize("ctx", [900, 3000, 40000])
def test_select_with_the_smallest_and_largest_numbers(td, ctx):
    """Subnormal and huge bounds: what is decided in 64 bits is decided there exactly."""
    lay = make([ctx], 4, 2, "hnd", seed=3)
    n, g = pages(ctx), gen(13)
    for scale in (2.0 ** -126, 2.0 ** -133, 2.0 ** 60):
        q = (torch.randint(-3, 4, (1, 4, D), generator=g, device=DEV).double() * (1.0 if scale < 1 else 2.0 ** 20)).to(torch.bfloat16)
        bounds = (torch.randint(-8, 9, (1, 2, n, 2, D), generator=g, device=DEV).sort(-2).values.double() * scale).to(torch.bfloat16)
        assert torch.equal(bounds.double() / scale, (bounds.double() / scale).round())      # (nothing was rounded away)
        s = torch.maximum(q.double().view(1, 2, 2, 1, D) * bounds[:, :, None, :, 0].double(),
                          q.double().view(1, 2, 2, 1, D) * bounds[:, :, None, :, 1].double()).sum(-1)
        for gran, score in ((0, s.reshape(1, 4, n)), (1, s.sum(2)), (2, s.sum((1, 2))[:, None])):
            idx, _ = td.block_select(lay, bounds, q, 11, gran)
            ref = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :11].sort(-1).values
            assert torch.equal(idx.long(), ref), (scale, gran)


def test_select_with_a_query_that_is_not_finite(td):
    for ctx in (3000, 60000):
        lay = make([ctx], 4, 2, "hnd", seed=7)
        q, n = query(lay, 7), pages(ctx)
        q[0, 1, 5] = float("nan")
        q[0, 2, 9] = float("inf")
        for gran in GRANS:
            idx, _ = td.block_select(lay, td.block_bounds(lay), q, 9, gran, keep_last=1)
            got = idx.cpu()
            assert (got[..., 1:] > got[..., :-1]).all() and (got >= 0).all() and (got < n).all() and (got[..., -1] == n - 1).all()
        ok, _ = td.block_select(lay, td.block_bounds(lay), q, 9, 0, keep_last=1)
        fine = query(lay, 7)                              # the heads without one keep their sets
        ref = ref_select(lay, fine, 9, 0, 0, 1)[0]
        assert torch.equal(ok.cpu()[0, 0], ref[0, 0]) and torch.equal(ok.cpu()[0, 3], ref[0, 3])


def test_pages_shared_by_sequences(td):
    """A common prefix of full pages: one set of bounds serves both."""
    lay = make([100, 70], 4, 2, "paged", seed=14)
    lay.page_table[1, :4] = lay.page_table[0, :4]
    lay.codes[1] = tuple(torch.cat((a[:, :64], b[:, 64:]), 1) for a, b in zip(lay.codes[0], lay.codes[1]))
    lay.dense[1] = lay.codes[1]
    q = query(lay, 14)
    idx, cnt = td.block_select(lay, td.block_bounds(lay), q, 3, 1)
    assert torch.equal(idx.cpu(), ref_select(lay, q, 3, 1, 0, 0)[0])
    ref, tol = ref_attn(lay, q, idx.cpu())
    close(td.block_attn(lay, q, idx, cnt), ref, tol, "shared pages")


def test_a_closed_context_refuses(td):
    t = binding.Tidal(0)
    lay = make([40], 2, 1, "hnd", seed=0)
    t.close()
    with pytest.raises(binding.TidalError) as e:
        t.block_bounds(lay)
    assert e.value.status == binding.ERR_INVALID


def test_select_score_is_a_bound_that_keeps_the_best_block(td):
    """With one block per head, it holds a key whose logit no other block's bound passes if it holds the dominant key."""
    lay = make([2000], 4, 2, "hnd", seed=21)
    q = query(lay, 2)
    at = [37, 1203]
    for g in range(2):
        lay.k[0, g, at[g]] = (8.0 * q[0, 2 * g].float()).to(torch.bfloat16)
    idx, _ = td.block_select(lay, td.block_bounds(lay), q, 1)
    assert idx[0, 0, 0] == at[0] // BLK and idx[0, 2, 0] == at[1] // BLK


# ---- attention -----------------------------------------------------------------------------------------------------

ATTN = [
    # lens, hq, hkv, m
    ([1], 1, 1, 1),
    ([16], 8, 1, 2),
    ([17, 0, 4000], 8, 2, 6),
    ([300, 40], 15, 3, 9),
    ([5000], 32, 8, 64),
    ([700, 1, 33, 512, 90], 14, 2, 33),
    ([9000], 4, 4, 300),
    ([12345, 800], 2, 1, 200),
]


def some_blocks(lens, hi, m, seed):
    """Blocks in no order, some twice, padding in between."""
    g = torch.Generator().manual_seed(seed)
    idx = torch.full((len(lens), hi, m), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        if n:
            idx[b] = torch.randint(0, pages(n), (hi, m), generator=g).to(torch.int32)
            idx[b, :, 0] = pages(n) - 1                   # the ragged block
            idx[b][torch.rand(hi, m, generator=g) < 0.2] = -1
    return idx


@pytest.mark.parametrize("layout", ["paged", "hnd", "nhd"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,hq,hkv,m", ATTN)
def test_attention_over_listed_blocks(td, layout, fp8, lens, hq, hkv, m):
    lay = make(lens, hq, hkv, layout, fp8, seed=m, sm_scale=0.11 if m == 9 else 0.0)
    q = query(lay, m)
    for hi in sorted({hq, hkv, 1}):
        idx = some_blocks(lens, hi, m, m + hi)
        cnt = torch.tensor([(m + 1) // 2 + i % 2 for i in range(len(lens))], dtype=torch.int32)
        for count in (None, cnt):
            guard = util.Guarded((len(lens), hq, D), torch.float32, DEV, fill=9e9)
            td.block_attn(lay, q, idx.to(DEV), None if count is None else count.to(DEV), out=guard.t)
            ref, tol = ref_attn(lay, q, idx, count)
            close(guard.t, ref, tol, f"hi {hi}, count {count is not None}")
            guard.check("out")
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("batch,hq,hkv,hi,m,ctx", [
    (10, 32, 32, 32, 3, 150), (20, 33, 33, 33, 5, 90), (60, 32, 8, 8, 2, 70), (80, 64, 8, 8, 3, 60), (19, 64, 8, 1, 9, 200),
    (3, 64, 8, 64, 70, 1500), (25, 56, 8, 8, 66, 1200), (12, 32, 4, 4, 70, 1300), (4, 64, 16, 1, 40, 900), (2, 16, 16, 16, 400, 7000), (5, 32, 32, 32, 30, 600),
    (12, 64, 16, 16, 70, 1300), (23, 8, 8, 8, 20, 500)])
def test_attention_of_many_items(td, fp8, batch, hq, hkv, hi, m, ctx):
    """One, two, four and eight warps to a CTA, alone and in clusters."""
    lens = [ctx - (ctx - 1) * i // (batch + 1) for i in range(batch)]
    lens[batch // 2] = 0
    lay = make(lens, hq, hkv, "paged", fp8, seed=batch)
    q, idx = query(lay, m), some_blocks(lens, hi, m, m)
    guard = util.Guarded((batch, hq, D), torch.float32, DEV, fill=9e9)
    td.block_attn(lay, q, idx.to(DEV), out=guard.t)
    ref, tol = ref_attn(lay, q, idx)
    close(guard.t, ref, tol, "many items")
    guard.check("out")
    assert td.device_status() == binding.OK


def test_attention_bf16_outputs(td):
    lay = make([900, 55], 8, 2, "paged", seed=1)
    q, idx = query(lay, 1), some_blocks([900, 55], 2, 20, 4)
    td.set_output_bf16(True)
    try:
        out = td.block_attn(lay, q, idx.to(DEV))
        assert out.dtype == torch.bfloat16
    finally:
        td.set_output_bf16(False)
    ref, tol = ref_attn(lay, q, idx)
    close(out, ref, tol, "bf16", bf16=True)


def test_rows_without_a_block_are_zero(td):
    lay = make([0, 50, 50], 4, 2, "paged", seed=2)
    q = query(lay, 2)
    idx = torch.full((3, 2, 5), -1, dtype=torch.int32, device=DEV)
    idx[2] = 1
    out = torch.full((3, 4, D), float("nan"), device=DEV)
    td.block_attn(lay, q, idx, torch.tensor([5, 5, 0], dtype=torch.int32, device=DEV), out=out)
    assert (out == 0).all()
    td.block_attn(lay, q, idx, torch.tensor([-3, 5, 5], dtype=torch.int32, device=DEV), out=out)
    assert (out[:2] == 0).all() and out[2].abs().sum() > 0


def test_bad_blocks_and_pages_are_skipped_and_reported(td):
    lay = make([100, 40], 4, 2, "paged", seed=6)
    q = query(lay, 6)
    idx = torch.tensor([[0, 2, 6], [2, 1, 0]], dtype=torch.int32)[:, None].repeat(1, 2, 1)
    ref, tol = ref_attn(lay, q, idx)
    assert td.device_status() == binding.OK
    for bad in (7, 3, -2, 2 ** 31 - 1, -2 ** 31):         # sequence 0 has blocks 0 .. 6, sequence 1 has 0 .. 2
        more = torch.cat((idx, torch.full((2, 2, 1), bad, dtype=torch.int32)), -1)
        r, t = ref_attn(lay, q, more)
        close(td.block_attn(lay, q, more.to(DEV)), r, t, f"block {bad}")
        assert td.device_status() == binding.ERR_INDEX
    good = lay.page_table[0, 2].clone()
    lay.page_table[0, 2] = lay.num_pages                  # a page outside the pool: its block drops out
    out = td.block_attn(lay, q, idx.to(DEV))
    assert td.device_status() == binding.ERR_INDEX
    less = idx.clone()
    less[0, :, 1] = -1
    r, t = ref_attn(lay, q, less)
    close(out, r, t, "bad page")
    bounds = torch.full(binding.block_bounds_shape(lay), 3.0, dtype=torch.bfloat16, device=DEV)
    td.block_bounds(lay, bounds)
    assert td.device_status() == binding.ERR_INDEX
    sel, cnt = td.block_select(lay, bounds, q, 3)
    assert td.device_status() == binding.ERR_INDEX
    assert cnt.tolist() == [3, 3] and ((sel >= 0) & (sel < 7)).all()
    lay.page_table[0, 2] = good
    td.block_select(lay, bounds, q, 3)
    assert td.device_status() == binding.OK


def test_all_blocks_equal_full_attention(td):
    lay = make([1000, 333], 8, 2, "paged", seed=8)
    q = query(lay, 8)
    idx, cnt = td.block_select(lay, td.block_bounds(lay), q, 63, binding.SEL_PER_KVHEAD)
    assert cnt.tolist() == [63, 21]
    ref, tol = ref_attn(lay, q, idx.cpu(), cnt.cpu())
    close(td.block_attn(lay, q, idx, cnt), ref, tol, "blocks")
    util.check_out(td.full_attn(lay, q).cpu().numpy(), ref.cpu().numpy(), "full")


def test_offsets_beyond_32_bits(td):
    """Pages more than 2^32 bytes apart, in every operator that follows a page id."""
    hkv, stride = 2, 1 << 27                              # 2^27 elements per page: page 40 starts 10.7 GB into the pool
    buf = torch.empty(41 * stride, dtype=torch.bfloat16, device=DEV)
    pool = buf.view(41, stride)[:, : hkv * BLK * 2 * D].view(41, hkv, BLK, 2, D)
    use = [40, 3, 17]
    for p in use:
        pool[p] = float("nan")
    lens = torch.tensor([40], dtype=torch.int32, device=DEV)
    table = torch.tensor([use], dtype=torch.int32, device=DEV)
    lay = synth.LayerKV(k=pool[..., 0, :], v=pool[..., 1, :], batch=1, num_q_heads=4, num_kv_heads=hkv, head_dim=D, ctx_lens=lens,
                        max_ctx_len=48, stride_pos=2 * D, stride_head=BLK * 2 * D, stride_page=stride, page_table=table,
                        max_pages_per_seq=3, keep=[buf])
    lay.num_pages = 41
    g = gen(5)
    k, v = (torch.randn(40, hkv, D, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    pos = torch.arange(40, device=DEV)
    td.kv_write(lay, k, v, table[0, pos // BLK].long() * BLK + pos % BLK)
    assert torch.equal(pool[40, :, :, 0].transpose(0, 1), k[:16]) and torch.equal(pool[17, :, :8, 1].transpose(0, 1), v[32:])
    lay.codes = lay.dense = [(k.double().transpose(0, 1), v.double().transpose(0, 1))]
    q = query(lay, 3)
    bounds = td.block_bounds(lay)
    assert torch.equal(bounds[40].double(), ref_bounds(lay, 0)[:, 0])
    idx, cnt = td.block_select(lay, bounds, q, 2)
    ref, _ = ref_select(lay, q, 2, 0, 0, 0)
    assert torch.equal(idx.cpu(), ref)
    r, t = ref_attn(lay, q, idx.cpu())
    close(td.block_attn(lay, q, idx, cnt), r, t, "far pages")
    assert td.device_status() == binding.OK


# ---- page maps -----------------------------------------------------------------------------------------------------

def ref_map(old, new, table, free, n_free):
    """The definition with lists: pages given back are pushed, then the growing sequences pop."""
    table, stack = [r[:] for r in table], free[:n_free]
    for o, n, row in zip(old, new, table):
        stack += row[pages(n): pages(o)]
    slots, positions, offsets = [], [], [0]
    for o, n, row in zip(old, new, table):
        for i in range(pages(o), pages(n)):
            row[i] = stack.pop()
        slots += [row[p // BLK] * BLK + p % BLK for p in range(o, n)]
        positions += list(range(o, n))
        offsets.append(len(slots))
    return table, stack, slots, positions, offsets


def map_case(old, width, total, seed):
    """A table that holds the old lengths, -1 elsewhere, and a stack of the other pages."""
    g = torch.Generator().manual_seed(seed)
    perm = torch.randperm(total, generator=g).tolist()
    table, at = [[-1] * width for _ in old], 0
    for row, o in zip(table, old):
        row[: pages(o)] = perm[at: at + pages(o)]
        at += pages(o)
    return table, perm[at:]


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def run_map(td, old, new, table, free, total, cap, alias=True):
    t, f = i32(table), torch.full((total,), -5, dtype=torch.int32, device=DEV)
    f[: len(free)] = i32(free)
    nf = i32([len(free)])
    out = nf if alias else i32([-9])
    gs, gp = util.Guarded((max(cap, 1),), torch.int64, DEV, fill=-77), util.Guarded((max(cap, 1),), torch.int32, DEV, fill=-77)
    go = util.Guarded((len(old) + 1,), torch.int32, DEV, fill=-77)
    td.page_map(i32(old), i32(new), t, f, nf, gs.t[:cap], num_free_out=out, positions=gp.t[:cap], token_offsets=go.t)
    for x in (gs, gp, go):
        x.check("page_map")
    return t, f, out, gs.t[:cap], gp.t[:cap], go.t


MAPS = [
    ([0], [1]), ([0], [0]), ([5], [16]), ([16], [17]), ([17], [16]), ([40], [0]),
    ([0, 31, 100, 64, 7], [50, 33, 0, 64, 8]),                                # grow, give back and stay in one call
    ([200, 200, 200], [0, 210, 17]),
    ([0, 0, 300, 0], [100, 0, 0, 200]),                                       # takes what is given back in the same call
    (list(range(1, 70)), [x + 1 for x in range(1, 70)]),
    ([1000] * 30 + [0] * 30, [0] * 30 + [990] * 30),
    ([0] * 7, [3000, 1, 0, 2999, 16, 15, 9000]),
]


@pytest.mark.parametrize("old,new", MAPS)
@pytest.mark.parametrize("pad", [0, 13])
def test_page_map(td, old, new, pad):
    width = max(map(pages, old + new)) + 2
    held, want = sum(map(pages, old)), sum(map(pages, new))
    total = max(held, want) + 3
    table, free = map_case(old, width, total, len(old))
    ref_t, ref_s, slots, positions, offsets = ref_map(old, new, table, free, len(free))
    t, f, nf, s, p, o = run_map(td, old, new, table, free, total, len(slots) + pad, alias=pad == 0)
    assert td.device_status() == binding.OK
    assert t.tolist() == ref_t
    assert int(nf) == len(ref_s) and f[: len(ref_s)].tolist() == ref_s
    assert s.tolist() == slots + [-1] * pad and p.tolist() == positions + [-1] * pad and o.tolist() == offsets


@pytest.mark.parametrize("batch", [1023, 1024, 1025, 4095, 4096])
def test_page_map_large_batches(td, batch):
    g = torch.Generator().manual_seed(batch)
    old = torch.randint(0, 60, (batch,), generator=g).tolist()
    new = [max(0, x + d) for x, d in zip(old, torch.randint(-40, 40, (batch,), generator=g).tolist())]
    width, total = 8, sum(map(pages, old)) + sum(map(pages, new)) + 1
    table, free = map_case(old, width, total, 3)
    ref_t, ref_s, slots, positions, offsets = ref_map(old, new, table, free, len(free))
    t, f, nf, s, p, o = run_map(td, old, new, table, free, total, len(slots) + 5)
    assert t.tolist() == ref_t and f[: len(ref_s)].tolist() == ref_s and int(nf) == len(ref_s)
    assert s.tolist() == slots + [-1] * 5 and p.tolist() == positions + [-1] * 5 and o.tolist() == offsets
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("fits", [True, False])
def test_page_map_with_the_largest_number_of_tokens(td, fits):
    """max_tokens next to 2^31: what is behind the last token is filled, and no counter wraps."""
    cap = 2 ** 31 - 1
    slots = torch.full((cap,), 7, dtype=torch.int64, device=DEV)
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    old, new = ints([3, 0]), ints([40, 17 if fits else 10 ** 6])
    table, free = torch.zeros(2, 4, dtype=torch.int32, device=DEV), torch.arange(9, dtype=torch.int32, device=DEV)
    td.page_map(old, new, table, free, ints([8]), slots)
    assert td.device_status() == (binding.OK if fits else binding.ERR_PAGES)
    used = 54 if fits else 0
    assert (slots[:used] >= 0).all()
    assert all(int((part != -1).sum()) == 0 for part in slots[used:].split(2 ** 28))
    del slots
    torch.cuda.empty_cache()


@pytest.mark.parametrize("why", ["pages", "tokens", "length", "negative", "count", "page", "overfull"])
@pytest.mark.parametrize("cap", [400, 20000])
def test_page_map_that_does_not_fit_changes_nothing(td, why, cap):
    old, new = [30, 0, 100], [45, 300, 10]
    table, free = map_case(old, 30, 60, 1)
    total = 60
    if why == "pages":
        free = free[:5]
    elif why == "tokens":
        cap = 314                                         # 15 + 300 tokens
    elif why == "length":
        new[1] = 30 * BLK + 1
    elif why == "negative":
        old[2] = -1
    elif why == "page":
        table[2][3] = 60                                  # would be given back
    elif why == "overfull":
        new, free = [0, 0, 0], free + list(range(60 - len(free)))
    t, f = i32(table), torch.full((total,), -5, dtype=torch.int32, device=DEV)
    f[: len(free)] = i32(free)
    nf = i32([61 if why == "count" else len(free)])
    t0, f0, nf0 = t.clone(), f.clone(), nf.clone()
    s, p, o = (torch.full((n,), 5, dtype=d, device=DEV) for n, d in ((cap, torch.int64), (cap, torch.int32), (4, torch.int32)))
    td.page_map(i32(old), i32(new), t, f, nf, s, positions=p, token_offsets=o)
    assert td.device_status() == binding.ERR_PAGES
    assert torch.equal(t, t0) and torch.equal(f, f0) and torch.equal(nf, nf0)
    assert (s == -1).all() and (p == -1).all() and (o == 0).all()
    assert td.device_status() == binding.OK


def test_page_map_reports_bad_ids_in_table_and_stack(td):
    t, f, nf = i32([[99, -1]]), i32([4, 77, 2, 3, 1]), i32([2])
    s = torch.zeros(20, dtype=torch.int64, device=DEV)
    td.page_map(i32([3]), i32([20]), t, f, nf, s)         # tokens 3..15 on page 99, 16..19 on page 77: both outside the pool
    assert td.device_status() == binding.ERR_INDEX
    assert (s == -1).all() and int(nf) == 1 and t.tolist() == [[99, 77]]


# ---- writing tokens ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("layout", ["paged", "hnd", "nhd"])
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hkv,T", [(1, 1), (3, 70), (8, 200), (2, 33)])
def test_kv_write(td, layout, fp8, hkv, T):
    lay = make([100, 130], hkv, hkv, layout, fp8, seed=T, spoil=False)
    cap = (lay.num_pages if lay.paged else 0) * BLK or 2 * lay.max_ctx_len
    g = gen(T)
    qkv = torch.randn(T, 3 * hkv, D, generator=g, device=DEV) * torch.exp2(torch.randint(-12, 6, (T, 3 * hkv, 1), generator=g, device=DEV).float())
    qkv = qkv.to(torch.bfloat16)
    k, v = qkv[:, hkv: 2 * hkv], qkv[:, 2 * hkv:]         # strided between tokens
    slots = torch.randperm(cap, generator=g, device=DEV)[:T].clone()
    slots[::7] = -1
    before = [x.clone() for x in lay.keep]
    td.kv_write(lay, k, v, slots)
    assert td.device_status() == binding.OK
    got, want = [x.view(torch.uint8 if fp8 else torch.int16) for x in lay.keep], [x.view(torch.uint8 if fp8 else torch.int16) for x in before]
    for i, (rows, sc) in enumerate(((k, lay.k_scale), (v, lay.v_scale))):
        if fp8:
            code = (rows.float().cpu() / sc.cpu()[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn)
            # the nearest value: off by at most half a step, 2^-4 of the value and 2^-10 near zero, up to saturation
            x = rows.double().cpu() / sc.double().cpu()[:, None]
            off = (code.float().double() - x.clamp(-448, 448)).abs()
            assert (off <= 2.0 ** -4 * x.abs() * (1 + 2.0 ** -20) + 2.0 ** -10).all()
            bits = code.view(torch.uint8).to(DEV)
        else:
            bits = rows.contiguous().view(torch.int16)
        for t in range(T):
            s = int(slots[t])
            if s < 0:
                continue
            if layout == "paged":
                want[0][s // BLK, :, s % BLK, i] = bits[t]
            elif layout == "hnd":
                want[0][s // lay.max_ctx_len, :, s % lay.max_ctx_len, i] = bits[t]
            else:
                want[i][s // lay.max_ctx_len, s % lay.max_ctx_len] = bits[t]
    for a, b in zip(got, want):
        assert torch.equal(a, b)                          # the whole buffer: nothing else was touched


def test_kv_write_saturates_and_rounds_to_even(td):
    lay = make([16], 1, 1, "hnd", True, seed=0, spoil=False)
    lay.k_scale.fill_(1.0)
    lay.v_scale.fill_(2.0)
    x = torch.zeros(1, 1, D)
    special = [448.0, 464.0, 500.0, -1e30, math.inf, -math.inf, math.nan, 17.0, 19.0, -17.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9, 1e-30, 0.0, 1.0625]
    x[0, 0, : len(special)] = torch.tensor(special)
    x = x.to(torch.bfloat16).to(DEV)
    td.kv_write(lay, x, x, torch.tensor([4], device=DEV))
    got = lay.k[0, 0, 4].float()[: len(special)].tolist()
    want = [448.0, 448.0, 448.0, -448.0, 448.0, -448.0, math.nan, 16.0, 20.0, -16.0, 0.0, 2.0 ** -8, 2.0 ** -9, 0.0, 0.0, 1.0]
    assert all((a == b) or (a != a and b != b) for a, b in zip(got, want)), got
    assert lay.v[0, 0, 4].float()[0] == 224.0


def test_kv_write_of_one_token_takes_any_token_stride(td):
    lay = make([16], 2, 2, "hnd", seed=0, spoil=False)
    k = torch.randn(2, D, 1, device=DEV).to(torch.bfloat16).permute(2, 0, 1)      # stride 1 between its one token
    k = torch.as_strided(k.contiguous(), (1, 2, D), (3, D, 1))
    td.kv_write(lay, k, k, torch.tensor([5], device=DEV))
    assert torch.equal(lay.k[0, :, 5], k[0]) and torch.equal(lay.v[0, :, 5], k[0])


def test_kv_write_skips_and_reports_slots_outside_the_cache(td):
    lay = make([64], 2, 2, "paged", seed=0)
    before = lay.keep[0].clone()
    k = torch.ones(3, 2, D, dtype=torch.bfloat16, device=DEV)
    for bad in (lay.num_pages * BLK, -2, 2 ** 62, -2 ** 63):
        td.kv_write(lay, k, k, torch.tensor([-1, bad, -1], device=DEV))
        assert td.device_status() == binding.ERR_INDEX
    assert torch.equal(lay.keep[0].view(torch.int16), before.view(torch.int16))
    td.kv_write(lay, k[:0], k[:0], torch.zeros(0, dtype=torch.int64, device=DEV))
    assert td.device_status() == binding.OK


# ---- the operators together ----------------------------------------------------------------------------------------

class Serving:
    """A pool, requests that come, grow and end, and one layer's cache, driven as a serving loop does it."""

    def __init__(self, td, batch, hq, hkv, fp8, total, width, cap):
        self.td, self.cap, self.fp8 = td, cap, fp8
        dt = torch.float8_e4m3fn if fp8 else torch.bfloat16
        pool = torch.zeros(total, hkv, BLK, 2, D, dtype=dt, device=DEV)
        (pool.view(torch.uint8) if fp8 else pool).fill_(0x7F if fp8 else float("nan"))
        self.old, self.new = torch.zeros(batch, dtype=torch.int32, device=DEV), torch.zeros(batch, dtype=torch.int32, device=DEV)
        self.table = torch.full((batch, width), -1, dtype=torch.int32, device=DEV)
        self.free = torch.randperm(total, generator=gen(1), device=DEV).to(torch.int32)
        self.n_free = i32([total])
        self.slots = torch.zeros(cap, dtype=torch.int64, device=DEV)
        self.rows = [torch.zeros(cap, hkv, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        self.q = torch.zeros(batch, hq, D, dtype=torch.bfloat16, device=DEV)
        sc = dict(k_scale=torch.full((hkv,), 0.02, device=DEV), v_scale=torch.full((hkv,), 0.015, device=DEV)) if fp8 else {}
        self.lay = synth.LayerKV(k=pool[..., 0, :], v=pool[..., 1, :], batch=batch, num_q_heads=hq, num_kv_heads=hkv, head_dim=D,
                                 ctx_lens=self.new, max_ctx_len=width * BLK, stride_pos=2 * D, stride_head=BLK * 2 * D,
                                 stride_page=hkv * BLK * 2 * D, page_table=self.table, max_pages_per_seq=width, keep=[pool],
                                 kv_dtype=int(fp8), **sc)
        self.lay.num_pages = total
        self.bounds = torch.zeros(binding.block_bounds_shape(self.lay), dtype=torch.bfloat16, device=DEV)
        self.dense = [(torch.zeros(hkv, 0, D, dtype=torch.float64, device=DEV),) * 2 for _ in range(batch)]

    def step(self, m, gran):
        td, lay = self.td, self.lay
        td.page_map(self.old, self.new, self.table, self.free, self.n_free, self.slots)
        td.kv_write(lay, self.rows[0], self.rows[1], self.slots)
        td.block_bounds(lay, self.bounds, start_lens=self.old)
        idx, cnt = td.block_select(lay, self.bounds, self.q, m, gran, keep_first=1, keep_last=1)
        return td.block_attn(lay, self.q, idx, cnt), idx, cnt

    def feed(self, lens, seed):
        """New lengths, new rows and a query; the dense copy follows."""
        g = gen(seed)
        self.old.copy_(self.new)
        self.new.copy_(i32(lens))
        for r in self.rows:
            r.normal_(generator=g)
        self.q.normal_(generator=g)
        at = 0
        for b, (o, n) in enumerate(zip(self.old.tolist(), lens)):
            new = [self.held(self.rows[i][at: at + max(n - o, 0)].transpose(0, 1), i) for i in range(2)]
            self.dense[b] = tuple(torch.cat((x[:, :n], y), 1) for x, y in zip(self.dense[b], new))
            at += max(n - o, 0)

    def held(self, x, which):
        if not self.fp8:
            return x.double()
        sc = (self.lay.v_scale if which else self.lay.k_scale)[:, None, None]
        return (x.float() / sc).clamp(-448, 448).to(torch.float8_e4m3fn).float().double() * sc.double()

    def check(self, out, idx, cnt, m, gran):
        lay = self.lay
        lay.dense = self.dense
        sk = lay.k_scale.double()[:, None, None] if self.fp8 else 1.0
        lay.codes = [(k / sk, v) for k, v in self.dense]
        ref, ref_cnt = ref_select(lay, self.q, m, gran, 1, 1)
        assert torch.equal(cnt.cpu(), ref_cnt) and torch.equal(idx.cpu(), ref)
        r, t = ref_attn(lay, self.q, idx.cpu(), cnt.cpu())
        close(out, r, t, "step")
        held = sum(pages(n) for n in self.new.tolist())
        assert int(self.n_free) == lay.num_pages - held


STEPS = [[200, 0, 37, 64], [201, 0, 38, 65], [202, 90, 0, 66], [0, 91, 0, 67], [16, 92, 130, 68], [17, 93, 131, 0], [18, 94, 132, 300]]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("gran", GRANS)
def test_a_serving_loop(td, fp8, gran):
    s = Serving(td, 4, 8, 2, fp8, total=40, width=20, cap=400)
    for i, lens in enumerate(STEPS):
        s.feed(lens, i)
        out, idx, cnt = s.step(5, gran)
        s.check(out, idx, cnt, 5, gran)
    assert td.device_status() == binding.OK


@pytest.mark.parametrize("fp8", [False, True])
def test_a_captured_step_replayed_over_changing_lengths(fp8):
    """The whole step as one graph from a fresh context's first call on; eager calls of another shape come in between."""
    t = binding.Tidal(0)
    try:
        s = Serving(t, 4, 8, 2, fp8, total=40, width=20, cap=400)
        side = torch.cuda.Stream()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                res = s.step(5, 1)
        for i, lens in enumerate(STEPS):
            s.feed(lens, 40 + i)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            s.check(*res, 5, 1)
            big = make([3000 * (i + 1)], 8, 2, "hnd", seed=i)
            qb = query(big, i)
            idx, _ = t.block_select(big, t.block_bounds(big), qb, 9)
            assert torch.equal(idx.cpu(), ref_select(big, qb, 9, 0, 0, 0)[0])
        assert t.device_status() == binding.OK
        del graph
    finally:
        t.close()


@pytest.mark.parametrize("ctx", [900, 40000])
def test_the_first_call_of_a_context_can_be_captured(ctx):
    """Short contexts need nothing reserved before a capture, long ones do."""
    t = binding.Tidal(0)
    try:
        lay = make([ctx], 8, 2, "hnd", seed=1)
        q = query(lay, 1)
        bounds = torch.zeros(binding.block_bounds_shape(lay), dtype=torch.bfloat16, device=DEV)
        idx, cnt = torch.zeros(1, 8, 4, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        out = torch.zeros(1, 8, D, device=DEV)
        if ctx > 16384:
            t.reserve(lay, 16)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                t.block_bounds(lay, bounds)
                t.block_select(lay, bounds, q, 4, idx=idx, idx_count=cnt)
                t.block_attn(lay, q, idx, cnt, out=out)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(idx.cpu(), ref_select(lay, q, 4, 0, 0, 0)[0])
        ref, tol = ref_attn(lay, q, idx.cpu())
        close(out, ref, tol, "captured")
        del graph
    finally:
        t.close()


def test_scratch_is_not_allocated_into_a_capture():
    t = binding.Tidal(0)
    try:
        lay = make([40000], 8, 2, "hnd", seed=1)
        q, bounds = query(lay, 1), t.block_bounds(lay)
        idx, cnt = torch.zeros(1, 8, 4, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        x = torch.zeros(8, device=DEV)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                x += 1
                with pytest.raises(binding.TidalError) as e:
                    t.block_select(lay, bounds, q, 4, idx=idx, idx_count=cnt)
                assert e.value.status == binding.ERR_NOMEM
        graph.replay()
        torch.cuda.synchronize()
        assert (x == 1).all()
        t.block_select(lay, bounds, q, 4, idx=idx, idx_count=cnt)
        assert torch.equal(idx.cpu(), ref_select(lay, q, 4, 0, 0, 0)[0])
        del graph
    finally:
        t.close()


def test_a_captured_selection_outlives_the_growth_of_its_scratch():
    t = binding.Tidal(0)
    try:
        lay = make([30000], 8, 2, "paged", seed=2)
        q, bounds = query(lay, 2), t.block_bounds(lay)
        idx, cnt = torch.zeros(1, 2, 50, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        t.block_select(lay, bounds, q, 50, 1, idx=idx, idx_count=cnt)
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            with torch.cuda.graph(graph, stream=side):
                t.block_select(lay, bounds, q, 50, 1, idx=idx, idx_count=cnt)
        big = make([60000, 50000, 70000], 8, 2, "paged", seed=3)
        qb = query(big, 3)
        big_idx, _ = t.block_select(big, t.block_bounds(big), qb, 30)
        assert torch.equal(big_idx.cpu(), ref_select(big, qb, 30, 0, 0, 0)[0])
        for i in range(3):
            q.copy_(query(lay, 10 + i))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(idx.cpu(), ref_select(lay, q, 50, 1, 0, 0)[0])
        del graph
    finally:
        t.close()


def test_two_contexts_on_two_streams():
    a, b = binding.Tidal(0), binding.Tidal(0)
    try:
        lay = make([5000, 1234], 8, 2, "paged", seed=13)
        qs = [query(lay, i) for i in range(2)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        bounds = a.block_bounds(lay)
        refs = [ref_select(lay, q, 40, 0, 0, 1) for q in qs]
        torch.cuda.synchronize()
        outs = []
        for _ in range(20):
            for t, st, q in zip((a, b), streams, qs):
                with torch.cuda.stream(st):
                    idx, cnt = t.block_select(lay, bounds, q, 40, keep_last=1)
                    outs.append((idx, t.block_attn(lay, q, idx, cnt)))
        torch.cuda.synchronize()
        for i, (idx, out) in enumerate(outs):
            assert torch.equal(idx.cpu(), refs[i % 2][0])
            assert torch.equal(out, outs[i % 2][1])       # no atomics: the same bits every time
    finally:
        a.close(); b.close()


def test_random_shapes(td):
    """Whole chains (bounds, selection, attention) over shapes drawn at random."""
    import random
    rng = random.Random(20)
    for i in range(40):
        hkv, G = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8])
        lens = [rng.choice([0, 1, rng.randint(1, 50), rng.randint(1, 3000)]) for _ in range(rng.randint(1, 5))]
        fp8, layout, gran = rng.random() < 0.5, rng.choice(["paged", "hnd", "nhd"]), rng.choice(GRANS)
        m, first, last = rng.randint(1, 60), rng.randint(0, 2), rng.randint(0, 2)
        lay = make(lens, hkv * G, hkv, layout, fp8, seed=i)
        q = query(lay, i)
        idx, cnt = td.block_select(lay, td.block_bounds(lay), q, m, gran, first, last)
        ref, ref_cnt = ref_select(lay, q, m, gran, first, last)
        assert torch.equal(idx.cpu(), ref) and torch.equal(cnt.cpu(), ref_cnt), (i, lens, hkv, G)
        r, t = ref_attn(lay, q, idx.cpu(), cnt.cpu())
        close(td.block_attn(lay, q, idx, cnt), r, t, f"{i}")
    assert td.device_status() == binding.OK


# ---- refusals of the binding ---------------------------------------------------------------------------------------

def test_the_binding_refuses_tensors_it_cannot_take(td):
    lay = make([100], 4, 2, "paged", seed=0)
    q, bounds = query(lay, 0), td.block_bounds(lay)
    idx = torch.zeros(1, 4, 3, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError, match="q:"):
        td.block_select(lay, bounds, q.float(), 3)
    with pytest.raises(ValueError, match="q:"):
        td.block_attn(lay, q.cpu(), idx)
    with pytest.raises(ValueError, match="bounds"):
        td.block_select(lay, bounds[:, :1], q, 3)
    with pytest.raises(ValueError, match="bounds"):
        td.block_bounds(lay, bounds.float())
    with pytest.raises(ValueError, match="idx"):
        td.block_attn(lay, q, idx.long())
    with pytest.raises(ValueError, match="out"):
        td.block_attn(lay, q, idx, out=torch.zeros(1, 4, D, dtype=torch.bfloat16, device=DEV))
    with pytest.raises(ValueError, match="k_new"):
        td.kv_write(lay, q, q, torch.zeros(1, dtype=torch.int64, device=DEV))
    with pytest.raises(ValueError, match="slots"):
        td.kv_write(lay, q[:, :2], q[:, :2], torch.zeros(1, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError, match="new_lens"):
        td.page_map(i32([1]), i32([1, 2]), i32([[0]]), i32([0]), i32([1]), torch.zeros(1, dtype=torch.int64, device=DEV))
    for m in (0, -1, 16385):
        with pytest.raises(binding.TidalError):
            td.block_select(lay, bounds, q, m)
    with pytest.raises(binding.TidalError):
        td.block_attn(lay, q, torch.zeros(1, 3, 3, dtype=torch.int32, device=DEV))
    assert td.device_status() == binding.OK
