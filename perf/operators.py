"""What is measured of the block-sparse decode path: page tables and slot maps from request lengths, the writing of
tokens into the cache, key summaries of blocks, the selection of blocks by a bound on their logits, and attention over
the selected blocks. Every operator stands here in its plain form (elementary torch operations) and as the call of the
framework's own operator; `own` says which of the two run() takes.

A block is 16 consecutive positions of a sequence, one page of a paged cache. Caches are bf16 or E4M3 codes with
a scale per KV head, a position's key row followed by its value row: [page][Hkv][16][2][128], or
[batch][Hkv][positions][2][128] where they are contiguous. Sizes are those of the benchmark's configurations (8/2 heads at
4096; 32/8 heads at 131072 with 4096 selected tokens; a ragged batch of 8 up to 65536 with 2048) and generic ones.
"""
import math
from types import SimpleNamespace

import torch

own = False

D = 128          # head dimension
BLK = 16         # positions per block and per page
DEV = "cuda:0"


# ---- cases -------------------------------------------------------------------------------------------------------

def _case(op, name=None, **over):
    c = {"op": op, "batch": 1, "hq": 32, "hkv": 8, "ctx_min": 0, "ctx": 4096, "paged": False, "fp8": False}
    c.update(over)
    c["ctx_min"] = c["ctx_min"] or c["ctx"]
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a decode step of 64 running requests: one token more for each, a page for about four of them
        _case("page_map", "map: 64 requests decode", batch=64, ctx_min=33, ctx=16384, new=1),
        # eight long prompts admitted at once: every page and slot of them
        _case("page_map", "map: 8 prompts to 65536", batch=8, ctx_min=8192, ctx=65536, new=0),
        # the new token's rows of 64 running requests
        _case("kv_write", "write: 64 tokens bf16", tokens=64, paged=True),
        # one long prompt quantised into an 8-bit cache
        _case("kv_write", "write: 65536 tokens fp8", tokens=65536, paged=True, fp8=True),
        # after a decode step: the summary of each request's newest block
        _case("block_bounds", "bounds: 64 newest blocks", batch=64, ctx_min=33, ctx=4096, paged=True, new=1),
        # after the prefill of a 128K prompt: every block
        _case("block_bounds", "bounds: prompt of 131072", ctx=131072, new=0),
        # a short context, a set of blocks per query head
        _case("block_select", "select: 4096, 16 per head", hq=8, hkv=2, ctx=4096, m=16, gran="qhead", first=0, last=1),
        # a 128K context, a set per KV head of as many tokens as the token selection keeps (4096)
        _case("block_select", "select: 131072, 256 per KV", ctx=131072, m=256, gran="kvhead", first=1, last=2),
        # a ragged paged batch, a set of 2048 tokens per query head
        _case("block_select", "select: 8x65536 paged", batch=8, ctx_min=8192, ctx=65536, paged=True, m=128, gran="qhead", first=0, last=1),
        # the attention that follows each of the three selections; the last one over an 8-bit cache
        _case("block_attn", "attn: 4096, 16 per head", hq=8, hkv=2, ctx=4096, m=16, gran="qhead"),
        _case("block_attn", "attn: 131072, 256 per KV", ctx=131072, m=256, gran="kvhead"),
        _case("block_attn", "attn: 8x65536 paged fp8", batch=8, ctx_min=8192, ctx=65536, paged=True, fp8=True, m=128, gran="qhead"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["page_map", "kv_write", "block_bounds", "block_select", "block_attn"])
    hkv, g = rng.choice([(1, 8), (2, 4), (3, 5), (4, 1), (4, 7), (8, 4), (8, 8), (8, 2), (32, 1)])
    c = dict(hq=hkv * g, hkv=hkv, paged=rng.random() < 0.6, fp8=rng.random() < 0.4)
    if op == "page_map":
        b = _log(rng, 1, 512)
        ctx = _log(rng, 16, min(65536, 300000 // b))
        c.update(batch=b, ctx=ctx, ctx_min=_log(rng, 1, ctx), new=rng.choice([1, 1, 0, _log(rng, 2, ctx)]), paged=True)
    elif op == "kv_write":
        c.update(tokens=_log(rng, 1, (65536 if c["fp8"] else 49152) * 8 // max(hkv, 8)), paged=True)
    else:
        most = 131072 * 8 // max(hkv, 8)
        b = _log(rng, 1, 48)
        ctx = _log(rng, 40, max(64, most // b))
        c.update(batch=b, ctx=ctx, ctx_min=_log(rng, 1, ctx))
        if op == "block_bounds":
            c.update(new=rng.choice([0, 1, _log(rng, 2, ctx)]))
        else:
            c.update(m=_log(rng, 1, max(2, min(512, 2 * ctx // BLK))), gran=rng.choice(["qhead", "kvhead", "kvhead", "shared"]))
            if op == "block_attn":                        # at most the bytes of the largest listed one
                hi = {"qhead": hkv * g, "kvhead": hkv, "shared": hkv}[c["gran"]]
                c["m"] = max(1, min(c["m"], (32768 if c["fp8"] else 16384) // (b * hi)))
            else:
                c.update(first=rng.choice([0, 0, 1, 3]), last=rng.choice([0, 1, 2]))
    return _case(op, **c)


def _lens(case):
    """The sequences' lengths: even steps from ctx_min to ctx (their order comes from the seed)."""
    b, lo, hi = case["batch"], case["ctx_min"], case["ctx"]
    return [hi - (hi - lo) * i // max(b - 1, 1) for i in range(b)]


def _old_lens(case):
    """The lengths before the `new` tokens of each sequence came; new = 0: all of them are new."""
    return [max(n - case["new"], 0) if case["new"] else 0 for n in _lens(case)]


def _pages(n):
    return (n + BLK - 1) // BLK


def _index_heads(case):
    return {"qhead": case["hq"], "kvhead": case["hkv"], "shared": 1}[case["gran"]]


def work(case):
    op, hq, hkv = case["op"], case["hq"], case["hkv"]
    esz = 1 if case["fp8"] else 2
    if op == "page_map":
        old, new = _old_lens(case), _lens(case)
        grown = sum(_pages(n) - _pages(o) for o, n in zip(old, new))
        tokens = sum(n - o for o, n in zip(old, new))
        return {"bytes": 8 * len(old) + 4 * (len(old) + 1) + 8 * grown + 12 * tokens, "flops": 0}
    if op == "kv_write":
        t = case["tokens"]
        return {"bytes": t * hkv * D * 2 * (2 + esz) + 8 * t, "flops": t * hkv * D * 2 if case["fp8"] else 0}
    lens = _lens(case)
    if op == "block_bounds":
        total = rows = 0
        for o, n in zip(_old_lens(case), lens):
            total += (_pages(n) - o // BLK) * hkv
            rows += (n - o // BLK * BLK) * hkv
        return {"bytes": rows * D * esz + total * 2 * D * 2, "flops": 2 * rows * D}
    hi, m = _index_heads(case), case["m"]
    if op == "block_select":
        blocks = sum(_pages(n) for n in lens)
        return {"bytes": blocks * hkv * 2 * D * 2 + len(lens) * (hq * D * 2 + hi * m * 4), "flops": 4 * D * hq * blocks}
    read = rows = 0
    for n in lens:
        cnt = min(m, _pages(n))
        read += min(cnt * max(hi, hkv), _pages(n) * hkv) * BLK
        rows += cnt * BLK * hq
    return {"bytes": read * 2 * D * esz + len(lens) * (hq * D * 6 + hi * m * 4), "flops": 4 * D * rows}


# ---- inputs ------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(1000003 * (seed + 1))


def _normal(g, *shape):
    return torch.empty(*shape, dtype=torch.bfloat16, device=DEV).normal_(generator=g)


def _cache(s, case, g, lens):
    """A filled cache: normal keys and values, a few key channels off centre as trained models have them."""
    b, hkv = case["batch"], case["hkv"]
    if case["paged"]:
        total = sum(_pages(n) for n in lens) + 5
        buf = _normal(g, total, hkv, BLK, 2, D)
        width = _pages(max(lens))
        table = torch.zeros(b, width, dtype=torch.int32, device=DEV)
        perm = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
        at = 0
        for i, n in enumerate(lens):
            table[i, : _pages(n)] = perm[at: at + _pages(n)]
            at += _pages(n)
        s["table"] = table
    else:
        buf = _normal(g, b, hkv, _pages(max(lens)), BLK, 2, D)
    off = torch.zeros(hkv, D, device=DEV)
    off[:, torch.randint(0, D, (4,), generator=g, device=DEV)] = 3.0 * torch.randn(hkv, 4, generator=g, device=DEV)
    shape = [1] * buf.dim()
    shape[1], shape[-1] = hkv, D
    buf.select(-2, 0).add_(off.to(torch.bfloat16).view(shape[:-2] + [D]))
    s["k_scale"] = s["v_scale"] = None
    if case["fp8"]:
        s["k_scale"] = 0.02 + 0.03 * torch.rand(hkv, generator=g, device=DEV)
        s["v_scale"] = 0.01 + 0.02 * torch.rand(hkv, generator=g, device=DEV)
        q8 = torch.empty(buf.shape, dtype=torch.float8_e4m3fn, device=DEV)
        for i, sc in ((0, s["k_scale"]), (1, s["v_scale"])):
            q8.select(-2, i).copy_((buf.select(-2, i).float() / sc.view(shape[:-2] + [1])).clamp(-448.0, 448.0))
        buf = q8
    s["buf"] = buf


def _layer(s, case):
    """The cache's descriptor as the framework's binding takes it."""
    buf, hkv = s["buf"], case["hkv"]
    paged = case["paged"]
    if not paged:
        buf = buf.view(case["batch"], hkv, -1, 2, D)
    st = buf.stride()
    return SimpleNamespace(
        k=buf.select(-2, 0), v=buf.select(-2, 1), batch=case["batch"], num_q_heads=case["hq"], num_kv_heads=hkv, head_dim=D,
        ctx_lens=s["lens"], max_ctx_len=s["max_len"], stride_b=0 if paged else st[0], stride_pos=2 * D, stride_head=st[1],
        stride_page=st[0] if paged else 0, page_table=s.get("table"), page_size=BLK,
        max_pages_per_seq=s["table"].shape[1] if paged else 0, num_pages=buf.shape[0] if paged else 0, sm_scale=0.0,
        keep=[s["buf"]], kv_dtype=1 if case["fp8"] else 0, k_scale=s["k_scale"], v_scale=s["v_scale"])


_handles = {}


def _handle():
    """The framework's context on this GPU: one for the whole program."""
    from paper_2410_05076_b200 import binding
    if "td" not in _handles:
        _handles["td"] = binding.Tidal(0)
    return binding, _handles["td"]


def _bounds_of(buf):
    keys = buf.select(-2, 0).to(torch.bfloat16)
    return torch.stack((keys.amin(-2), keys.amax(-2)), -2).contiguous()


def prepare(case, seed):
    g = _gen(seed)
    op, b, hq, hkv = case["op"], case["batch"], case["hq"], case["hkv"]
    s = {"case": case, "op": op}
    order = torch.randperm(b, generator=torch.Generator().manual_seed(seed + 17)).tolist()
    lens = [_lens(case)[i] for i in order]
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    s["lens"], s["max_len"] = ints(lens), max(lens)
    if op == "page_map":
        old = [_old_lens(case)[i] for i in order]
        held, want = sum(map(_pages, old)), sum(map(_pages, lens))
        total = want + 7
        perm = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
        table = torch.full((b, _pages(case["ctx"])), -1, dtype=torch.int32, device=DEV)
        at = 0
        for i, n in enumerate(old):
            table[i, : _pages(n)] = perm[at: at + _pages(n)]
            at += _pages(n)
        free = torch.full((total,), -1, dtype=torch.int32, device=DEV)
        free[: total - held] = perm[held:]
        tokens = sum(n - o for o, n in zip(old, lens))
        s.update(old=ints(old), table=table, free=free, n_free=ints([total - held]), n_free_out=ints([0]), tokens=tokens,
                 slots=torch.full((tokens,), -1, dtype=torch.int64, device=DEV), pos=torch.zeros(tokens, dtype=torch.int32, device=DEV),
                 offsets=torch.zeros(b + 1, dtype=torch.int32, device=DEV))
    elif op == "kv_write":
        t = case["tokens"]
        pages = _pages(t) + 3
        s["lens"], s["max_len"] = ints([pages * BLK]), pages * BLK
        one = dict(case, batch=1)
        _cache(s, one, g, [pages * BLK])
        at = torch.randperm(pages, generator=g, device=DEV)[:, None] * BLK + torch.arange(BLK, device=DEV)
        s["slots"] = at.reshape(-1)[:t].contiguous()
        qkv = _normal(g, t, hq + 2 * hkv, D)              # the rows are slices of a fused projection's output
        s["k_new"], s["v_new"] = qkv[:, hq: hq + hkv], qkv[:, hq + hkv:]
        if own:
            s["kv"] = _handle()[0].kv_struct(_layer(s, one))
        return s
    elif op == "block_bounds":
        _cache(s, case, g, lens)
        old = [_old_lens(case)[i] for i in order]
        s["old"], s["max_new"] = ints(old), max(n - o for o, n in zip(old, lens))
        s["bounds"] = torch.zeros(s["buf"].shape[:-3] + (2, D), dtype=torch.bfloat16, device=DEV)
    else:
        _cache(s, case, g, lens)
        s["q"] = _normal(g, b, hq, D)
        hi, m = _index_heads(case), case["m"]
        s["count"] = torch.tensor([min(m, _pages(n)) for n in lens], dtype=torch.int32, device=DEV)
        s["idx"] = torch.full((b, hi, m), -1, dtype=torch.int32, device=DEV)
        if op == "block_select":
            s["bounds"] = _bounds_of(s["buf"])
            s["count"].zero_()
        else:
            r = torch.rand(b, hi, _pages(max(lens)), generator=g, device=DEV)
            for i, n in enumerate(lens):                  # a set of each sequence's blocks, the newest among them
                have = _pages(n)
                r[i, :, have - 1] = 2.0
                c = min(m, have)
                s["idx"][i, :, :c] = r[i, :, :have].topk(c, dim=-1).indices.sort(-1).values.to(torch.int32)
            s["out"] = torch.zeros(b, hq, D, dtype=torch.float32, device=DEV)
    if own and op != "page_map":
        s["kv"] = _handle()[0].kv_struct(_layer(s, case))
    elif own:
        _handle()
    return s


# ---- the framework's operators -----------------------------------------------------------------------------------

def _own(s):
    binding, td = _handle()
    op, c = s["op"], s["case"]
    if op == "page_map":
        td.page_map(s["old"], s["lens"], s["table"], s["free"], s["n_free"], s["slots"], num_free_out=s["n_free_out"],
                    positions=s["pos"], token_offsets=s["offsets"])
        return [s["table"], s["slots"], s["pos"], s["offsets"], s["free"], s["n_free_out"]]
    if op == "kv_write":
        td.kv_write(s["kv"], s["k_new"], s["v_new"], s["slots"])
        return s["buf"]
    if op == "block_bounds":
        return td.block_bounds(s["kv"], s["bounds"], start_lens=s["old"], max_new=s["max_new"])
    if op == "block_select":
        gran = {"qhead": binding.SEL_PER_QHEAD, "kvhead": binding.SEL_PER_KVHEAD, "shared": binding.SEL_SHARED}[c["gran"]]
        return list(td.block_select(s["kv"], s["bounds"], s["q"], c["m"], gran, keep_first=c["first"], keep_last=c["last"],
                                    idx=s["idx"], idx_count=s["count"]))
    return td.block_attn(s["kv"], s["q"], s["idx"], s["count"], out=s["out"])


# ---- the plain forms ---------------------------------------------------------------------------------------------

def _page_map(s):
    """Pages that grow are popped off the stack of free pages in the order of sequence and position; a token's
    slot is its page times 16 and its place there."""
    old, new, table, free = s["old"].long(), s["lens"].long(), s["table"], s["free"]
    have, need = (old + BLK - 1) // BLK, (new + BLK - 1) // BLK
    zero = torch.zeros(1, dtype=torch.long, device=DEV)
    ends = torch.cat((zero, (need - have).cumsum(0)))
    n_free = s["n_free"].long()
    col = torch.arange(table.shape[1], device=DEV)[None, :]
    fresh = (col >= have[:, None]) & (col < need[:, None])
    at = (n_free - 1 - (ends[:-1, None] + col - have[:, None])).clamp(0, free.numel() - 1)
    table.copy_(torch.where(fresh, free[at], table))
    offsets = torch.cat((zero, (new - old).cumsum(0)))
    t = torch.arange(s["tokens"], device=DEV)
    seq = torch.searchsorted(offsets, t, right=True) - 1
    pos = old[seq] + t - offsets[seq]
    s["slots"].copy_(table[seq, pos // BLK].long() * BLK + pos % BLK)
    s["pos"].copy_(pos)
    s["offsets"].copy_(offsets)
    s["n_free_out"].copy_(n_free - ends[-1:])
    return [table, s["slots"], s["pos"], s["offsets"], free, s["n_free_out"]]


def _kv_write(s):
    """Each token's rows to its slot; for an 8-bit cache the quotient by the head's scale, rounded to the nearest code."""
    page, place = s["slots"] // BLK, s["slots"] % BLK
    buf, fp8 = s["buf"], s["case"]["fp8"]
    held = buf.view(torch.uint8) if fp8 else buf
    heads = torch.arange(buf.shape[1], device=DEV)[None, :]
    for i, new, scale in ((0, s["k_new"], s["k_scale"]), (1, s["v_new"], s["v_scale"])):
        if fp8:
            new = (new.float() / scale[:, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        held[:, :, :, i][page[:, None], heads, place[:, None]] = new
    return buf


def _rows(s, which, blk):
    """The key (0) or value (1) rows of blocks `blk` [B, heads, n] of each sequence and KV head: [B, Hkv, n, 16, 128]
    in 32 bits, without the scale of an 8-bit cache."""
    buf, hkv = s["buf"], s["case"]["hkv"]
    heads = torch.arange(hkv, device=DEV).view(1, hkv, 1)
    if blk.shape[1] not in (1, hkv):
        heads = heads.repeat_interleave(blk.shape[1] // hkv, 1)
    seq = torch.arange(blk.shape[0], device=DEV).view(-1, 1, 1)
    held = buf.view(torch.uint8) if buf.dtype == torch.float8_e4m3fn else buf
    held = held.select(-2, which)
    rows = held[s["table"][seq, blk].long(), heads] if "table" in s else held[seq, heads, blk]
    return rows.view(torch.float8_e4m3fn).float() if buf.dtype == torch.float8_e4m3fn else rows.float()


def _block_bounds(s):
    """The least and the greatest key of each channel over the cached positions of a block."""
    lens, first = s["lens"].long(), s["old"].long() // BLK
    n = (s["max_new"] + BLK - 1) // BLK + 1
    last = (lens + BLK - 1) // BLK - 1
    blk = torch.minimum(first[:, None] + torch.arange(n, device=DEV), last[:, None])[:, None, :]
    rows = _rows(s, 0, blk)
    there = (blk[..., None] * BLK + torch.arange(BLK, device=DEV) < lens.view(-1, 1, 1, 1))[..., None]
    lo = rows.masked_fill(~there, math.inf).amin(-2)
    hi = rows.masked_fill(~there, -math.inf).amax(-2)
    both = torch.stack((lo, hi), -2).to(torch.bfloat16)
    heads = torch.arange(rows.shape[1], device=DEV).view(1, -1, 1)
    seq = torch.arange(rows.shape[0], device=DEV).view(-1, 1, 1)
    if "table" in s:
        s["bounds"][s["table"][seq, blk].long(), heads] = both
    else:
        s["bounds"][seq, heads, blk] = both
    return s["bounds"]


def _own_bounds(s):
    """The bounds of every block of every sequence: [B, Hkv, n, 2, 128]."""
    b = s["bounds"]
    return b[s["table"].long()].transpose(1, 2) if "table" in s else b


def _block_select(s):
    """An upper bound of a block's logits, sum_c max(q_c lo_c, q_c hi_c), as two products (the query's positive part
    with the greatest keys, its negative part with the least): in 64 bits, since values next to the border decide."""
    c = s["case"]
    b, hq, hkv, hi, m = c["batch"], c["hq"], c["hkv"], _index_heads(c), c["m"]
    bounds = _own_bounds(s).double()
    q = s["q"].double().view(b, hkv, hq // hkv, D)
    score = q.clamp(min=0) @ bounds[..., 1, :].transpose(-1, -2) + q.clamp(max=0) @ bounds[..., 0, :].transpose(-1, -2)
    if c["fp8"]:
        score = score * s["k_scale"].double().view(1, hkv, 1, 1)
    n = score.shape[-1]
    score = score.reshape(b, hi, hq // hi, n).sum(2)
    blk = torch.arange(n, device=DEV)
    have = ((s["lens"].long() + BLK - 1) // BLK).view(b, 1, 1)
    kept = (blk < c["first"]) | (blk >= have - c["last"])
    score = torch.where(kept, math.inf, score).masked_fill(blk >= have, -math.inf)
    best = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., :m]
    if best.shape[-1] < m:
        best = torch.cat((best, best.new_full((b, hi, m - best.shape[-1]), n)), -1)
    count = have.clamp(max=m)
    best = torch.where(torch.arange(m, device=DEV) < count, best, n).sort(-1).values
    s["idx"].copy_(torch.where(best < n, best, -1))
    s["count"].copy_(count.view(b))
    return [s["idx"], s["count"]]


def _block_attn(s):
    """Softmax over the cached positions of each query head's blocks."""
    c = s["case"]
    b, hq, hkv, hi = c["batch"], c["hq"], c["hkv"], _index_heads(c)
    idx = s["idx"].long()
    if hi == 1:
        idx = idx.expand(b, hkv, -1)
    items = idx.shape[1]
    blk = idx.clamp(min=0)
    k, v = _rows(s, 0, blk).flatten(2, 3), _rows(s, 1, blk).flatten(2, 3)
    per = hkv // items if items < hkv else items // hkv
    if c["fp8"]:
        k = k * s["k_scale"].repeat_interleave(per)[None, :, None, None]
        v = v * s["v_scale"].repeat_interleave(per)[None, :, None, None]
    q = s["q"].float().view(b, items, hq // items, D)
    logits = (q @ k.transpose(-1, -2)) / math.sqrt(D)
    pos = (blk[..., None] * BLK + torch.arange(BLK, device=DEV)).flatten(2)
    there = (idx >= 0).repeat_interleave(BLK, -1) & (pos < s["lens"].long().view(b, 1, 1))
    logits = logits.masked_fill(~there[:, :, None], -math.inf)
    p = torch.exp(logits - logits.amax(-1, keepdim=True))
    s["out"].copy_(((p / p.sum(-1, keepdim=True)) @ v).view(b, hq, D))
    return s["out"]


_PLAIN = {"page_map": _page_map, "kv_write": _kv_write, "block_bounds": _block_bounds, "block_select": _block_select,
          "block_attn": _block_attn}


def run(state):
    return _own(state) if own else _PLAIN[state["op"]](state)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

def _e4m3(x):
    """The nearest E4M3 value of each number in 64 bits, ties to the even code, from the format's definition:
    steps of 2^(e-3) between 2^e and 2^(e+1), of 2^-9 below 2^-6, at most 448."""
    a = x.abs().clamp(max=448.0)
    e = (torch.frexp(a).exponent - 1).clamp(min=-6)
    step = torch.exp2(e.double() - 3.0)
    n = a / step
    low = torch.floor(n)
    up = (n - low > 0.5) | ((n - low == 0.5) & (low % 2 == 1))
    return torch.sign(x) * (low + up) * step


def _sequence(s, which, b):
    """All keys or values of sequence b in 64 bits, [Hkv, positions, 128], scales taken in."""
    c, n = s["case"], int(s["lens"][b])
    held = s["buf"].view(torch.uint8) if c["fp8"] else s["buf"]
    if "table" in s:
        x = held[s["table"][b, : _pages(n)].long()][..., which, :].permute(1, 0, 2, 3)
    else:
        x = held[b][..., which, :]
    x = x.reshape(c["hkv"], -1, D)[:, :n].contiguous()
    if c["fp8"]:
        x = x.view(torch.float8_e4m3fn).to(torch.float32)
    x = x.double()
    scale = s["v_scale" if which else "k_scale"]
    return x, (x if scale is None else x * scale.double()[:, None, None])


def exact(case, seed):
    if case["op"] == "page_map":
        return None                                        # whole numbers only
    s = prepare(case, seed)
    op, b, hq, hkv = case["op"], case["batch"], case["hq"], case["hkv"]
    if op == "kv_write":
        out = s["buf"].float().double() if not case["fp8"] else s["buf"].to(torch.float32).double()
        for i, new, scale in ((0, s["k_new"], s["k_scale"]), (1, s["v_new"], s["v_scale"])):
            new = new.double() if scale is None else _e4m3(new.double() / scale.double()[:, None])
            view = out[:, :, :, i].transpose(1, 2)         # [page, 16, Hkv, 128]
            view[s["slots"] // BLK, s["slots"] % BLK] = new
        return out
    if op == "block_bounds":
        out = s["bounds"].double()
        for i in range(b):
            keys, n, first = _sequence(s, 0, i)[0], int(s["lens"][i]), int(s["old"][i]) // BLK
            for j in range(first, _pages(n)):
                if j == first and n // BLK > first:        # the whole blocks at once, the ragged one by itself
                    whole = keys[:, first * BLK: n // BLK * BLK].reshape(hkv, -1, BLK, D)
                    both = torch.stack((whole.amin(2), whole.amax(2)), 2)
                    if "table" in s:
                        out[s["table"][i, first: n // BLK].long()] = both.transpose(0, 1)
                    else:
                        out[i, :, first: n // BLK] = both
                if j >= n // BLK:
                    rows = keys[:, j * BLK: n]
                    at = (int(s["table"][i, j]),) if "table" in s else (i, slice(None), j)
                    out[at] = torch.stack((rows.amin(1), rows.amax(1)), 1)
        return out
    hi = _index_heads(case)
    if op == "block_select":
        idx = torch.full((b, hi, case["m"]), -1, dtype=torch.int64, device=DEV)
        count = torch.zeros(b, dtype=torch.int64, device=DEV)
        bounds = s["bounds"]
        for i in range(b):
            have = _pages(int(s["lens"][i]))
            mine = (bounds[s["table"][i, :have].long()].transpose(0, 1) if "table" in s else bounds[i, :, :have]).double()
            total = torch.zeros(hi, have, dtype=torch.float64, device=DEV)
            for h in range(hq):
                g = h // (hq // hkv)
                q = s["q"][i, h].double()
                one = torch.maximum(q * mine[g, :, 0], q * mine[g, :, 1]).sum(-1)
                total[h * hi // hq] += one if s["k_scale"] is None else one * s["k_scale"][g].double()
            blk = torch.arange(have, device=DEV)
            total[:, (blk < case["first"]) | (blk >= have - case["last"])] = math.inf
            c = min(case["m"], have)
            idx[i, :, :c] = torch.sort(total, dim=-1, descending=True, stable=True).indices[:, :c].sort(-1).values
            count[i] = c
        return [idx, count]
    out = torch.zeros(b, hq, D, dtype=torch.float64, device=DEV)
    for i in range(b):
        k, v, n = _sequence(s, 0, i)[1], _sequence(s, 1, i)[1], int(s["lens"][i])
        for h in range(hq):
            blk = s["idx"][i, h * hi // hq].long()
            pos = (blk[blk >= 0][:, None] * BLK + torch.arange(BLK, device=DEV)).flatten()
            pos = pos[pos < n]
            g = h // (hq // hkv)
            out[i, h] = torch.softmax((k[g, pos] @ s["q"][i, h].double()) / math.sqrt(D), 0) @ v[g, pos]
    return out
