"""What is measured of a served prompt's way through the cache: queries and keys normed, rotated to their positions and written
(rope), attention of a chunk of new tokens over everything cached (attn), the attention weight that every cached position
receives (weights), and the eviction of the positions that received least (evict). Every operator stands here in its plain form
(elementary torch operations) and as the calls of the framework's own operators; `own` says which of the two run() takes.

Caches are those of perf/operators.py: bf16, or E4M3 codes with a scale per KV head, a position's key row followed by its value
row, [page][Hkv][16][2][128] paged or [batch][Hkv][positions][2][128]. Queries, keys and values of new tokens are slices of a
fused projection's output [tokens][Hq + 2 Hkv][128]. Sizes are those of the benchmark's configurations (8/2 heads at 4096; 32/8
heads at 131072 with 4096 selected tokens; a ragged batch of 8 up to 65536 with 2048) and generic ones.
"""
import math
from types import SimpleNamespace

import torch

own = False

D = 128          # head dimension
PAGE = 16        # positions per page
EPS = 1e-6
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
        # a decode step of 64 running requests: queries and keys rotated, frequencies scaled by wavelength
        _case("rope", "rope: 64 tokens", tokens=64, far=131072, rotary=128, half=True, scaling="bands", norm=False, write=False),
        # a long prompt's queries and keys, normed per head, half of each head rotated in the interleaved layout
        _case("rope", "rope: 16384 tokens normed", tokens=16384, far=16384, rotary=64, half=False, scaling="none", norm=True, write=False),
        # the same on the way into an 8-bit paged cache: keys normed, rotated and quantised, values quantised
        _case("rope", "rope: 32768 tokens into fp8", tokens=32768, far=32768, rotary=128, half=True, scaling="ramp", norm=True, write=True,
              paged=True, fp8=True),
        # a short chunk after a short context: speculative tokens to be verified
        _case("attn", "attn: 7 after 4096", hq=8, hkv=2, ctx=4103, new_min=7, new=7),
        # a decode step of 64 running requests, one token each
        _case("attn", "attn: 64 requests, 1 token", batch=64, ctx_min=33, ctx=16384, new_min=1, new=1, paged=True),
        # a batch in which some sequences bring a chunk of their prompt and others a token, over an 8-bit cache
        _case("attn", "attn: 8x65536 ragged fp8", batch=8, ctx_min=8192, ctx=65536, new_min=1, new=1000, paged=True, fp8=True),
        # the last chunk of a 128K prompt
        _case("attn", "attn: 4096 of 131072", ctx=131072, new_min=4096, new=4096),
        # a decode step of 64 running requests: what every cached position received from the new token
        _case("weights", "weights: 64 requests, 1 token", batch=64, ctx_min=33, ctx=16384, new_min=1, new=1, paged=True),
        # the last 64 queries of a 128K prompt decide what is kept of it
        _case("weights", "weights: 64 of 131072", ctx=131072, new_min=64, new=64),
        # 64 running requests that have grown a page past their budget, one set of positions for all heads
        _case("evict", "evict: 64 requests to 2048", batch=64, ctx_min=1000, ctx=2064, m=2048, shared=True, first=4, last=64, paged=True),
        # a 128K prompt down to as many tokens as the token selection keeps, a set per KV head
        _case("evict", "evict: 131072 to 4096", ctx=131072, m=4096, shared=False, first=4, last=64),
        # a ragged 8-bit batch
        _case("evict", "evict: 8x65536 fp8 to 2048", batch=8, ctx_min=8192, ctx=65536, m=2048, shared=False, first=0, last=32, paged=True, fp8=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "attn", "attn", "weights", "evict"])
    hkv, g = rng.choice([(1, 8), (2, 4), (3, 5), (4, 1), (4, 7), (8, 4), (8, 8), (8, 2), (16, 1), (5, 3)])
    c = dict(hq=hkv * g, hkv=hkv, paged=rng.random() < 0.6, fp8=rng.random() < 0.4)
    if op == "rope":
        write = rng.random() < 0.5
        c.update(tokens=_log(rng, 1, 32768 * 48 // max(hkv * (g + 2), 48)), far=_log(rng, 16, 262144), rotary=rng.choice([128, 128, 64, 32, 96, 16]),
                 half=rng.random() < 0.6, scaling=rng.choice(["none", "linear", "base", "bands", "ramp"]), norm=rng.random() < 0.5, write=write)
        c.update(paged=True, fp8=c["fp8"] and write)
        return _case(op, **c)
    b = _log(rng, 1, 64)
    ctx = _log(rng, 20, max(64, min(131072, 1048576 * 8 // (max(hkv, 8) * b))))
    c.update(batch=b, ctx=ctx, ctx_min=_log(rng, 1, ctx))
    if op == "evict":
        c.update(m=_log(rng, 1, max(2, min(8192, ctx, 65536 // b))), shared=rng.random() < 0.3, first=rng.choice([0, 0, 1, 4]), last=rng.choice([0, 1, 32, 64]))
        return _case(op, **c)
    # at most the work of the largest listed one (rows of all heads times positions)
    most = 32 * 4096 * 100000 if op == "attn" else 32 * 64 * 131072
    new = _log(rng, 1, max(1, min(ctx, 4096, most // (b * hkv * g * ctx))))
    c.update(new=new, new_min=rng.choice([new, 1, _log(rng, 1, new)]))
    return _case(op, **c)


def _steps(lo, hi, n):
    return [hi - (hi - lo) * i // max(n - 1, 1) for i in range(n)]


def _lens(case):
    """The sequences' lengths, new tokens included: even steps from ctx_min to ctx (their order comes from the seed)."""
    return _steps(case["ctx_min"], case["ctx"], case["batch"])


def _new(case):
    """New tokens of each sequence: the longest chunk beside the shortest context, as far as that holds it."""
    return [min(a, n) for a, n in zip(_steps(case["new_min"], case["new"], case["batch"])[::-1], _lens(case))]


def _pages(n):
    return (n + PAGE - 1) // PAGE


def _visible(case):
    """Pairs of a query and a position that it sees, of one head."""
    return sum(a * (n - a) + a * (a + 1) // 2 for a, n in zip(_new(case), _lens(case)))


def work(case):
    op, hq, hkv = case["op"], case["hq"], case["hkv"]
    esz = 1 if case["fp8"] else 2
    if op == "rope":
        t = case["tokens"]
        rows = t * (hq + hkv)
        size = rows * D * 2 + t * hq * D * 2 + t * 4
        size += t * hkv * D * (2 + 2 * esz) + t * 8 if case["write"] else t * hkv * D * 2
        return {"bytes": size, "flops": rows * (3 * case["rotary"] + (4 * D if case["norm"] else 0))}
    lens = _lens(case)
    if op == "attn":
        rows = sum(_new(case)) * hq
        return {"bytes": sum(lens) * hkv * 2 * D * esz + rows * (2 * D * 2 + 4), "flops": 4 * D * hq * _visible(case)}
    if op == "weights":
        rows = sum(_new(case)) * hq
        return {"bytes": sum(lens) * hkv * (D * esz + 4) + rows * (D * 2 + 4), "flops": 2 * D * hq * _visible(case)}
    ha, kept = 1 if case["shared"] else hkv, sum(min(case["m"], n) for n in lens)
    return {"bytes": sum(lens) * ha * 4 + kept * (2 * hkv * 2 * D * esz + 8 * ha), "flops": 0}


# ---- inputs ------------------------------------------------------------------------------------------------------

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(1000003 * (seed + 1))


def _normal(g, *shape):
    return torch.empty(*shape, dtype=torch.bfloat16, device=DEV).normal_(generator=g)


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device=DEV)


def _table(g, lens, total):
    table = torch.zeros(len(lens), max(_pages(max(lens)), 1), dtype=torch.int32, device=DEV)
    perm = torch.randperm(total, generator=g, device=DEV).to(torch.int32)
    at = 0
    for i, n in enumerate(lens):
        table[i, : _pages(n)] = perm[at: at + _pages(n)]
        at += _pages(n)
    return table


def _cache(s, case, g, lens):
    """A filled cache: normal keys and values, a few key channels off centre as trained models have them."""
    hkv = case["hkv"]
    if case["paged"]:
        total = sum(map(_pages, lens)) + 5
        buf = _normal(g, total, hkv, PAGE, 2, D)
        s["table"] = _table(g, lens, total)
    else:
        buf = _normal(g, len(lens), hkv, _pages(max(lens)) * PAGE, 2, D)
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


def _layer(s, case, buf, table, lens, max_len):
    """The descriptor of a cache as the framework's binding takes it."""
    hkv, paged = case["hkv"], table is not None
    if not paged:
        buf = buf.view(buf.shape[0], hkv, -1, 2, D)
    st = buf.stride()
    return SimpleNamespace(
        k=buf.select(-2, 0), v=buf.select(-2, 1), batch=lens.numel(), num_q_heads=case["hq"], num_kv_heads=hkv, head_dim=D,
        ctx_lens=lens, max_ctx_len=max_len, stride_b=0 if paged else st[0], stride_pos=2 * D, stride_head=st[1],
        stride_page=st[0] if paged else 0, page_table=table, page_size=PAGE, max_pages_per_seq=table.shape[1] if paged else 0,
        num_pages=buf.shape[0] if paged else 0, sm_scale=0.0, keep=[buf], kv_dtype=1 if case["fp8"] else 0, k_scale=s["k_scale"],
        v_scale=s["v_scale"])


_handles = {}


def _handle(half):
    """The framework's contexts on this GPU, for the whole program: one that writes fp32 outputs, one that writes bf16."""
    from paper_2410_05076_b200 import binding
    if half not in _handles:
        _handles[half] = binding.Tidal(0)
        _handles[half].set_output_bf16(half)
    return binding, _handles[half]


# How rotary frequencies are stretched for contexts beyond the trained one: (factor, low, high, trained length).
BASE = 500000.0
STRETCH = {"none": (1.0, 0.0, 0.0, 0.0), "linear": (4.0, 0.0, 0.0, 0.0), "base": (8.0, 0.0, 0.0, 0.0),
           "bands": (8.0, 1.0, 4.0, 8192.0), "ramp": (16.0, 1.0, 32.0, 8192.0)}


def _frequencies(case):
    """Radians per position of every pair of channels, and the factor on cosines and sines."""
    n, (factor, low, high, trained) = case["rotary"], STRETCH[case["scaling"]]
    base = BASE * factor ** (n / (n - 2)) if case["scaling"] == "base" else BASE
    f = [base ** (-2.0 * i / n) for i in range(n // 2)]
    if case["scaling"] == "linear":
        f = [x / factor for x in f]
    if case["scaling"] == "bands":                        # long wavelengths are stretched, short ones are not
        mix = [min(max((trained * x / (2 * math.pi) - low) / (high - low), 0.0), 1.0) for x in f]
        f = [(1 - m) * x / factor + m * x for m, x in zip(mix, f)]
    if case["scaling"] == "ramp":                         # a ramp over the channels that turn `high` to `low` times
        at = lambda turns: n * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(BASE))  # noqa: E731
        lo, hi = max(math.floor(at(high)), 0), min(math.ceil(at(low)), n - 1)
        ramp = [min(max((i - lo) / max(hi - lo, 0.001), 0.0), 1.0) for i in range(n // 2)]
        f = [x / factor * r + x * (1 - r) for r, x in zip(ramp, f)]
        return f, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _prepare_rope(s, case, g):
    t, hq, hkv = case["tokens"], case["hq"], case["hkv"]
    qkv = _normal(g, t, hq + 2 * hkv, D)
    s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq: hq + hkv], qkv[:, hq + hkv:]
    s["pos"] = torch.randint(0, case["far"], (t,), generator=g, device=DEV, dtype=torch.int32)
    if t > case["far"] // 2:                              # a prompt's positions, in order
        s["pos"] = torch.arange(t, device=DEV, dtype=torch.int32) % case["far"]
    s["qw"] = s["kw"] = None
    if case["norm"]:
        s["qw"], s["kw"] = [(1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(torch.bfloat16) for _ in range(2)]
    s["q_out"] = torch.zeros(t, hq, D, dtype=torch.bfloat16, device=DEV)
    f, s["factor"] = _frequencies(case)
    s["freq"] = _ints(f, torch.float64)
    if case["write"]:
        pages = _pages(t) + 3
        _cache(s, dict(case, batch=1), g, [pages * PAGE])
        at = torch.randperm(pages, generator=g, device=DEV)[:, None] * PAGE + torch.arange(PAGE, device=DEV)
        s["slots"] = at.reshape(-1)[:t].contiguous()
    else:
        s["k_out"] = torch.zeros(t, hkv, D, dtype=torch.bfloat16, device=DEV)
    if own:
        binding = _handle(False)[0]
        kinds = {"none": binding.ROPE_PLAIN, "linear": binding.ROPE_LINEAR, "base": binding.ROPE_BASE, "bands": binding.ROPE_BANDS,
                 "ramp": binding.ROPE_RAMP}
        factor, low, high, trained = STRETCH[case["scaling"]]
        s["plan"] = binding.rope_plan(case["rotary"], base=BASE, layout=binding.ROPE_HALF if case["half"] else binding.ROPE_INTERLEAVED,
                                      scaling=kinds[case["scaling"]], factor=factor, low=low, high=high, trained_len=trained)
        if case["write"]:
            lens = _ints([s["table"].shape[1] * PAGE])
            s["lens"] = lens
            s["kv"] = binding.kv_struct(_layer(s, case, s["buf"], s["table"], lens, s["table"].shape[1] * PAGE))


def prepare(case, seed):
    g = _gen(seed)
    op, b, hq, hkv = case["op"], case["batch"], case["hq"], case["hkv"]
    s = {"case": case, "op": op}
    if op == "rope":
        _prepare_rope(s, case, g)
        return s
    order = torch.randperm(b, generator=torch.Generator().manual_seed(seed + 17)).tolist()
    lens = [_lens(case)[i] for i in order]
    s["host_lens"], s["lens"] = lens, _ints(lens)
    _cache(s, case, g, lens)
    table = s.get("table")
    if own:
        s["kv"] = _handle(op == "attn")[0].kv_struct(_layer(s, case, s["buf"], table, s["lens"], max(lens)))
    if op == "evict":
        ha, m = 1 if case["shared"] else hkv, case["m"]
        wide = (max(lens) + 63) // 64 * 64
        w = torch.rand(b, ha, wide, generator=g, device=DEV)
        s["w"] = (w * w * w).pow_(4)                      # most positions receive little, few a lot
        s["w"][..., ::7] = 0.0                            # and some nothing: ties
        s["w_out"] = torch.zeros(b, ha, m, device=DEV)
        s["kept"] = torch.zeros(b, ha, m, dtype=torch.int32, device=DEV)
        s["count"] = torch.zeros(b, dtype=torch.int32, device=DEV)
        outs = [min(m, n) for n in lens]
        shape = list(s["buf"].shape)                      # kept rows go to fresh pages, as where prompts share theirs
        shape[0 if case["paged"] else 2] = sum(map(_pages, outs)) + 3 if case["paged"] else _pages(max(outs)) * PAGE
        s["to"] = torch.zeros(shape, dtype=torch.uint8 if case["fp8"] else torch.bfloat16, device=DEV)
        if case["fp8"]:
            s["to"] = s["to"].view(torch.float8_e4m3fn)
        s["to_table"] = _table(g, outs, shape[0]) if case["paged"] else None
        if own:
            s["kv_to"] = _handle(False)[0].kv_struct(_layer(s, case, s["to"], s["to_table"], s["count"], max(outs)))
        return s
    new = [_new(case)[i] for i in order]
    s["new"], s["max_new"] = new, max(new)
    t = sum(new)
    s["offsets"] = _ints([sum(new[:i]) for i in range(b + 1)])
    s["q"] = _normal(g, t, hq + 2 * hkv, D)[:, :hq]
    if op == "attn":
        s["out"] = torch.zeros(t, hq, D, dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.zeros(t, hq, device=DEV)
    else:
        s["lse"] = _chunks(s, torch.float32, None, None, torch.zeros(t, hq, device=DEV))
        s["w"] = torch.zeros(b, hkv, (max(lens) + 63) // 64 * 64, device=DEV)
    return s


# ---- the framework's operators -----------------------------------------------------------------------------------

def _own(s):
    op, c = s["op"], s["case"]
    td = _handle(op == "attn")[1]
    if op == "rope":
        if c["write"]:
            td.rope_write(s["kv"], s["plan"], s["q"], s["k"], s["v"], s["pos"], s["slots"], q_weight=s["qw"], k_weight=s["kw"], eps=EPS, q_out=s["q_out"])
            return [s["q_out"], s["buf"]]
        return list(td.rope(s["plan"], s["q"], s["k"], s["pos"], q_weight=s["qw"], k_weight=s["kw"], eps=EPS, q_out=s["q_out"], k_out=s["k_out"]))
    if op == "attn":
        td.chunk_attn(s["kv"], s["q"], s["offsets"], max_new=s["max_new"], out=s["out"], lse=s["lse"])
        return [s["out"], s["lse"]]
    if op == "weights":
        return td.chunk_weights(s["kv"], s["q"], s["offsets"], s["lse"], s["w"], decay=0.0, max_new=s["max_new"])
    td.evict_select(s["kv"], s["w"], c["m"], keep_first=c["first"], keep_last=c["last"], kept=s["kept"], new_lens=s["count"])
    td.kv_gather(s["kv"], s["kept"], s["count"], into=s["kv_to"], weights=s["w"], weights_out=s["w_out"])
    return [s["kept"], s["count"], s["to"], s["w_out"]]


# ---- the plain forms ---------------------------------------------------------------------------------------------

def _turned(s, x, weight):
    """Rows [T, H, 128] normed and rotated, in 32 bits; the angles in 64."""
    c = s["case"]
    n = c["rotary"]
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    angle = s["pos"].double()[:, None] * s["freq"][None]
    cos, sin = [(f(angle) * s["factor"]).float()[:, None] for f in (torch.cos, torch.sin)]
    head = x[..., :n]
    a, b = (head[..., : n // 2], head[..., n // 2:]) if c["half"] else (head[..., ::2], head[..., 1::2])
    a, b = a * cos - b * sin, b * cos + a * sin
    head = torch.cat((a, b), -1) if c["half"] else torch.stack((a, b), -1).flatten(-2)
    return torch.cat((head, x[..., n:]), -1)


def _rope(s):
    c = s["case"]
    s["q_out"].copy_(_turned(s, s["q"], s["qw"]))
    k = _turned(s, s["k"], s["kw"])
    if not c["write"]:
        s["k_out"].copy_(k)
        return [s["q_out"], s["k_out"]]
    page, place = s["slots"] // PAGE, s["slots"] % PAGE
    buf, fp8 = s["buf"], c["fp8"]
    held = buf.view(torch.uint8) if fp8 else buf
    heads = torch.arange(buf.shape[1], device=DEV)[None, :]
    for i, new, scale in ((0, k, s["k_scale"]), (1, s["v"].float(), s["v_scale"])):
        if fp8:
            new = (new / scale[:, None]).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
        held[:, :, :, i][page[:, None], heads, place[:, None]] = new.to(held.dtype)
    return [s["q_out"], buf]


def _rows(s, which, b, dtype):
    """The keys (0) or values (1) of sequence b, [Hkv, positions, 128], scales taken in."""
    c, n = s["case"], s["host_lens"][b]
    held = s["buf"].view(torch.uint8) if c["fp8"] else s["buf"]
    if c["paged"]:
        x = held[s["table"][b, : _pages(n)].long()][..., which, :].permute(1, 0, 2, 3)
    else:
        x = held[b][..., which, :]
    x = x.reshape(c["hkv"], -1, D)[:, :n].contiguous()
    if not c["fp8"]:
        return x.to(dtype)
    return x.view(torch.float8_e4m3fn).float().to(dtype) * s["v_scale" if which else "k_scale"].to(dtype)[:, None, None]


def _chunks(s, dtype, out, weights, lse):
    """Softmax over the positions up to each query's own, sequence by sequence, KV head by KV head and a block of queries at a
    time: `out` and `lse` are filled, or, given lse, `weights` with the sums of exp(logit - lse) over a KV head's queries."""
    c = s["case"]
    hkv, G = c["hkv"], c["hq"] // c["hkv"]
    at = 0
    for b, (n, new) in enumerate(zip(s["host_lens"], s["new"])):
        keys, values = _rows(s, 0, b, dtype), _rows(s, 1, b, dtype) if out is not None else None
        together = hkv if hkv * new * G * n <= 1 << 26 else 1          # all heads at once where they are small
        step = max(1, (1 << 29) // (together * G * n))
        pos = torch.arange(n, device=DEV)
        for h in range(0, hkv, together):
            for t in range(0, new, step):
                m = min(step, new - t)
                rows = slice(at + t, at + t + m)
                q = s["q"][rows, h * G: (h + together) * G].to(dtype).view(m, together, G, D).permute(1, 2, 0, 3)
                logits = q.reshape(together, G * m, D) @ keys[h: h + together].transpose(-1, -2)
                logits = logits.mul_(1 / math.sqrt(D)).view(together, G, m, n)
                hidden = pos > (n - new + t + torch.arange(m, device=DEV))[:, None]
                logits.masked_fill_(hidden, -math.inf)
                if weights is not None:
                    given = lse[rows, h * G: (h + together) * G].to(dtype).view(m, together, G).permute(1, 2, 0)
                    weights[b, h: h + together, :n] += torch.exp(logits - given[..., None]).sum((1, 2))
                    continue
                top = logits.amax(-1, keepdim=True)
                p = torch.exp_(logits.sub_(top))
                total = p.sum(-1, keepdim=True)
                back = lambda x, w: x.reshape(together, G, m, w).permute(2, 0, 1, 3).reshape(m, together * G, w)  # noqa: E731
                lse[rows, h * G: (h + together) * G] = back(top + torch.log(total), 1)[..., 0].to(lse.dtype)
                if out is not None:
                    o = (p.view(together, G * m, n) @ values[h: h + together]).view(together, G, m, D) / total
                    out[rows, h * G: (h + together) * G] = back(o, D).to(out.dtype)
        at += new
    return weights if weights is not None else lse


def _attn(s):
    _chunks(s, torch.float32, s["out"], None, s["lse"])
    return [s["out"], s["lse"]]


def _weights(s):
    w = s["w"]
    w.copy_(_chunks(s, torch.float32, None, torch.zeros_like(w), s["lse"]))
    return w


def _evict(s):
    """The positions of the largest weights, the first and last ones among them, in ascending order; then their rows."""
    c = s["case"]
    b, hkv, m, w = c["batch"], c["hkv"], c["m"], s["w"]
    ha, n = w.shape[1:]
    have = s["lens"].long().view(b, 1, 1)
    pos = torch.arange(n, device=DEV)
    rank = torch.where((pos < c["first"]) | (pos >= have - c["last"]), math.inf, w).masked_fill(pos >= have, -math.inf)
    best = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :m]
    if best.shape[-1] < m:
        best = torch.cat((best, best.new_full((b, ha, m - best.shape[-1]), n)), -1)
    there = torch.arange(m, device=DEV) < have
    best = torch.where(there, best, n).sort(-1).values
    s["kept"].copy_(torch.where(best < n, best, -1))
    s["count"].copy_(have.clamp(max=m).view(b))
    s["w_out"].copy_(torch.where(there, w.gather(-1, best.clamp(max=n - 1)), s["w_out"]))
    held, to = [x.view(torch.uint8) if c["fp8"] else x for x in (s["buf"], s["to"])]
    for i in range(b):
        k = min(m, s["host_lens"][i])
        src, dst = best[i, :, :k].expand(hkv, k), torch.arange(k, device=DEV)
        heads = torch.arange(hkv, device=DEV)[:, None]
        rows = held[s["table"][i, src // PAGE].long(), heads, src % PAGE] if c["paged"] else held[i, heads, src]
        if c["paged"]:
            to[s["to_table"][i, dst // PAGE].long()[None], heads, (dst % PAGE)[None]] = rows
        else:
            to[i, :, :k] = rows
    return [s["kept"], s["count"], s["to"], s["w_out"]]


_PLAIN = {"rope": _rope, "attn": _attn, "weights": _weights, "evict": _evict}


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


def _exact_rope(s, case):
    n = case["rotary"]
    turn = torch.polar(torch.full_like(s["freq"], s["factor"]), torch.zeros_like(s["freq"]))[None] * torch.exp(
        1j * torch.outer(s["pos"].double(), s["freq"]))
    ways = torch.arange(n, device=DEV).view(2, -1) if case["half"] else torch.arange(n, device=DEV).view(-1, 2).t()

    def rows(x, weight):
        x = x.double()
        if weight is not None:
            x = x / torch.sqrt((x ** 2).sum(-1, keepdim=True) / D + EPS) * weight.double()
        out = x.clone()
        for h in range(x.shape[1]):                       # a pair of channels is a complex number, the rotation a product
            z = torch.complex(x[:, h, ways[0]], x[:, h, ways[1]]) * turn
            out[:, h, ways[0]], out[:, h, ways[1]] = z.real, z.imag
        return out

    q, k = rows(s["q"], s["qw"]), rows(s["k"], s["kw"])
    if not case["write"]:
        return [q, k]
    buf = s["buf"].to(torch.float32).double()
    for i, new, scale in ((0, k, s["k_scale"]), (1, s["v"].double(), s["v_scale"])):
        if scale is not None:
            new = _e4m3(new / scale.double()[:, None])
        buf[:, :, :, i].transpose(1, 2)[s["slots"] // PAGE, s["slots"] % PAGE] = new
    return [q, buf]


def exact(case, seed):
    op, hq, hkv = case["op"], case["hq"], case["hkv"]
    if op == "evict":
        return None                                        # positions, and rows moved as they are
    s = prepare(case, seed)
    if op == "rope":
        return _exact_rope(s, case)
    if hq * _visible(case) > 2e10:
        return None
    t, G = sum(s["new"]), hq // hkv
    out, lse = torch.zeros(t, hq, D, dtype=torch.float64, device=DEV), torch.zeros(t, hq, dtype=torch.float64, device=DEV)
    w = torch.zeros(s["w"].shape, dtype=torch.float64, device=DEV) if op == "weights" else None
    at = 0
    for b, (n, new) in enumerate(zip(s["host_lens"], s["new"])):
        k, v = _rows(s, 0, b, torch.float64), _rows(s, 1, b, torch.float64)
        for h in range(hq):
            for t0 in range(0, new, max(1, (1 << 28) // n)):
                t1 = min(new, t0 + max(1, (1 << 28) // n))
                x = s["q"][at + t0: at + t1, h].double() @ k[h // G].t() / math.sqrt(D)
                own_pos = torch.arange(n - new + t0, n - new + t1, device=DEV)
                x = torch.where(torch.arange(n, device=DEV)[None] <= own_pos[:, None], x, -math.inf)
                if w is not None:
                    w[b, h // G, :n] += torch.exp(x - s["lse"][at + t0: at + t1, h].double()[:, None]).sum(0)
                else:
                    lse[at + t0: at + t1, h] = torch.logsumexp(x, 1)
                    out[at + t0: at + t1, h] = torch.softmax(x, 1) @ v[h // G]
        at += new
    return w if w is not None else [out, lse]
