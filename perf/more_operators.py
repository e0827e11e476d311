"""The operators between a language-model block's q/k/v product and its output product, as measurable cases.

rope    norms of queries and keys for each head and the rotation by their positions in one pass, keys and values written
        into the pages of a cache (``dsq_qk_norm_rope``): a serving step.
rtrain  the same in a training step, with positions of several axes: forward, then ``dsq_qk_norm_rope_bwd``.
attn    attention over whole prompts, packed one behind the other, causal, grouped heads (``dsq_attention``).
atrain  the same in a training step: forward, then ``dsq_attention_bwd``.
cache   attention of single tokens or of trees of drafted tokens over a paged cache (``dsq_attention_cache``).

Queries, keys and values are the parts of one tensor, as the product before them leaves it.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6

# Most of a drawn case: elements of a norm, padded scores of a prompt and of a training step, operations of a prompt, elements of a cache.
MAX_NORM = 8192 * 40 * 128
MAX_SCORES, MAX_TRAIN_SCORES = 16 * 16384 * 16384, 1 << 30
MAX_FLOPS = 4 * 128 * 16 * 16384 * 16384 // 2
MAX_CACHE = 32 * 8192 * 8 * 128


def listed():
    return [
        # A decoding batch of a few requests: the smallest call, latency.
        dict(name="rope.tokens.8", kind="rope", rows=8, q_heads=32, kv_heads=8, dim=128, rope_dim=128, axes=1, interleaved=False, page=64, dtype="bf16"),
        # A prompt.
        dict(name="rope.prompt.4096", kind="rope", rows=4096, q_heads=32, kv_heads=8, dim=128, rope_dim=128, axes=1, interleaved=False, page=64, dtype="bf16"),
        # A training step over images: time, height and width, some of each head's elements not rotated, full precision.
        dict(name="rtrain.images.f32", kind="rtrain", rows=5000, q_heads=12, kv_heads=4, dim=80, rope_dim=48, axes=3, interleaved=True, dtype="f32"),
        # One prompt of ordinary length.
        dict(name="attn.prompt.4096", kind="attn", sequences=1, longest=4096, ragged=False, context=0, q_heads=32, kv_heads=8, dim=128, causal=True, dtype="bf16"),
        # Short prompts of many lengths, small heads.
        dict(name="attn.packed.16x1000", kind="attn", sequences=16, longest=1000, ragged=True, context=0, q_heads=16, kv_heads=16, dim=64, causal=True, dtype="f16"),
        # A long prompt.
        dict(name="attn.long.16384", kind="attn", sequences=1, longest=16384, ragged=False, context=0, q_heads=16, kv_heads=2, dim=128, causal=True, dtype="bf16"),
        # A training step's micro-batch.
        dict(name="atrain.4x2048", kind="atrain", sequences=4, longest=2048, ragged=False, context=0, q_heads=16, kv_heads=4, dim=128, causal=True, dtype="bf16"),
        # Odd lengths, more keys than queries, a head of 80 elements, full precision.
        dict(name="atrain.odd.f32", kind="atrain", sequences=3, longest=701, ragged=True, context=50, q_heads=6, kv_heads=2, dim=80, causal=True, dtype="f32"),
        # One token over a short context: latency.
        dict(name="cache.token.1x500", kind="cache", sequences=1, longest=500, ragged=False, drafted=1, q_heads=32, kv_heads=8, dim=128, page=16, dtype="bf16"),
        # A decoding batch of requests of many lengths: the cache comes from memory.
        dict(name="cache.batch.32x8192", kind="cache", sequences=32, longest=8192, ragged=True, drafted=1, q_heads=32, kv_heads=8, dim=128, page=64, dtype="bf16"),
        # One token over a long context.
        dict(name="cache.long.1x131072", kind="cache", sequences=1, longest=131072, ragged=False, drafted=1, q_heads=32, kv_heads=4, dim=128, page=128, dtype="bf16"),
        # Trees of drafted tokens.
        dict(name="cache.tree.8x4096", kind="cache", sequences=8, longest=4096, ragged=True, drafted=48, q_heads=32, kv_heads=8, dim=128, page=64, dtype="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "rtrain", "attn", "attn", "atrain", "cache", "cache"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    while True:
        kv_heads = rng.choice([1, 2, 4, 8, rng.randint(1, 16)])
        q_heads = kv_heads * rng.choice([1, 2, 4, 8, rng.randint(1, 12)])
        dim = rng.choice([64, 128, 128, 8 * rng.randint(4, 16)])
        if q_heads > 64:
            continue
        heads = dict(q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=dtype)
        if kind in ("rope", "rtrain"):
            if rng.random() < 0.2:
                dim = heads["dim"] = rng.choice([192, 256])
            rows = _log(rng, 1, 16384)
            case = dict(kind=kind, rows=rows, rope_dim=rng.choice([dim // 16 * 16, 16 * rng.randint(1, dim // 16)]),
                        axes=rng.choice([1, 1, 2, 3]), interleaved=rng.random() < 0.4, **heads)
            if kind == "rope":
                case["page"] = rng.choice([1, 16, 64, 256])
            if rows * (q_heads + 2 * kv_heads) * dim <= MAX_NORM // (2 if dtype == "f32" else 1):
                return case
        elif kind in ("attn", "atrain"):
            longest, ragged = _log(rng, 1, 16384), rng.random() < 0.5
            case = dict(kind=kind, sequences=rng.choice([1, 1, _log(rng, 2, 64)]), longest=longest, ragged=ragged,
                        context=rng.choice([0, 0, _log(rng, 1, 1000)]), causal=rng.random() < 0.8, **heads)
            scores = case["sequences"] * q_heads * longest * (longest + case["context"])
            if scores <= (MAX_SCORES if kind == "attn" else MAX_TRAIN_SCORES) // (8 if dtype == "f32" else 1) and work(case)["flops"] <= MAX_FLOPS:
                return case
        else:
            drafted = rng.choice([1, 1, _log(rng, 2, 64)])
            case = dict(kind=kind, sequences=rng.choice([1, _log(rng, 2, 64)]), longest=drafted + _log(rng, 1, 131072), ragged=rng.random() < 0.6,
                        drafted=drafted, page=rng.choice([16, 64, 128, 256]), **heads)
            keys = case["sequences"] * case["longest"]
            if keys * kv_heads * dim <= MAX_CACHE // (2 if dtype == "f32" else 1) and keys * q_heads * drafted <= MAX_SCORES // 8:
                return case


def _sizes(case):
    """Rows and keys of each sequence: all the longest, or the first the longest and the others spread below it."""
    rng = random.Random(case["longest"] * 1009 + case["sequences"])
    if case["kind"] == "cache":
        n = case["drafted"]
        keys = [case["longest"] if i == 0 or not case["ragged"] else rng.randint(n, case["longest"]) for i in range(case["sequences"])]
        return [n if i == 0 or not case["ragged"] else rng.randint(1, n) for i in range(case["sequences"])], keys
    rows = [case["longest"] if i == 0 or not case["ragged"] else rng.randint(1, case["longest"]) for i in range(case["sequences"])]
    return rows, [n + case["context"] for n in rows]


# ---- inputs --------------------------------------------------------------------------------------

def _starts(sizes):
    at = [0]
    for n in sizes:
        at.append(at[-1] + n)
    return at


def _inputs(case, seed):
    """The tensors of a case, from its seed."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    dt, i32 = DTYPES[case["dtype"]], dict(dtype=torch.int32, device="cuda")
    hq, hk, dim = case["q_heads"], case["kv_heads"], case["dim"]
    if case["kind"] in ("rope", "rtrain"):
        rows, pairs = case["rows"], case["rope_dim"] // 2
        qkv = (normal(rows, hq + 2 * hk, dim) * torch.exp(0.5 * normal(1, hq + 2 * hk, 1))).to(dt)
        d = {"q": qkv[:, :hq], "k": qkv[:, hq:hq + hk], "v": qkv[:, hq + hk:], "q_weight": (1.0 + 0.2 * normal(dim)).to(dt),
             "k_weight": (1.0 + 0.2 * normal(dim)).to(dt),
             "positions": torch.randint(0, 32768, (case["axes"], rows), generator=g, **i32),
             "frequencies": torch.tensor([1e4 ** (-j / pairs) for j in range(pairs)], device="cuda"),
             # (the axes take turns from pair to pair)
             "pair_axis": (torch.arange(pairs, device="cuda") % case["axes"]).to(torch.uint8) if case["axes"] > 1 else None}
        if case["kind"] == "rope":
            pages = -(-rows // case["page"]) + 3
            d["slots"] = torch.randperm(pages * case["page"], generator=g, device="cuda")[:rows]
            d["k_cache"], d["v_cache"] = (torch.zeros(pages, hk, case["page"], dim, dtype=dt, device="cuda") for _ in range(2))
        else:
            d["grad_q_out"], d["grad_k_out"] = normal(rows, hq, dim).to(dt), normal(rows, hk, dim).to(dt)
        return d
    rows, keys = _sizes(case)
    d = {"q_starts": torch.tensor(_starts(rows), **i32)}
    if case["kind"] == "cache":
        page = case["page"]
        pages = [-(-n // page) for n in keys]
        order = torch.randperm(sum(pages), generator=g, device="cuda").to(torch.int32)
        table = torch.full((len(pages), max(pages)), -1, **i32)
        there = torch.arange(max(pages), device="cuda")[None] < torch.tensor(pages, device="cuda")[:, None]
        table[there] = order
        rng, words = random.Random(seed), []
        for n in rows:
            seen = []
            for i in range(n):
                parent = rng.randint(-1, i - 1)
                seen.append((seen[parent] if parent >= 0 else 0) | 1 << i)
            words += [[w - (1 << 64) if w >> 63 else w] for w in seen]
        d.update(q=(1.5 * normal(sum(rows), hq, dim)).to(dt), k_cache=normal(sum(pages), hk, page, dim).to(dt),
                 v_cache=normal(sum(pages), hk, page, dim).to(dt), table=table, lengths=torch.tensor(keys, **i32),
                 tree=torch.tensor(words, dtype=torch.int64, device="cuda") if case["drafted"] > 1 else None)
        return d
    if case["context"]:
        d["q"], kv = (1.5 * normal(sum(rows), hq, dim)).to(dt), normal(sum(keys), 2 * hk, dim).to(dt)
        d["k"], d["v"], d["k_starts"] = kv[:, :hk], kv[:, hk:], torch.tensor(_starts(keys), **i32)
    else:
        qkv = normal(sum(rows), hq + 2 * hk, dim)
        qkv[:, :hq] *= 1.5
        qkv = qkv.to(dt)
        d["q"], d["k"], d["v"], d["k_starts"] = qkv[:, :hq], qkv[:, hq:hq + hk], qkv[:, hq + hk:], d["q_starts"]
    if case["kind"] == "atrain":
        d["grad_out"] = normal(sum(rows), hq, dim).to(dt)
    return d


def prepare(case, seed):
    d = _inputs(case, seed)
    state = {"case": case, "in": d, "scale": case["dim"] ** -0.5}
    if own:
        from paper_1908_05033_amd import binding as B
        state["B"] = B
        like = lambda t: torch.empty(t.shape, dtype=t.dtype, device="cuda")
        buffer = lambda n: torch.empty(n, dtype=torch.uint8, device="cuda")
        hq, hk, dim = case["q_heads"], case["kv_heads"], case["dim"]
        out = state["out"] = {}
        if case["kind"] == "rope":
            out.update(q=like(d["q"]), k_cache=d["k_cache"], v_cache=d["v_cache"])
        elif case["kind"] == "rtrain":
            out.update(q=like(d["q"]), k=like(d["k"]), grad_q=like(d["q"]), grad_k=like(d["k"]),
                       grad_q_weight=torch.empty(dim, device="cuda"), grad_k_weight=torch.empty(dim, device="cuda"))
            state["workspace"] = buffer(B.dsq_qk_norm_rope_bwd_bytes(case["rows"], hq, hk, dim))
        else:
            out["out"] = like(d["q"])
            if case["kind"] == "atrain":
                out.update(grad_q=like(d["q"]), grad_k=like(d["k"]), grad_v=like(d["v"]))
                state["lse"] = torch.empty(hq, d["q"].shape[0], device="cuda")
                state["workspace"] = buffer(B.dsq_attention_bwd_bytes(d["q"].shape[0], hq))
            elif case["kind"] == "cache":
                state["workspace"] = buffer(B.dsq_attention_cache_bytes(case["sequences"], case["drafted"], hq, hk, dim))
    return state


# ---- one pass ------------------------------------------------------------------------------------

def _own(state):
    case, d, out, B = state["case"], state["in"], state["out"], state["B"]
    if case["kind"] == "rope":
        B.dsq_qk_norm_rope(d["q"], d["k"], d["v"], d["q_weight"], d["k_weight"], EPS, d["positions"], d["pair_axis"], d["frequencies"],
                           case["interleaved"], out["q"], None, d["k_cache"], d["v_cache"], d["slots"])
    elif case["kind"] == "rtrain":
        B.dsq_qk_norm_rope(d["q"], d["k"], None, d["q_weight"], d["k_weight"], EPS, d["positions"], d["pair_axis"], d["frequencies"],
                           case["interleaved"], out["q"], out["k"], None, None, None)
        B.dsq_qk_norm_rope_bwd(d["q"], d["k"], d["q_weight"], d["k_weight"], EPS, d["positions"], d["pair_axis"], d["frequencies"],
                               case["interleaved"], d["grad_q_out"], d["grad_k_out"], out["grad_q"], out["grad_k"],
                               out["grad_q_weight"], out["grad_k_weight"], state["workspace"])
    elif case["kind"] == "cache":
        B.dsq_attention_cache(d["q"], d["q_starts"], case["drafted"], d["k_cache"], d["v_cache"], d["table"], d["lengths"], d["tree"],
                              state["scale"], out["out"], state["workspace"])
    else:
        B.dsq_attention(d["q"], d["k"], d["v"], d["q_starts"], d["k_starts"], case["causal"], state["scale"], out["out"], state.get("lse"))
        if case["kind"] == "atrain":
            B.dsq_attention_bwd(d["q"], d["k"], d["v"], out["out"], state["lse"], d["grad_out"], d["q_starts"], d["k_starts"],
                                case["causal"], state["scale"], out["grad_q"], out["grad_k"], out["grad_v"], state["workspace"])
    return out


def _turn(case, d, x, back=False):
    """Heads x [rows, heads, dim] rotated by their positions, or back."""
    half, rd = case["rope_dim"] // 2, case["rope_dim"]
    at = d["positions"][d["pair_axis"].long()] if case["axes"] > 1 else d["positions"].expand(half, -1)
    # (angles in 64 bits: far positions)
    angle = at.double().t() * d["frequencies"].double()
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    s = -s if back else s
    a, b = (x[..., 0:rd:2], x[..., 1:rd:2]) if case["interleaved"] else (x[..., :half], x[..., half:rd])
    u, v = a * c - b * s, b * c + a * s
    turned = torch.stack((u, v), -1).flatten(-2) if case["interleaved"] else torch.cat((u, v), -1)
    return torch.cat((turned, x[..., rd:]), -1)


def _norm(x, w):
    xf = x.float()
    r = torch.rsqrt((xf * xf).mean(-1, keepdim=True) + EPS)
    return xf * r, r, w.float()


def _norm_back(x, w, g):
    n, r, w = _norm(x, w)
    t = g * w
    return (r * (t - n * (t * n).mean(-1, keepdim=True))).to(x.dtype), (g * n).double().sum((0, 1)).float()


def _scores(q, k, q_len, k_len, seen, scale):
    """Probabilities [sequences, kv heads, group * rows, keys] of padded rows q [sequences, rows, heads, dim] and keys
    k [sequences, keys, kv heads, dim], ``seen`` [sequences, rows, keys]; and the rows in that order."""
    S, L, hq, dim = q.shape
    hk = k.shape[2]
    qt = q.view(S, L, hk, hq // hk, dim).permute(0, 2, 3, 1, 4).reshape(S, hk, hq // hk * L, dim)
    kt = k.permute(0, 2, 3, 1).contiguous()
    s = torch.matmul(qt, kt).mul_(scale)
    hide = ~seen[:, None, None]
    s.view(S, hk, hq // hk, L, -1).masked_fill_(hide, -math.inf)
    s.sub_(s.amax(-1, keepdim=True).clamp_min(-1e30)).exp_()
    total = s.sum(-1, keepdim=True)
    return s.div_(torch.where(total > 0, total, 1.0)), qt


def _padded(t, starts, sizes, longest):
    """[sequences, longest, ...] of packed rows, zeros behind a sequence's last; and which places are rows."""
    place = torch.arange(longest, device="cuda")
    there = place[None] < sizes[:, None]
    at = torch.where(there, starts[:-1, None].long() + place, 0)
    return t[at].float() * there.view(*there.shape, *[1] * (t.dim() - 1)), there


def _rows_back(o, like):
    """Rows in their order [sequences, rows, heads, dim] of [sequences, kv heads, group * rows, dim]."""
    S, L, hq, dim = like.shape
    return o.view(S, o.shape[1], -1, L, dim).permute(0, 3, 1, 2, 4).reshape(S, L, hq, dim)


def _cache(state):
    case, d = state["case"], state["in"]
    dt, starts = DTYPES[case["dtype"]], d["q_starts"]
    q, there = _padded(d["q"], starts, starts.diff(), case["drafted"])
    place = torch.arange(case["longest"], device="cuda")
    pages = d["table"].clamp_min(0).long()[:, place // case["page"]]
    live = (place[None] < d["lengths"][:, None])
    k, v = ((t[pages, :, place % case["page"]].float() * live[..., None, None]) for t in (d["k_cache"], d["v_cache"]))
    bit = place[None] - (d["lengths"] - starts.diff())[:, None]            # a key's place among the drafted
    row = torch.arange(case["drafted"], device="cuda")
    if d["tree"] is None:
        seen = bit[:, None] <= row[:, None]
    else:
        word = torch.where(there, d["tree"][torch.where(there, starts[:-1, None] + row, 0), 0], 0)
        seen = (bit[:, None] < 0) | ((word[..., None] >> bit[:, None].clamp(0, 63)) & 1).bool()
    p, qt = _scores(q, k, None, None, seen & live[:, None], state["scale"])
    o = torch.matmul(p, v.permute(0, 2, 1, 3).contiguous())
    return {"out": _rows_back(o, q)[there].to(dt)}


def run(state):
    if own:
        return _own(state)
    case, d = state["case"], state["in"]
    dt = DTYPES[case["dtype"]]
    if case["kind"] == "cache":
        return _cache(state)
    if case["kind"] in ("rope", "rtrain"):
        q, k = ((lambda n, r, w: _turn(case, d, n * w).to(dt))(*_norm(d[x], d[x + "_weight"])) for x in "qk")
        if case["kind"] == "rope":
            page, at = d["slots"] // case["page"], d["slots"] % case["page"]
            d["k_cache"][page, :, at] = k
            d["v_cache"][page, :, at] = d["v"]
            return {"q": q, "k_cache": d["k_cache"], "v_cache": d["v_cache"]}
        gq, gqw = _norm_back(d["q"], d["q_weight"], _turn(case, d, d["grad_q_out"].float(), True))
        gk, gkw = _norm_back(d["k"], d["k_weight"], _turn(case, d, d["grad_k_out"].float(), True))
        return {"q": q, "k": k, "grad_q": gq, "grad_k": gk, "grad_q_weight": gqw, "grad_k_weight": gkw}
    longest, keys = case["longest"], case["longest"] + case["context"]
    q_len, k_len = d["q_starts"].diff(), d["k_starts"].diff()
    q, there = _padded(d["q"], d["q_starts"], q_len, longest)
    k, live = _padded(d["k"], d["k_starts"], k_len, keys)
    v, _ = _padded(d["v"], d["k_starts"], k_len, keys)
    seen = live[:, None]
    if case["causal"]:
        row, key = torch.arange(longest, device="cuda"), torch.arange(keys, device="cuda")
        seen = seen & (key[None, None] <= row[None, :, None] + (k_len - q_len)[:, None, None])
    else:
        seen = seen.expand(-1, longest, -1)
    p, qt = _scores(q, k, q_len, k_len, seen, state["scale"])
    vt = v.permute(0, 2, 1, 3).contiguous()
    o = torch.matmul(p, vt)
    out = {"out": _rows_back(o, q)[there].to(dt)}
    if case["kind"] == "atrain":
        S, hk = o.shape[:2]
        g, _ = _padded(d["grad_out"], d["q_starts"], q_len, longest)
        gt = g.view(S, longest, hk, -1, case["dim"]).permute(0, 2, 3, 1, 4).reshape(o.shape)
        grad_v = torch.matmul(p.transpose(-1, -2).contiguous(), gt)
        ds = torch.matmul(gt, vt.transpose(-1, -2).contiguous()).sub_((gt * o).sum(-1, keepdim=True)).mul_(p).mul_(state["scale"])
        grad_q = torch.matmul(ds, k.permute(0, 2, 1, 3).contiguous())
        grad_k = torch.matmul(ds.transpose(-1, -2).contiguous(), qt)
        out.update(grad_q=_rows_back(grad_q, q)[there].to(dt), grad_k=grad_k.permute(0, 2, 1, 3)[live].to(dt),
                   grad_v=grad_v.permute(0, 2, 1, 3)[live].to(dt))
    return out


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    hq, hk, dim = case["q_heads"], case["kv_heads"], case["dim"]
    if case["kind"] == "rope":
        # queries, keys and values in and out; positions, slots, weights, frequencies
        n = case["rows"] * (hq + 2 * hk) * dim
        return {"bytes": 2 * e * n + case["rows"] * (4 * case["axes"] + 8) + 2 * dim * e + 2 * case["rope_dim"], "flops": 8 * n}
    if case["kind"] == "rtrain":
        # forward: heads in and out; backward: heads and gradients in, gradients out
        n = case["rows"] * (hq + hk) * dim
        return {"bytes": 5 * e * n + 8 * case["rows"] * case["axes"] + 2 * dim * (2 * e + 4) + 4 * case["rope_dim"], "flops": 24 * n}
    rows, keys = _sizes(case)
    if case["kind"] == "cache":
        pairs = sum(n * k for n, k in zip(rows, keys))
        return {"bytes": e * dim * (2 * hk * sum(keys) + 2 * hq * sum(rows)) + 4 * sum(-(-k // case["page"]) for k in keys),
                "flops": 4 * dim * hq * pairs}
    # (a causal row sees the keys before it: half of a square)
    pairs = sum(n * k - (n * (n - 1) // 2 if case["causal"] else 0) for n, k in zip(rows, keys))
    q, kv = e * dim * hq * sum(rows), e * dim * hk * sum(keys)
    if case["kind"] == "attn":
        return {"bytes": 2 * q + 2 * kv, "flops": 4 * dim * hq * pairs}
    return {"bytes": 6 * q + 6 * kv + 8 * hq * sum(rows), "flops": 14 * dim * hq * pairs}


# ---- the definition in 64 bits -------------------------------------------------------------------

def _exact_heads(case, d):
    pairs = case["rope_dim"] // 2
    axis = torch.arange(pairs, device="cuda") % case["axes"]
    angle = torch.stack([d["positions"][int(axis[j])].double() * d["frequencies"][j].double() for j in range(pairs)], 1)
    unit = torch.polar(torch.ones_like(angle), angle)[:, None]

    def pairs_of(x):
        y = x[..., :2 * pairs]
        y = y.unflatten(-1, (pairs, 2)) if case["interleaved"] else y.unflatten(-1, (2, pairs)).transpose(-1, -2)
        return torch.complex(y[..., 0], y[..., 1])

    def whole(z, x):
        y = torch.view_as_real(z)
        y = y if case["interleaved"] else y.transpose(-1, -2)
        return torch.cat((y.flatten(-2), x[..., 2 * pairs:]), -1)

    result = {}
    for name in "qk":
        x, w = d[name].double(), d[name + "_weight"].double()
        rms = torch.sqrt(torch.sum(x ** 2, -1, keepdim=True) / case["dim"] + EPS)
        n = x / rms
        result[name] = whole(pairs_of(n * w) * unit, n * w)
        if case["kind"] == "rtrain":
            g = d["grad_%s_out" % name].double()
            g = whole(pairs_of(g) * unit.conj(), g)
            along = torch.sum(g * w * n, -1, keepdim=True) / case["dim"]
            result["grad_" + name] = (g * w - n * along) / rms
            result["grad_%s_weight" % name] = torch.einsum("thd,thd->d", g, n)
    return result


def exact(case, seed):
    d = _inputs(case, seed)
    if case["kind"] == "rtrain":
        r = _exact_heads(case, d)
        return {k: r[k] for k in ("q", "k", "grad_q", "grad_k", "grad_q_weight", "grad_k_weight")}
    if case["kind"] == "rope":
        r = _exact_heads(case, d)
        cache = {}
        for name, heads in (("k_cache", r["k"]), ("v_cache", d["v"].double())):
            c = torch.zeros(d[name].shape, dtype=torch.float64, device="cuda").transpose(1, 2).contiguous()
            c.flatten(0, 1).index_copy_(0, d["slots"], heads)
            cache[name] = c.transpose(1, 2).contiguous()
        return {"q": r["q"], **cache}
    rows, keys = _sizes(case)
    group, scale, dim = case["q_heads"] // case["kv_heads"], case["dim"] ** -0.5, case["dim"]
    new = lambda t: torch.zeros(t.shape, dtype=torch.float64, device="cuda")
    out = {"out": new(d["q"])}
    if case["kind"] == "atrain":
        out.update(grad_q=new(d["q"]), grad_k=new(d["k"]), grad_v=new(d["v"]))
    q0 = k0 = 0
    for s, (n, m) in enumerate(zip(rows, keys)):
        at = torch.arange(m, device="cuda")
        if case["kind"] == "cache":
            page = d["table"][s, :-(-m // case["page"])].long()
            k, v = (d[c][page].transpose(1, 2).flatten(0, 1)[:m].double() for c in ("k_cache", "v_cache"))
            mask = torch.ones(n, m, dtype=torch.bool, device="cuda")
            if d["tree"] is None:
                mask[:, m - n:] = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
            else:
                mask[:, m - n:] = torch.bitwise_and(d["tree"][q0:q0 + n], torch.bitwise_left_shift(torch.ones((), dtype=torch.int64, device="cuda"), at[:n])) != 0
        else:
            k, v = d["k"][k0:k0 + m].double(), d["v"][k0:k0 + m].double()
            mask = torch.ones(n, m, dtype=torch.bool, device="cuda")
            mask = mask.tril(m - n) if case["causal"] else mask
        for h in range(case["q_heads"]):
            q, kh, vh = d["q"][q0:q0 + n, h].double(), k[:, h // group], v[:, h // group]
            p = torch.softmax(torch.where(mask, scale * torch.mm(q, kh.t()), -math.inf), 1)
            out["out"][q0:q0 + n, h] = torch.mm(p, vh)
            if case["kind"] == "atrain":
                g = d["grad_out"][q0:q0 + n, h].double()
                gp = torch.mm(g, vh.t())
                gs = p * (gp - torch.sum(p * gp, 1, keepdim=True)) * scale
                out["grad_v"][k0:k0 + m, h // group] += torch.mm(p.t(), g)
                out["grad_q"][q0:q0 + n, h] = torch.mm(gs, kh)
                out["grad_k"][k0:k0 + m, h // group] += torch.mm(gs.t(), q)
        q0, k0 = q0 + n, k0 + m
    return out
