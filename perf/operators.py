"""The 8-bit serving operators as measurable cases.

  linear     activations quantized per token, then the 8-bit product with a
             scale for each token and each output channel
  experts    the same product grouped by expert: rows gathered from the tokens
             by a router's decision, ragged group sizes
  append     rotate queries and keys, append keys and values to the paged
             8-bit cache (a power-of-two scale for each page and head, old
             codes re-rounded where it grows), read the touched pages back
  attention  softmax attention over such a cache, one or several new tokens
             per sequence, grouped heads, causal

``run`` computes them in their plain form (elementary torch operations in 32
bits) or, where ``own`` is set, through the framework's entry points.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
FLOOR = 2.0 ** -100  # magnitudes below this count as this when a scale is chosen


def listed():
    return [
        # one token through the classifier layer of the ResNet-50 workload: bound by latency
        dict(name="linear_1x2048x1000", kind="linear", rows=1, k=2048, n=1000, type="bf16", rule="max", bias=True),
        # AlexNet's first FC layer at the benchmark's batch: a small batch streams its weights
        dict(name="linear_64x9216x4096", kind="linear", rows=64, k=9216, n=4096, type="f16", rule="dfx", bias=True),
        # an odd number of rows, depth and columns, full-precision values
        dict(name="linear_777x2050x1533", kind="linear", rows=777, k=2050, n=1533, type="f32", rule="max", bias=False),
        # a prompt batch through a wide projection: bound by the matrix cores
        dict(name="linear_8192x4096x8192", kind="linear", rows=8192, k=4096, n=8192, type="bf16", rule="max", bias=False),
        # one decoding step of 64 sequences, two experts a token: few rows per expert
        dict(name="experts_64x2_e32", kind="experts", tokens=64, top=2, experts=32, k=2048, n=4096, type="bf16", skew=0.5),
        # a prompt of 8192 tokens: large ragged groups, some experts far more popular
        dict(name="experts_8192x2_e16", kind="experts", tokens=8192, top=2, experts=16, k=2048, n=4096, type="bf16", skew=1.0),
        # one new token for each of 64 sequences
        dict(name="append_64x1", kind="append", seqs=64, new=1, ctx=4096, page=16, q_heads=32, heads=8, dim=128, rot=128, type="bf16"),
        # prompts of up to 2048 tokens, some continuing an earlier context
        dict(name="append_8x2048", kind="append", seqs=8, new=2048, ctx=1000, page=64, q_heads=32, heads=8, dim=128, rot=64, type="f16"),
        # one short conversation: latency
        dict(name="attention_1x1_300", kind="attention", seqs=1, new=1, ctx=300, page=16, q_heads=16, heads=16, dim=64, type="bf16"),
        # a full serving batch, lengths from a few tokens to 8192
        dict(name="attention_64x1_8192", kind="attention", seqs=64, new=1, ctx=8192, page=16, q_heads=32, heads=8, dim=128, type="bf16"),
        # one very long context: the cache is split among the compute units
        dict(name="attention_1x1_131072", kind="attention", seqs=1, new=1, ctx=131072, page=64, q_heads=32, heads=8, dim=128, type="bf16"),
        # prompts appended in chunks: causal inside the chunk, everything before it visible
        dict(name="attention_4x1024_4000", kind="attention", seqs=4, new=1024, ctx=4000, page=32, q_heads=32, heads=8, dim=128, type="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = {c["kind"]: max((_cost(x) for x in listed() if x["kind"] == c["kind"])) for c in listed()}
    kind = rng.choice(["linear", "experts", "append", "attention"])
    while True:
        t = rng.choice(["bf16", "bf16", "f16", "f32"])
        if kind == "linear":
            c = dict(kind=kind, rows=_log(rng, 1, 8192), k=_log(rng, 64, 9216), n=_log(rng, 16, 8192), type=t,
                     rule=rng.choice(["max", "dfx"]), bias=rng.random() < 0.5)
        elif kind == "experts":
            e = rng.choice([4, 8, 16, 32, 64])
            c = dict(kind=kind, tokens=_log(rng, 1, 8192), top=rng.choice([1, 2, 4]), experts=e, k=16 * _log(rng, 16, 256),
                     n=_log(rng, 128, 4096), type=t, skew=rng.choice([0.0, 0.5, 1.0, 2.0]))
        else:
            heads = rng.choice([1, 2, 4, 8, 16])
            c = dict(kind=kind, seqs=_log(rng, 1, 64), new=rng.choice([1, 1, _log(rng, 2, 2048)]), ctx=_log(rng, 16, 131072),
                     page=rng.choice([16, 32, 64, 128]), q_heads=heads * rng.choice([1, 2, 4, 6, 8]), heads=heads,
                     dim=rng.choice([64, 96, 128, 256]), type=t)
            if kind == "append":
                c["rot"] = rng.choice([c["dim"], c["dim"] // 2])
                c["ctx"] = min(c["ctx"], 8192)
        if _cost(c) <= top[kind]:
            return c


def _cost(c):
    """What bounds a draw: the time a plain form would take, roughly (padded sizes included)."""
    if c["kind"] == "linear":
        return 2.0 * c["rows"] * c["k"] * c["n"] + 400.0 * (c["rows"] + c["n"]) * c["k"]
    if c["kind"] == "experts":
        return (2.0 * max(_sizes(c)) + 800.0) * c["experts"] * c["k"] * c["n"]
    pages = c["seqs"] * (c["ctx"] + c["new"])
    if c["kind"] == "append":
        return c["seqs"] * (c["new"] + c["page"]) * (c["q_heads"] + 2.0 * c["heads"]) * c["dim"] + 0.05 * pages * c["heads"] * c["dim"]
    return 180.0 * pages * c["heads"] * c["dim"] + 1.0 * pages * c["new"] * c["q_heads"] * (c["dim"] + 20)


def _sizes(c):
    """Host sizes of a case that the seed does not change: rows of each expert, lengths and new tokens of each sequence."""
    if c["kind"] == "experts":
        w = [1.0 / (1 + e) ** c["skew"] for e in range(c["experts"])]
        rows = c["tokens"] * c["top"]
        cum, total, counts, at = 0.0, sum(w), [], 0
        for e in range(c["experts"]):
            cum += w[e]
            to = rows if e + 1 == c["experts"] else int(round(rows * cum / total))
            counts.append(to - at)
            at = to
        return counts
    s, new, length = c["seqs"], [], []
    for i in range(s):
        # a ragged batch: the first sequence has the largest sizes, the others spread below them
        n = c["new"] if i % 3 == 0 else max(1, (c["new"] * (2 * i + 1)) // (2 * s + 1))
        new.append(n)
        length.append(n + (c["ctx"] if i == 0 else (c["ctx"] * ((i * 37) % (s + 1))) // (s + 1)))
    return new, length


def work(c):
    b = 4 if c["type"] == "f32" else 2
    if c["kind"] == "linear":
        m, k, n = c["rows"], c["k"], c["n"]
        return {"bytes": m * k * b + n * k + 4 * n * (2 if c["bias"] else 1) + m * n * b, "flops": 2 * m * n * k}
    if c["kind"] == "experts":
        counts = _sizes(c)
        rows, used = sum(counts), sum(1 for x in counts if x)
        return {"bytes": c["tokens"] * c["k"] * b + used * c["n"] * (c["k"] + 4) + rows * c["n"] * b + 4 * rows,
                "flops": 2 * rows * c["n"] * c["k"]}
    new, length = _sizes(c)
    t, d = sum(new), c["dim"]
    if c["kind"] == "append":
        # read q, k, v; write rotated q and the codes; read the touched pages' codes and write their values
        back = sum(x - (x - n) // c["page"] * c["page"] for n, x in zip(new, length))
        return {"bytes": t * d * (2 * c["q_heads"] + 2 * c["heads"]) * b + t * 2 * c["heads"] * d + back * 2 * c["heads"] * d * (1 + b),
                "flops": 3 * t * c["rot"] * (c["q_heads"] + c["heads"])}
    seen = sum(n * x - n * (n - 1) // 2 for n, x in zip(new, length))
    return {"bytes": sum(length) * c["heads"] * 2 * d + 2 * t * c["q_heads"] * d * b + sum(8 * c["heads"] * -(-x // c["page"]) for x in length),
            "flops": 4 * seen * c["q_heads"] * d}


class _State(dict):
    __getattr__ = dict.__getitem__


def prepare(case, seed):
    c = _State(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = TYPES[c.type]
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    s = _State(case=c, dt=dt)
    if c.kind == "linear":
        kp = -(-c.k // 16) * 16
        # activations with a few channels far larger than the rest, as hidden states have
        x = randn(c.rows, c.k) * torch.exp(1.0 * randn(1, c.k))
        w = torch.zeros(c.n, kp, dtype=torch.int8, device=DEV)
        w[:, : c.k] = (randn(c.n, c.k) * 40).round().clamp(-127, 127).to(torch.int8)
        s |= dict(x=x.to(dt), w=w, sb=torch.rand(c.n, generator=g, device=DEV) * 1e-3 + 1e-4,
                  bias=randn(c.n) if c.bias else None, kp=kp)
    elif c.kind == "experts":
        counts = _sizes(c)
        rows = sum(counts)
        x = randn(c.tokens, c.k) * torch.exp(1.0 * randn(1, c.k))
        w = (torch.randn(c.experts, c.n, c.k, generator=g, device=DEV, dtype=torch.float16) * 40).round().clamp(-127, 127).to(torch.int8)
        off = torch.zeros(c.experts + 1, dtype=torch.int32)
        off[1:] = torch.tensor(counts).cumsum(0)
        # which token each row of an expert's group comes from
        pick = torch.randperm(rows, generator=g, device=DEV) % c.tokens
        s |= dict(x=x.to(dt), w=w, sb=torch.rand(c.experts, c.n, generator=g, device=DEV) * 1e-3 + 1e-4, off=off.to(DEV),
                  pick=pick.to(torch.int32), rows=rows, most=max(counts))
    else:
        new, length = _sizes(c)
        s |= _cache(c, g, new, length)
        t, d = sum(new), c.dim
        if c.kind == "append":
            # one fused projection's output: queries, keys and values side by side in a row
            s.qkv = (randn(t, (c.q_heads + 2 * c.heads) * d)).to(dt)
            ang = torch.arange(max(length), device=DEV, dtype=torch.float64)[:, None] * 10000.0 ** (
                -torch.arange(0, c.rot, 2, device=DEV, dtype=torch.float64) / c.rot)
            s.cos, s.sin = ang.cos().float(), ang.sin().float()
            back = [x - (x - n) // c.page * c.page for n, x in zip(new, length)]
            s.back_tokens, s.back_most = sum(back), max(back)
            s.back_start = torch.tensor([0] + back).cumsum(0).to(torch.int32).to(DEV)
        else:
            s.q = randn(t, c.q_heads * d).to(dt)
    if own:
        _handles(s)
    return s


def _cache(c, g, new, length):
    """A paged cache that holds the context, its pages in no order, and the batch that describes its sequences."""
    need = [-(-x // c.page) for x in length]
    pages, width = sum(need), max(need)
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    table = torch.zeros(c.seqs, width, dtype=torch.int32, device=DEV)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at : at + n]
        at += n
    codes = lambda *sh: (torch.randn(*sh, generator=g, device=DEV, dtype=torch.float16) * 30).round().clamp(-127, 127).to(torch.int8)  # noqa: E731
    scale = lambda: 2.0 ** -(torch.randint(4, 7, (pages, c.heads), generator=g, device=DEV).float())  # noqa: E731
    return dict(k=codes(pages, c.heads, c.page, c.dim), v=codes(pages, c.heads, c.page // 16, c.dim, 16), ks=scale(), vs=scale(),
                table=table, start=torch.tensor([0] + new).cumsum(0).to(torch.int32).to(DEV),
                length=torch.tensor(length, dtype=torch.int32, device=DEV), pages=pages, width=width, tokens=sum(new),
                most_new=max(new), most_len=max(length))


def _handles(s):
    """What a user's program keeps beside its data: the handle, descriptors, result and work space."""
    from paper_2203_12091_amd import fxpq as fx
    global _handle
    if _handle is None:
        _handle = fx.Handle(0)
    c, empty = s.case, lambda sh, dt: torch.empty(sh, dtype=dt, device=DEV)
    s.fx, s.h, s.t = fx, _handle, {"f32": fx.F32, "f16": fx.F16, "bf16": fx.BF16}[c.type]
    if c.kind in ("linear", "experts"):
        m = c.rows if c.kind == "linear" else c.tokens
        kp = s.kp if c.kind == "linear" else c.k
        rows = c.rows if c.kind == "linear" else s.rows
        s |= dict(codes=empty((m, kp), torch.int8), sa=empty((m,), torch.float32), y=empty((rows, c.n), s.dt))
        need = fx.token_gemm_workspace(c.rows, c.n, s.kp) if c.kind == "linear" else 0
        s.ws, s.ws_bytes = empty((max(need, 16),), torch.uint8), need
        return
    s.cache = fx.kv_cache(s.k, s.v, s.ks, s.vs, s.pages, c.page, c.heads, c.dim)
    s.batch = fx.kv_batch(s.start, s.length, s.table, c.seqs, s.width, s.tokens, s.most_new, s.most_len)
    if c.kind == "append":
        s.rotary = fx.rotary(s.cos, s.sin, s.cos.shape[0], c.rot, 0)
        s.back = fx.kv_batch(s.back_start, s.length, s.table, c.seqs, s.width, s.back_tokens, s.back_most, s.most_len)
        s |= dict(q_out=empty((s.tokens, c.q_heads * c.dim), s.dt), k_out=empty((s.back_tokens, c.heads, c.dim), s.dt),
                  v_out=empty((s.back_tokens, c.heads, c.dim), s.dt))
    else:
        s.out = empty((s.tokens, c.q_heads * c.dim), s.dt)
        s.ws_bytes = fx.cache_attention_workspace(s.h, s.cache, s.batch, c.q_heads)
        s.ws = empty((max(s.ws_bytes, 16),), torch.uint8)


_handle = None


def run(s):
    c = s.case
    if own:
        return _OWN[c.kind](s, c, s.fx)
    return _PLAIN[c.kind](s, c)


# ---- through the framework ----------------------------------------------------

def _own_linear(s, c, fx):
    fx.token_quantize(s.h, s.x, s.t, c.rows, c.k, c.k, fx.SCALE_DFX if c.rule == "dfx" else fx.SCALE_MAX, s.codes, s.kp, s.sa)
    fx.token_gemm(s.h, c.rows, c.n, s.kp, s.codes, s.kp, s.sa, s.w, s.sb, s.bias, s.y, s.t, c.n, s.ws, s.ws_bytes)
    return s.y


def _own_experts(s, c, fx):
    fx.token_quantize(s.h, s.x, s.t, c.tokens, c.k, c.k, fx.SCALE_MAX, s.codes, c.k, s.sa)
    fx.expert_gemm(s.h, s.rows, c.n, c.k, c.experts, s.codes, c.tokens, c.k, s.sa, s.pick, s.off, s.w, s.sb, None, s.y, s.t, c.n)
    return s.y


def _own_append(s, c, fx):
    d, ld = c.dim, s.qkv.shape[1]
    at = s.qkv.data_ptr()
    size = s.qkv.element_size()
    q, k, v = at, at + c.q_heads * d * size, at + (c.q_heads + c.heads) * d * size
    fx.cache_append(s.h, s.cache, s.batch, s.rotary, k, ld, v, ld, q, ld, s.q_out, c.q_heads * d, c.q_heads, s.t)
    fx.cache_read(s.h, s.cache, s.back, s.k_out, s.v_out, s.t)
    return s.q_out, s.k_out, s.v_out


def _own_attention(s, c, fx):
    w = c.q_heads * c.dim
    fx.cache_attention(s.h, s.cache, s.batch, s.q, w, c.q_heads, c.dim ** -0.5, 1, s.out, w, s.t, s.ws, s.ws_bytes)
    return s.out


_OWN = {"linear": _own_linear, "experts": _own_experts, "append": _own_append, "attention": _own_attention}


# ---- plain forms ----------------------------------------------------------------

def _quantize(x, rule):
    """Codes (as fp32 integers) and the scale of each row."""
    a = x.abs().amax(-1, keepdim=True).clamp_min(FLOOR)
    if rule == "dfx":
        scale = _dfx_scale(a)
        return (x / scale).round(), scale
    return (x * (torch.full_like(a, 127.0) / a)).round(), a / 127.0


def _dfx_scale(a):
    """The smallest power of two whose 8-bit codes reach the magnitude a."""
    m, e = torch.frexp(a)
    fl = 7 - e - (m * 128.0 >= 127.5).to(e.dtype)
    return torch.ldexp(torch.ones_like(a), -fl)


def _plain_linear(s, c):
    q, sa = _quantize(s.x.float(), c.rule)
    y = q @ s.w[:, : c.k].float().t() * sa * s.sb
    if c.bias:
        y = y + s.bias
    return y.to(s.dt)


def _plain_experts(s, c):
    q, sa = _quantize(s.x.float(), "max")
    row = torch.arange(s.rows, device=DEV, dtype=torch.int32)
    e = torch.searchsorted(s.off, row, right=True) - 1
    at = row - s.off[e]  # the row's place in its expert's group
    pad = torch.zeros(c.experts, s.most, c.k, device=DEV)
    pad[e, at] = q[s.pick.long()]
    y = torch.bmm(pad, s.w.float().transpose(1, 2).contiguous())[e, at]
    return (y * sa[s.pick.long()] * s.sb[e]).to(s.dt)


def _rotate(x, cos, sin, rot):
    h = rot // 2
    x1, x2 = x[..., :h], x[..., h:rot]
    return torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin, x[..., rot:]], -1)


def _rows_of(v):
    """The values of a page's V codes as [..., page, dim] (stored 16 tokens side by side for each dimension)."""
    return v.transpose(-1, -2).flatten(-3, -2)


def _plain_append(s, c):
    t, d, P = s.tokens, c.dim, c.page
    length, start = s.length.long(), s.start.long()
    n = start[1:] - start[:-1]
    tok = torch.arange(t, device=DEV)
    seq = torch.searchsorted(start, tok, right=True) - 1
    pos = length[seq] - n[seq] + tok - start[seq]
    x = s.qkv.float().view(t, c.q_heads + 2 * c.heads, d)
    cos, sin = s.cos[pos][:, None], s.sin[pos][:, None]
    q = _rotate(x[:, : c.q_heads], cos, sin, c.rot)
    k, v = _rotate(x[:, c.q_heads : c.q_heads + c.heads], cos, sin, c.rot), x[:, c.q_heads + c.heads :]
    # the pages that new tokens fall in: [seqs, most touched]; a sequence that touches fewer names its last one again
    first, last = (length - n) // P, (length - 1) // P
    j = torch.arange((s.most_new + P - 2) // P + 1, device=DEV)
    nth = torch.minimum(first[:, None] + j, last[:, None])
    page = s.table.gather(1, nth).long()
    at = nth[:, :, None] * P + torch.arange(P, device=DEV)  # the positions their slots stand for
    is_new = (at >= (length - n)[:, None, None]) & (at < length[:, None, None])
    src = (at - (length - n)[:, None, None] + start[:-1, None, None]).clamp(0, t - 1)
    kept = (nth * P < (length - n)[:, None])[:, :, None]
    got = []
    for x, codes, scale in ((k, s.k, s.ks), (v, s.v, s.vs)):
        new = x[src].movedim(3, 2)  # [seqs, pages, heads, slots, dim]
        mask = is_new[:, :, None, :, None]
        a = torch.where(mask, new.abs(), 0.0).amax((-1, -2)).clamp_min(FLOOR)
        old = scale[page]
        grown = torch.where(kept, torch.maximum(old, _dfx_scale(a)), _dfx_scale(a))
        was = codes[page].float()
        was = _rows_of(was) if codes is s.v else was
        now = torch.where(mask, (new / grown[..., None, None]).round(), (was * (old / grown)[..., None, None]).round().clamp(-128, 127))
        now = torch.where((at < length[:, None, None])[:, :, None, :, None], now, was).to(torch.int8)
        codes[page] = now.unflatten(-2, (P // 16, 16)).transpose(-1, -2) if codes is s.v else now
        scale[page] = grown
        # what the touched pages hold now, sequence by sequence, up to its length
        i = torch.arange(s.back_tokens, device=DEV)
        q_seq = torch.searchsorted(s.back_start, i.to(torch.int32), right=True) - 1
        p = first[q_seq] * P + i - s.back_start[q_seq]
        pg, slot = s.table[q_seq, p // P].long(), p % P
        held = codes[pg, :, slot // 16, :, slot % 16] if codes is s.v else codes[pg, :, slot]
        got.append((held.float() * scale[pg][..., None]).to(s.dt))
    return q.flatten(1).to(s.dt), got[0], got[1]


def _plain_attention(s, c):
    S, H, G, D, N = c.seqs, c.heads, c.q_heads // c.heads, c.dim, s.most_new
    length, start = s.length.long(), s.start.long()
    n = start[1:] - start[:-1]
    page = s.table.long()
    k = s.k[page].float() * s.ks[page][..., None, None]  # [S, width, H, P, D]
    v = _rows_of(s.v[page].float()) * s.vs[page][..., None, None]
    k, v = (z.transpose(1, 2).reshape(S, H, -1, D) for z in (k, v))
    i = torch.arange(N, device=DEV)
    src = (start[:-1, None] + torch.minimum(i, n[:, None] - 1)).clamp_min(0)
    q = s.q.float().view(-1, H, G, D)[src].permute(0, 2, 3, 1, 4).reshape(S, H, G * N, D)
    sc = (q @ k.transpose(-1, -2).contiguous()).view(S, H, G, N, -1) * D ** -0.5
    at = torch.arange(sc.shape[-1], device=DEV)
    see = at <= ((length - n)[:, None] + i)[:, :, None]  # [S, N, L]
    sc = sc.masked_fill(~see[:, None, None], float("-inf"))
    p = torch.exp(sc - sc.amax(-1, keepdim=True))
    # pages past a sequence's end hold other sequences' codes: their weight is zero
    o = (p / p.sum(-1, keepdim=True)).view(S, H, G * N, -1) @ v
    o = o.view(S, H, G, N, D).permute(0, 3, 1, 2, 4).reshape(S, N, H * G * D)
    tok = torch.arange(s.tokens, device=DEV)
    seq = torch.searchsorted(start, tok, right=True) - 1
    return o[seq, tok - start[seq]].to(s.dt)


_PLAIN = {"linear": _plain_linear, "experts": _plain_experts, "append": _plain_append, "attention": _plain_attention}


# ---- definitions in 64 bits ----------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return _EXACT[s.case.kind](s, s.case)


def _exact_codes(x, rule):
    x = x.double()
    top = x.abs().max(dim=-1).values.clamp(min=FLOOR)
    if rule == "max":
        step = top / 127
    else:
        step = torch.exp2(torch.floor(torch.log2(top)) - 6)
        step = torch.where(torch.round(top / step) > 127, 2 * step, step)
    return torch.round(x / step[:, None]), step


def _exact_linear(s, c):
    q, step = _exact_codes(s.x, c.rule)
    y = torch.matmul(q, s.w[:, : c.k].double().t()) * torch.outer(step, s.sb.double())
    return y + s.bias.double() if c.bias else y


def _exact_experts(s, c):
    q, step = _exact_codes(s.x, "max")
    off, out = s.off.tolist(), torch.zeros(s.rows, c.n, dtype=torch.float64, device=DEV)
    for e in range(c.experts):
        rows = s.pick[off[e] : off[e + 1]].long()
        out[off[e] : off[e + 1]] = torch.matmul(q[rows], s.w[e].double().t()) * torch.outer(step[rows], s.sb[e].double())
    return out


def _exact_append(s, c):
    d, P, start, length = c.dim, c.page, s.start.tolist(), s.length.tolist()
    x = s.qkv.double().view(s.tokens, -1, d).clone()
    turned = c.q_heads + c.heads
    ks, vs, queries = [], [], []
    for i in range(c.seqs):
        n = start[i + 1] - start[i]
        p0 = length[i] - n
        y = x[start[i] : start[i + 1]]
        z = torch.view_as_complex(torch.stack([y[:, :turned, : c.rot // 2], y[:, :turned, c.rot // 2 : c.rot]], -1))
        w = torch.complex(s.cos[p0 : length[i]].double(), s.sin[p0 : length[i]].double())
        z = torch.view_as_real(z * w[:, None])
        y[:, :turned, : c.rot] = torch.cat([z[..., 0], z[..., 1]], -1)
        queries.append(y[:, : c.q_heads].reshape(n, -1))
        begin = p0 // P * P
        many = -(-length[i] // P) - begin // P
        page = s.table[i, begin // P : begin // P + many].long()
        for new, codes, scale, out in ((y[:, c.q_heads : turned], s.k, s.ks, ks), (y[:, turned:], s.v, s.vs, vs)):
            was = codes[page].double()
            was = was if was.dim() == 4 else was.permute(0, 1, 2, 4, 3).reshape(many, c.heads, P, d)
            was = was.permute(0, 2, 1, 3).reshape(many * P, c.heads, d)
            old = scale[page].double()
            full = torch.zeros(many * P, c.heads, d, dtype=torch.float64, device=DEV)
            full[p0 - begin : length[i] - begin] = new
            top = full.view(many, P, c.heads, d).abs().amax((1, 3)).clamp(min=FLOOR)
            step = torch.exp2(torch.floor(torch.log2(top)) - 6)
            step = torch.where(torch.round(top / step) > 127, 2 * step, step)
            if p0 > begin:
                step[0] = torch.maximum(step[0], old[0])
            wide = step.repeat_interleave(P, 0)[..., None]
            held = torch.round(was * (old.repeat_interleave(P, 0)[..., None] / wide)).clamp(-128, 127)
            held[p0 - begin :] = torch.round(full[p0 - begin :] / wide[p0 - begin :])
            out.append((held * wide)[: length[i] - begin])
    return torch.cat(queries), torch.cat(ks), torch.cat(vs)


def _exact_attention(s, c):
    start, length, G = s.start.tolist(), s.length.tolist(), c.q_heads // c.heads
    out = torch.zeros(s.tokens, c.q_heads, c.dim, dtype=torch.float64, device=DEV)
    for i in range(c.seqs):
        page = s.table[i, : -(-length[i] // c.page)].long()
        n = start[i + 1] - start[i]
        for h in range(c.heads):
            k = (s.k[page, h].double() * s.ks[page, h].double()[:, None, None]).reshape(-1, c.dim)[: length[i]]
            v = s.v[page, h].double().permute(0, 1, 3, 2).reshape(len(page), c.page, c.dim) * s.vs[page, h].double()[:, None, None]
            v = v.reshape(-1, c.dim)[: length[i]]
            for g in range(h * G, h * G + G):
                q = s.q[start[i] : start[i + 1]].view(n, c.q_heads, c.dim)[:, g].double()
                z = torch.matmul(q, k.t().contiguous()) / math.sqrt(c.dim)
                if n > 1:
                    z += torch.full_like(z, -math.inf).triu(length[i] - n + 1)
                out[start[i] : start[i + 1], g] = torch.matmul(torch.softmax(z, -1), v)
    return out.flatten(1)


_EXACT = {"linear": _exact_linear, "experts": _exact_experts, "append": _exact_append, "attention": _exact_attention}
