"""The paged 8-bit cache of latents (append with rotation, read) and the two forms of
attention over it, against plain implementations: codes and scales bit for bit
(each step is one fp32 or fp64 rounding), attention against 64 bits.

Absorbed attention's tolerance, per output value, with S = max |value| of the visible
tokens and L of them: a logit is off by at most d = |softmax_scale| sum |q k| *
((latent + rope + 8) * 2^-24 (fp32 sums) + 2^-22 in f32 (q as two f16 terms of 2^-11 each))
+ |softmax_scale| sum |k| * 2^-38 max |q| (the end of f16's range) + 4 * 2^-24 |logit|;
a weight by 2 d + 4 * 2^-23 (exp2), by its rounding before the second product uP (2^-11
one f16 term, 2^-22 two), and by 2^-31 of the largest weight (f16's range again); the sums
by 2 (L + 64) * 2^-24.  All of it weighs at most S; the type's rounding comes last.
For 16-bit q the first product's sums may start from a constant per query, up to (1152 +
127) s_max sum |q| in all; every step of 8 dimensions rounds by 2^-24 of that at most.  With
q of random signs the partial sums stay near sqrt(latent) * 1152 |q|, below the products'
magnitudes sum |q k| that are counted already; q of one sign is tested with the term.
Expanded attention: products exact or rounded in fp32 sums, uP the type's own rounding."""
import math

import numpy as np
import pytest

from gpu_util import DEV, note

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
HALF_ULP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module")
def fx():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2203_12091_amd import fxpq
    return fxpq


@pytest.fixture(scope="module")
def h(fx):
    hd = fx.Handle(0)
    yield hd
    hd.close()


def code_of(fx, t):
    return {"f32": fx.F32, "f16": fx.F16, "bf16": fx.BF16}[t]


class Cache:
    """A cache whose unused memory holds the worst there is: code -128, NaN scales, page
    numbers outside the cache past each sequence's end."""

    def __init__(self, fx, lens_max, latent, rope, page, seed=0, spare=2):
        self.fx, self.latent, self.rope, self.page, self.seqs = fx, latent, rope, page, len(lens_max)
        need = [-(-n // page) for n in lens_max]
        self.width, self.pages = max(max(need), 1), sum(need) + spare
        order = np.random.default_rng(seed).permutation(self.pages)
        self.table = np.full((self.seqs, self.width), 2 ** 31 - 1, dtype=np.int32)
        at = 0
        for s, n in enumerate(need):
            self.table[s, :n] = order[at : at + n]
            at += n
        self.codes = torch.full((self.pages, page, latent + rope), -128, dtype=torch.int8, device=DEV)
        self.scale = torch.full((self.pages, page), float("nan"), device=DEV)
        self.rope_scale = torch.full((self.pages, page), float("nan"), device=DEV)
        self.desc = fx.latent_cache(self.codes, self.scale, self.rope_scale, self.pages, page, latent, rope)
        self.dtable = torch.from_numpy(self.table).to(DEV)

    def batch(self, new, length, max_new=None, max_len=None, tokens=None):
        start = torch.tensor([0] + list(new)).cumsum(0).to(torch.int32).to(DEV)
        ln = torch.tensor(list(length), dtype=torch.int32, device=DEV)
        return self.fx.kv_batch(start, ln, self.dtable, len(new), self.width, int(sum(new)) if tokens is None else tokens,
                                max(new) if max_new is None else max_new, max(length) if max_len is None else max_len)

    def fill(self, lens, seed, spread=0.3):
        """Codes and scales of the sequences' tokens, on the host too."""
        g = torch.Generator().manual_seed(seed)
        codes, scale, rope_scale = self.codes.cpu(), self.scale.cpu(), self.rope_scale.cpu()
        for s, n in enumerate(lens):
            for nth in range(-(-n // self.page)):
                k, p = min(self.page, n - nth * self.page), int(self.table[s, nth])
                codes[p, :k] = (torch.randn(k, self.latent + self.rope, generator=g) * 40).round().clamp(-127, 127).to(torch.int8)
                scale[p, :k] = 0.02 * torch.exp(spread * torch.randn(k, generator=g))
                rope_scale[p, :k] = 0.03 * torch.exp(spread * torch.randn(k, generator=g))
        for to, x in ((self.codes, codes), (self.scale, scale), (self.rope_scale, rope_scale)):
            to.copy_(x)

    def held(self, s, n):
        """Codes, latent values and key values (64 bits) of a sequence's first n tokens."""
        p = torch.from_numpy(self.table[s, : -(-n // self.page)].astype(np.int64))
        c = self.codes.cpu()[p].flatten(0, 1)[:n]
        v = c[:, : self.latent].double() * self.scale.cpu()[p].flatten()[:n, None].double()
        return c, v, c[:, self.latent :].double() * self.rope_scale.cpu()[p].flatten()[:n, None].double()


def tables(positions, dims, stretch=1.0):
    ang = torch.arange(positions, dtype=torch.float64)[:, None] / stretch * 10000.0 ** (-torch.arange(0, dims, 2).double() / dims)
    return ang.cos().float(), ang.sin().float()


def rotate(x, cos, sin, interleaved):
    """Products of fp32 numbers are exact in fp64; one rounding there, one to fp32."""
    x, cos, sin = x.double(), cos.double(), sin.double()
    k = x.shape[-1] // 2
    x1, x2 = (x[..., 0::2], x[..., 1::2]) if interleaved else (x[..., :k], x[..., k:])
    y = (x1 * cos - x2 * sin, x2 * cos + x1 * sin)
    return (torch.stack(y, -1).flatten(-2) if interleaved else torch.cat(y, -1)).float()


def quantized(x, rule):
    """Codes and scale of rows of finite fp32 values, in fp32 steps."""
    a = x.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -100)
    if rule == "max":
        return (x * (torch.full_like(a, 127.0) / a)).round(), (a / 127.0)[:, 0]
    m, e = torch.frexp(a)
    s = torch.ldexp(torch.ones_like(a), e - 7 + (m * 128.0 >= 127.5).int())
    return (x / s).round(), s[:, 0]


APPEND = [  # (page, latent, rope, heads, nope, interleaved, rule, steps of new tokens of each sequence)
    (16, 512, 64, 4, 128, 1, "max", [(5, 0, 16), (1, 1, 1), (12, 33, 0), (1, 0, 1)]),
    (64, 256, 32, 3, 64, 0, "dfx", [(70, 1), (1, 130)]),
    (128, 512, 16, 1, 16, 1, "dfx", [(1,), (1,), (200,)]),
    (32, 256, 48, 17, 64, 0, "max", [(31, 32, 33), (40, 1, 64)]),
]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("gap", [0, 3], ids=["aligned", "odd strides"])
@pytest.mark.parametrize("case", APPEND, ids=str)
def test_append_and_read(fx, h, t, case, gap):
    page, latent, rope, heads, nope, interleaved, rule, steps = case
    note("latent append", t, case, gap)
    S, T = len(steps[0]), TYPES[t]
    lens = [0] * S
    total = [sum(st[s] for st in steps) for s in range(S)]
    cache = Cache(fx, total, latent, rope, page, seed=latent + rope)
    want_codes, want_scale, want_rope = cache.codes.cpu(), cache.scale.cpu(), cache.rope_scale.cpu()
    cos, sin = tables(max(total) + 3, rope, stretch=4.0)
    rot = fx.rotary(cos.to(DEV), sin.to(DEV), cos.shape[0], rope, interleaved)
    g = torch.Generator().manual_seed(page + latent)
    d, off = nope + rope, 1 if gap else 0
    for new in steps:
        lens = [a + b for a, b in zip(lens, new)]
        n = sum(new)
        width = latent + rope + gap
        x = (torch.randn(n, width, generator=g) * torch.exp(torch.randn(n, 1, generator=g))).to(T)
        q = torch.randn(n, heads * d + gap, generator=g).to(T)
        xd, qd = (torch.cat([torch.zeros(off, dtype=T), v.flatten()]).to(DEV) for v in (x, q))
        q_out = torch.full((n, heads, rope + gap), 5.0, dtype=T, device=DEV)
        batch = cache.batch(new, lens)
        fx.latent_append(h, cache.desc, batch, rot, fx.SCALE_DFX if rule == "dfx" else fx.SCALE_MAX, xd[off:], width,
                         xd[off + latent :], width, qd[off + nope :], heads * d + gap, d, q_out, heads * (rope + gap), rope + gap,
                         heads, code_of(fx, t))
        outs = [torch.full((n, w + gap), 5.0, dtype=T, device=DEV) for w in (latent, rope)]
        fx.latent_read(h, cache.desc, batch, None, n, None, 0, None, outs[0], latent + gap, outs[1], rope + gap, code_of(fx, t))
        assert fx.sync_status(h) == 0
        pos = torch.cat([torch.arange(a - b, a) for a, b in zip(lens, new)])
        turned = rotate(q[:, : heads * d].float().view(n, heads, d)[..., nope:], cos[pos][:, None], sin[pos][:, None], interleaved)
        assert torch.equal(q_out[..., :rope].cpu(), turned.to(T)) and (q_out[..., rope:] == 5.0).all()
        lc, ls = quantized(x[:, :latent].float(), rule)
        kc, ks = quantized(rotate(x[:, latent : latent + rope], cos[pos], sin[pos], interleaved), rule)
        seq = torch.cat([torch.full((b,), s) for s, b in enumerate(new)]).long()
        p, slot = torch.from_numpy(cache.table)[seq, pos // page].long(), pos % page
        want_codes[p, slot] = torch.cat([lc, kc], 1).to(torch.int8)
        want_scale[p, slot], want_rope[p, slot] = ls, ks
        assert torch.equal(cache.codes.cpu(), want_codes)
        for got, want in ((cache.scale, want_scale), (cache.rope_scale, want_rope)):
            assert torch.equal(torch.nan_to_num(got.cpu(), -1.0), torch.nan_to_num(want, -1.0))
        assert torch.equal(outs[0][:, :latent].cpu(), (lc * ls[:, None]).to(T)) and (outs[0][:, latent:] == 5.0).all()
        assert torch.equal(outs[1][:, :rope].cpu(), (kc * ks[:, None]).to(T)) and (outs[1][:, rope:] == 5.0).all()
    # all tokens of the sequences: the operand of the 8-bit product
    held = sum(lens)
    kv_start = torch.tensor([0] + lens).cumsum(0).to(torch.int32).to(DEV)
    rows = torch.full((held + 1, latent + 16), 77, dtype=torch.int8, device=DEV)
    steps_out = torch.full((held + 1,), 5.0, device=DEV)
    keys = torch.full((held + 1, rope), 5.0, dtype=T, device=DEV)
    empty = cache.batch([0] * S, lens, max_new=0)
    fx.latent_read(h, cache.desc, empty, kv_start, held, rows, latent + 16, steps_out, None, 0, keys, rope, code_of(fx, t))
    assert fx.sync_status(h) == 0
    at = 0
    for s, n in enumerate(lens):
        c, _, k = cache.held(s, n)
        assert torch.equal(rows[at : at + n, :latent].cpu(), c[:, :latent])
        p = torch.from_numpy(cache.table[s, : -(-n // page)].astype(np.int64))
        assert torch.equal(steps_out[at : at + n].cpu(), want_scale[p].flatten()[:n])
        assert torch.equal(keys[at : at + n].cpu(), (c[:, latent:].float() * want_rope[p].flatten()[:n, None]).to(T))
        at += n
    assert (rows[held] == 77).all() and (rows[:, latent:] == 77).all() and steps_out[held] == 5.0 and (keys[held] == 5.0).all()


def test_append_in_place_without_rotation_and_nonfinite(fx, h):
    """Queries rotated where they lie; a NaN or an infinity in a latent or a key is stored
    as 0 and takes no part in the scale; rows of zeros; without rotation keys as they are."""
    cache = Cache(fx, [16], 256, 64, 16)
    x = torch.randn(4, 320, generator=torch.Generator().manual_seed(1))
    x[0, 5], x[1, 300], x[3] = float("nan"), float("-inf"), 0.0
    q = torch.randn(4, 2, 64, generator=torch.Generator().manual_seed(2))
    for rot in (None, tables(16, 64)):
        r = None if rot is None else fx.rotary(rot[0].to(DEV), rot[1].to(DEV), 16, 64, 1)
        xd, qd = x.to(DEV), q.to(DEV)
        fx.latent_append(h, cache.desc, cache.batch([4], [9]), r, fx.SCALE_MAX, xd, 320, xd[:, 256:], 320, qd, 128, 64, qd, 128,
                         64, 2, fx.F32)
        assert fx.sync_status(h) == fx.FLAG_NONFINITE
        p = int(cache.table[0, 0])
        clean = x.clone()
        clean[0, 5] = 0.0
        turn = lambda v: v if rot is None else rotate(v, rot[0][5:9], rot[1][5:9], 1)  # noqa: E731
        key = torch.nan_to_num(turn(clean[:, 256:]), nan=0.0, posinf=0.0, neginf=0.0)
        lc, ls = quantized(clean[:, :256], "max")
        kc, ks = quantized(key, "max")
        assert torch.equal(cache.codes[p, 5:9].cpu(), torch.cat([lc, kc], 1).to(torch.int8))
        assert torch.equal(cache.scale[p, 5:9].cpu(), ls) and torch.equal(cache.rope_scale[p, 5:9].cpu(), ks)
        want = q if rot is None else rotate(q, rot[0][5:9][:, None], rot[1][5:9][:, None], 1)
        assert torch.equal(qd.cpu(), want)
        assert (cache.codes[p, :5] == -128).all() and (cache.codes[p, 9:] == -128).all() and cache.scale[p, 9:].isnan().all()


def test_calls_skip_what_contradicts(fx, h):
    """Sequences whose numbers contradict the bounds, the table or the rotation are left
    alone and the others served; pages outside the cache are not touched."""
    cache = Cache(fx, [40, 40, 40, 40], 256, 32, 16)
    g = torch.Generator().manual_seed(4)
    x, q = torch.randn(12, 288, generator=g).to(DEV), torch.randn(12, 3, 32, generator=g).to(DEV)
    cos, sin = tables(30, 32)
    rot = fx.rotary(cos.to(DEV), sin.to(DEV), 30, 32)
    start = torch.tensor([0, 3, 6, 9, 12], dtype=torch.int32, device=DEV)
    length = torch.tensor([20, 31, 2, 25], dtype=torch.int32, device=DEV)  # the second is past the rotation, the third shorter than its new tokens
    cache.dtable[3, 1] = 10 ** 6
    batch = fx.kv_batch(start, length, cache.dtable, 4, cache.width, 12, 3, 31)
    out = torch.full((12, 3, 32), 5.0, device=DEV)
    fx.latent_append(h, cache.desc, batch, rot, fx.SCALE_MAX, x, 288, x[:, 256:], 288, q, 96, 32, out, 96, 32, 3, fx.F32)
    assert fx.sync_status(h) == fx.FLAG_RANGE
    assert (out[3:9] == 5.0).all() and (out[:3] != 5.0).any(-1).all() and (out[9:] != 5.0).any(-1).all()
    touched = cache.scale.cpu().isnan().logical_not()
    assert touched.sum() == 3 and touched[int(cache.table[0, 1]), 1:4].all()
    back = torch.full((12, 256), 5.0, device=DEV)
    fx.latent_read(h, cache.desc, batch, None, 12, None, 0, None, back, 256, None, 0, fx.F32)
    assert fx.sync_status(h) == fx.FLAG_RANGE
    assert (back[6:9] == 5.0).all() and (back[9:] == 0.0).all() and (back[:3] != 5.0).any(-1).all()
    # rows that do not match a sequence's length, or pass the bound
    kv_start = torch.tensor([0, 20, 51, 53, 78], dtype=torch.int32, device=DEV)
    good = fx.kv_batch(torch.zeros(5, dtype=torch.int32, device=DEV), length, cache.dtable, 4, cache.width, 0, 0, 31)
    rows = torch.full((78, 256), 77, dtype=torch.int8, device=DEV)
    fx.latent_read(h, cache.desc, good, kv_start + torch.tensor([0, 0, 0, 1, 0], device=DEV, dtype=torch.int32), 60, rows, 256, None, None,
                   0, None, 0, fx.F32)
    assert fx.sync_status(h) == fx.FLAG_RANGE
    assert (rows[51:] == 77).all() and (rows[:51, 0] != 77).any()


# ---- attention over the latents ---------------------------------------------------

def want_latent(cache, s, n, fresh, q, qr, scale, causal):
    """64-bit result and tolerance of one sequence: q, qr [fresh, heads, ...] doubles."""
    _, v, k = cache.held(s, n)
    x = (q @ v.t() + qr @ k.t()) * scale
    mag = abs(scale) * (q.abs() @ v.abs().t() + qr.abs() @ k.abs().t())
    seen = torch.arange(n) <= (n - fresh + torch.arange(fresh))[:, None] if causal else torch.ones(fresh, n, dtype=torch.bool)
    w = torch.softmax(x.masked_fill(~seen[:, None], -math.inf), -1)
    out = w @ v
    keep = seen[:, None].expand_as(x)
    tops = torch.cat([q, qr], -1).abs().amax(-1)
    return out, (mag * keep).amax(-1), (x.abs() * keep).amax(-1), tops * (v.abs().sum(1).max() + k.abs().sum(1).max()) * abs(scale), v.abs().max()


def check_latent(got, cache, lens, new, q, qr, scale, causal, t, more=0.0):
    at = 0
    for s, (n, fresh) in enumerate(zip(lens, new)):
        if fresh == 0:
            continue
        want, mag, x, ends, S = want_latent(cache, s, n, fresh, q[at : at + fresh].double(), qr[at : at + fresh].double(), scale, causal)
        d = mag * ((cache.latent + cache.rope + 8) * 2.0 ** -24 + (2.0 ** -22 if t == "f32" else 0)) + ends * 2.0 ** -38 + 4 * 2.0 ** -24 * x + more
        uP = 2.0 ** -22 if t == "f32" else 2.0 ** -11
        tol = S * (2 * d + 4 * 2.0 ** -23 + uP + n * 2.0 ** -31 + 2 * (n + 64) * 2.0 ** -24)[..., None] + 1.01 * HALF_ULP[t] * want.abs()
        off = (got[at : at + fresh].double() - want).abs()
        assert (off <= tol).all(), (s, float((off / tol).max()))
        at += fresh


def run_latent(fx, h, cache, new, lens, q, qr, scale, causal, t, layout="token", **bounds):
    T, H, W, R = sum(new), q.shape[1], cache.latent, cache.rope
    dt = TYPES[t]
    out = torch.full((T * H * (W + 4) + 8,), 5.0, dtype=dt, device=DEV)
    if layout == "token":
        a, b, strides, o_strides, off = q.to(DEV), qr.to(DEV), (H * W, W, H * R, R), (H * W, W), 0
    elif layout == "head":  # each head's tokens side by side
        a, b = q.transpose(0, 1).contiguous().to(DEV), qr.transpose(0, 1).contiguous().to(DEV)
        strides, o_strides, off = (W, T * W, R, T * R), (W, T * W), 0
    else:  # odd strides and an odd start: rows of latent and key beside each other
        both = torch.cat([q, qr, torch.zeros(T, H, 3, dtype=dt)], -1)
        a = torch.cat([torch.zeros(1, dtype=dt), both.flatten()]).to(DEV)[1:]
        b, D = a[W:], W + R + 3
        strides, o_strides, off = (H * D, D, H * D, D), (H * (W + 3), W + 3), 1
    batch = cache.batch(new, lens, **bounds)
    need = fx.latent_attention_workspace(h, cache.desc, batch, H)
    ws = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device=DEV)
    fx.latent_attention(h, cache.desc, batch, a, strides[0], strides[1], b, strides[2], strides[3], H, scale, causal, out[off:],
                        o_strides[0], o_strides[1], code_of(fx, t), ws, need)
    got = torch.as_strided(out, (T, H, W), (o_strides[0], o_strides[1], 1), off).cpu()
    rest = out.clone()
    torch.as_strided(rest, (T, H, W), (o_strides[0], o_strides[1], 1), off).fill_(5.0)
    assert (rest == 5.0).all()
    return got


LATENT = [  # (latent, rope, page, heads, new, lengths, causal)
    (512, 64, 16, 1, [1], [1], 1),
    (512, 64, 16, 16, [1, 1, 1, 1], [300, 17, 16, 1], 1),
    (256, 32, 32, 7, [3, 0, 1], [129, 40, 64], 1),
    (512, 16, 128, 16, [1, 1], [63, 65], 0),
    (256, 48, 64, 33, [1, 2], [513, 31], 1),
    (512, 64, 64, 12, [5, 70], [2100, 70], 1),
    (512, 64, 64, 40, [2], [5000], 0),
    (256, 64, 16, 128, [1, 1], [200, 3000], 1),
    (512, 32, 64, 128, [3], [1000], 1),
]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", LATENT, ids=str)
def test_latent_attention(fx, h, t, case):
    latent, rope, page, heads, new, lens, causal = case
    note("latent attention", t, case)
    cache = Cache(fx, lens, latent, rope, page, seed=latent + page)
    cache.fill(lens, 7)
    g = torch.Generator().manual_seed(11)
    q = torch.randn(sum(new), heads, latent, generator=g).to(TYPES[t])
    qr = torch.randn(sum(new), heads, rope, generator=g).to(TYPES[t])
    for layout in ("token", "head", "odd"):
        got = run_latent(fx, h, cache, new, lens, q, qr, 0.07, causal, t, layout)
        assert fx.sync_status(h) == 0
        check_latent(got, cache, lens, new, q, qr, 0.07, causal, t)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("new", [[0, 3, 2, 1], [1, 1, 1, 1]], ids=str)
def test_latent_attention_of_short_sequences_under_wide_bounds(fx, h, t, new):
    """More splits than there is work, and tensors with rows behind the last sequence."""
    lens = [4, 3, 2, 1]
    cache = Cache(fx, [4096] * 4, 512, 64, 16)
    cache.fill(lens, 3)
    g = torch.Generator().manual_seed(1)
    q, qr = torch.randn(sum(new), 20, 512, generator=g).to(TYPES[t]), torch.randn(sum(new), 20, 64, generator=g).to(TYPES[t])
    for bounds in (dict(), dict(max_len=4096)):
        got = run_latent(fx, h, cache, new, lens, q, qr, 0.3, 1, t, **bounds)
        assert fx.sync_status(h) == 0
        check_latent(got, cache, lens, new, q, qr, 0.3, 1, t)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("case", [(256, 100, 128, 90, 3000), (512, 150, 40, 40, 1500), (256, 230, 20, 200, 900), (512, 40, 70, 64, 64)], ids=str)
def test_latent_attention_of_many_uneven_sequences(fx, h, t, case):
    """More sequences than run at a time, one of them far longer, some without new tokens."""
    latent, S, heads, most, longest = case
    note("latent attention", t, case)
    rng = np.random.default_rng(S)
    lens = rng.integers(1, most + 1, S).tolist()
    lens[S // 3] = longest
    new = [0 if i % 17 == 3 else 1 for i in range(S)]
    cache = Cache(fx, lens, latent, 32, 64, seed=S)
    cache.fill(lens, 21)
    g = torch.Generator().manual_seed(S)
    q = torch.randn(sum(new), heads, latent, generator=g).to(TYPES[t])
    qr = torch.randn(sum(new), heads, 32, generator=g).to(TYPES[t])
    got = run_latent(fx, h, cache, new, lens, q, qr, 0.05, 1, t)
    assert fx.sync_status(h) == 0
    check_latent(got, cache, lens, new, q, qr, 0.05, 1, t)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads", [4, 33])
def test_latent_attention_extremes(fx, h, t, heads):
    """Scale 0 and below 0, one token that takes all, a query of zeros, a lone huge
    dimension, tiny queries; a NaN and an infinity make their own rows NaN only."""
    lens = [400]
    cache = Cache(fx, lens, 512, 64, 16)
    cache.fill(lens, 5)
    g = torch.Generator().manual_seed(8)
    q, qr = torch.randn(2, heads, 512, generator=g), torch.randn(2, heads, 64, generator=g)
    q[0, 0], qr[0, 0] = 0, 0
    q[0, 1, 7] = 3000.0
    q[0, 2] *= 1e-3
    q, qr = q.to(TYPES[t]), qr.to(TYPES[t])
    for scale in (0.0, 2.0, -0.2):
        got = run_latent(fx, h, cache, [2], lens, q, qr, scale, 1, t)
        assert fx.sync_status(h) == 0
        check_latent(got, cache, lens, [2], q, qr, scale, 1, t)
    q[0, 2, 3], qr[1, 3, 1] = float("nan"), float("inf")
    got = run_latent(fx, h, cache, [2], lens, q, qr, 0.1, 1, t)
    bad = got.isnan()
    assert bad[0, 2].all() and bad[1, 3].all() and bad.sum() == 2 * 512


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("latent,heads", [(512, 16), (256, 64), (512, 40)])
def test_latent_attention_of_queries_of_one_sign(fx, h, t, latent, heads):
    lens = [900, 70]
    cache = Cache(fx, lens, latent, 64, 16)
    cache.fill(lens, 12)
    g = torch.Generator().manual_seed(14)
    q, qr = (torch.rand(2, heads, latent, generator=g) + 1).to(TYPES[t]), -(torch.rand(2, heads, 64, generator=g) + 1).to(TYPES[t])
    got = run_latent(fx, h, cache, [1, 1], lens, q, qr, 0.1, 1, t)
    assert fx.sync_status(h) == 0
    at_most = max(float(cache.scale.nan_to_num().max()), float(cache.rope_scale.nan_to_num().max()))
    d = 0.1 * at_most * 1279 * float((q.double().abs().sum(-1) + qr.double().abs().sum(-1)).max()) * (latent + 64) / 8 * 2.0 ** -24
    check_latent(got, cache, lens, [1, 1], q, qr, 0.1, 1, t, more=0.0 if t == "f32" else d)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_latent_attention_of_uneven_scales(fx, h, t):
    """Token scales that differ by 2^40 and grow along the cache, tokens of zeros (the
    smallest scale there is) that take most of the weight through the shared key."""
    lens = [700]
    cache = Cache(fx, lens, 256, 32, 64)
    cache.fill(lens, 9)
    g = torch.Generator().manual_seed(3)
    p = torch.from_numpy(cache.table[0].astype(np.int64)).to(DEV)
    step = torch.exp2(torch.arange(704) / 704 * 40 - 46)
    cache.scale[p] = step.view(11, 64).to(DEV)
    cache.codes[p[2], :, :256] = 0
    cache.scale[p[2]] = 2.0 ** -100 / 127
    cache.rope_scale[p[2]] = 0.5
    q = torch.randn(1, 20, 256, generator=g).to(TYPES[t])
    qr = torch.randn(1, 20, 32, generator=g).to(TYPES[t])
    q = (q.float() * 2.0 ** 4).to(TYPES[t])
    got = run_latent(fx, h, cache, [1], lens, q, qr, 0.07, 1, t)
    assert fx.sync_status(h) == 0
    check_latent(got, cache, lens, [1], q, qr, 0.07, 1, t)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_latent_attention_of_huge_logits(fx, h, t, sign):
    """Equal tokens give equal logits, here near 2^110 either way: every weight is the
    same and the result the tokens' one value."""
    lens = [1500]
    cache = Cache(fx, lens, 256, 32, 64)
    cache.codes.fill_(100)
    cache.scale.fill_(2.0 ** -6)
    cache.rope_scale.fill_(2.0 ** -6)
    q = torch.full((1, 4, 256), sign * 2.0 ** 102).to(TYPES[t])
    qr = torch.zeros(1, 4, 32).to(TYPES[t])
    got = run_latent(fx, h, cache, [1], lens, q, qr, 1.0, 0, t)
    assert fx.sync_status(h) == 0
    want = 100 * 2.0 ** -6
    assert ((got.double() - want).abs() <= want * ((lens[0] + 64) * 2.0 ** -23 + HALF_ULP[t] + 2.0 ** -22)).all()


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("heads", [4, 20])
@pytest.mark.parametrize("size", [2.0 ** 14, 2.0 ** 30, 2.0 ** 70], ids=["2^14", "2^30", "2^70"])
def test_latent_attention_of_large_logits_takes_the_largest(fx, h, t, heads, size):
    """Logits past 2^24, which fp32 holds in steps above one: one token takes all.  The
    logits of a row differ by 2^-9 of their size and more, so that all other weights are 0;
    the result is off by the weight's rounding, which the sum does not share, and its own."""
    lens = [1000]
    cache = Cache(fx, lens, 256, 32, 64)
    cache.fill(lens, 31, spread=0.6)
    g = torch.Generator().manual_seed(2)
    up = min(size, 2.0 ** 15) if t == "f16" else size
    for scale in (0.7 * size / up, -0.7 * size / up) if size > 2.0 ** 14 else (0.7 * 2.0 ** 14, -0.7 * 2.0 ** 13):
        q = (torch.rand(1, heads, 256, generator=g) + 1).mul(up).mul(torch.rand(1, heads, 256, generator=g).sub(0.5).sign()).to(TYPES[t])
        qr = torch.zeros(1, heads, 32).to(TYPES[t])
        _, v, _ = cache.held(0, lens[0])
        x = q[0].double() @ v.t() * scale
        top = x.topk(2, -1)
        told = (top.values[:, 0] - top.values[:, 1]) / x.abs().amax(-1) > 2.0 ** -9
        assert told.sum() >= heads // 2
        want = v[top.indices[:, 0]]
        got = run_latent(fx, h, cache, [1], lens, q, qr, scale, 0, t)[0].double()
        assert fx.sync_status(h) == 0
        uP = 2.0 ** -22 if t == "f32" else 2.0 ** -11
        assert ((got - want).abs() <= want.abs() * (uP + 8 * 2.0 ** -24 + 1.01 * HALF_ULP[t]))[told].all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("power", [20, 24, 28, 60, 105])
def test_latent_attention_of_equal_large_logits(fx, h, t, sign, power):
    """Equal tokens, of logits that no float holds exactly: every weight is the same."""
    lens = [700]
    cache = Cache(fx, lens, 256, 32, 64)
    cache.codes.fill_(101)
    cache.scale.fill_(0.0137)
    cache.rope_scale.fill_(0.0137)
    q = torch.full((1, 20, 256), sign * 0.37 * 2.0 ** power).to(TYPES[t])
    got = run_latent(fx, h, cache, [1], lens, q, torch.zeros(1, 20, 32).to(TYPES[t]), 1.1, 0, t)
    assert fx.sync_status(h) == 0
    want = 101 * float(torch.tensor(0.0137))
    uP = 2.0 ** -22 if t == "f32" else 2.0 ** -11
    assert ((got.double() - want).abs() <= want * ((lens[0] + 64) * 2.0 ** -23 + HALF_ULP[t] * 1.01 + uP + 2.0 ** -22)).all()


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("below", [3, 9, 21, 34, 45])
def test_latent_attention_of_large_logits_and_uneven_scales(fx, h, t, below):
    """One token takes all through the shared key, and its latent's scale is 2^-below of
    the others', whose logits are 0.  Weights are written as f16 and a scale's power of two
    is in them: the result is off by 2^-24 of the others' values, besides its roundings."""
    lens = [300]
    cache = Cache(fx, lens, 256, 32, 64)
    cache.codes.fill_(90)
    cache.codes[..., 256:] = 0
    cache.scale.fill_(1.0)
    cache.rope_scale.fill_(1.0)
    page = int(cache.table[0, 2])
    cache.codes[page, 5, 256:] = 101
    cache.scale[page, 5] = 2.0 ** -below
    want = 90 * 2.0 ** -below
    for power in range(20, 33):
        for heads in (4, 20):
            qr = torch.full((1, heads, 32), 0.37).to(TYPES[t])
            scale = 2.0 ** power / (0.37 * 32 * 101)
            got = run_latent(fx, h, cache, [1], lens, torch.zeros(1, heads, 256).to(TYPES[t]), qr, scale, 0, t).double()
            assert fx.sync_status(h) == 0
            uP = 2.0 ** -22 if t == "f32" else 2.0 ** -11
            assert ((got - want).abs() <= 90 * 2.0 ** -24 + want * (uP + 8 * 2.0 ** -24 + 1.01 * HALF_ULP[t])).all(), (power, heads)


def test_latent_attention_page_outside_the_cache(fx, h):
    """Its tokens are not seen, and the flag is raised; a query that sees nothing gets 0."""
    lens = [100]
    cache = Cache(fx, lens, 256, 32, 16)
    cache.fill(lens, 6)
    g = torch.Generator().manual_seed(9)
    q, qr = torch.randn(1, 4, 256, generator=g), torch.randn(1, 4, 32, generator=g)
    cache.dtable[0, 2] = -5
    got = run_latent(fx, h, cache, [1], lens, q, qr, 0.06, 1, "f32")
    assert fx.sync_status(h) == fx.FLAG_RANGE
    _, v, k = cache.held(0, 100)
    keep = torch.from_numpy(np.r_[0:32, 48:100])
    w = torch.softmax((q[0].double() @ v[keep].t() + qr[0].double() @ k[keep].t()) * 0.06, -1)
    assert ((got[0].double() - w @ v[keep]).abs() <= 1e-5 * v.abs().max()).all()
    cache.dtable.fill_(10 ** 6)
    got = run_latent(fx, h, cache, [1], lens, q, qr, 0.06, 1, "f32")
    assert fx.sync_status(h) == fx.FLAG_RANGE and (got == 0).all()


# ---- attention over expanded keys and values ----------------------------------------

EXPANDED = [  # (nope, rope, vdim, heads, new, lengths, causal)
    (64, 32, 64, 1, [1], [1], 1),
    (128, 64, 128, 3, [130, 1], [130, 300], 1),
    (64, 64, 128, 2, [65, 0, 64], [100, 40, 64], 1),
    (128, 32, 64, 5, [3, 200], [900, 200], 0),
    (128, 64, 128, 2, [17], [1000], 1),
    (64, 32, 128, 8, [300], [333], 1),
    (128, 32, 128, 1, [129, 33], [129, 1025], 1),
    (128, 64, 64, 4, [31, 32, 33], [31, 95, 97], 1),
    (64, 64, 64, 3, [16, 2], [4000, 129], 1),
    # many rows: 64 and 128 of them a block
    (128, 64, 128, 40, [90, 3], [200, 77], 1),
    (128, 64, 128, 64, [150, 129, 140, 1], [400, 129, 150, 300], 1),
    (64, 32, 64, 64, [140, 150, 1, 0], [150, 170, 40, 9], 0),
    (64, 32, 128, 70, [65, 129, 128, 64], [65, 130, 300, 64], 1),
]


def run_expanded(fx, h, c, new, lens, q, k, key, v, scale, t, odd=False, rows=None):
    nope, rope, vdim, heads, causal = c
    held, T, dt = sum(lens), sum(new), TYPES[t]
    gap, off = (3, 1) if odd else (0, 0)
    lead = lambda x: torch.cat([torch.zeros(off, dtype=dt), x.flatten()]).to(DEV)[off:]  # noqa: E731
    wide = lambda x: lead(torch.cat([x, torch.full((*x.shape[:-1], gap), float("nan"), dtype=dt)], -1))  # noqa: E731
    kv = wide(torch.cat([k, v], -1))  # each head's key and value beside each other
    w = nope + vdim + gap
    qd, kd = wide(q.flatten(1)), wide(key)
    ldo = heads * vdim + gap
    out = torch.full((T * ldo + 8,), 5.0, dtype=dt, device=DEV)
    rows = torch.tensor([0] + list(lens)).cumsum(0).to(torch.int32).to(DEV) if rows is None else rows
    desc = fx.expanded_kv(kv, heads * w, w, kd, rope + gap, kv[nope:], heads * w, w, rows, held, heads, nope, rope, vdim)
    start = torch.tensor([0] + list(new)).cumsum(0).to(torch.int32).to(DEV)
    batch = fx.kv_batch(start, torch.tensor(lens, dtype=torch.int32, device=DEV), None, len(new), 0, T, max(new), max(lens))
    fx.expanded_attention(h, desc, batch, qd, heads * (nope + rope) + gap, scale, causal, out[off:], ldo, code_of(fx, t))
    o = out.cpu()
    assert (o[:off] == 5.0).all() and (o[off + T * ldo :] == 5.0).all()
    o = o[off : off + T * ldo].view(T, ldo)
    assert (o[:, heads * vdim :] == 5.0).all()
    return o[:, : heads * vdim].reshape(T, heads, vdim)


def check_expanded(got, c, new, lens, q, k, key, v, scale, t):
    nope, rope, vdim, heads, causal = c
    at = first = 0
    for n, fresh in zip(lens, new):
        if fresh:
            kk = torch.cat([k[first : first + n], key[first : first + n, None].expand(n, heads, rope)], -1).double().permute(1, 2, 0).contiguous()
            vv = v[first : first + n].double().transpose(0, 1).contiguous()
            qq = q[at : at + fresh].double().transpose(0, 1).contiguous()
            x = qq @ kk * scale
            seen = torch.arange(n) <= (n - fresh + torch.arange(fresh))[:, None] if causal else torch.ones(fresh, n, dtype=torch.bool)
            want = (torch.softmax(x.masked_fill(~seen, -math.inf), -1) @ vv).transpose(0, 1)
            mag = ((qq.abs() @ kk.abs()) * abs(scale) * seen).amax(-1).t()
            d = mag * (nope + rope + 8) * 2.0 ** -24 + 4 * 2.0 ** -24 * (x.abs() * seen).amax(-1).t()
            tol = vv.abs().amax((1, 2))[:, None] * (2 * d + 4 * 2.0 ** -23 + HALF_ULP[t] + n * 2.0 ** -31 + 2 * (n + 64) * 2.0 ** -24)[..., None]
            tol = tol + 1.01 * HALF_ULP[t] * want.abs()
            off = (got[at : at + fresh].double() - want).abs()
            assert (off <= tol).all(), (n, fresh, float((off / tol).max()))
        at += fresh
        first += n


def heads_of(c, new, lens, t, seed):
    nope, rope, vdim, heads, _ = c
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g).to(TYPES[t])  # noqa: E731
    return r(sum(new), heads, nope + rope), r(sum(lens), heads, nope), r(sum(lens), rope), r(sum(lens), heads, vdim)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", EXPANDED, ids=str)
def test_expanded_attention(fx, h, t, case):
    *c, new, lens, causal = case
    c = (*c, causal)
    note("expanded attention", t, case)
    q, k, key, v = heads_of(c, new, lens, t, 5)
    for odd in (False, True):
        for scale in (0.1, -0.3) if odd else (0.1, 0.0):
            got = run_expanded(fx, h, c, new, lens, q, k, key, v, scale, t, odd)
            assert fx.sync_status(h) == 0
            check_expanded(got, c, new, lens, q, k, key, v, scale, t)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("fresh,before,q0,heads", [(90, 110, 50, 2), (128, 0, 5, 2), (200, 7, 130, 2), (3, 300, 1, 2), (90, 110, 50, 40),
                                                   (150, 60, 20, 40), (200, 7, 130, 256), (150, 30, 20, 256)])
def test_expanded_attention_sees_nothing_of_masked_places(fx, h, t, fresh, before, q0, heads):
    """NaN and infinities in keys, shared keys and values that a query does not see leave
    its result alone, bit for bit; a query that sees one in a value has it in that dimension
    only, one that sees one in a key is NaN."""
    c, new, lens = (128, 64, 128, heads, 1), [fresh, 40], [before + fresh, 40]
    q, k, key, v = heads_of(c, new, lens, t, 6)
    clean = run_expanded(fx, h, c, new, lens, q, k, key, v, 0.1, t)
    at = before + q0  # the place of the first sequence's query q0
    for what, x in (("value", v), ("key", k), ("shared", key)):
        for bad in (float("nan"), float("inf")):
            y = x.clone()
            y[at, ..., 7] = bad
            args = [y if x is z else z for z in (k, key, v)]
            got = run_expanded(fx, h, c, new, lens, q, *args, 0.1, t)
            assert fx.sync_status(h) == 0
            assert torch.equal(got[:q0], clean[:q0]) and torch.equal(got[fresh:], clean[fresh:])
            if what == "value":
                assert not got[q0:fresh, :, 7].isfinite().any()
                keep = [i for i in range(128) if i != 7]
                assert torch.equal(got[q0:fresh][..., keep], clean[q0:fresh][..., keep])
            elif bad != bad:
                assert got[q0:fresh].isnan().all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_expanded_attention_of_huge_logits(fx, h, t, sign):
    """Equal keys, logits near 2^100 either way: the mean of the values."""
    c, new, lens = (64, 32, 64, 1, 0), [70], [700]
    q, k, key, v = heads_of(c, new, lens, t, 7)
    q = torch.full_like(q, sign * 2.0 ** 50)
    k, key = torch.full_like(k, 2.0 ** 44), torch.full_like(key, 2.0 ** 44)
    got = run_expanded(fx, h, c, new, lens, q, k, key, v, 1.0, t)
    want = v[:, 0].double().mean(0)
    tol = v.double().abs().max() * ((700 + 64) * 2.0 ** -23) + HALF_ULP[t] * want.abs() * 1.01
    assert ((got[:, 0].double() - want).abs() <= tol).all()


def test_expanded_attention_skips_what_contradicts(fx, h):
    c, new, lens = (64, 32, 64, 2, 1), [5, 6, 7], [50, 60, 70]
    q, k, key, v = heads_of(c, new, lens, "f32", 8)
    rows = torch.tensor([0, 50, 111, 181], dtype=torch.int32, device=DEV)  # 61 and 70 rows, the last past the bound of 180
    got = run_expanded(fx, h, c, new, lens, q, k, key, v, 0.1, "f32", rows=rows)
    assert fx.sync_status(h) == fx.FLAG_RANGE
    assert (got[5:] == 5.0).all() and torch.isfinite(got[:5]).all() and (got[:5] != 5.0).all()
