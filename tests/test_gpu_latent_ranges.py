"""Latent attention at the ends of its range: codes that a few channels leave
small, queries and scales of any size, row tiles that are not cut, values that cancel.

The tolerance is the one of test_gpu_latent.py, held to what each dimension's own tokens
weigh: a weight off by a share e moves dimension d by at most e sum_j w_j |v_jd|, not by e
times the largest value of all dimensions."""
import math

import pytest

from gpu_util import DEV, note
from test_gpu_latent import HALF_ULP, TYPES, Cache, check_latent, fx, h, heads_of, run_expanded, run_latent  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def weighed(cache, s, n, fresh, q, qr, scale):
    """Of one sequence's causal queries, in 64 bits: weights, values, and of each query the
    largest sum of a logit's magnitudes."""
    _, v, k = cache.held(s, n)
    seen = (torch.arange(n) <= (n - fresh + torch.arange(fresh))[:, None])[:, None]
    x = torch.where(seen, (q @ v.t() + qr @ k.t()) * scale, -math.inf)
    mag = (q.abs() @ v.abs().t() + qr.abs() @ k.abs().t()) * abs(scale) * seen
    return torch.softmax(x, -1), v, mag.amax(-1, keepdim=True)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("one_sign", [True, False], ids=["one sign", "both signs"])
@pytest.mark.parametrize("rms", [1.0, 6.0])
@pytest.mark.parametrize("latent,heads", [(512, 16), (512, 40), (256, 16), (256, 64)])
def test_latent_attention_of_few_large_channels(fx, h, t, one_sign, rms, latent, heads):
    """Two channels of every latent are +-127 and its scale follows them, the others have a
    few steps; queries are small there, so that the logits (of deviation 8) come from the
    small codes.  The error's norm against that of its parts: the result's rounding, the
    weights' (2^-11, a share of each by itself), and the logits': fewer than 81 sums, each off
    by 2^-24 of the magnitudes, at random 9 times that, for a weight and for the sum of all.
    (Sums that start at or pass a constant of 1152 times the query are off by 0.05 here.)"""
    note("few large channels", t, one_sign, rms, latent, heads)
    lens = [700, 90]
    cache = Cache(fx, lens, latent, 32, 64, seed=2)
    cache.fill(lens, 17, spread=0.0)
    g = torch.Generator().manual_seed(23)
    few = [40, 200]
    codes = (torch.randn(*cache.codes.shape, generator=g) * rms).round()
    codes[..., few] = 127 * torch.randn(*cache.codes.shape[:2], 2, generator=g).sign()
    cache.codes.copy_(codes)
    make = (lambda *s: torch.rand(*s, generator=g) + 1) if one_sign else (lambda *s: torch.randn(*s, generator=g))
    q, qr = make(2, heads, latent), 1e-3 * make(2, heads, 32)
    q[..., few] *= 2.0 ** -10
    q, qr = q.to(TYPES[t]), qr.to(TYPES[t])
    _, v, _ = cache.held(0, lens[0])
    scale = float(8 / (q[0].double() @ v.t()).std())
    got = run_latent(fx, h, cache, [1, 1], lens, q, qr, scale, 1, t)
    assert fx.sync_status(h) == 0
    for s, n in enumerate(lens):
        w, v, mag = weighed(cache, s, n, 1, q[s : s + 1].double(), qr[s : s + 1].double(), scale)
        want = w @ v
        rounding = (want.to(TYPES[t]).double() - want).norm()
        uP = 2.0 ** -22 if t == "f32" else 2.0 ** -11
        logits = 2 * (9 * 2.0 ** -24 + (2.0 ** -22 if t == "f32" else 0)) * (mag * (w @ v.abs())).norm()
        sums = 2 * (n + 64) * 2.0 ** -24 * (w @ v.abs()).norm()
        assert (got[s : s + 1].double() - want).norm() <= rounding + uP * ((w * w) @ (v * v)).sqrt().norm() + logits + sums


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("latent,heads", [(256, 4), (512, 20)])
@pytest.mark.parametrize("power,scale,token", [(126, 2.0 ** -100, 1.0), (127, 2.0 ** -100, 1.0), (127, -(2.0 ** -90), 2.0 ** -14)])
def test_latent_attention_of_the_largest_queries(fx, h, t, latent, heads, power, scale, token):
    """Queries up to the end of their type.  Logits past 2^24 that differ by 2^-9 of their size
    and more: one token takes all, as in the test of large logits."""
    takes_the_largest(fx, h, t, latent, heads, 2.0 ** power, scale, token)


def takes_the_largest(fx, h, t, latent, heads, size, scale, token):
    note("one takes all", t, latent, heads, size, scale, token)
    lens = [500]
    cache = Cache(fx, lens, latent, 32, 64)
    cache.fill(lens, 31, spread=0.6)
    cache.scale *= token
    g = torch.Generator().manual_seed(2)
    q = (0.9 * torch.rand(1, heads, latent, generator=g) + 1) * torch.rand(1, heads, latent, generator=g).sub(0.5).sign()
    q, qr = (q * size).to(TYPES[t]), torch.zeros(1, heads, 32).to(TYPES[t])
    _, v, _ = cache.held(0, lens[0])
    x = q[0].double() @ v.t() * scale
    top = x.topk(2, -1)
    told = (top.values[:, 0] - top.values[:, 1]) / x.abs().amax(-1) > 2.0 ** -9
    assert told.sum() >= heads // 2 and x.abs().max() > 2.0 ** 24
    want = v[top.indices[:, 0]]
    got = run_latent(fx, h, cache, [1], lens, q, qr, scale, 1, t)[0].double()
    assert fx.sync_status(h) == 0
    uP = 2.0 ** -22 if t == "f32" else 2.0 ** -11
    assert ((got - want).abs() <= want.abs() * (uP + 8 * 2.0 ** -24 + 1.01 * HALF_ULP[t]))[told].all()


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("latent,heads", [(256, 4), (512, 20)])
@pytest.mark.parametrize("size,scale,token", [(1.0, 2.0 ** 14, 2.0 ** 100), (1.0, -(2.0 ** 20), 2.0 ** 94), (2.0 ** -90, 2.0 ** 40, 2.0 ** 95),
                                              (2.0 ** 100, 2.0 ** 110, 2.0 ** -100), (2.0 ** 110, 2.0 ** -126, 2.0 ** 60)])
def test_latent_attention_of_large_logits_of_any_factors(fx, h, t, latent, heads, size, scale, token):
    """Logits that fp32 holds, whichever of query, latent and softmax scale they owe it to."""
    takes_the_largest(fx, h, t, latent, heads, size, scale, token)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [4, 20])
@pytest.mark.parametrize("size,scale,token", [(2.0 ** 120, 2.0 ** -60, 2.0 ** -60), (2.0 ** 100, 2.0 ** -110, 2.0 ** 10),
                                              (2.0 ** -90, 2.0 ** 90, 1.0), (2.0 ** -60, 2.0 ** -30, 2.0 ** 90)])
def test_latent_attention_of_ordinary_logits_of_any_factors(fx, h, t, heads, size, scale, token):
    note("factors", t, heads, size, scale, token)
    lens = [500]
    cache = Cache(fx, lens, 256, 32, 64)
    cache.fill(lens, 18)
    cache.scale *= token
    cache.rope_scale *= token
    g = torch.Generator().manual_seed(4)
    q, qr = ((torch.randn(1, heads, d, generator=g) * size).to(TYPES[t]) for d in (256, 32))
    got = run_latent(fx, h, cache, [1], lens, q, qr, 0.2 * scale, 1, t)
    assert fx.sync_status(h) == 0
    check_latent(got, cache, lens, [1], q, qr, float(torch.tensor(0.2 * scale)), 1, t)


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [1, 40, 560])
@pytest.mark.parametrize("n,small,large", [(64, 0.0, 2.0 ** 20), (64, 0.0, 2.0 ** 90), (3000, 0.0, 2.0 ** 40), (256, 2.0 ** -90, 2.0 ** 30),
                                           (256, 2.0 ** -40, 2.0 ** 90), (1000, 1.0, 2.0 ** 60), (300, 1.0, 2.0 ** 50), (65, 2.0 ** -20, 2.0 ** 30)])
def test_latent_attention_of_scales_far_apart(fx, h, t, heads, n, small, large):
    """The last token's scale is that many times the others'.  The query before it does not
    see it: its result, and the last one's, are right by their own measure.  (small 0: tokens of
    zeros as append writes them.)"""
    note("scales apart", t, heads, n, small, large)
    lens, new = [n + 1], [2]
    cache = Cache(fx, lens, 256, 32, 64)
    cache.fill(lens, 13)
    last = torch.arange(n + 1)
    page = torch.from_numpy(cache.table[0])[last // 64].long().to(DEV)
    slot = (last % 64).to(DEV)
    cache.scale[page[:n], slot[:n]] = small or 2.0 ** -100 / 127
    if not small:
        cache.codes[page[:n], slot[:n], :256] = 0
    cache.scale[page[n], slot[n]] = large
    g = torch.Generator().manual_seed(6)
    q, qr = torch.zeros(2, heads, 256).to(TYPES[t]), torch.randn(2, heads, 32, generator=g).to(TYPES[t])
    got = run_latent(fx, h, cache, new, lens, q, qr, 0.2, 1, t).double()
    assert fx.sync_status(h) == 0
    w, v, mag = weighed(cache, 0, n + 1, 2, q.double(), qr.double(), float(torch.tensor(0.2)))
    d = mag * (40 * 2.0 ** -24 + (2.0 ** -22 if t == "f32" else 0)) + 4 * 2.0 ** -24 * mag
    uP = 2.0 ** -22 if t == "f32" else 2.0 ** -11
    for i in range(2):
        vi = v[: n + i]
        wi = w[i, :, : n + i]
        tol = (2 * d[i] + 4 * 2.0 ** -23 + uP + 2 * (n + 64) * 2.0 ** -24) * (wi @ vi.abs()) + n * 2.0 ** -31 * vi.abs().max()
        off = (got[i] - wi @ vi).abs()
        assert (off <= tol + 1.01 * HALF_ULP[t] * (wi @ vi).abs()).all(), (i, float(off.max()))


def test_latent_attention_of_bounds_past_what_is_counted(fx, h):
    """Sequences of more than 2^31 chunks in all, by their bounds, are not cut: a cut's counts
    would not fit 32 bits.  (Only the work space is asked for, which cut calls need.)"""
    codes, scale = torch.zeros(1, 128, 288, dtype=torch.int8, device=DEV), torch.zeros(1, 128, device=DEV)
    cache = fx.latent_cache(codes, scale, scale, 1, 128, 256, 32)
    some = torch.zeros(257, dtype=torch.int32, device=DEV)
    for seqs, most, cut in ((256, 1 << 30, False), (128, 1 << 30, False), (127, 1 << 30, True), (256, 1 << 28, True)):
        batch = fx.kv_batch(some, some, some, seqs, 1 << 23, seqs, 1, most)
        assert (fx.latent_attention_workspace(h, cache, batch, 1) > 0) == cut


WHOLE = [  # more than 32 row tiles of a sequence, more than 256 sequences: (latent, rope, page, heads, new, lengths)
    (512, 64, 64, 64, [20, 3], [300, 70]),
    (512, 32, 16, 16, [70], [400]),
    (512, 16, 32, 128, [9], [1000]),
    (256, 64, 32, 128, [20], [900]),
    (256, 48, 16, 33, [40, 0, 7], [41, 60, 500]),
    (512, 64, 16, 16, [1] * 260, [(7 * i) % 90 + 1 for i in range(260)]),
    (256, 32, 64, 70, [i % 3 for i in range(258)], [(5 * i) % 130 + 2 for i in range(258)]),
    # four row tiles a block, cut
    (256, 32, 128, 128, [4], [24600]),
]


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("case", WHOLE, ids=lambda c: f"{c[0]} {c[3]} heads {len(c[4])} x {max(c[4])} over {max(c[5])}")
def test_latent_attention_of_many_row_tiles_or_sequences(fx, h, t, case):
    latent, rope, page, heads, new, lens = case
    note("many row tiles", t, case)
    cache = Cache(fx, lens, latent, rope, page, seed=heads)
    cache.fill(lens, 27)
    g = torch.Generator().manual_seed(28)
    q, qr = (torch.randn(sum(new), heads, d, generator=g).to(TYPES[t]) for d in (latent, rope))
    for layout in ("token", "odd") if sum(lens) < 20000 else ("token",):
        got = run_latent(fx, h, cache, new, lens, q, qr, 0.07, 1, t, layout)
        assert fx.sync_status(h) == 0
        check_latent(got, cache, lens, new, q, qr, 0.07, 1, t)


TERMS = [  # (nope, rope, vdim, heads, new, lengths): waves that share tokens, 64 and 128 rows a block
    (128, 64, 128, 2, [16, 3], [700, 90]),
    (64, 32, 64, 5, [9], [1500]),
    (64, 32, 64, 20, [140, 60], [700, 90]),
    (128, 32, 128, 24, [150], [900]),
    (128, 64, 128, 70, [150, 129, 140, 1], [600, 129, 150, 300]),
    (64, 64, 64, 128, [129, 100], [700, 130]),
]


@pytest.mark.parametrize("t", ["f16", "bf16"])
@pytest.mark.parametrize("case", TERMS, ids=str)
def test_expanded_attention_weights_in_more_bits_than_the_result(fx, h, t, case):
    """Values that cancel to a small part of themselves tell weights of the result's own type
    from two terms of it (2^-16 of a weight at most).  The error's norm against that of its
    parts: the result's rounding; the weights' terms and exponentials, each by itself; the
    logits' sums as above; sums of n products, at random the square root of their number."""
    nope, rope, vdim, heads, new, lens = case
    note("expanded terms", t, case)
    c, scale = (nope, rope, vdim, heads, 1), 0.2 * (nope + rope) ** -0.5
    q, k, key, v = heads_of(c, new, lens, t, 33)
    got = run_expanded(fx, h, c, new, lens, q, k, key, v, scale, t)
    assert fx.sync_status(h) == 0
    at = first = 0
    parts = torch.zeros(4, dtype=torch.float64)
    off = torch.zeros((), dtype=torch.float64)
    for n, fresh in zip(lens, new):
        kk = torch.cat([k[first : first + n], key[first : first + n, None].expand(n, heads, rope)], -1).double().permute(1, 2, 0).contiguous()
        vv = v[first : first + n].double().transpose(0, 1).contiguous()
        qq = q[at : at + fresh].double().transpose(0, 1).contiguous()
        seen = torch.arange(n) <= (n - fresh + torch.arange(fresh))[:, None]
        w = torch.softmax((qq @ kk * scale).masked_fill(~seen, -math.inf), -1)
        mag = ((qq.abs() @ kk.abs()) * scale * seen).amax(-1, keepdim=True)
        want, size = w @ vv, w @ vv.abs()
        off += (got[at : at + fresh].double().transpose(0, 1) - want).square().sum()
        for i, x in enumerate((want.to(TYPES[t]).double() - want, (2.0 ** -16 + 2.0 ** -22) * ((w * w) @ (vv * vv)).sqrt(),
                               2 * 9 * 2.0 ** -24 * mag * size, 2 * (n + 64) ** 0.5 * 2.0 ** -24 * size)):
            parts[i] += x.square().sum()
        at += fresh
        first += n
    assert off.sqrt() <= parts.sqrt().sum(), (float(off.sqrt()), parts.sqrt().tolist())


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("nope,rope,vdim,heads,new,lens", [(128, 64, 128, 2, [16], [700]), (64, 32, 64, 5, [70], [400]), (64, 32, 128, 40, [90], [300]),
                                                           (128, 64, 128, 70, [150, 129, 140, 1], [600, 129, 150, 300])])
def test_expanded_attention_of_infinite_values(fx, h, t, nope, rope, vdim, heads, new, lens):
    """A query that sees an infinite value, in whatever chunk, has it in that dimension, NaN
    where it sees both infinities or a NaN; its other dimensions and what does not see them
    stay as they are."""
    note("infinite values", t, nope, rope, vdim, heads, new, lens)
    c, scale = (nope, rope, vdim, heads, 1), 0.05
    q, k, key, v = heads_of(c, new, lens, t, 35)
    want = run_expanded(fx, h, c, new, lens, q, k, key, v, scale, t)
    put = [(3, 7, math.inf), (130, 9, -math.inf), (lens[0] - 5, 7, math.inf), (40, 11, math.inf), (60, 11, -math.inf), (80, 13, math.nan)]
    seen = lens[0] - new[0] + torch.arange(new[0])  # the first sequence's queries
    for at, d, x in put:
        v[at, :, d] = x
    for d in {d for _, d, _ in put}:
        total = torch.zeros(new[0])
        for at, e, x in put:
            if e == d:
                total = torch.where(seen >= at, total + x, total)
        want[: new[0], :, d] = torch.where((total == 0)[:, None], want[: new[0], :, d].float(), total[:, None]).to(want.dtype)
    got = run_expanded(fx, h, c, new, lens, q, k, key, v, scale, t)
    assert fx.sync_status(h) == 0
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0, math.inf, -math.inf), want.nan_to_num(0.0, math.inf, -math.inf))
