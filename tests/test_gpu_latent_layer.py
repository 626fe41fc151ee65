"""The latent attention operators together: append, both forms of attention and the 8-bit
product against 64 bits on the codes that lie in the cache, the decoder layer that runs
them, replays in captured graphs, other streams, two calls that share nothing."""
import math

import pytest

from gpu_util import DEV, note

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dec():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2203_12091_amd import decoder
    return decoder


@pytest.fixture(scope="module")
def fx(dec):
    from paper_2203_12091_amd import fxpq
    return fxpq


@pytest.mark.parametrize("new", [1, 40])
def test_both_forms_against_64_bits(fx, dec, new):
    """From the codes in the cache on: keys and values of each head out of the 8-bit
    product, and the query carried through the keys' weights instead, both against 64 bits
    (f32: products, sums and roundings of 2^-22 of their magnitudes each, 600 fp32 additions
    in a logit; the tolerance takes their sum)."""
    note("both forms", new)
    H, nope, rope, vdim, latent, ctx, S = 5, 64, 32, 64, 256, 70, 2
    g = torch.Generator(device=DEV).manual_seed(3)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    h = fx.Handle(0)
    cache = dec.LatentCache(40, 16, latent, rope, 20, S)
    ang = torch.arange(256, device=DEV).double()[:, None] * 10000.0 ** (-torch.arange(0, rope, 2, device=DEV).double() / rope)
    rot = fx.rotary(ang.cos().float(), ang.sin().float(), 256, rope, 1)
    w, ws = dec.quantize_rows(h, randn(H * (nope + vdim), latent) * latent ** -0.5)
    for n in (ctx, new):
        batch = cache.extend(list(range(S)), [n, max(n - 3, 1)])
        t = batch.tokens
        cr, q = randn(t, latent + rope), randn(t, H, nope + rope)
        fx.latent_append(h, cache.desc, batch, rot, fx.SCALE_MAX, cr, latent + rope, cr[:, latent:], latent + rope, q[:, :, nope:],
                         H * (nope + rope), nope + rope, q[:, :, nope:], H * (nope + rope), nope + rope, H, fx.F32)
    held, scale = batch.held, (nope + rope) ** -0.5
    codes, cs = torch.empty(held, latent, dtype=torch.int8, device=DEV), torch.empty(held, device=DEV)
    key, kv = torch.empty(held, rope, device=DEV), torch.empty(held, H, nope + vdim, device=DEV)
    fx.latent_read(h, cache.desc, batch, batch.rows, held, codes, latent, cs, None, 0, key, rope, fx.F32)
    need = fx.token_gemm_workspace(held, H * (nope + vdim), latent)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    fx.token_gemm(h, held, H * (nope + vdim), latent, codes, latent, cs, w, ws, None, kv, fx.F32, H * (nope + vdim), work, need)
    desc = fx.expanded_kv(kv, H * (nope + vdim), nope + vdim, key, rope, kv[:, :, nope:], H * (nope + vdim), nope + vdim, batch.rows,
                          held, H, nope, rope, vdim)
    out = torch.empty(t, H, vdim, device=DEV)
    fx.expanded_attention(h, desc, batch, q, H * (nope + rope), scale, 1, out, H * vdim, fx.F32)
    # absorbed, with the very weights that the product used
    W = (w.double() * ws.double()[:, None]).view(H, nope + vdim, latent)
    ql = torch.stack([q[:, i, :nope].double() @ W[i, :nope] for i in range(H)], 1).float()
    lat = torch.empty(t, H, latent, device=DEV)
    need = fx.latent_attention_workspace(h, cache.desc, batch, H)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    fx.latent_attention(h, cache.desc, batch, ql, H * latent, latent, q[:, :, nope:], H * (nope + rope), nope + rope, H, scale, 1, lat,
                        H * latent, latent, fx.F32, work, need)
    assert fx.sync_status(h) == 0
    got = torch.stack([lat[:, i].double() @ W[i, nope:].t().contiguous() for i in range(H)], 1)
    c, rows, start = codes.double() * cs.double()[:, None], batch.rows.tolist(), [0, new, t]
    for s in range(S):
        a, b, lo, hi = start[s], start[s + 1], rows[s], rows[s + 1]
        see = torch.arange(hi - lo, device=DEV) <= (hi - lo - (b - a) + torch.arange(b - a, device=DEV))[:, None]
        for i in range(H):
            k, v = c[lo:hi] @ W[i, :nope].t().contiguous(), c[lo:hi] @ W[i, nope:].t().contiguous()
            qn, qr = q[a:b, i, :nope].double(), q[a:b, i, nope:].double()
            x = (qn @ k.t().contiguous() + qr @ key[lo:hi].double().t().contiguous()) * scale
            mag = (qn.abs() @ (c[lo:hi].abs() @ W[i, :nope].abs().t().contiguous()).t().contiguous()
                   + qr.abs() @ key[lo:hi].double().abs().t().contiguous()) * scale
            want = torch.softmax(x.masked_fill(~see, -math.inf), -1) @ v
            S_v = (c[lo:hi].abs() @ W[i, nope:].abs().t().contiguous()).max()
            tol = S_v * (2 * (mag * see).amax(-1, keepdim=True) * (600 * 2.0 ** -24 + 3 * 2.0 ** -22) + 300 * 2.0 ** -24 + 4 * 2.0 ** -22)
            assert ((out[a:b, i].double() - want).abs() <= tol).all()
            assert ((got[a:b, i] - want).abs() <= tol).all()
    h.close()


def layer_of(dec, dtype):
    layer = dec.LatentLayer(256, 6, 64, 32, 64, 256, experts=4, top=2, inner=160, dtype=dtype, seed=3)
    return layer, dec.LatentCache(pages=60, page=16, latent=256, rope=32, max_pages_per_seq=20, max_seqs=4)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_of_the_layer_in_one_call_against_several(dec, fx, dtype):
    """Prompts in one call (keys and values made of the latents), and the same tokens in
    small calls (queries through the keys' weights): the codes in the cache are the same.
    The attention halves differ by the 8-bit roundings that only one of the forms has, each
    of an rms of max / (127 * 12^0.5) of a row, for rows whose largest value is three times
    their rms 0.7 % of it: queries and weights on the way to the logits (of rms 1), so 0.9 % of
    a weight and of the weighted sum; that sum's own rounding 0.7 %; the roundings that the
    output product starts from, which differ once their inputs do, 0.7 % on each side.  Together
    1.6 %; bf16 adds five roundings of 0.2 %.  The tolerance is twice that, and a row's largest
    value may be four times its rms.  (The experts behind it are left out: a token near the
    border of two experts takes another one, whatever the difference.)"""
    note("latent layer", dtype)
    layer, whole = layer_of(dec, dtype)
    _, parts = layer_of(dec, dtype)
    new = [64, 40, 48]
    x = [torch.randn(n, 256, generator=torch.Generator().manual_seed(n)).to(dtype).to(DEV) for n in new]
    want = layer.attend(torch.cat(x), whole, whole.extend([0, 1, 2], new)).split(new)
    got = [[], [], []]
    at = 0
    while at < max(new):
        seqs = [s for s in range(3) if at < new[s]]
        step = [min(layer.FEW, 16, new[s] - at) for s in seqs]
        y = layer.attend(torch.cat([x[s][at : at + n] for s, n in zip(seqs, step)]), parts, parts.extend(seqs, step)).split(step)
        for s, v in zip(seqs, y):
            got[s].append(v)
        at += 16
    for w, v, s in zip(want, got, range(3)):
        v = torch.cat(v).float()
        assert (v - w.float()).norm() <= 4.5e-2 * w.float().norm()
        a, b = whole.owned[s], parts.owned[s]
        n = new[s]
        assert torch.equal(whole.codes[a].flatten(0, 1)[:n], parts.codes[b].flatten(0, 1)[:n])
        assert torch.equal(whole.scale[a].flatten()[:n], parts.scale[b].flatten()[:n])
    assert fx.sync_status(layer.h) == 0
    layer.h.close()


def test_layer_steps_and_a_batch_made_by_hand(dec, fx):
    layer, cache = layer_of(dec, torch.float16)
    layer.forward(torch.randn(50, 256, device=DEV).half(), cache, cache.extend([7, 9], [36, 14]))
    for _ in range(3):
        y = layer.forward(torch.randn(2, 256, device=DEV).half(), cache, cache.extend([7, 9], [1, 1]))
        assert torch.isfinite(y).all()
    assert layer.forward(torch.zeros(0, 256, device=DEV).half(), cache, cache.extend([7], [0])).shape == (0, 256)
    told = cache.extend([7], [40])
    start, length, table = told._refs
    hand = fx.kv_batch(start, length, table, 1, cache.max_pages, 40, 40, told.max_len)
    x = torch.randn(40, 256, device=DEV).half()
    a, b = layer.attend(x, cache, told), layer.attend(x, cache, hand)  # made of the latents, over the latents
    assert (a.float() - b.float()).norm() <= 4.5e-2 * a.float().norm()  # as above
    assert fx.sync_status(layer.h) == 0
    layer.h.close()


def test_layer_on_another_stream(dec, fx):
    layer, cache = layer_of(dec, torch.bfloat16)
    _, other = layer_of(dec, torch.bfloat16)
    x = torch.randn(45, 256, device=DEV).bfloat16()
    want = layer.forward(x, cache, cache.extend([0], [45]))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer.forward(x, other, other.extend([0], [45]))
    side.synchronize()
    assert torch.equal(got, want)
    layer.h.close()


def test_example_runs(dec, capsys):
    assert dec.main(prompt=40, steps=2, seqs=3, latent=True) == 0
    assert "step: 3 tokens" in capsys.readouterr().out


@pytest.mark.parametrize("new,H,t", [(1, 16, "bf16"), (3, 40, "f16"), (50, 2, "f32")])
def test_operators_in_a_graph(fx, dec, new, H, t):
    """Append, read and both attentions captured once and replayed with new inputs and
    lengths: every replay equals the calls made directly, bit for bit; the work space holds
    anything before each of them."""
    dt = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[t]
    code = {"bf16": fx.BF16, "f16": fx.F16, "f32": fx.F32}[t]
    latent, rope, nope, vdim, S, page = 512, 64, 64, 64, 3, 32
    h = fx.Handle(0)
    g = torch.Generator(device=DEV).manual_seed(4)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV).to(dt)  # noqa: E731
    caches = [dec.LatentCache(60, page, latent, rope, 20, S) for _ in range(2)]
    for c in caches:
        c.codes.copy_(torch.randint(-99, 99, c.codes.shape, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV))
        c.scale.fill_(0.02)
        c.rope_scale.fill_(0.03)
    T = S * new
    cr, q, ql = randn(T, latent + rope), randn(T, H, nope + rope), randn(T, H, latent)
    start = torch.arange(S + 1, dtype=torch.int32, device=DEV) * new
    length = torch.tensor([new + 5, new + 340, new + 100], dtype=torch.int32, device=DEV)
    rows = torch.zeros(S + 1, dtype=torch.int32, device=DEV)
    table = torch.arange(60, dtype=torch.int32, device=DEV).view(3, 20)
    batch = fx.kv_batch(start, length, table, S, 20, T, new, 640)
    most = 3 * 640
    ang = torch.arange(640, device=DEV)[:, None] * 10000.0 ** (-torch.arange(0, rope, 2, device=DEV) / rope)
    rot = fx.rotary(ang.cos().contiguous(), ang.sin().contiguous(), 640, rope)
    codes, cs = torch.zeros(most, latent, dtype=torch.int8, device=DEV), torch.zeros(most, device=DEV)
    key, kv = torch.zeros(most, rope, dtype=dt, device=DEV), randn(most, H, nope + vdim)
    qr = torch.zeros(T, H, rope, dtype=dt, device=DEV)
    out, ex = torch.zeros(T, H, latent, dtype=dt, device=DEV), torch.zeros(T, H, vdim, dtype=dt, device=DEV)
    need = fx.latent_attention_workspace(h, caches[0].desc, batch, H)
    work = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)
    desc = fx.expanded_kv(kv, H * (nope + vdim), nope + vdim, key, rope, kv[:, :, nope:], H * (nope + vdim), nope + vdim, rows, most, H,
                          nope, rope, vdim)
    w = nope + rope

    def step(cache):
        fx.latent_append(h, cache.desc, batch, rot, fx.SCALE_DFX, cr, latent + rope, cr[:, latent:], latent + rope, q[:, :, nope:],
                         H * w, w, qr, H * rope, rope, H, code)
        fx.latent_read(h, cache.desc, batch, rows, most, codes, latent, cs, None, 0, key, rope, code)
        fx.latent_attention(h, cache.desc, batch, ql, H * latent, latent, qr, H * rope, rope, H, 0.06, 1, out, H * latent, latent, code,
                            work, need)
        fx.expanded_attention(h, desc, batch, q, H * w, 0.1, 1, ex, H * vdim, code)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fx.set_stream(h, side)
    rows[1:] = length.cumsum(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(caches[1])  # before the capture: everything is loaded
        step(caches[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(caches[0])
    for i in range(4):
        cr.copy_(randn(T, latent + rope) * 2.0 ** i)
        q.copy_(randn(T, H, w))
        length += torch.tensor([new, 1, 60], dtype=torch.int32, device=DEV)
        rows[1:] = length.cumsum(0)
        work.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (qr, codes, cs, key, out, ex)]
        work.fill_(0x7F)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step(caches[1])
        torch.cuda.synchronize()
        for a, b in zip(got, (qr, codes, cs, key, out, ex)):
            assert torch.equal(a, b)
        assert torch.equal(caches[0].codes, caches[1].codes) and torch.equal(caches[0].scale, caches[1].scale)
    fx.set_stream(h, None)
    assert fx.sync_status(h) == 0
    h.close()


@pytest.mark.parametrize("S", [3, 100, 300])
def test_many_sequences_and_rows_behind_the_last(fx, dec, S):
    """More sequences than are shared among the blocks, most of them without new tokens or
    without any; the tensors have rows behind the last sequence, which stay as they were."""
    note("many sequences", S)
    H, latent, rope = 20, 256, 32
    h = fx.Handle(0)
    g = torch.Generator(device=DEV).manual_seed(S)
    length = torch.randint(0, 200, (S,), generator=torch.Generator().manual_seed(S)).tolist()
    length[0], length[-1] = 0, 150
    new = [min(n, 1 if i % 3 else 0) for i, n in enumerate(length)]
    new[-1] = 2
    T = sum(new)
    need_pages = [-(-n // 16) for n in length]
    table = torch.full((S, max(need_pages)), 2 ** 31 - 1, dtype=torch.int32)
    at = 0
    for i, n in enumerate(need_pages):
        table[i, :n] = torch.arange(at, at + n)
        at += n
    codes = torch.randint(-127, 128, (at, 16, latent + rope), generator=g, device=DEV).to(torch.int8)
    scale = torch.rand(at, 16, generator=g, device=DEV) * 0.02 + 0.01
    cache = fx.latent_cache(codes, scale, scale, at, 16, latent, rope)
    start = torch.tensor([0] + new).cumsum(0).to(torch.int32).to(DEV)
    batch = fx.kv_batch(start, torch.tensor(length, dtype=torch.int32, device=DEV), table.to(DEV), S, table.shape[1], T + 5, 3, max(length))
    q, qr = torch.randn(T + 5, H, latent, generator=g, device=DEV), torch.randn(T + 5, H, rope, generator=g, device=DEV)
    out = torch.full((T + 5, H, latent), 5.0, device=DEV)
    need = fx.latent_attention_workspace(h, cache, batch, H)
    work = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device=DEV)
    fx.latent_attention(h, cache, batch, q, H * latent, latent, qr, H * rope, rope, H, 0.06, 1, out, H * latent, latent, fx.F32, work, need)
    assert fx.sync_status(h) == 0 and (out[T:] == 5.0).all()
    row = 0
    for i, (n, k) in enumerate(zip(length, new)):
        for e in range(k):
            seen = n - k + 1 + e
            p = table[i, : need_pages[i]].long().to(DEV)
            c = codes[p].flatten(0, 1)[:seen].double() * scale[p].flatten()[:seen, None].double()
            x = (q[row].double() @ c[:, :latent].t().contiguous() + qr[row].double() @ c[:, latent:].t().contiguous()) * 0.06
            want = torch.softmax(x, -1) @ c[:, :latent].contiguous()
            # logits below 30 in magnitude of sums below 100: 2 * 100 * 300 * 2^-24 and the f16 terms' 2^-20
            assert ((out[row].double() - want).abs() <= c.abs().max() * (60000 * 2.0 ** -24 + 2.0 ** -19)).all()
            row += 1
    h.close()


@pytest.mark.parametrize("nope,rope,vdim", [(80, 16, 32), (64, 48, 96), (16, 32, 16)])
def test_layer_of_heads_that_are_not_expanded(dec, fx, nope, rope, vdim):
    """Heads that attention over keys and values does not take: a prompt in one call and in
    small ones, over the latents both ways.  They differ in the order of fp32 sums, by which
    a value may get the next code: one in 10^4 of them, of a step of 1 / 127 of the row's
    largest (four times its rms), 3e-4 of a row's norm in each of four products."""
    note("latent layer", nope, rope, vdim)
    layer = dec.LatentLayer(256, 6, nope, rope, vdim, 256, experts=4, top=2, inner=160, dtype=torch.float32, seed=4)
    caches = [dec.LatentCache(pages=60, page=16, latent=256, rope=rope, max_pages_per_seq=20, max_seqs=4) for _ in range(2)]
    x = torch.randn(layer.FEW + 30, 256, generator=torch.Generator().manual_seed(5)).to(DEV)
    whole = layer.attend(x, caches[0], caches[0].extend([0], [len(x)]))
    parts = torch.cat([layer.attend(y, caches[1], caches[1].extend([0], [len(y)])) for y in x.split(16)])
    assert fx.sync_status(layer.h) == 0
    assert (whole - parts).norm() <= 1.2e-3 * whole.norm()
    layer.h.close()


def test_prompts_and_single_tokens_in_one_batch(dec, fx):
    """Each sequence's result is what it is alone (the orders of fp32 sums differ: as above)."""
    layer, cache = layer_of(dec, torch.float32)
    g = torch.Generator().manual_seed(6)
    make = lambda n: torch.randn(n, 256, generator=g).to(DEV)  # noqa: E731
    layer.attend(make(150), cache, cache.extend([0, 1, 2], [50, 70, 30]))
    new = [1, layer.FEW + 8, 0, layer.FEW]
    x = make(sum(new))
    batch = cache.extend([0, 1, 2, 3], new)
    got = layer.attend(x, cache, batch).split(new)
    start, length, table = batch._refs
    for i, (n, y) in enumerate(zip(new, x.split(new))):
        if not n:
            continue
        # the tokens are in the cache already: writing them again writes the same
        one = cache._batch([n], [int(length[i])], table[i : i + 1].cpu())
        want = layer.attend(y, cache, one)
        assert (got[i] - want).norm() <= 1.2e-3 * want.norm()
    assert fx.sync_status(layer.h) == 0
    layer.h.close()
