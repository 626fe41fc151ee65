"""The decoder layer that runs the 8-bit serving operators together: each product
against 64 bits on the codes it was given, the layer in one call against the same
tokens in several, replays in a captured graph, and the cache's book-keeping."""
import pytest

from gpu_util import DEV, note

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def dec():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2203_12091_amd import decoder
    return decoder


def make(dec, dtype, page=16):
    layer = dec.Layer(256, 8, 2, 64, experts=4, top=2, inner=160, dtype=dtype, seed=3)
    cache = dec.Cache(pages=40, page=page, heads=2, dim=64, max_pages_per_seq=16, max_seqs=4)
    return layer, cache


def value(codes, scale):
    return codes.double() * scale.double()[:, None]


def product(a, a_scale, b, b_scale):
    """The integer sum, exact in fp64, then the scales."""
    return (a.double() @ b.double().t()) * torch.outer(a_scale.double(), b_scale.double())


@pytest.mark.gpu
def test_products_of_the_layer(dec):
    """Rounding of the activations is the operators' own; the products on the codes
    are exact up to fp32 scaling: 2^-22 of each value (four roundings)."""
    layer, _ = make(dec, torch.float32)
    x = torch.randn(33, 256, device=DEV)
    codes, scale = dec.quantize_rows(layer.h, x)
    assert (value(codes, scale)[:, :256] - x.double()).abs().max() <= 0.5001 * scale.max()
    y = layer._linear(x, layer.qkv)
    want = product(codes, scale, *layer.qkv)
    assert ((y.double() - want).abs() <= 2.0 ** -22 * want.abs()).all()
    weight, token, place, offsets = layer.route(x)
    assert offsets.tolist()[0] == 0 and offsets.tolist()[-1] == 66
    up = layer._grouped(codes, scale, token, offsets, layer.up, 320)
    w, w_scale = layer.up[0].view(4, 320, -1), layer.up[1].view(4, 320)
    for e in range(4):
        at = token[int(offsets[e]) : int(offsets[e + 1])].long()
        want = product(codes[at], scale[at], w[e], w_scale[e])
        assert ((up[int(offsets[e]) : int(offsets[e + 1])].double() - want).abs() <= 2.0 ** -22 * want.abs()).all()
    assert torch.equal(token[place.view(33, 2)].long(), torch.arange(33, device=DEV)[:, None].expand(33, 2))
    layer.h.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,tol", [(torch.float32, 2e-3), (torch.bfloat16, 5e-2)])
def test_one_call_against_several(dec, dtype, tol):
    """Prompts in one call, and cut where pages end (the cache is then the same, code
    for code): the outputs differ by the attention's rounding and by the codes of
    later quantizations that it moves, each by one step of 1 / 127 of a row's
    largest value.  fp32: about one code in 10^4 moves; bf16: a rounding of 2^-9
    moves one code in three, 2 % of a row's values on the whole through the two
    quantizations that follow; the tolerance is a little over twice that."""
    note("decoder", dtype)
    layer, whole = make(dec, dtype)
    _, parts = make(dec, dtype)
    new = [64, 17, 48]
    x = [torch.randn(n, 256, device=DEV).to(dtype) for n in new]
    want = layer.forward(torch.cat(x), whole, whole.extend([0, 1, 2], new)).split(new)
    cut = [32, 16, 16]
    first = layer.forward(torch.cat([a[:c] for a, c in zip(x, cut)]), parts, parts.extend([0, 1, 2], cut)).split(cut)
    rest = [n - c for n, c in zip(new, cut)]
    second = layer.forward(torch.cat([a[c:] for a, c in zip(x, cut)]), parts, parts.extend([0, 1, 2], rest)).split(rest)
    for w, a, b in zip(want, first, second):
        got = torch.cat([a, b]).float()
        assert (got - w.float()).norm() <= tol * w.float().norm()
    for s in range(3):
        a, b = whole.owned[s], parts.owned[s]
        assert torch.equal(whole.k_scale[a], parts.k_scale[b]) or dtype != torch.float32
    layer.h.close()


@pytest.mark.gpu
def test_decoding_steps_and_pages(dec):
    layer, cache = make(dec, torch.float16)
    y = layer.forward(torch.randn(30, 256, device=DEV).half(), cache, cache.extend([7, 9], [16, 14]))
    for _ in range(5):
        y = layer.forward(torch.randn(2, 256, device=DEV).half(), cache, cache.extend([7, 9], [1, 1]))
    assert torch.isfinite(y).all() and cache.length == {7: 21, 9: 19}
    assert len(cache.owned[7]) == 2 and len(cache.free) == 36
    from paper_2203_12091_amd import fxpq as fx
    assert fx.sync_status(layer.h) == 0
    cache.release(7)
    assert len(cache.free) == 38
    with pytest.raises(MemoryError):
        cache.extend([1], [16 * 17])
    with pytest.raises(ValueError):
        cache.extend([1, 2, 3, 4, 5], [1] * 5)
    layer.h.close()


@pytest.mark.gpu
def test_operators_in_a_graph(dec):
    """One decoding step's calls captured and replayed, with new inputs and lengths
    between the replays: every replay equals the calls made directly."""
    from paper_2203_12091_amd import fxpq as fx
    heads, dim, page, q_heads, seqs, hidden = 2, 64, 16, 8, 3, 512
    h = fx.Handle(0)
    g = torch.Generator(device=DEV).manual_seed(4)
    randn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    caches = [dec.Cache(30, page, heads, dim, 10, seqs) for _ in range(2)]
    for c in caches:
        c.k.copy_(torch.randint(-99, 99, c.k.shape, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV))
        c.v.copy_(torch.randint(-99, 99, c.v.shape, generator=torch.Generator(device=DEV).manual_seed(6), device=DEV))
        c.k_scale.fill_(2.0 ** -6)
        c.v_scale.fill_(2.0 ** -5)
    w, ws = dec.quantize_rows(h, randn((q_heads + 2 * heads) * dim, hidden))
    x = randn(seqs, hidden).bfloat16()
    start = torch.arange(seqs + 1, dtype=torch.int32, device=DEV)
    length = torch.tensor([5, 40, 100], dtype=torch.int32, device=DEV)
    table = torch.arange(30, dtype=torch.int32, device=DEV).view(3, 10)
    batch = fx.kv_batch(start, length, table, seqs, 10, seqs, 1, 160)
    width = w.shape[0]
    ang = torch.arange(160, device=DEV)[:, None] * 10000.0 ** (-torch.arange(0, dim, 2, device=DEV) / dim)
    rot = fx.rotary(ang.cos().contiguous(), ang.sin().contiguous(), 160, dim)
    codes, sa = torch.empty(seqs, hidden, dtype=torch.int8, device=DEV), torch.empty(seqs, device=DEV)
    qkv, out = torch.empty(seqs, width, dtype=torch.bfloat16, device=DEV), torch.empty(seqs, q_heads * dim, dtype=torch.bfloat16, device=DEV)
    need = max(fx.token_gemm_workspace(seqs, width, hidden), fx.cache_attention_workspace(h, caches[0].desc, batch, q_heads))
    work = torch.empty(max(need, 256), dtype=torch.uint8, device=DEV)

    def step(cache):
        fx.token_quantize(h, x, fx.BF16, seqs, hidden, hidden, fx.SCALE_MAX, codes, hidden, sa)
        fx.token_gemm(h, seqs, width, hidden, codes, hidden, sa, w, ws, None, qkv, fx.BF16, width, work, work.numel())
        k, v = qkv[:, q_heads * dim :], qkv[:, (q_heads + heads) * dim :]
        fx.cache_append(h, cache.desc, batch, rot, k, width, v, width, qkv, width, qkv, width, q_heads, fx.BF16)
        fx.cache_attention(h, cache.desc, batch, qkv, width, q_heads, dim ** -0.5, 1, out, q_heads * dim, fx.BF16,
                           work, work.numel())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    fx.set_stream(h, side)
    with torch.cuda.stream(side):
        step(caches[1])  # before the capture: everything is loaded
        step(caches[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(caches[0])
    for i in range(5):
        x.copy_(randn(seqs, hidden).bfloat16() * 2.0 ** i)
        length += 1
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), qkv.clone()
        with torch.cuda.stream(side):
            step(caches[1])
        torch.cuda.synchronize()
        assert torch.equal(got[0], out) and torch.equal(got[1], qkv)
        assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v)
        assert torch.equal(caches[0].k_scale, caches[1].k_scale) and torch.equal(caches[0].v_scale, caches[1].v_scale)
    fx.set_stream(h, None)
    assert fx.sync_status(h) == 0
    h.close()


@pytest.mark.gpu
def test_example_runs(dec, capsys):
    assert dec.main(prompt=40, steps=2, seqs=3) == 0
    assert "step: 3 tokens" in capsys.readouterr().out


def test_serving_calls_reject_bad_arguments_without_a_device():
    """Host checks come before any device call."""
    import ctypes as C
    import os

    from paper_2203_12091_amd import fxpq as fx
    if not os.path.exists(fx.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    L = fx.lib()
    assert C.sizeof(fx.KvCache) == 48 and C.sizeof(fx.KvBatch) == 48 and C.sizeof(fx.Rotary) == 32
    bad = fx.ERR_INVALID_ARG
    assert L.fxpq_token_quantize(None, None, fx.F32, 1, 1, 1, 0, None, 16, None) == bad
    assert L.fxpq_token_gemm(None, 1, 1, 16, None, 16, None, None, None, None, None, fx.F32, 1, None, 0) == bad
    assert L.fxpq_expert_gemm(None, 1, 1, 16, 1, None, 1, 16, None, None, None, None, None, None, None, fx.F32, 1) == bad
    cache, batch = fx.KvCache(), fx.KvBatch()
    p = C.byref
    assert L.fxpq_cache_append(None, p(cache), p(batch), None, None, 0, None, 0, None, 0, None, 0, 0, fx.F32) == bad
    assert L.fxpq_cache_read(None, p(cache), p(batch), None, None, fx.F32) == bad
    assert L.fxpq_cache_attention(None, p(cache), p(batch), None, 0, 1, 1.0, 1, None, 0, fx.F32, None, 0) == bad
    n = C.c_int64(-1)
    assert L.fxpq_cache_attention_workspace(None, p(cache), p(batch), 1, p(n)) == bad and n.value == 0
    assert L.fxpq_token_gemm_workspace(64, 4096, 9216, p(n)) == fx.OK and n.value == 4 * 64 * 4096 * 4
    assert L.fxpq_token_gemm_workspace(1, 1000, 2048, p(n)) == fx.OK and n.value == 0
    for m, k, want in ((1, 24, bad), (-1, 16, bad), (1, 131072, fx.ERR_OVERFLOW)):
        assert L.fxpq_token_gemm_workspace(m, 8, k, p(n)) == want and n.value == 0
    assert L.fxpq_token_gemm_workspace(1, 8, 16, None) == bad


@pytest.mark.parametrize("n", [1, 4096, 4097, 5000, 2 ** 31 - 1])
@pytest.mark.parametrize("k", [16, 64, 9216])
def test_products_of_no_rows_need_no_work_space(n, k):
    """The query answers for M = 0, which the product accepts, at any width."""
    import ctypes as C
    import os

    from paper_2203_12091_amd import fxpq as fx
    if not os.path.exists(fx.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    need = C.c_int64(-1)
    assert fx.lib().fxpq_token_gemm_workspace(0, n, k, C.byref(need)) == fx.OK and need.value == 0


@pytest.mark.gpu
def test_layer_of_another_stream(dec):
    """A layer made and run inside another stream gives what one made and run on the
    default stream gives."""
    x = torch.randn(40, 256, device=DEV)
    layer, cache = make(dec, torch.float32)
    want = [layer.forward(x, cache, cache.extend([0, 1], [30, 10])), layer.forward(x[:2], cache, cache.extend([0, 1], [1, 1]))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other, pages = make(dec, torch.float32)
        got = [other.forward(x, pages, pages.extend([0, 1], [30, 10])), other.forward(x[:2], pages, pages.extend([0, 1], [1, 1]))]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip((layer.qkv, layer.out, layer.up, layer.down), (other.qkv, other.out, other.up, other.down)):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    layer.h.close()
    other.h.close()


@pytest.mark.gpu
def test_step_without_tokens_of_a_wide_layer(dec):
    """No new tokens, in a layer whose projection has 4608 channels, between steps
    that have some: no rows come back and the cache stays as it was."""
    from paper_2203_12091_amd import fxpq as fx
    layer = dec.Layer(64, 64, 4, 64, experts=4, top=2, inner=48, dtype=torch.bfloat16)
    cache = dec.Cache(pages=4, page=16, heads=4, dim=64, max_pages_per_seq=2, max_seqs=2)
    x = torch.randn(6, 64, device=DEV).bfloat16()
    layer.forward(x, cache, cache.extend([0, 1], [4, 2]))
    kept = [t.clone() for t in (cache.k, cache.v, cache.k_scale, cache.v_scale)]
    y = layer.forward(x[:0], cache, cache.extend([0, 1], [0, 0]))
    assert y.shape == (0, 64) and all(torch.equal(a, b) for a, b in zip(kept, (cache.k, cache.v, cache.k_scale, cache.v_scale)))
    y = layer.forward(x[:1], cache, cache.extend([0, 1], [0, 1]))
    assert y.shape == (1, 64) and torch.isfinite(y).all() and fx.sync_status(layer.h) == 0
    layer.h.close()


def test_rotation_tables_are_checked_for_alignment():
    """cos and sin are floats; checked before any device call (the handle's memory is
    never looked at: the batch has no tokens)."""
    import ctypes as C
    import os

    from paper_2203_12091_amd import fxpq as fx
    if not os.path.exists(fx.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    at = 1 << 20  # stands for device addresses, none of which is read
    cache = fx.KvCache(k=at, v=at, k_scale=at, v_scale=at, pages=1, page=16, heads=1, dim=32)
    batch = fx.KvBatch(start=at, length=at, table=at, seqs=1, table_ld=1, tokens=0, max_new=0, max_len=16)
    handle = C.create_string_buffer(1 << 16)
    p = C.byref
    for shift, want in ((0, fx.OK), (4, fx.OK), (2, fx.ERR_INVALID_ARG), (1, fx.ERR_INVALID_ARG)):
        for rot in (fx.Rotary(cos=at + shift, sin=at, positions=16, dims=32), fx.Rotary(cos=at, sin=at + shift, positions=16, dims=32)):
            assert fx.lib().fxpq_cache_append(p(handle), p(cache), p(batch), p(rot), None, 32, None, 32, None, 0, None, 0, 0,
                                              fx.F32) == want, shift


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
def test_cache_of_one_call_against_several(dec, dtype):
    """Rows quantized one by one, exact sums, scales of whole pages: prompts that are
    cut where pages end leave the same codes and scales as in one call.  The norm, a
    reduction of torch's whose order may depend on the number of rows, is left out."""
    note("decoder cache", dtype)
    layer, whole = make(dec, dtype)
    other, parts = make(dec, dtype)
    new, cut = [64, 17, 48], [32, 16, 16]
    rest = [n - c for n, c in zip(new, cut)]
    x = [torch.randn(n, 256, device=DEV).to(dtype) for n in new]
    layer.attend(torch.cat(x), whole, whole.extend([0, 1, 2], new))
    layer.attend(torch.cat([a[:c] for a, c in zip(x, cut)]), parts, parts.extend([0, 1, 2], cut))
    layer.attend(torch.cat([a[c:] for a, c in zip(x, cut)]), parts, parts.extend([0, 1, 2], rest))
    torch.cuda.synchronize()
    for s in range(3):
        a, b = whole.owned[s], parts.owned[s]
        assert len(a) == len(b) == -(-new[s] // 16)
        for one, several in zip((whole.k, whole.v, whole.k_scale, whole.v_scale), (parts.k, parts.v, parts.k_scale, parts.v_scale)):
            assert torch.equal(one[a], several[b])  # slots past the end are 0 in both
    layer.h.close()
    other.h.close()
