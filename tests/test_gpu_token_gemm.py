"""Per-token quantization and the 8-bit products with token and channel scales,
plain and grouped by expert, against plain implementations in 64 bits.

Tolerances: a scale is one fp32 division (2^-24 relative); a code's product
x * (127 / a) carries two fp32 roundings of a value of at most 127, so the code
is within 1/2 + 127 * 2^-23 * 1.5 of the exact quotient; an output carries the
conversion of the exact sum, two products and an addition (each 2^-24 of its
result, the products' magnitude where the bias cancels them) and the rounding
to its type."""
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


def gen(seed):
    return torch.Generator().manual_seed(seed)


# ---- token_quantize ---------------------------------------------------------------

def dfx_step(a):
    step = 2.0 ** (np.floor(np.log2(a)) - 6)
    return np.where(np.round(a / step) > 127, 2 * step, step)


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rule", ["max", "dfx"])
@pytest.mark.parametrize("rows,cols,ldx,shift", [(1, 1, 1, 0), (3, 15, 15, 0), (2, 16, 24, 0), (5, 17, 40, 0),
                                                 (4, 4099, 4104, 0), (2, 4096, 4096, 0), (3, 333, 335, 1),
                                                 (1, 20000, 20000, 0)])
def test_token_quantize(fx, h, t, rule, rows, cols, ldx, shift):
    note("token_quantize", t, rule, rows, cols, ldx, shift)
    x = torch.randn(rows, ldx, generator=gen(rows * cols)) * torch.exp2(torch.randint(-12, 9, (rows, 1), generator=gen(3)).float())
    x = x.to(TYPES[t])
    buf = torch.zeros(rows * ldx + 8, dtype=TYPES[t])
    buf[shift : shift + rows * ldx] = x.flatten()  # shift: an address aligned to the type only
    d = buf.to(DEV)
    ldc = -(-cols // 16) * 16 + 16
    codes = torch.full((rows, ldc), 77, dtype=torch.int8, device=DEV)
    scale = torch.zeros(rows, device=DEV)
    fx.token_quantize(h, d[shift:], code_of(fx, t), rows, cols, ldx, fx.SCALE_DFX if rule == "dfx" else fx.SCALE_MAX,
                      codes, ldc, scale)
    assert fx.sync_status(h) == 0
    xs = x[:, :cols].double().numpy()
    a = np.maximum(np.abs(xs).max(1), 2.0 ** -100)
    step = a / 127 if rule == "max" else dfx_step(a)
    got, s = codes.cpu().numpy(), scale.cpu().double().numpy()
    np.testing.assert_allclose(s, step, rtol=2.0 ** -24 if rule == "max" else 0)
    q = got[:, :cols].astype(np.float64)
    slack = 1.5 * 127 * 2.0 ** -23 if rule == "max" else 0.0
    assert np.abs(q - xs / step[:, None]).max() <= 0.5 + slack
    assert np.abs(q).max() <= 127
    up = -(-cols // 16) * 16
    assert (got[:, cols:up] == 0).all() and (got[:, up:] == 77).all()


def test_token_quantize_ties_and_edges(fx, h):
    """Exact ties go to the even code; zeros, magnitudes under the floor, the
    largest finite values; the magnitude at which the DFX scale steps up."""
    big = float(torch.finfo(torch.float32).max)
    rows = torch.zeros(8, 16)
    rows[0, :5] = torch.tensor([127.0, 0.5, 1.5, -2.5, -0.0])
    rows[2, :2] = torch.tensor([2.0 ** -110, -(2.0 ** -140)])
    rows[3, :3] = torch.tensor([big, -big, 1.0])
    rows[4, :2] = torch.tensor([127.49, -3.0])
    rows[5, :2] = torch.tensor([127.5, 1.0])
    rows[6, :3] = torch.tensor([1e-39, -1e-45, 2.0 ** -100])
    rows[7, :1] = -0.0
    d = rows.to(DEV)
    for rule in (fx.SCALE_MAX, fx.SCALE_DFX):
        codes, scale = torch.zeros(8, 16, dtype=torch.int8, device=DEV), torch.zeros(8, device=DEV)
        fx.token_quantize(h, d, fx.F32, 8, 16, 16, rule, codes, 16, scale)
        assert fx.sync_status(h) == 0
        c, s = codes.cpu().numpy().astype(np.int64), scale.cpu().double().numpy()
        assert c[0, :5].tolist() == [127, 0, 2, -2, 0] and s[0] == 1.0
        assert (c[1] == 0).all() and (c[7] == 0).all()
        xs = rows.double().numpy()
        a = np.maximum(np.abs(xs).max(1), 2.0 ** -100)
        step = a / 127 if rule == fx.SCALE_MAX else dfx_step(a)
        np.testing.assert_allclose(s, step, rtol=2.0 ** -23)
        assert np.abs(c - xs / step[:, None]).max() <= 0.5 + 1.5 * 127 * 2.0 ** -23
    assert s[4] == 1.0 and s[5] == 2.0 and c[5, 0] == 64


@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_token_quantize_nonfinite_rows(fx, h, t):
    x = torch.randn(4, 50, generator=gen(9)).to(TYPES[t])
    x[1, 49], x[2, 0], x[2, 1] = float("nan"), float("-inf"), 3.0
    codes, scale = torch.full((4, 64), 5, dtype=torch.int8, device=DEV), torch.zeros(4, device=DEV)
    fx.token_quantize(h, x.to(DEV), code_of(fx, t), 4, 50, 50, fx.SCALE_MAX, codes, 64, scale)
    assert fx.sync_status(h) == fx.FLAG_NONFINITE
    c, s = codes.cpu(), scale.cpu()
    assert torch.isnan(s).tolist() == [False, True, True, False]
    assert (c[1:3] == 0).all() and c[0].abs().max() == 127 and c[3].abs().max() == 127


# ---- products ----------------------------------------------------------------------

def reference(a, sa, b, sb, bias):
    p = (a.astype(np.float64) @ b.astype(np.float64).T) * sa.astype(np.float64)[:, None] * sb.astype(np.float64)
    return p, p + (bias.astype(np.float64) if bias is not None else 0.0)


def check(got, p, want, t, biased):
    tol = 4 * 2.0 ** -24 * np.abs(p) + (2 * 2.0 ** -24 * np.abs(want) if biased else 0) + HALF_ULP[t] * np.abs(want) * 1.01 + (2.0 ** -25 if t == "f16" else 1e-40)
    err = np.abs(got.astype(np.float64) - want)
    assert (err <= tol).all(), (err / tol).max()


SIZES = [(1, 1000, 2048), (1, 1, 16), (2, 37, 48), (7, 16, 64), (16, 129, 144), (17, 64, 4096), (33, 1533, 2064),
         (64, 48, 112), (65, 300, 1008), (128, 128, 128), (129, 130, 272), (300, 515, 400), (513, 270, 1040),
         (1100, 1030, 256)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
def test_token_gemm(fx, h, m, n, k, t):
    note("token_gemm", m, n, k, t)
    g = gen(m * 7 + n * 3 + k)
    lda, ldy = k + (16 if m % 2 else 0), n + (5 if n % 2 else 0)
    a = torch.randint(-128, 128, (m, lda), generator=g, dtype=torch.int16).to(torch.int8)
    b = torch.randint(-128, 128, (n, k), generator=g, dtype=torch.int16).to(torch.int8)
    sa, sb = torch.rand(m, generator=g) * 1e-2, torch.rand(n, generator=g) * 1e-2
    bias = torch.randn(n, generator=g) if (m + n) % 3 else None
    y = torch.full((m, ldy), 123.0, dtype=TYPES[t], device=DEV)
    need = fx.token_gemm_workspace(m, n, k)
    ws = torch.full((max(need, 16),), 0x5A, dtype=torch.uint8, device=DEV)
    args = (h, m, n, k, a.to(DEV), lda, sa.to(DEV), b.to(DEV), sb.to(DEV), bias.to(DEV) if bias is not None else None,
            y, code_of(fx, t), ldy, ws, need)
    fx.token_gemm(*args)
    assert fx.sync_status(h) == 0
    p, want = reference(a[:, :k].numpy(), sa.numpy(), b.numpy(), sb.numpy(), bias.numpy() if bias is not None else None)
    got = y.cpu()
    check(got[:, :n].float().numpy(), p, want, t, bias is not None)
    assert (got[:, n:] == 123.0).all()
    fx.token_gemm(*args)  # a second call finds the work space as the first left it
    assert torch.equal(y.cpu(), got)


@pytest.mark.parametrize("m,n,k", [(20, 70, 4112), (64, 203, 9216), (17, 16, 20000), (130, 1025, 2064), (400, 2100, 272),
                                   (1000, 4100, 144), (4000, 2100, 144), (16, 4096, 1040), (16, 4097, 1040)])
def test_token_gemm_every_tile(fx, h, m, n, k):
    """Sizes that reach each tile shape, the split depth (its last share shorter)
    and both sides of the few-rows rule; bf16 results, reference sums in 64 bits on
    the device."""
    note("token_gemm tiles", m, n, k)
    a = torch.randint(-128, 128, (m, k), device=DEV, dtype=torch.int16).to(torch.int8)
    b = torch.randint(-128, 128, (n, k), device=DEV, dtype=torch.int16).to(torch.int8)
    sa, sb, bias = torch.rand(m, device=DEV), torch.rand(n, device=DEV), torch.randn(n, device=DEV)
    y = torch.zeros(m, n, device=DEV)
    need = fx.token_gemm_workspace(m, n, k)
    ws = torch.full((max(need, 16),), 0x5A, dtype=torch.uint8, device=DEV)
    fx.token_gemm(h, m, n, k, a, k, sa, b, sb, bias, y, fx.F32, n, ws, need)
    assert fx.sync_status(h) == 0
    p = (a.double() @ b.double().t()) * sa.double()[:, None] * sb.double()
    want = p + bias.double()
    assert ((y.double() - want).abs() <= 2.0 ** -24 * (4 * p.abs() + 3 * want.abs())).all()


def test_token_gemm_deepest_sum(fx, h):
    """All codes -128 at the deepest contraction: 2^14 a term, just inside int32."""
    k = 131056
    a, b = torch.full((3, k), -128, dtype=torch.int8, device=DEV), torch.full((5, k), -128, dtype=torch.int8, device=DEV)
    one = torch.ones(8, device=DEV)
    y = torch.zeros(3, 5, device=DEV)
    need = fx.token_gemm_workspace(3, 5, k)
    ws = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    fx.token_gemm(h, 3, 5, k, a, k, one, b, one, None, y, fx.F32, 5, ws, need)
    assert (y.cpu() == float(16384 * k)).all()


@pytest.mark.parametrize("m", [3, 70])
def test_nonfinite_token_gives_a_nan_row(fx, h, m):
    """A token with a NaN or an infinity makes its own output row NaN, no other."""
    x = torch.randn(m, 64, generator=gen(1))
    x[1, 5], x[2, 9] = float("inf"), float("nan")
    codes, scale = torch.empty(m, 64, dtype=torch.int8, device=DEV), torch.empty(m, device=DEV)
    fx.token_quantize(h, x.to(DEV), fx.F32, m, 64, 64, fx.SCALE_DFX, codes, 64, scale)
    y, one = torch.zeros(m, 20, device=DEV), torch.ones(20, device=DEV)
    b = torch.ones(20, 64, dtype=torch.int8, device=DEV)
    fx.token_gemm(h, m, 20, 64, codes, 64, scale, b, one, None, y, fx.F32, 20)
    assert fx.sync_status(h) == fx.FLAG_NONFINITE
    bad = torch.isnan(y.cpu())
    assert bad[1:3].all() and bad.sum() == 40


def test_token_gemm_on_another_stream(fx, h):
    """Inputs made on one stream, the product on the handle's: ordered by an event."""
    side = torch.cuda.Stream()
    fx.set_stream(h, side)
    try:
        a = torch.randint(-127, 128, (70, 256), device=DEV, dtype=torch.int16).to(torch.int8)
        b = torch.randint(-127, 128, (50, 256), device=DEV, dtype=torch.int16).to(torch.int8)
        one, y = torch.ones(70, device=DEV), torch.zeros(70, 50, device=DEV)
        need = fx.token_gemm_workspace(70, 50, 256)
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
        side.wait_stream(torch.cuda.current_stream())
        fx.token_gemm(h, 70, 50, 256, a, 256, one, b, one, None, y, fx.F32, 50, ws, need)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(y.cpu(), (a.cpu().float() @ b.cpu().float().T))
    finally:
        fx.set_stream(h, None)


GROUPS = [[1], [0, 5, 0], [3, 0, 130, 1, 64], [17] * 9, [0, 0, 300], [200, 1, 1, 1], [1] * 70, [0] * 40 + [65] + [0] * 40 + [2]]


@pytest.mark.parametrize("counts", GROUPS, ids=str)
@pytest.mark.parametrize("t,n,k,gather,biased", [("bf16", 130, 272, True, False), ("f32", 37, 144, False, True),
                                                 ("f16", 257, 128, True, True)])
def test_expert_gemm(fx, h, counts, t, n, k, gather, biased):
    note("expert_gemm", counts, t, n, k)
    g = gen(len(counts) + n)
    e, used = len(counts), sum(counts)
    rows = used + 3  # rows past the last group are nobody's
    count = max(1, used // 2) if gather else rows
    a = torch.randint(-128, 128, (count, k), generator=g, dtype=torch.int16).to(torch.int8)
    b = torch.randint(-128, 128, (e, n, k), generator=g, dtype=torch.int16).to(torch.int8)
    sa, sb = torch.rand(count, generator=g) * 1e-2, torch.rand(e, n, generator=g) * 1e-2
    bias = torch.randn(e, n, generator=g) if biased else None
    pick = torch.randint(0, count, (rows,), generator=g, dtype=torch.int32) if gather else None
    off = torch.tensor([0] + counts).cumsum(0).to(torch.int32)
    y = torch.full((rows, n), 9.0, dtype=TYPES[t], device=DEV)
    fx.expert_gemm(h, rows, n, k, e, a.to(DEV), count, k, sa.to(DEV), pick.to(DEV) if gather else None, off.to(DEV),
                   b.to(DEV), sb.to(DEV), bias.to(DEV) if biased else None, y, code_of(fx, t), n)
    assert fx.sync_status(h) == 0
    got = y.cpu()
    src = pick.long() if gather else torch.arange(rows)
    for i in range(e):
        lo, hi = int(off[i]), int(off[i + 1])
        if lo == hi:
            continue
        p, want = reference(a[src[lo:hi]].numpy(), sa[src[lo:hi]].numpy(), b[i].numpy(), sb[i].numpy(),
                            bias[i].numpy() if biased else None)
        check(got[lo:hi].float().numpy(), p, want, t, biased)
    assert (got[used:] == 9.0).all()


@pytest.mark.parametrize("e,rows,n,k,skew", [(4, 4000, 515, 272, 1.0), (8, 900, 130, 144, 2.0), (16, 2000, 300, 400, 0.0),
                                             (3, 16, 200, 1040, 1.0)])
def test_expert_gemm_large_groups(fx, h, e, rows, n, k, skew):
    note("expert_gemm large", e, rows, n, k, skew)
    w = torch.tensor([(1 + i) ** -skew for i in range(e)])
    off = torch.cat([torch.zeros(1), (w.cumsum(0) / w.sum() * rows).round()]).to(torch.int32)
    a = torch.randint(-128, 128, (rows, k), device=DEV, dtype=torch.int16).to(torch.int8)
    b = torch.randint(-128, 128, (e, n, k), device=DEV, dtype=torch.int16).to(torch.int8)
    sa, sb = torch.rand(rows, device=DEV), torch.rand(e, n, device=DEV)
    pick = torch.randperm(rows, device=DEV).to(torch.int32)
    y = torch.zeros(rows, n, device=DEV)
    fx.expert_gemm(h, rows, n, k, e, a, rows, k, sa, pick, off.to(DEV), b, sb, None, y, fx.F32, n)
    assert fx.sync_status(h) == 0
    for i in range(e):
        at = pick[int(off[i]) : int(off[i + 1])].long()
        want = (a[at].double() @ b[i].double().t()) * sa[at].double()[:, None] * sb[i].double()
        assert ((y[int(off[i]) : int(off[i + 1])].double() - want).abs() <= 2.0 ** -24 * 4 * want.abs()).all()


def test_expert_gemm_bad_rows_and_offsets(fx, h):
    """A row index outside the activations gives a row of NaN; offsets that go
    back or pass the rows leave their expert's rows alone; both raise the flag."""
    n, k, rows = 40, 64, 20
    a = torch.ones(4, k, dtype=torch.int8, device=DEV)
    b = torch.ones(3, n, k, dtype=torch.int8, device=DEV)
    one, sb = torch.ones(4, device=DEV), torch.ones(3, n, device=DEV)
    pick = torch.zeros(rows, dtype=torch.int32)
    pick[3], pick[11] = 4, -1
    off = torch.tensor([0, 8, 14, 20], dtype=torch.int32, device=DEV)
    y = torch.full((rows, n), 9.0, device=DEV)
    fx.expert_gemm(h, rows, n, k, 3, a, 4, k, one, pick.to(DEV), off, b, sb, None, y, fx.F32, n)
    assert fx.sync_status(h) == fx.FLAG_RANGE
    got = y.cpu()
    bad = torch.isnan(got).all(1)
    assert bad.nonzero().flatten().tolist() == [3, 11] and (got[~bad] == 64.0).all()
    for values, kept in (([0, 8, 6, 20], (0, 8)), ([0, 8, 14, 21], (0, 14)), ([-1, 8, 14, 20], (8, 20))):
        y.fill_(9.0)
        o = torch.tensor(values, dtype=torch.int32, device=DEV)
        fx.expert_gemm(h, rows, n, k, 3, a, 4, k, one, torch.zeros(rows, dtype=torch.int32, device=DEV), o, b, sb, None,
                       y, fx.F32, n)
        assert fx.sync_status(h) == fx.FLAG_RANGE
        got = y.cpu()
        assert (got[kept[0] : kept[1]] == 64.0).all()
        assert ((got == 64.0) | (got == 9.0)).all()


def test_products_reject_bad_calls(fx, h):
    a, f = torch.zeros(64 * 64, dtype=torch.int8, device=DEV), torch.zeros(64, device=DEV)
    y = torch.zeros(64 * 64, device=DEV)
    ok = dict(M=4, N=8, K=32, a=a, lda=32, a_scale=f, b=a, b_scale=f, bias=None, y=y, y_type=fx.F32, ldy=8)
    call = lambda **kw: fx.token_gemm(h, **{**ok, **kw})  # noqa: E731
    call()
    call(M=0)
    for kw in (dict(K=24), dict(K=0), dict(M=-1), dict(N=0), dict(lda=16), dict(lda=40), dict(ldy=7), dict(a=None),
               dict(a=a[1:]), dict(b=a[8:]), dict(b_scale=None), dict(y=None), dict(y_type=fx.I8), dict(K=131072, lda=131072)):
        with pytest.raises(fx.FxpqError) as e:
            call(**kw)
        assert e.value.status == (fx.ERR_OVERFLOW if kw.get("K") == 131072 else fx.ERR_INVALID_ARG), kw
    q = dict(x=f, x_type=fx.F32, rows=2, cols=20, ldx=20, rule=fx.SCALE_MAX, codes=a, ldc=32, scale=y)
    quant = lambda **kw: fx.token_quantize(h, **{**q, **kw})  # noqa: E731
    quant()
    for kw in (dict(x_type=fx.I32), dict(rule=2), dict(ldx=19), dict(ldc=16), dict(ldc=40), dict(cols=0), dict(rows=-1),
               dict(x=None), dict(codes=a[4:]), dict(scale=None)):
        with pytest.raises(fx.FxpqError):
            quant(**kw)
    off = torch.zeros(3, dtype=torch.int32, device=DEV)
    g = dict(rows=4, N=8, K=32, experts=2, a=a, a_count=4, lda=32, a_scale=f, a_rows=None, offsets=off, b=a, b_scale=f,
             bias=None, y=y, y_type=fx.F32, ldy=8)
    group = lambda **kw: fx.expert_gemm(h, **{**g, **kw})  # noqa: E731
    group()
    for kw in (dict(experts=0), dict(a_count=3), dict(a_count=0, a_rows=off), dict(offsets=None), dict(K=30), dict(ldy=4)):
        with pytest.raises(fx.FxpqError):
            group(**kw)
    assert fx.sync_status(h) == 0


def test_products_of_no_rows_of_a_wide_layer(fx, h):
    """M = 0 is accepted at a width that more than one block column takes, and
    writes nothing."""
    b, f = torch.zeros(5000, 64, dtype=torch.int8, device=DEV), torch.zeros(5000, device=DEV)
    y = torch.full((4, 5000), 9.0, device=DEV)
    need = fx.token_gemm_workspace(0, 5000, 64)
    assert need == 0
    fx.token_gemm(h, 0, 5000, 64, None, 64, None, b, f, None, y, fx.F32, 5000, None, need)
    assert fx.sync_status(h) == 0 and (y == 9.0).all()


def check_on_device(y, p, want, t):
    tol = 4 * 2.0 ** -24 * p.abs() + (2 * 2.0 ** -24 + 1.01 * HALF_ULP[t]) * want.abs() + (2.0 ** -25 if t == "f16" else 1e-40)
    err = (y.double() - want).abs()
    assert (err <= tol).all(), (err / tol).max()


def codes_of(seed, *shape):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-128, 128, shape, generator=g, device=DEV, dtype=torch.int16).to(torch.int8)


def scales_of(seed, *shape):
    return torch.rand(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV) * 1e-2


@pytest.mark.parametrize("m,n,k", [(130, 1025, 2064), (600, 2100, 272), (513, 4097, 144), (4097, 2101, 272), (4000, 2100, 144)])
@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("aligned", [True, False], ids=["aligned", "odd"])
def test_token_gemm_results_of_every_tile(fx, h, m, n, k, t, aligned):
    """Each tile shape (64 x 64, 128 x 64, 128 x 128, 256 x 256 twice) in each type of
    result, its rows 16-byte aligned (whole pieces, the last one of an odd N in part)
    and not (element by element); partly filled tiles on both sides."""
    note("token_gemm results", m, n, k, t, aligned)
    a, b, sa, sb = codes_of(1, m, k), codes_of(2, n, k), scales_of(3, m), scales_of(4, n)
    bias = torch.randn(n, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV)
    ldy = (n + 7) // 8 * 8 if aligned else n + 1 + n % 2
    y = torch.full((m, ldy), 123.0, dtype=TYPES[t], device=DEV)
    need = fx.token_gemm_workspace(m, n, k)
    ws = torch.full((max(need, 16),), 0x5A, dtype=torch.uint8, device=DEV)
    fx.token_gemm(h, m, n, k, a, k, sa, b, sb, bias, y, code_of(fx, t), ldy, ws, need)
    assert fx.sync_status(h) == 0
    p = (a.double() @ b.double().t().contiguous()) * sa.double()[:, None] * sb.double()
    check_on_device(y[:, :n], p, p + bias.double(), t)
    assert (y[:, n:] == 123.0).all()


@pytest.mark.parametrize("counts,n,k", [([257, 0, 2561, 1182], 2101, 144), ([3000, 1, 255, 744], 2100, 144),
                                        ([129, 0, 1, 640, 230], 1101, 144), ([385, 3, 0, 511, 1], 2101, 144)],
                         ids=["256x256 odd", "256x256", "128x64", "128x128"])
@pytest.mark.parametrize("t", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("aligned", [True, False], ids=["aligned", "odd"])
def test_expert_gemm_results_of_every_tile(fx, h, counts, n, k, t, aligned):
    """Ragged groups, some of one row, none, or one row past a whole tile, in the tiles
    that large groups take: every row by its own expert's weights, none past the last
    group."""
    note("expert_gemm results", counts, n, k, t, aligned)
    e, rows = len(counts), sum(counts)
    count = rows // 2
    a, b = codes_of(1, count, k), codes_of(2, e, n, k)
    sa, sb = scales_of(3, count), scales_of(4, e, n)
    bias = torch.randn(e, n, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV)
    pick = (torch.randperm(rows, generator=gen(6)) % count).to(torch.int32).to(DEV)
    off = torch.tensor([0] + counts).cumsum(0).to(torch.int32)
    ldy = (n + 7) // 8 * 8 if aligned else n + 1 + n % 2
    y = torch.full((rows + 2, ldy), 123.0, dtype=TYPES[t], device=DEV)
    fx.expert_gemm(h, rows, n, k, e, a, count, k, sa, pick, off.to(DEV), b, sb, bias, y, code_of(fx, t), ldy)
    assert fx.sync_status(h) == 0
    for i in range(e):
        lo, hi = int(off[i]), int(off[i + 1])
        at = pick[lo:hi].long()
        p = (a[at].double() @ b[i].double().t().contiguous()) * sa[at].double()[:, None] * sb[i].double()
        if lo < hi:
            check_on_device(y[lo:hi, :n], p, p + bias[i].double(), t)
    assert (y[rows:] == 123.0).all() and (y[:, n:] == 123.0).all()
