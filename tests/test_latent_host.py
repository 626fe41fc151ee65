"""Argument checks of the latent attention calls, before any device call: a block of
zeros stands for a handle, which no call gets to use."""
import ctypes as C
import os

import pytest


@pytest.fixture(scope="module")
def fx():
    from paper_2203_12091_amd import fxpq
    if not os.path.exists(fxpq.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    fxpq.lib()
    return fxpq


class Calls:
    """Each call with good arguments (addresses that are never followed), some replaced."""

    def __init__(self, fx):
        self.fx, self.L = fx, fx.lib()
        self.h = C.cast(C.create_string_buffer(1 << 16), C.c_void_p)
        self.a = 1 << 20  # an aligned address

    def cache(self, **kw):
        return self.fx.LatentCache(**{**dict(codes=self.a, scale=self.a, rope_scale=self.a, pages=8, page=16, latent=512, rope=64), **kw})

    def batch(self, **kw):
        return self.fx.KvBatch(**{**dict(start=self.a, length=self.a, table=self.a, seqs=2, table_ld=4, tokens=5, max_new=3,
                                         max_len=64), **kw})

    def rotary(self, **kw):
        return self.fx.Rotary(**{**dict(cos=self.a, sin=self.a, positions=64, dims=64), **kw})

    def append(self, cache=None, batch=None, rot=None, **kw):
        v = {**dict(h=self.h, rule=0, c=self.a, ldc=576, r=self.a, ldr=576, q=self.a, ldq=512, hdq=128, q_out=2 * self.a, ldqo=256,
                    hdqo=64, heads=4, t=self.fx.F32), **kw}
        rot = self.rotary() if rot is None else rot
        return self.L.fxpq_latent_append(v["h"], C.byref(cache or self.cache()), C.byref(batch or self.batch()), C.byref(rot),
                                         v["rule"], v["c"], v["ldc"], v["r"], v["ldr"], v["q"], v["ldq"], v["hdq"], v["q_out"],
                                         v["ldqo"], v["hdqo"], v["heads"], v["t"])

    def read(self, cache=None, batch=None, **kw):
        v = {**dict(h=self.h, start=self.a, tokens=80, codes=self.a, ldc=512, scale=self.a, latent=self.a, ldl=512, key=self.a,
                    ldk=64, t=self.fx.F32), **kw}
        return self.L.fxpq_latent_read(v["h"], C.byref(cache or self.cache()), C.byref(batch or self.batch()), v["start"],
                                       v["tokens"], v["codes"], v["ldc"], v["scale"], v["latent"], v["ldl"], v["key"], v["ldk"], v["t"])

    def attention(self, cache=None, batch=None, **kw):
        v = {**dict(h=self.h, q=self.a, ldq=2048, hdq=512, qr=self.a, ldqr=256, hdqr=64, heads=4, scale=0.1, causal=1, out=self.a,
                    ldo=2048, hdo=512, t=self.fx.F32), **kw}
        return self.L.fxpq_latent_attention(v["h"], C.byref(cache or self.cache()), C.byref(batch or self.batch()), v["q"], v["ldq"],
                                            v["hdq"], v["qr"], v["ldqr"], v["hdqr"], v["heads"], v["scale"], v["causal"], v["out"],
                                            v["ldo"], v["hdo"], v["t"], None, 0)

    def expanded(self, batch=None, **kw):
        d = dict(k=self.a, key=self.a, v=self.a, ldk=1024, hdk=256, ld_key=64, ldv=1024, hdv=256, start=self.a, tokens=100, heads=4,
                 nope=128, rope=64, vdim=128)
        c = {**dict(h=self.h, q=self.a, ldq=768, scale=0.1, causal=1, out=self.a, ldo=512, t=self.fx.F32)}
        for k, x in kw.items():
            (d if k in d else c)[k] = x
        return self.L.fxpq_expanded_attention(c["h"], C.byref(self.fx.ExpandedKv(**d)), C.byref(batch or self.batch()), c["q"], c["ldq"],
                                              c["scale"], c["causal"], c["out"], c["ldo"], c["t"])


@pytest.fixture
def calls(fx):
    return Calls(fx)


def test_struct_sizes(fx):
    assert C.sizeof(fx.LatentCache) == 40 and C.sizeof(fx.ExpandedKv) == 96


def test_bad_caches_and_batches(calls):
    bad = calls.fx.ERR_INVALID_ARG
    odd = calls.a + 4
    for kw in (dict(codes=None), dict(codes=odd), dict(scale=None), dict(scale=odd), dict(rope_scale=None), dict(rope_scale=odd),
               dict(pages=0), dict(page=8), dict(page=48), dict(latent=384), dict(latent=0), dict(rope=0), dict(rope=80), dict(rope=24)):
        cache = calls.cache(**kw)
        assert [f(cache) for f in (calls.append, calls.read, calls.attention)] == [bad] * 3, kw
        n = C.c_int64(-1)
        assert calls.L.fxpq_latent_attention_workspace(calls.h, C.byref(cache), C.byref(calls.batch()), 4, C.byref(n)) == bad
        assert n.value == 0
    for kw in (dict(start=None), dict(length=None), dict(start=calls.a + 2), dict(seqs=0), dict(seqs=65536), dict(tokens=-1),
               dict(max_new=6), dict(max_new=0), dict(max_len=2), dict(max_len=2 ** 30 + 1)):
        batch = calls.batch(**kw)
        assert calls.expanded(batch) == bad, kw
        assert [f(None, batch) for f in (calls.append, calls.read, calls.attention)] == [bad] * 3, kw
    for kw in (dict(table=None), dict(table=calls.a + 1), dict(table_ld=0), dict(max_len=65)):
        batch = calls.batch(**kw)
        assert [f(None, batch) for f in (calls.append, calls.read, calls.attention)] == [bad] * 3, kw


def test_bad_arguments(calls):
    fx, bad, a = calls.fx, calls.fx.ERR_INVALID_ARG, calls.a
    for kw in (dict(h=None), dict(t=fx.I8), dict(rule=2), dict(ldc=511), dict(ldr=63), dict(c=None), dict(r=None), dict(c=a + 2),
               dict(r=a + 1), dict(q=a + 2), dict(q_out=None), dict(q_out=a + 2), dict(heads=0), dict(heads=65536), dict(ldq=63),
               dict(hdq=63), dict(ldqo=63), dict(hdqo=32), dict(ldqo=128), dict(q_out=a)):  # the last two: rows that overlap
        assert calls.append(**kw) == bad, kw
    for kw in (dict(dims=32), dict(dims=0), dict(cos=None), dict(sin=None), dict(sin=a + 2), dict(positions=-1)):
        assert calls.append(rot=calls.rotary(**kw)) == bad, kw
    for kw in (dict(h=None), dict(t=fx.I32), dict(tokens=-1), dict(start=a + 2), dict(start=None), dict(codes=a + 8), dict(ldc=496),
               dict(ldc=520), dict(scale=a + 1), dict(latent=a + 2), dict(ldl=500), dict(key=a + 1), dict(ldk=60)):
        assert calls.read(**kw) == bad, kw
    for kw in (dict(h=None), dict(t=fx.I64), dict(heads=0), dict(heads=65536), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(ldq=511), dict(hdq=500), dict(ldqr=63), dict(hdqr=0), dict(ldo=511), dict(hdo=256), dict(ldo=1024), dict(q=None),
               dict(qr=None), dict(out=None), dict(q=a + 2), dict(qr=a + 1), dict(out=a + 2)):
        assert calls.attention(**kw) == bad, kw
    assert calls.attention(None, calls.batch(tokens=1 << 24, max_new=1 << 24, max_len=1 << 24, table_ld=1 << 20), heads=64) == bad
    for kw in (dict(h=None), dict(t=fx.I16), dict(nope=96), dict(vdim=32), dict(rope=16), dict(rope=128), dict(heads=0),
               dict(heads=65536), dict(tokens=-1), dict(ldk=127), dict(hdk=64), dict(ldv=100), dict(hdv=127), dict(ld_key=63),
               dict(ldq=767), dict(ldo=511), dict(scale=float("nan")), dict(q=None), dict(out=None), dict(k=None), dict(key=None),
               dict(v=None), dict(start=None), dict(start=a + 2), dict(k=a + 2), dict(out=a + 1)):
        assert calls.expanded(**kw) == bad, kw
    n = C.c_int64(-1)
    size = calls.L.fxpq_latent_attention_workspace
    assert size(None, C.byref(calls.cache()), C.byref(calls.batch()), 4, C.byref(n)) == bad and n.value == 0
    assert size(calls.h, C.byref(calls.cache()), C.byref(calls.batch()), 4, None) == bad


def test_calls_without_tokens_return_at_once(calls):
    """Nothing is launched, and nothing needs to be there."""
    none = calls.batch(tokens=0, max_new=0)
    assert calls.append(None, none, c=None, r=None, q=None) == calls.fx.OK
    assert calls.read(None, none, start=None, tokens=0) == calls.fx.OK
    assert calls.read(None, None, codes=None, scale=None, latent=None, key=None) == calls.fx.OK
    assert calls.attention(None, none, q=None, qr=None, out=None) == calls.fx.OK
    assert calls.expanded(none, q=None, out=None, k=None, key=None, v=None) == calls.fx.OK
    n = C.c_int64(-1)
    assert calls.L.fxpq_latent_attention_workspace(calls.h, C.byref(calls.cache()), C.byref(none), 4, C.byref(n)) == calls.fx.OK
    assert n.value == 0


def test_rows_that_overlap_whatever_the_strides(calls):
    """2^31 - 1 tokens 2^33 apart: the last begins past 2^63, far behind the next head's first."""
    batch = calls.batch(tokens=2 ** 31 - 1)
    assert calls.attention(None, batch, ldo=2 ** 33, hdo=2 ** 34) == calls.fx.ERR_INVALID_ARG
    assert calls.append(None, batch, ldqo=2 ** 33, hdqo=2 ** 34) == calls.fx.ERR_INVALID_ARG
