"""The decoder layer's host side, without a device: the library is replaced by one
that records its calls, torch's streams by a name."""
import types

import pytest

torch = pytest.importorskip("torch")

STREAM = "the current stream"


class Recorder:
    """Stands for the library's binding: every call is noted and does nothing; work
    spaces are wanted by every product."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def Handle(self, device):
        return types.SimpleNamespace(value=None, device=device, close=lambda: None)

    def token_gemm_workspace(self, *args):
        return 4096

    def cache_attention_workspace(self, *args):
        return 8192

    def kv_cache(self, k, v, k_scale, v_scale, pages, page, heads, dim):
        return types.SimpleNamespace(pages=pages, page=page, heads=heads, dim=dim)

    def kv_batch(self, start, length, table, seqs, table_ld, tokens, max_new, max_len):
        return types.SimpleNamespace(seqs=seqs, tokens=tokens, max_new=max_new, max_len=max_len)

    def rotary(self, cos, sin, positions, dims, interleaved=0):
        return types.SimpleNamespace(positions=positions, dims=dims)

    def __getattr__(self, name):
        what = getattr(self.real, name)
        return (lambda *args: self.calls.append((name, args))) if callable(what) else what

    def names(self):
        return [n for n, _ in self.calls]


@pytest.fixture
def dec(monkeypatch):
    from paper_2203_12091_amd import decoder
    monkeypatch.setattr(decoder, "fx", Recorder(decoder.fx))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: STREAM)
    return decoder


def make(dec, **kw):
    layer = dec.Layer(64, 4, 2, 16, experts=4, top=2, inner=48, dtype=torch.float32, device="cpu", **kw)
    cache = dec.Cache(pages=8, page=16, heads=2, dim=16, max_pages_per_seq=4, max_seqs=3, device="cpu")
    return layer, cache


def test_quantization_runs_on_the_stream_of_its_values(dec):
    """What torch computed on its current stream is quantized on that stream: the
    weights of a new layer, and rows given to the helper."""
    layer, _ = make(dec)
    names = dec.fx.names()
    assert "token_quantize" in names and names.index("set_stream") < names.index("token_quantize")
    dec.fx.calls.clear()
    dec.quantize_rows(layer.h, torch.zeros(2, 64))
    assert dec.fx.names() == ["set_stream", "token_quantize"]
    assert dec.fx.calls[0][1] == (layer.h, STREAM)


def test_each_call_has_a_work_space_of_its_own(dec):
    """Calls in flight on two streams must not share one: two products' work spaces,
    both still held here, are different memory of the size asked for."""
    layer, _ = make(dec)
    dec.fx.calls.clear()
    for _ in range(2):
        layer._linear(torch.zeros(3, 64), layer.qkv)
    spaces = [args[-2] for name, args in dec.fx.calls if name == "token_gemm"]
    assert [s.numel() for s in spaces] == [4096, 4096]
    assert spaces[0].data_ptr() != spaces[1].data_ptr()
    assert layer._workspace(0) is None


def test_step_without_new_tokens(dec):
    """Cache.extend accepts one; the layer answers with no rows."""
    layer, cache = make(dec)
    for new in ([0, 0], [5, 0]):
        y = layer.forward(torch.zeros(sum(new), 64), cache, cache.extend([0, 1], new))
        assert y.shape == (sum(new), 64) and y.dtype == torch.float32
    assert cache.length == {0: 5, 1: 0}


def test_rows_of_any_strides_are_quantized_as_they_read(dec):
    """The library takes rows of neighbouring values: what it is given has the
    tensor's values at the row stride that is named."""
    base = torch.arange(24 * 12, dtype=torch.float32).view(24, 12)
    for x in (base, base[:, ::2], base[:, 3:9], base.t(), base[:1].expand(5, 12), base[0].expand(1, 12), base[3:4, 2:5],
              base[::5], base[:0]):
        dec.fx.calls.clear()
        dec.quantize_rows(None, x)
        _, given, _, rows, cols, ldx, _, codes, ldc, scale = dec.fx.calls[-1][1]
        assert (rows, cols) == x.shape and ldx >= cols and ldc == codes.shape[1] >= cols and scale.numel() == rows
        got = torch.as_strided(given, (rows, cols), (ldx, 1)) if rows else given
        assert torch.equal(got, x)


def test_cache_refuses_lists_that_do_not_match(dec):
    """A count for each sequence, and one sequence at least: the device reads as many
    starts and lengths as there are sequences."""
    _, cache = make(dec)
    for seqs, new in (([0, 1], [5]), ([0], [5, 6]), ([], [])):
        with pytest.raises(ValueError):
            cache.extend(seqs, new)
    assert cache.length == {} and cache.owned == {} and len(cache.free) == 8


def test_layer_refuses_what_does_not_fit_the_batch(dec):
    """The kernels take the number of rows, heads and dimensions from the batch and
    the cache: none may go past x or the layer's own.  Nothing is launched."""
    layer, cache = make(dec)
    other = dec.Cache(pages=8, page=16, heads=4, dim=16, max_pages_per_seq=4, max_seqs=3, device="cpu")
    wide = dec.Cache(pages=8, page=16, heads=2, dim=32, max_pages_per_seq=4, max_seqs=3, device="cpu")
    dec.fx.calls.clear()
    for x, c in ((torch.zeros(4, 64), cache), (torch.zeros(6, 64), cache), (torch.zeros(5, 48), cache),
                 (torch.zeros(5), cache), (torch.zeros(5, 64), other), (torch.zeros(5, 64), wide)):
        with pytest.raises(ValueError):
            layer.forward(x, c, c.extend([0], [5]))
        c.release(0)
    assert dec.fx.calls == []


def test_layer_refuses_sequences_past_its_positions(dec):
    """The append would skip such a sequence, and the attention run over slots that
    were never written.  The last position is still fine."""
    layer, cache = make(dec, positions=20)
    layer.forward(torch.zeros(24, 64), cache, cache.extend([0, 1], [20, 4]))
    dec.fx.calls.clear()
    with pytest.raises(ValueError):
        layer.forward(torch.zeros(2, 64), cache, cache.extend([0, 1], [1, 1]))
    assert dec.fx.calls == []


def test_failed_forward_takes_back_the_batch(dec, monkeypatch):
    """Lengths and pages are what they were before the extend whose tokens did not
    get through, whether they were refused or a call failed on the way."""
    layer, cache = make(dec, positions=40)
    layer.forward(torch.zeros(22, 64), cache, cache.extend([0, 1], [20, 2]))

    def state():
        return dict(cache.length), {s: list(p) for s, p in cache.owned.items()}, sorted(cache.free)

    before = state()
    with pytest.raises(ValueError):  # a new sequence, a page more, too many tokens
        layer.forward(torch.zeros(39, 64), cache, cache.extend([0, 2, 1], [21, 17, 1]))
    assert state() == before

    def fails(*args):
        raise dec.fx.real.FxpqError("fxpq_cache_attention", 5)

    monkeypatch.setattr(dec.fx, "cache_attention", fails, raising=False)
    with pytest.raises(dec.fx.real.FxpqError):
        layer.forward(torch.zeros(14, 64), cache, cache.extend([1], [14]))
    assert state() == before
    batch = cache.extend([1], [3])
    cache.release(1)
    cache.retract(batch)  # a sequence that is gone stays gone
    assert 1 not in cache.length and len(cache.free) == 6


def test_failed_forward_of_a_batch_made_by_hand(dec):
    """A batch that no extend made has nothing to take back: the error is its own."""
    layer, cache = make(dec)
    batch = dec.fx.kv_batch(None, None, None, 1, 4, 5, 5, 5)
    with pytest.raises(ValueError):
        layer.forward(torch.zeros(4, 64), cache, batch)
    assert cache.length == {} and len(cache.free) == 8
