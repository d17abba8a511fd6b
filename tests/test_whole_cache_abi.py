"""Caches held whole on the host: the structs mirror the header, bad arguments are refused before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2406_02542_amd import api
from tests.test_cache_operators_abi import BIG, P, _layout, _members, by


@pytest.mark.parametrize("name,struct", [("loki_cache", api.CacheArgs), ("loki_span_args", api.SpanArgs)])
def test_structs_match_the_header(name, struct):
    assert [f[0].rstrip("_") for f in struct._fields_] == _members(name)


def _cache(**kw):
    return api.CacheArgs(**{**dict(k=P, v=P), **kw})


BAD_CACHES = [(dict(k=None), 1), (dict(v=None), 1), (dict(k_scales=P), 1), (dict(v_scales=P), 1), (dict(k=P + 8), 3), (dict(v=P + 4), 3),
              (dict(k_scales=P + 2, v_scales=P), 3), (dict(k_scales=P, v_scales=P + 8), 3),
              (dict(page_table=P, page_rows=8, pages_per_seq=64, n_pages=9), 1), (dict(page_table=P, page_rows=48, pages_per_seq=64, n_pages=9), 1),
              (dict(page_table=P, page_rows=16, pages_per_seq=31, n_pages=9), 1), (dict(page_table=P, page_rows=0, pages_per_seq=32, n_pages=9), 1),
              (dict(page_table=P, page_rows=16, pages_per_seq=0, n_pages=9), 1), (dict(page_table=P, page_rows=16, pages_per_seq=32, n_pages=0), 1),
              (dict(page_table=P, page_rows=256, pages_per_seq=2, n_pages=1 << 23), 2), (dict(page_table=P + 2, page_rows=16, pages_per_seq=32, n_pages=9), 3)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(kw, status):
    L, lay, n, span = api.lib(), _layout(), ctypes.c_size_t(), api.SpanArgs()
    c = _cache(**kw)
    assert L.dense_cache_workspace_bytes(by(lay), by(c), 512, by(span), by(n)) == status
    assert L.dense_decode_cache(by(lay), P, by(c), 512, by(span), P, BIG, P, None) == status
    assert L.loki_read_rows(by(lay), by(c), 4, P, P, P, None) == status
    assert L.loki_append(by(lay), by(c), 4, by(_append()), None) == status


def _append(**kw):
    t = lambda i, o: api.RotaryTensor(i, o, 1024, 256, 128, 1024, 256, 128)
    a = api.RotaryArgs(t(P, 2 * P), t(4 * P, None), t(5 * P, None), P, P, P, 0, 128, 0, 0, 1.0)
    for name, x in kw.items():
        part, _, member = name.partition("__")
        if member:
            setattr(getattr(a, part), member, x)
        else:
            setattr(a, part, x)
    return a


def test_attention_refusals():
    L, lay, n = api.lib(), _layout(), ctypes.c_size_t()

    def call(S=512, q=P, ws=P, nbytes=BIG, out=P, lay=lay, **kw):
        return L.dense_decode_cache(by(lay), q, by(_cache()), S, by(api.SpanArgs(**kw)), ws, nbytes, out, None)

    for kw in (dict(q=None), dict(ws=None), dict(out=None), dict(S=0), dict(S=513), dict(queries_per_seq=-1), dict(window=-1), dict(sinks=-1),
               dict(queries_per_seq=(1 << 23) + 1), dict(queries_per_seq=1 << 23, lay=_layout(Hq=16, Hkv=2))):
        assert call(**kw) == 1, kw
    for kw in (dict(q=P + 8), dict(out=P + 4), dict(ws=P + 16), dict(seq_lens=P + 2)):
        assert call(**kw) == 3, kw
    assert call(lay=_layout(D=64)) == 2
    assert L.dense_cache_workspace_bytes(by(lay), by(_cache()), 512, by(api.SpanArgs()), by(n)) == 0
    assert call(nbytes=n.value - 1) == 4
    assert L.dense_cache_workspace_bytes(by(lay), by(_cache()), 512, by(api.SpanArgs()), None) == 1
    assert L.dense_cache_workspace_bytes(by(lay), by(_cache()), 512, None, by(n)) == 1
    assert L.dense_cache_workspace_bytes(by(lay), None, 512, by(api.SpanArgs()), by(n)) == 1
    assert L.dense_cache_workspace_bytes(None, by(_cache()), 512, by(api.SpanArgs()), by(n)) == 1
    long = _layout(S_cap=(1 << 30) + 1)
    assert L.dense_cache_workspace_bytes(by(long), by(_cache()), 1 << 30, by(api.SpanArgs()), by(n)) == 0
    assert L.dense_cache_workspace_bytes(by(long), by(_cache()), (1 << 30) + 1, by(api.SpanArgs()), by(n)) == 1


def test_append_refusals():
    L, lay = api.lib(), _layout()
    call = lambda n=4, lay=lay, **kw: L.loki_append(by(lay), by(_cache()), n, by(_append(**kw)), None)
    for kw in (dict(n=0), dict(n=(1 << 23) + 1), dict(k__in_=None), dict(v__in_=None), dict(k__out=P), dict(v__out=P), dict(rows=None),
               dict(rotary_dims=-2), dict(rotary_dims=3), dict(rotary_dims=130), dict(positions=None), dict(frequencies=None), dict(q__out=None),
               dict(q__in_batch=-8), dict(k__in_token=-8), dict(q__out=P, q__out_head=256), dict(k__in_=P)):
        assert call(**kw) == 1, kw  # (k__in_: out of the cache itself)
    for kw in (dict(q__in_=P + 2), dict(k__in_=P + 8), dict(v__in_=P + 4), dict(k__in_head=3), dict(q__out_token=2), dict(rows=P + 2),
               dict(positions=P + 1), dict(frequencies=P + 4)):
        assert call(**kw) == 3, kw
    assert L.loki_append(by(lay), by(_cache()), 4, None, None) == 1


def test_read_refusals():
    L, lay = api.lib(), _layout()
    call = lambda n=4, rows=P, k=P, v=P, lay=lay: L.loki_read_rows(by(lay), by(_cache()), n, rows, k, v, None)
    assert call(n=0) == call(rows=None) == call(k=None, v=None) == call(n=(1 << 23) + 1) == call(n=1 << 23, lay=_layout(Hq=16, Hkv=16)) == 1
    assert call(rows=P + 2) == call(k=P + 8) == call(v=P + 2) == 3


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("scales", [None, P])
@pytest.mark.parametrize("B,Hq,Hkv", [(1, 8, 8), (3, 8, 1), (64, 64, 8), (2, 64, 8), (5, 32, 8)])
def test_workspace_of_the_longest_length_serves_shorter_ones(B, Hq, Hkv, scales, dtype):
    lay = api.make_layout(B, Hq, Hkv, 128, 128, 1 << 20, dtype)
    c, n = _cache(k_scales=scales, v_scales=scales), ctypes.c_size_t()

    def size(S, **kw):
        assert api.lib().dense_cache_workspace_bytes(by(lay), by(c), S, by(api.SpanArgs(**kw)), by(n)) == 0
        return n.value

    for kw in (dict(), dict(window=1), dict(window=1000, sinks=4), dict(queries_per_seq=5), dict(queries_per_seq=8), dict(queries_per_seq=13, window=20000), dict(queries_per_seq=300, window=4096), dict(queries_per_seq=3000)):
        sizes = [size(S, **kw) for S in (1, 2, 31, 64, 65, 127, 128, 129, 255, 700, 1100, 4186, 8192, 16384, 100000, 1 << 20)]
        assert sizes == sorted(sizes), kw


def test_binding_refuses_what_does_not_fit():
    lay = api.make_layout(2, 4, 2, 128, 128, 64, torch.float32)
    t = torch.zeros(2, 2, 64, 128)
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    for args, kw, what in (((t, t), {}, "GPU"), ((t[:, :, :63], t), {}, "k must be"), ((t, t[:1]), {}, "v must be"), ((t, t), dict(k_scales=t), "together"),
                           ((t, t), dict(page_table=i(3, 4)), "page_table"), ((t, t), dict(page_table=i(2)), "page_table"),
                           ((t[0], t), dict(page_table=i(2, 4)), "k must be"), ((t, t), dict(k_scales=t, v_scales=t), "k must be")):
        with pytest.raises(ValueError, match=what):
            api.Cache(lay, *args, **kw)
    x, rows, pos, f = torch.zeros(2, 3, 2, 128), i(2, 3), i(2, 3), torch.zeros(64, dtype=torch.float64)
    with pytest.raises(ValueError, match="rows"):
        api.loki_append(lay, None, i(3, 3), x, x)
    with pytest.raises(ValueError, match="q_out"):
        api.loki_append(lay, None, rows, x, x, q=x)
    with pytest.raises(ValueError, match="frequencies"):
        api.loki_append(lay, None, rows, x, x, positions=pos)
    with pytest.raises(ValueError, match="frequencies"):
        api.loki_append(lay, None, rows, x, x, frequencies=f)
    with pytest.raises(ValueError, match="GPU"):
        api.loki_append(lay, None, rows, x, x)
    with pytest.raises(ValueError, match="rows"):
        api.loki_read_rows(lay, None, i(3, 3), x)
