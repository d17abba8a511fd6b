"""Rotary positions, weighed rows, eviction and shared prefixes on the host: the structs mirror the header, the
frequencies follow their formulas, and bad arguments are refused before anything is launched (no GPU needed)."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2406_02542_amd import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000  # non-null, aligned, never dereferenced
by = ctypes.byref
BIG = 1 << 40


def _members(name):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "loki.h")).read(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text)[1]
    return [re.sub(r"[\s*]", "", m) for line in body.split(";") if line.strip()
            for m in re.sub(r"^\s*(const\s+)?\w+\s*\**", "", line.strip()).split(",")]


@pytest.mark.parametrize("name,struct", [("loki_rotary_tensor", api.RotaryTensor), ("loki_rotary_args", api.RotaryArgs),
                                         ("loki_evict_args", api.EvictArgs)])
def test_structs_match_the_header(name, struct):
    assert [f[0].rstrip("_") for f in struct._fields_] == _members(name)


def test_struct_sizes():
    assert ctypes.sizeof(api.RotaryTensor) == 64
    assert ctypes.sizeof(api.RotaryArgs) == 3 * 64 + 3 * 8 + 5 * 4 + 4
    assert ctypes.sizeof(api.EvictArgs) == 12 * 8 + 4 * 4


# ---- frequencies --------------------------------------------------------------------------------
def _freqs(R, *a, **kw):
    f, scale = api.loki_rotary_frequencies(R, *a, device="cpu", **kw)
    return f.tolist(), scale


@pytest.mark.parametrize("R", [2, 20, 64, 128])
def test_frequencies_unscaled_and_linear(R):
    f, scale = _freqs(R, 10000.0)
    assert scale == 1.0 and f == pytest.approx([10000.0 ** (-2 * i / R) for i in range(R // 2)], rel=1e-14)
    g, _ = _freqs(R, 10000.0, api.ROTARY_LINEAR, 4.0)
    assert g == pytest.approx([x / 4 for x in f], rel=1e-14)


def test_frequencies_larger_base():
    f, _ = _freqs(64, 10000.0)
    g, _ = _freqs(64, 10000.0, api.ROTARY_BASE, 8.0)
    assert g[0] == f[0] == 1.0
    assert g[-1] == pytest.approx(f[-1] / 8, rel=1e-12)


def test_frequencies_bands():
    f, _ = _freqs(128, 500000.0)
    g, _ = _freqs(128, 500000.0, api.ROTARY_BANDS, 8.0, 8192.0, 1.0, 4.0)
    seen = set()
    for x, y in zip(f, g):
        turns = 8192.0 * x / (2 * math.pi)
        if turns > 4:
            seen.add("short")
            assert y == x
        elif turns < 1:
            seen.add("long")
            assert y == pytest.approx(x / 8, rel=1e-14)
        else:
            seen.add("mixed")
            m = (turns - 1) / 3
            assert y == pytest.approx(m * x + (1 - m) * x / 8, rel=1e-13)
    assert seen == {"short", "long", "mixed"}


def test_frequencies_ramp():
    R, base, factor, ctx, low, high = 128, 10000.0, 4.0, 4096.0, 1.0, 32.0
    f, _ = _freqs(R, base)
    g, scale = _freqs(R, base, api.ROTARY_RAMP, factor, ctx, low, high)
    assert scale == pytest.approx(0.1 * math.log(4.0) + 1.0, rel=1e-6)
    # the pair that makes `turns` turns in the original context, as a real number
    pair = lambda turns: R * math.log(ctx / (2 * math.pi * turns)) / (2 * math.log(base))
    a, b = math.floor(pair(high)), math.ceil(pair(low))
    assert 0 < a < b < R // 2
    for i, (x, y) in enumerate(zip(f, g)):
        r = min(max((i - a) / (b - a), 0.0), 1.0)
        assert y == pytest.approx(x * (1 - r) + x / factor * r, rel=1e-12)


@pytest.mark.parametrize("a", [(3, 10000.0, 0, 1.0, 0, 0, 0), (0, 10000.0, 0, 1.0, 0, 0, 0), (130, 10000.0, 0, 1.0, 0, 0, 0),
                               (64, 1.0, 0, 1.0, 0, 0, 0), (64, float("nan"), 0, 1.0, 0, 0, 0), (64, 1e4, 5, 1.0, 0, 0, 0),
                               (64, 1e4, -1, 1.0, 0, 0, 0), (64, 1e4, 1, 0.5, 0, 0, 0), (64, 1e4, 1, float("nan"), 0, 0, 0),
                               (2, 1e4, 2, 2.0, 0, 0, 0), (64, 1e4, 3, 8.0, 0, 1, 4), (64, 1e4, 3, 8.0, 8192, 4, 4),
                               (64, 1e4, 4, 8.0, 8192, 0, 4), (64, 1e4, 4, 8.0, 8192, 8, 4)])
def test_frequencies_refusals(a):
    buf = (ctypes.c_double * 64)()
    assert api.lib().loki_rotary_frequencies(*a, ctypes.addressof(buf), None) == 1
    assert api.lib().loki_rotary_frequencies(64, 1e4, 0, 1.0, 0, 0, 0, None, None) == 1


# ---- refusals -----------------------------------------------------------------------------------
LAY = dict(B=2, Hq=8, Hkv=2, D=128, d_split=32, S_cap=512, dtype=api.LOKI_BF16)


def _layout(**kw):
    return api.Layout(**{**LAY, **kw})


def _rotary_args(**kw):
    t = lambda h: api.RotaryTensor(P, P, 4 * h * 128, h * 128, 128, 4 * h * 128, h * 128, 128)
    a = api.RotaryArgs(t(8), t(2), t(2), P, None, P, 4, 128, 0, 0, 1.0)
    for k, v in kw.items():
        o, names = a, k.split("__")
        for n in names[:-1]:
            o = getattr(o, n)
        setattr(o, names[-1], v)
    return a


@pytest.mark.parametrize("status,n,kw", [
    (1, 0, {}), (1, -1, {}), (1, 1 << 30, {}), (1, 4, dict(positions=None)), (1, 4, dict(frequencies=None)),
    (1, 4, dict(rotary_dims=0)), (1, 4, dict(rotary_dims=129)), (1, 4, dict(rotary_dims=130)), (1, 4, dict(rotary_dims=63)),
    (1, 4, dict(q__out=None)), (1, 4, dict(v__out=None)), (1, 4, dict(q__in_=None, k__in_=None, v__in_=None)),
    (1, 4, dict(rows=P, n_rows=0)), (1, 4, dict(k__in_token=-8)), (3, 4, dict(k__in_token=132)), (3, 4, dict(q__out_head=4)),
    (3, 4, dict(q__in_=P + 8)), (3, 4, dict(v__out=P + 2)), (3, 4, dict(positions=P + 2)), (3, 4, dict(rows=P + 1)),
    (3, 4, dict(frequencies=P + 4))])
def test_rotary_refusals(status, n, kw):
    assert api.lib().loki_rotary(by(_layout()), n, by(_rotary_args(**kw)), None) == status


def test_layout_refusals_of_every_entry_point():
    L, n = api.lib(), ctypes.c_size_t()
    ev = api.EvictArgs(weights=P, klo=P, khi=P, v=P)
    for lay, status in ((None, 1), (_layout(D=64), 2), (_layout(Hq=6, Hkv=4), 1), (_layout(dtype=7), 2), (_layout(Hq=6), 2),
                        (_layout(B=0), 1), (_layout(B=8192), 2)):
        p = by(lay) if lay is not None else None
        assert L.loki_rotary(p, 4, by(_rotary_args()), None) == status
        assert L.dense_weights_workspace_bytes(p, 64, by(n)) == status
        assert L.dense_decode_weights(p, P, P, P, 64, None, None, P, P, BIG, P, None) == status
        assert L.loki_evict_workspace_bytes(p, 64, 8, by(n)) == status
        assert L.loki_evict(p, by(ev), 64, 8, 0, 0, P, BIG, None) == status
        assert L.dense_shared_workspace_bytes(p, 64, 64, by(n)) == status
        assert L.dense_decode_shared(p, P, P, P, 64, 64, P, P, 64, None, P, BIG, P, None) == status
    assert L.loki_rotary(by(_layout()), 4, None, None) == 1


def test_weights_refusals():
    L, lay, n = api.lib(), _layout(), ctypes.c_size_t()
    ok = dict(q=P, k=P, v=P, S=512, lens=None, w_in=P, w_out=P, ws=P, bytes=BIG, out=P)

    def call(**kw):
        a = {**ok, **kw}
        return L.dense_decode_weights(by(lay), a["q"], a["k"], a["v"], a["S"], a["lens"], a["w_in"], a["w_out"], a["ws"],
                                      a["bytes"], a["out"], None)

    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(w_out=None), dict(ws=None), dict(out=None), dict(S=0), dict(S=513)):
        assert call(**kw) == 1, kw
    for kw in (dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(out=P + 8), dict(ws=P + 16), dict(lens=P + 2), dict(w_out=P + 2)):
        assert call(**kw) == 3, kw
    assert L.dense_weights_workspace_bytes(by(lay), 512, by(n)) == 0
    assert call(bytes=n.value - 1) == 4
    assert L.dense_weights_workspace_bytes(by(lay), 513, by(n)) == 1
    assert L.dense_weights_workspace_bytes(by(lay), 512, None) == 1


def test_evict_refusals():
    L, lay, n = api.lib(), _layout(), ctypes.c_size_t()

    def call(S=512, budget=64, sinks=4, recent=16, ws=P, nbytes=BIG, **kw):
        a = {**dict(weights=P, klo=P, khi=P, v=P), **kw}
        return L.loki_evict(by(lay), by(api.EvictArgs(**a)), S, budget, sinks, recent, ws, nbytes, None)

    Q = 2 * P
    moved = dict(klo_out=Q, khi_out=Q, v_out=Q, S_cap_out=64)
    for kw in (dict(S=0), dict(S=513), dict(budget=0), dict(sinks=-1), dict(recent=-1), dict(sinks=32, recent=33), dict(ws=None),
               dict(weights=None), dict(klo=None), dict(khi=None), dict(v=None),
               {**moved, "klo_out": None}, {**moved, "khi_out": None}, {**moved, "v_out": None}, {**moved, "S_cap_out": 63},
               {**moved, "klo_out": P}, {**moved, "v_out": P}, {**moved, "khi_out": P}, {**moved, "weights_out": P},
               dict(weights_out=Q), dict(page_table=P, page_rows=200, pages_per_seq=4, n_pages=8),
               dict(page_table=P, page_rows=256, pages_per_seq=1, n_pages=8), dict(page_table=P, page_rows=256, pages_per_seq=2, n_pages=0)):
        assert call(**kw) == 1, kw
    for kw in (dict(klo=P + 8), dict(v=P + 2), {**moved, "v_out": Q + 4}, dict(weights=P + 2), dict(seq_lens=P + 1), dict(ws=P + 16),
               dict(out_idx=P + 2), dict(lens_out=P + 2)):
        assert call(**kw) == 3, kw
    assert call(page_table=P, page_rows=256, pages_per_seq=2, n_pages=1 << 23) == 2
    assert L.loki_evict_workspace_bytes(by(lay), 512, 64, by(n)) == 0
    assert call(nbytes=n.value - 1) == 4
    assert L.loki_evict(by(lay), None, 512, 64, 0, 0, P, BIG, None) == 1
    assert L.loki_evict_workspace_bytes(by(lay), 512, 0, by(n)) == 1


def test_shared_refusals():
    L, lay, n = api.lib(), _layout(), ctypes.c_size_t()
    ok = dict(q=P, kp=P, vp=P, rows=100, cap=128, k=P, v=P, S=512, lens=None, ws=P, bytes=BIG, out=P)

    def call(**kw):
        a = {**ok, **kw}
        return L.dense_decode_shared(by(lay), a["q"], a["kp"], a["vp"], a["rows"], a["cap"], a["k"], a["v"], a["S"], a["lens"],
                                     a["ws"], a["bytes"], a["out"], None)

    for kw in (dict(q=None), dict(kp=None), dict(vp=None), dict(k=None), dict(v=None), dict(ws=None), dict(out=None),
               dict(rows=-1), dict(rows=129), dict(S=-1), dict(S=513)):
        assert call(**kw) == 1, kw
    for kw in (dict(q=P + 8), dict(kp=P + 2), dict(vp=P + 4), dict(k=P + 8), dict(v=P + 8), dict(ws=P + 16), dict(lens=P + 2)):
        assert call(**kw) == 3, kw
    assert L.dense_shared_workspace_bytes(by(lay), 100, 512, by(n)) == 0
    assert call(bytes=n.value - 1) == 4
    assert L.dense_shared_workspace_bytes(by(lay), -1, 512, by(n)) == 1
    assert L.dense_shared_workspace_bytes(by(lay), 0, 513, by(n)) == 1


def test_sizes_past_what_the_kernels_count_are_refused():
    L, lay, n = api.lib(), _layout(), ctypes.c_size_t()
    most, ev = 1 << 30, api.EvictArgs(weights=P, klo=P, khi=P, v=P)
    assert L.loki_rotary(by(lay), (1 << 23) + 1, by(_rotary_args()), None) == 1  # two sequences
    assert L.loki_evict_workspace_bytes(by(lay), 512, most, by(n)) == 0 and n.value == 4 * most * 4 + 256
    assert L.loki_evict_workspace_bytes(by(lay), 512, most + 1, by(n)) == 1
    assert L.loki_evict(by(lay), by(ev), 512, most + 1, 0, 0, P, BIG, None) == 1
    assert L.dense_shared_workspace_bytes(by(lay), most, 512, by(n)) == 0
    assert L.dense_shared_workspace_bytes(by(lay), most + 1, 512, by(n)) == 1
    assert L.dense_decode_shared(by(lay), P, P, P, most + 1, most + 1, P, P, 512, None, P, BIG, P, None) == 1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_workspace_of_the_longest_length_serves_shorter_ones(dtype):
    for B, Hq, Hkv in ((1, 8, 8), (6, 32, 8), (16, 64, 8), (48, 32, 32)):
        lay = api.make_layout(B, Hq, Hkv, 128, 128, 16384, dtype)
        sizes = [api.dense_weights_workspace_bytes(lay, S) for S in (1, 63, 64, 65, 255, 700, 4186, 8192, 16384)]
        assert sizes == sorted(sizes)


def test_binding_refuses_what_does_not_fit():
    lay = api.make_layout(1, 1, 1, 128, 128, 64, torch.float32)
    t, pos, f = torch.zeros(1, 2, 1, 128), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(64, dtype=torch.float64)
    with pytest.raises(ValueError, match="GPU"):
        api.loki_rotary(lay, pos, f, q=t, q_out=t)
    with pytest.raises(ValueError, match="output"):
        api.loki_rotary(lay, pos, f, q=t)
    with pytest.raises(ValueError, match="positions"):
        api.loki_rotary(lay, torch.zeros(2, 2, dtype=torch.int32), f, q=t, q_out=t)
    with pytest.raises(ValueError, match="rows"):
        api.loki_rotary(lay, pos, f, q=t, q_out=t, rows=pos)
    with pytest.raises(ValueError, match="GPU"):
        api.loki_evict(lay, t, t, None, t, 64, 8, 0, 0, torch.zeros(256, dtype=torch.uint8))
    with pytest.raises(ValueError, match="GPU"):
        api.dense_decode_weights(lay, t, t, t, 64, None, None, t, t, t)
    with pytest.raises(ValueError, match="GPU"):
        api.dense_decode_shared(lay, t, t, t, 1, None, None, 0, None, t, t)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,Hq,Hkv", [(1, 8, 8), (3, 4, 1), (8, 32, 8), (44, 64, 8), (64, 64, 8), (20, 32, 32), (130, 8, 1)])
def test_shared_workspace_of_the_longest_lengths_serves_shorter_ones(B, Hq, Hkv, dtype):
    """Of the prefix and of the sequences' own rows: runs get longer in steps, and the own rows have two rules."""
    lay = api.make_layout(B, Hq, Hkv, 128, 128, 16384, dtype)
    prefixes = (0, 1, 127, 128, 129, 500, 1000, 2048, 4096, 4097, 8192, 8193, 20000, 33000, 1 << 20)
    lens = (0, 1, 63, 64, 65, 300, 301, 700, 1171, 1172, 1500, 2048, 4186, 8192, 16384)
    size = [[api.dense_shared_workspace_bytes(lay, P, S) for S in lens] for P in prefixes]
    assert all(row == sorted(row) for row in size)
    assert all(list(col) == sorted(col) for col in zip(*size))


@pytest.mark.parametrize("R,base,factor,ctx,low,high", [(128, 10000.0, 4.0, 100.0, 1.0, 32.0), (128, 10000.0, 4.0, 1e9, 1.0, 32.0),
                                                        (64, 500000.0, 8.0, 4.0, 1.0, 4.0), (64, 10000.0, 2.0, 1e-3, 1.0, 4.0),
                                                        (20, 100.0, 16.0, 1e12, 1.0, 2.0), (2, 10000.0, 4.0, 50.0, 1.0, 32.0),
                                                        (128, 10000.0, 4.0, 4096.0, 1.0, 1.0 + 1e-12)])
def test_frequencies_ramp_with_ends_outside_the_pairs(R, base, factor, ctx, low, high):
    """The mix is linear between the pairs that make `high` and `low` turns, also where there are no such pairs: contexts in which
    even the first pair makes fewer turns, or the last one more."""
    f, _ = _freqs(R, base)
    g, _ = _freqs(R, base, api.ROTARY_RAMP, factor, ctx, low, high)
    pair = lambda turns: R * math.log(ctx / (2 * math.pi * turns)) / (2 * math.log(base))
    a, b = math.floor(pair(high)), math.ceil(pair(low))
    assert a < b
    for i, (x, y) in enumerate(zip(f, g)):
        r = min(max((i - a) / (b - a), 0.0), 1.0)
        assert y == pytest.approx(x * (1 - r) + x / factor * r, rel=1e-12), i


def test_binding_refuses_caches_of_different_lengths():
    """The calls take one number of rows for all parts of a cache; what would be read or written at the wrong places is refused."""
    lay, units = api.make_layout(2, 4, 4, 128, 32, 64, torch.bfloat16), 8
    t = lambda rows, x: torch.zeros(units * rows * x, dtype=torch.bfloat16)
    w, ws = torch.zeros(units * 64), torch.zeros(1 << 20, dtype=torch.uint8)
    evict = lambda **kw: api.loki_evict(lay, w, t(64, 32), t(64, 96), t(64, 128), 64, 8, 0, 0, ws, **kw)
    ok = dict(klo_out=t(10, 32), khi_out=t(10, 96), v_out=t(10, 128), weights_out=torch.zeros(units * 10))
    for name, other in (("klo_out", t(10, 32)[:-8]), ("khi_out", t(11, 96)), ("khi_out", t(9, 96)), ("v_out", t(11, 128)), ("v_out", t(9, 128)),
                        ("weights_out", torch.zeros(units * 11)), ("weights_out", torch.zeros(units * 64))):
        with pytest.raises(ValueError, match=name):
            evict(**{**ok, name: other})
    with pytest.raises(ValueError, match="GPU"):
        evict(**ok)
    q, out = torch.zeros(2, 4, 128, dtype=torch.bfloat16), torch.zeros(2, 4, 128, dtype=torch.bfloat16)
    p = lambda rows: torch.zeros(4, rows, 128, dtype=torch.bfloat16)
    shared = lambda kp, vp: api.dense_decode_shared(lay, q, kp, vp, 8, None, None, 0, None, ws, out)
    for kp, vp in ((p(8), p(9)), (p(9), p(8)), (p(8).flatten()[:-1], p(8)), (p(8), None), (None, p(8))):
        with pytest.raises(ValueError, match="_prefix"):
            shared(kp, vp)
    with pytest.raises(ValueError, match="GPU"):
        shared(p(8), p(8))


def test_binding_refuses_rotary_outputs_without_their_inputs():
    lay = api.make_layout(1, 1, 1, 128, 128, 64, torch.float32)
    t, pos, f = torch.zeros(1, 2, 1, 128), torch.zeros(1, 2, dtype=torch.int32), torch.zeros(64, dtype=torch.float64)
    for name in "qkv":
        with pytest.raises(ValueError, match=f"{name}_out"):
            api.loki_rotary(lay, pos, f, **{name + "_out": t})


def test_rotary_refuses_to_move_rows_in_place():
    """A block that writes a token's row may not be another's that has yet to be read: in place only where it lies."""
    call = lambda n, lay=_layout(), **kw: api.lib().loki_rotary(by(lay), n, by(_rotary_args(**kw)), None)
    for kw in (dict(rows=P, n_rows=64), dict(k__out_token=512, k__out_head=1024), dict(q__out_batch=1 << 20), dict(v__out_head=256)):
        assert call(4, **kw) == 1, kw


def test_rotary_uses_no_more_of_the_layout_than_it_says():
    """The rows of a cache and its split are no concern of a call that may know of no cache: what is refused is what follows."""
    for lay in (_layout(S_cap=0), _layout(S_cap=-1, d_split=0), _layout(d_split=200)):
        assert api.lib().loki_rotary(by(lay), 4, by(_rotary_args(positions=P + 2)), None) == 3
