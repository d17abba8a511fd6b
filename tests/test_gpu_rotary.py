"""loki_rotary against the rotation in 64 bits: layouts, partial heads, strides, rows of a cache, both directions."""
import pytest
import torch

from paper_2406_02542_amd import api
from tests.attention_bound import DT

pytestmark = pytest.mark.gpu


def turned(x, positions, f, R, interleaved, inverse, scale):
    """x [B, n, H, 128] in 64 bits, and a bound of an fp32 computation before its last rounding."""
    x = x.double()
    t = positions.double()[..., None, None] * f * (-1.0 if inverse else 1.0)
    c, s = torch.cos(t) * scale, torch.sin(t) * scale
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])
    y, e = x.clone(), torch.zeros_like(x)
    first, second = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    # the angle in quarter turns, at most 1/2, is rounded to fp32 and multiplied (3 2^-24 of 0.79), the polynomials leave
    # 2^-29 and three roundings of at most 2^-24: 2^-21 for a cosine; two products and a sum: 3 2^-24
    size = abs(scale) * (a.abs() + b.abs()) * (2.0 ** -21 + 3 * 2.0 ** -24)
    e[..., first], e[..., second] = size, size
    return y, e


def check(got, ref, e, dtype, R):
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    over = (got.double() - ref).abs() - (e + step * (ref.abs() + e))
    over[..., R:] = (got.double() - ref)[..., R:].abs()  # the other columns are copied
    assert float(over.max()) <= 0, float(over.max())


def inputs(B, n, Hq, Hkv, dtype, R, far, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(1000 * B + 10 * n + R + seed)
    q, k, v = (torch.randn((B, n, h, 128), generator=gen, device="cuda").to(DT[dtype]) for h in (Hq, Hkv, Hkv))
    pos = torch.randint(0, far + 1, (B, n), generator=gen, device="cuda", dtype=torch.int32)
    f, _ = api.loki_rotary_frequencies(R, 10000.0)
    return q, k, v, pos, f


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,n,Hq,Hkv,R,far,inverse,scale", [
    (1, 1, 1, 1, 128, 0, False, 1.0), (1, 1, 8, 8, 128, 5, False, 1.0), (2, 1, 32, 8, 64, 1 << 20, False, 1.0),
    (3, 7, 8, 2, 2, 100, True, 1.0), (1, 33, 24, 24, 20, 4000, False, 1.25), (5, 3, 4, 1, 126, 99999, True, 0.5),
    (1, 1500, 8, 4, 96, 131072, False, 1.0), (64, 1, 64, 8, 16, 70, False, 1.0), (2, 1031, 16, 2, 34, 2000, False, 1.1)])
def test_against_64_bits(B, n, Hq, Hkv, R, far, inverse, scale, interleaved, dtype):
    print("case", B, n, Hq, Hkv, R, far, inverse, scale, interleaved, dtype, flush=True)
    q, k, v, pos, f = inputs(B, n, Hq, Hkv, dtype, R, far)
    lay = api.make_layout(B, Hq, Hkv, 128, 128, 64, DT[dtype])
    q_out, k_out, v_out = torch.full_like(q, 9.0), *(torch.full((B, Hkv, n, 128), 9.0, dtype=DT[dtype], device="cuda") for _ in "kv")
    api.loki_rotary(lay, pos, f, q=q, q_out=q_out, k=k, k_out=k_out, v=v, v_out=v_out, interleaved=interleaved, inverse=inverse, scale=scale)
    torch.cuda.synchronize()
    for x, got in ((q, q_out), (k, k_out.transpose(1, 2))):
        ref, e = turned(x, pos, f, R, interleaved, inverse, scale)
        check(got, ref, e, dtype, R)
    assert torch.equal(v_out, v.transpose(1, 2))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("R", [128, 20])
def test_in_place_strided_and_one_tensor_at_a_time(R, interleaved, dtype):
    """Slices of one projection's output, turned where they are; only the tensors given are touched."""
    B, n, Hq, Hkv = 3, 5, 8, 2
    gen = torch.Generator(device="cuda").manual_seed(5)
    qkv = torch.randn((B, n, (Hq + 2 * Hkv + 1) * 128), generator=gen, device="cuda").to(DT[dtype])
    old = qkv.clone()
    part = lambda t, a, h: t[..., a * 128:(a + h) * 128].unflatten(-1, (h, 128))
    pos = torch.arange(B * n, dtype=torch.int32, device="cuda").view(B, n) * 77
    f, _ = api.loki_rotary_frequencies(R, 10000.0)
    lay = api.make_layout(B, Hq, Hkv, 128, 128, 64, DT[dtype])
    q, k = part(qkv, 0, Hq), part(qkv, Hq, Hkv)
    api.loki_rotary(lay, pos, f, q=q, q_out=q, interleaved=interleaved)
    api.loki_rotary(lay, pos, f, k=k, k_out=k, token_major=True, interleaved=interleaved)
    torch.cuda.synchronize()
    for a, h in ((0, Hq), (Hq, Hkv)):
        ref, e = turned(part(old, a, h), pos, f, R, interleaved, False, 1.0)
        check(part(qkv, a, h), ref, e, dtype, R)
    assert torch.equal(qkv[..., (Hq + Hkv) * 128:], old[..., (Hq + Hkv) * 128:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_into_the_rows_of_a_cache(dtype):
    """Padded tokens (rows outside the cache) are not written, nor any other row; a cache may be a slice."""
    B, n, Hq, Hkv, cap = 2, 6, 4, 2, 40
    q, k, v, pos, f = inputs(B, n, Hq, Hkv, dtype, 128, 3000)
    rows = torch.tensor([[3, 4, 5, 6, -1, 40], [39, 0, 17, 2147483647, -2147483648, 1]], dtype=torch.int32, device="cuda")
    both = torch.full((B, Hkv, 2, cap, 128), 7.0, dtype=DT[dtype], device="cuda")
    kc, vc = both[:, :, 0], both[:, :, 1]
    lay = api.make_layout(B, Hq, Hkv, 128, 128, cap, DT[dtype])
    q_out = torch.empty_like(q)
    api.loki_rotary(lay, pos, f, q=q, q_out=q_out, k=k, k_out=kc, v=v, v_out=vc, rows=rows)
    torch.cuda.synchronize()
    ref, e = turned(q, pos, f, 128, False, False, 1.0)
    check(q_out, ref, e, dtype, 128)
    ref, e = turned(k, pos, f, 128, False, False, 1.0)
    written = set()
    for b in range(B):
        for j in range(n):
            r = int(rows[b, j])
            if 0 <= r < cap:
                written.add((b, r))
                check(kc[b, :, r], ref[b, j], e[b, j], dtype, 128)
                assert torch.equal(vc[b, :, r], v[b, j])
    for b in range(B):
        rest = [r for r in range(cap) if (b, r) not in written]
        assert bool((both[b, :, :, rest] == 7.0).all())


def test_inverse_is_the_gradient_and_undoes():
    """<g, rotate(x)> = <rotate_inverse(g), x>, also by differences; with scale 1 the inverse undoes the rotation."""
    B, n, H, R, scale = 2, 9, 4, 64, 1.3
    x, g, _, pos, f = inputs(B, n, H, H, "f32", R, 50000)
    lay = api.make_layout(B, H, H, 128, 128, 64, torch.float32)

    def turn(t, inverse, s):
        y = torch.empty_like(t)
        api.loki_rotary(lay, pos, f, q=t, q_out=y, inverse=inverse, scale=s)
        return y

    y, dx = turn(x, False, scale), turn(g, True, scale)
    a, b = float((g.double() * y.double()).sum()), float((dx.double() * x.double()).sum())
    size = float((g.double() * y.double()).abs().sum())
    assert abs(a - b) <= 2 * size * 2.0 ** -20
    d = torch.randn_like(x)
    moved = turn(x + d, False, scale).double() - y.double()  # linear: the difference is exact but for roundings
    assert abs(float((g.double() * moved).sum()) - float((dx.double() * d.double()).sum())) <= 8 * float(g.double().abs().sum()) * 4 * 2.0 ** -20
    back = turn(turn(x, False, 1.0), True, 1.0)
    assert float((back - x).abs().max()) <= float(x.abs().max()) * 2 * 2.0 ** -19


def test_input_broadcast_over_heads():
    """One key for all heads, a stride of zero."""
    B, n, H = 2, 5, 6
    one, pos = torch.randn((B, n, 1, 128), device="cuda").bfloat16(), torch.arange(B * n, dtype=torch.int32, device="cuda").view(B, n)
    f, _ = api.loki_rotary_frequencies(128, 10000.0)
    lay = api.make_layout(B, H, H, 128, 128, 64, torch.bfloat16)
    k, k_out = one.expand(B, n, H, 128), torch.empty((B, H, n, 128), dtype=torch.bfloat16, device="cuda")
    api.loki_rotary(lay, pos, f, k=k, k_out=k_out)
    torch.cuda.synchronize()
    ref, e = turned(k, pos, f, 128, False, False, 1.0)
    check(k_out.transpose(1, 2), ref, e, "bf16", 128)


def test_stream_and_graph():
    """On a stream of its own, captured once and replayed with new positions between."""
    B, n, Hq, Hkv = 2, 1, 8, 2
    q, k, v, pos, f = inputs(B, n, Hq, Hkv, "bf16", 128, 1000)
    lay = api.make_layout(B, Hq, Hkv, 128, 128, 64, torch.bfloat16)
    q_out, k_out, v_out = torch.empty_like(q), *(torch.empty((B, Hkv, n, 128), dtype=q.dtype, device="cuda") for _ in "kv")

    def call():
        api.loki_rotary(lay, pos, f, q=q, q_out=q_out, k=k, k_out=k_out, v=v, v_out=v_out)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(4):
        pos.add_(1)
        graph.replay()
        torch.cuda.synchronize()
        a, b = q_out.clone(), k_out.clone()
        call()
        torch.cuda.synchronize()
        assert torch.equal(a, q_out) and torch.equal(b, k_out)
        ref, e = turned(q, pos, f, 128, False, False, 1.0)
        check(q_out, ref, e, "bf16", 128)
