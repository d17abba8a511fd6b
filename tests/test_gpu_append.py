"""loki_append and loki_read_rows: rotated rows into contiguous and paged caches, in the storage type and in 4 bits, and back."""
import pytest
import torch

from paper_2406_02542_amd import api
from tests.attention_bound import DT, worst
from tests.whole_cache import Case, make_table, quantise64, reference, unpack, values64

pytestmark = pytest.mark.gpu


def turned(x, positions, f, R, interleaved, inverse, scale):
    """x [B, n, H, 128] in 64 bits, and a bound of an fp32 computation before its last rounding: cosines and sines rounded once and
    times the scale (2^-23), each product and the sum rounded (2 2^-24 of their magnitudes)."""
    x = x.double()
    if not R:
        return x, torch.zeros_like(x)
    t = positions.double()[..., None, None] * f * (-1.0 if inverse else 1.0)
    c, s = torch.cos(t) * scale, torch.sin(t) * scale
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])
    y, e = x.clone(), torch.zeros_like(x)
    first, second = (slice(0, R, 2), slice(1, R, 2)) if interleaved else (slice(0, R // 2), slice(R // 2, R))
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    size = abs(scale) * (a.abs() + b.abs()) * (4 * 2.0 ** -24)
    e[..., first], e[..., second] = size, size
    return y, e


def within(got, ref, e, dtype):
    step = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    return bool(((got.double() - ref).abs() <= e + step * (ref.abs() + e)).all())


class Tokens:
    def __init__(self, B, n, Hq, Hkv, dtype, R, far, seed=0, fused=False):
        gen = torch.Generator(device="cuda").manual_seed(1000 * B + 10 * n + R + seed)
        dt = DT[dtype]
        if fused:  # slices of one projection's output
            x = torch.randn((B, n, (Hq + 2 * Hkv) * 128 + 8), generator=gen, device="cuda").to(dt)
            part = lambda a, h: x[..., a * 128:(a + h) * 128].unflatten(-1, (h, 128))
            self.q, self.k, self.v = part(0, Hq), part(Hq, Hkv), part(Hq + Hkv, Hkv)
        else:
            self.q, self.k, self.v = (torch.randn((B, n, h, 128), generator=gen, device="cuda").to(dt) for h in (Hq, Hkv, Hkv))
        self.positions = torch.randint(0, far + 1, (B, n), generator=gen, device="cuda", dtype=torch.int32)
        self.f = api.loki_rotary_frequencies(R, 10000.0)[0] if R else None
        self.rot = dict(positions=self.positions, frequencies=self.f) if R else {}


def unpaged(t, table, S):
    return t if table is None else t[table.long()].transpose(1, 2).flatten(2, 3)[:, :, :S]


@pytest.mark.parametrize("bits", [0, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,n,Hq,Hkv,S,page_rows,R,far,inverse,scale,fused", [
    (1, 1, 1, 1, 1, 0, 128, 0, False, 1.0, False), (1, 1, 32, 32, 300, 256, 128, 5000, False, 1.0, False), (3, 7, 8, 2, 40, 16, 2, 100, True, 1.0, True),
    (64, 1, 64, 8, 90, 32, 64, 1 << 20, False, 1.0, True), (2, 33, 24, 24, 70, 0, 20, 4000, False, 1.25, True), (5, 3, 4, 1, 30, 16, 126, 99999, True, 0.5, False),
    (2, 600, 8, 4, 700, 64, 96, 131072, False, 1.0, True), (1, 1100, 2, 1, 1100, 0, 16, 70, False, 1.0, False), (2, 9, 16, 2, 50, 16, 0, 0, False, 1.0, True)])
def test_against_64_bits(B, n, Hq, Hkv, S, page_rows, R, far, inverse, scale, fused, interleaved, dtype, bits):
    print("case", B, n, Hq, Hkv, S, page_rows, R, far, inverse, scale, interleaved, dtype, bits, flush=True)
    x = Tokens(B, n, Hq, Hkv, dtype, R, far, fused=fused)
    gen = torch.Generator(device="cuda").manual_seed(7)
    lay = api.make_layout(B, Hq, Hkv, 128, 128, S, DT[dtype])
    table, n_pages = make_table(B, S, page_rows, gen) if page_rows else (None, 0)
    cache = api.alloc_whole_cache(lay, bits == 4, table, page_rows, n_pages)
    for t in cache.tensors[:4]:
        if t is not None:
            t.fill_(7)
    # rows in no order; some tokens are padding, some sequences' last pages are not there yet
    rows = torch.stack([torch.randperm(S, generator=gen, device="cuda")[:n] for _ in range(B)]).int()
    rows[torch.rand((B, n), generator=gen, device="cuda") < (0.2 if n > 1 else 0.0)] = -1
    rows[B - 1, n - 1] = S if n > 2 else rows[B - 1, n - 1]
    there = (rows >= 0) & (rows < S)
    if page_rows and B > 1:
        gone = (S - 1) // page_rows
        table[1, gone] = -1
        there[1] &= rows[1] // page_rows != gone
    q_out = torch.full((B, n, Hq, 128), 9.0, dtype=DT[dtype], device="cuda")
    api.loki_append(lay, cache, rows, x.k, x.v, q=x.q, q_out=q_out, interleaved=interleaved, inverse=inverse, scale=scale, **x.rot)
    back = [torch.full((B, Hkv, n, 128), 9.0, dtype=DT[dtype], device="cuda") for _ in "kv"]
    api.loki_read_rows(lay, cache, rows, *back)
    torch.cuda.synchronize()
    assert within(q_out, *turned(x.q, x.positions, x.f, R, interleaved, inverse, scale), dtype)
    k, e = turned(x.k, x.positions, x.f, R, interleaved, inverse, scale)
    at = there[:, None].expand(B, Hkv, n)
    assert all(bool((y[~at] == 9.0).all()) for y in back)
    if page_rows and B > 1:
        table[1, gone] = 0  # (to look at the whole pool below)
    if not bits:
        assert within(back[0][at], k.transpose(1, 2)[at], e.transpose(1, 2)[at], dtype)
        assert torch.equal(back[1][at], x.v.transpose(1, 2)[at])
    else:
        for t, (y, off) in enumerate(((k, e), (x.v.double(), torch.zeros_like(e)))):
            y, off = y.transpose(1, 2)[at], off.transpose(1, 2)[at]
            # lowest is off by half a step of fp16 (2^-11 of it) and what the value was off, step by 2^-11; a code by half a step,
            # and past 15 by what the smaller step leaves of the range
            lo, hi = y.unflatten(-1, (4, 32)).amin(-1, True), y.unflatten(-1, (4, 32)).amax(-1, True)
            step = (hi - lo) / 15
            near = step * (0.5 + 15 * 2.0 ** -11 + 2.0 ** -10) + lo.abs() * 2.0 ** -10 + 2.0 ** -24
            bound = near.expand(*near.shape[:-1], 32).flatten(-2) + 2 * off
            assert within(back[t][at], y, bound, dtype)
    # nothing else was written
    new = 0
    for b in range(B):
        new += int(there[b].sum())
    for t in cache.tensors[:4]:
        if t is not None:
            changed = (t != 7).flatten(3).any(-1)
            assert int(changed.sum()) <= new * Hkv


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_codes_and_scales_are_those_of_the_definition(dtype):
    """Without a rotation the row is exact, and so are its codes; rows of one value, of two far apart, tiny, huge and half-way ones."""
    B, H, n = 1, 2, 64
    dt = DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(1)
    k = torch.randn((B, n, H, 128), generator=gen, device="cuda")
    k[0, 0] = 0.0
    k[0, 1] = -3.25
    k[0, 2, :, 5] = 1000.0
    k[0, 3] *= 1e-7
    k[0, 4] *= 1e-3
    k[0, 5] = k[0, 5] * 1e4
    k[0, 6] = 0.25 * torch.arange(128, device="cuda") % 7.75  # values half-way between two codes
    k[0, 7] = torch.arange(128, device="cuda") % 31 * 0.5
    k[0, 8, :, ::2] = 60000.0
    k = k.to(dt)
    v = k.flip(1).contiguous()
    lay = api.make_layout(B, H, H, 128, 128, n, dt)
    cache = api.alloc_whole_cache(lay, four_bits=True)
    rows = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    api.loki_append(lay, cache, rows, k, v)
    back = [torch.empty((B, H, n, 128), dtype=dt, device="cuda") for _ in "kv"]
    api.loki_read_rows(lay, cache, rows, *back)
    torch.cuda.synchronize()
    for i, x in enumerate((k, v)):
        codes, scales = quantise64(x.transpose(1, 2))
        # the range's fifteenth is rounded to fp32 in front of fp16, and a quotient to fp32 in front of its code: where that
        # ends half-way they may be one off; everywhere else they are the same
        assert float((cache.tensors[2 + i] != scales).float().mean()) <= 1e-3
        same = (cache.tensors[2 + i] == scales).all(-1).repeat_interleave(32, -1)
        got = unpack(cache.tensors[i])
        assert float((got != codes)[same].float().mean()) <= 1e-5
        assert torch.equal(back[i], values64(got, cache.tensors[2 + i]).to(dt)) or \
            float((back[i].double() - values64(got, cache.tensors[2 + i])).abs().max()) <= 2.0 ** -8 * float(back[i].abs().max())


@pytest.mark.parametrize("bits", [0, 4])
@pytest.mark.parametrize("dtype,B,n,Hq,Hkv,R,interleaved", [("bf16", 6, 1300, 32, 8, 128, False), ("f32", 3, 1100, 32, 8, 64, True), ("bf16", 7, 1030, 32, 8, 20, False),
                                                               ("bf16", 6, 1100, 32, 8, 96, False), ("bf16", 9, 1000, 32, 8, 16, False), ("f32", 3, 1100, 32, 8, 48, False)])
def test_large_appends(dtype, B, n, Hq, Hkv, R, interleaved, bits):
    """Enough for rows past the caches."""
    x = Tokens(B, n, Hq, Hkv, dtype, R, 100000)
    S = n + 30
    gen = torch.Generator(device="cuda").manual_seed(8)
    lay = api.make_layout(B, Hq, Hkv, 128, 128, S, DT[dtype])
    table, n_pages = make_table(B, S, 64, gen)
    cache = api.alloc_whole_cache(lay, bits == 4, table, 64, n_pages)
    rows = (17 + torch.arange(n, device="cuda", dtype=torch.int32))[None].repeat(B, 1)
    rows[1, n // 2:] = -1
    q_out = torch.empty_like(x.q)
    api.loki_append(lay, cache, rows, x.k, x.v, q=x.q, q_out=q_out, interleaved=interleaved, **x.rot)
    k, e = turned(x.k, x.positions, x.f, R, interleaved, False, 1.0)
    assert within(q_out, *turned(x.q, x.positions, x.f, R, interleaved, False, 1.0), dtype)
    held = [None if t is None else unpaged(t, table, S) for t in cache.tensors[:4]]
    for b in range(B):
        m = n // 2 if b == 1 else n
        at = slice(17, 17 + m)
        if not bits:
            assert within(held[0][b, :, at], k[b, :m].transpose(0, 1), e[b, :m].transpose(0, 1), dtype)
            assert torch.equal(held[1][b, :, at], x.v[b, :m].transpose(0, 1))
        else:
            for t, y, off in ((0, k, e), (1, x.v.double(), torch.zeros_like(e))):
                y, off = y[b, :m].transpose(0, 1), off[b, :m].transpose(0, 1)
                got = values64(unpack(held[t][b, :, at]), held[2 + t][b, :, at])
                lo, hi = y.unflatten(-1, (4, 32)).amin(-1, True), y.unflatten(-1, (4, 32)).amax(-1, True)
                near = (hi - lo) / 15 * (0.5 + 15 * 2.0 ** -11 + 2.0 ** -10) + lo.abs() * 2.0 ** -10 + 2.0 ** -24  # (as above)
                assert bool(((got - y).abs() <= near.expand(*near.shape[:-1], 32).flatten(-2) + 2 * off).all())
    assert bool((held[0][1, :, 17 + n // 2:] == 0).all()) and bool((held[1][:, :, :17] == 0).all())


def test_reads_of_one_tensor_and_of_rows_that_are_not_there():
    c = Case(2, 4, 2, 50, "bf16", 16)
    rows = torch.tensor([[49, 0, 0, 50], [-1, 17, 2 ** 31 - 1, -2 ** 31]], dtype=torch.int32, device="cuda")
    out = torch.full((2, 2, 4, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    api.loki_read_rows(c.lay, c.cache, rows, k_out=out)
    v_out = torch.full_like(out, 9.0)
    api.loki_read_rows(c.lay, c.cache, rows, v_out=v_out)
    for got, x in ((out, c.k), (v_out, c.v)):
        for b, j, r in ((0, 0, 49), (0, 1, 0), (0, 2, 0), (1, 1, 17)):
            assert torch.equal(got[b, :, j], x[b, :, r])
        for b, j in ((0, 3), (1, 0), (1, 2), (1, 3)):
            assert bool((got[b, :, j] == 9.0).all())


@pytest.mark.parametrize("bits", [0, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_prompt_and_then_token_by_token(dtype, bits):
    """As they are used together: chunks of a prompt appended and attended, then tokens one at a time, through a window with sinks, on
    pages; eager and as a captured step whose inputs change."""
    B, Hq, Hkv, S, window, sinks, chunk, page_rows = 2, 8, 2, 400, 64, 4, 60, 16
    gen = torch.Generator(device="cuda").manual_seed(9)
    dt = DT[dtype]
    lay = api.make_layout(B, Hq, Hkv, 128, 128, S, dt)
    table, n_pages = make_table(B, S, page_rows, gen)
    cache = api.alloc_whole_cache(lay, bits == 4, table, page_rows, n_pages)
    f, _ = api.loki_rotary_frequencies(128, 10000.0)
    lens = torch.tensor([chunk, chunk - 13])
    start = torch.zeros(B, dtype=torch.long)

    def inputs(m, real):
        j = torch.arange(m)[None]
        pos = start[:, None] + j
        rows = torch.where(j < real[:, None], pos, -1).int().cuda()
        sees = torch.where(j < real[:, None], pos + 1, 0).int().cuda()
        x = [torch.randn((B, m, h, 128), generator=gen, device="cuda").to(dt) for h in (Hq, Hkv, Hkv)]
        return x, pos.int().cuda(), rows, sees

    def step(x, pos, rows, sees, q_out, out, ws):
        m = pos.shape[1]
        api.loki_append(lay, cache, rows, x[1], x[2], positions=pos, frequencies=f, q=x[0], q_out=q_out)
        api.dense_decode_cache(lay, cache, q_out, S, ws, out, seq_lens=sees, queries_per_seq=m, window=window, sinks=sinks)

    def held():
        """What the cache holds, in 64 bits."""
        t = [None if t is None else unpaged(t, table, S) for t in cache.tensors[:4]]
        if not bits:
            return t[0], t[1], None
        return values64(unpack(t[0]), t[2]), values64(unpack(t[1]), t[3]), t[2:]

    graph = static = None
    for turn in range(12):
        m, real = (chunk, lens) if turn < 2 else (1, torch.ones(2, dtype=torch.long))
        x, pos, rows, sees = inputs(m, real)
        need = api.dense_cache_workspace_bytes(lay, cache, S, m, window, sinks)
        if turn >= 6:  # from here on as one graph
            if graph is None:
                static = [[t.clone() for t in x], pos.clone(), rows.clone(), sees.clone(), torch.empty_like(x[0]), torch.empty_like(x[0]),
                          torch.empty(need, dtype=torch.uint8, device="cuda")]
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph):
                    step(*static)
            for a, b in zip(static[0] + static[1:4], x + [pos, rows, sees]):
                a.copy_(b)
            graph.replay()
            q_out, out = static[4], static[5]
        else:
            q_out, out = torch.empty_like(x[0]), torch.empty_like(x[0])
            step(x, pos, rows, sees, q_out, out, torch.empty(need, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        assert within(q_out, *turned(x[0], pos, f, 128, False, False, 1.0), dtype)
        back = [torch.zeros((B, Hkv, m, 128), dtype=dt, device="cuda") for _ in "kv"]
        api.loki_read_rows(lay, cache, rows, *back)
        k, e = turned(x[1], pos, f, 128, False, False, 1.0)
        if not bits:
            at = (rows >= 0)[:, None].expand(B, Hkv, m)
            assert within(back[0][at], k.transpose(1, 2)[at], e.transpose(1, 2)[at], dtype) and torch.equal(back[1][at], x[2].transpose(1, 2)[at])
        k, v, scales = held()
        ref, bound = reference(q_out, k, v, sees.cpu(), window, sinks, scales)
        assert worst(out, ref, bound, dtype) <= 0, turn
        start += real


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_groups_with_a_value_that_is_no_number(dtype):
    """In 4 bits their step and lowest are NaN; the other groups, rows and heads are as without."""
    B, H, n = 2, 3, 37
    dt = DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn((B, n, H, 128), generator=gen, device="cuda").to(dt) for _ in "kv")
    spoilt = torch.zeros((B, H, n, 4), dtype=torch.bool, device="cuda")
    for b, j, h, col in ((0, 0, 0, 0), (0, 5, 2, 31), (1, 36, 1, 32), (1, 20, 0, 127), (1, 20, 0, 70)):
        spoilt[b, h, j, col // 32] = True
        v[b, j, h, col] = float("nan")
    lay = api.make_layout(B, H, H, 128, 128, n, dt)
    rows = torch.arange(n, dtype=torch.int32, device="cuda").repeat(B, 1)
    held = []
    for x in (v, torch.nan_to_num(v, nan=0.0)):
        cache = api.alloc_whole_cache(lay, four_bits=True)
        api.loki_append(lay, cache, rows, k, x)
        held.append(cache.tensors)
    torch.cuda.synchronize()
    assert torch.equal(held[0][0], held[1][0]) and torch.equal(held[0][2], held[1][2])
    assert bool(torch.isnan(held[0][3][spoilt]).all())
    assert torch.equal(held[0][3][~spoilt], held[1][3][~spoilt])
    clean = (~spoilt).repeat_interleave(32, -1)
    assert torch.equal(unpack(held[0][1])[clean], unpack(held[1][1])[clean])


@pytest.mark.parametrize("bits", [0, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved,R", [(False, 128), (True, 96), (False, 20)])
def test_queries_turned_in_place(interleaved, R, dtype, bits):
    B, n, Hq, H = 2, 300, 8, 2
    t = Tokens(B, n, Hq, H, dtype, R, 5000)
    lay = api.make_layout(B, Hq, H, 128, 128, n, DT[dtype])
    rows = torch.arange(n, dtype=torch.int32, device="cuda").repeat(B, 1)
    q_out, q = torch.empty_like(t.q), t.q.clone()
    caches = [api.alloc_whole_cache(lay, four_bits=bits == 4) for _ in range(2)]
    api.loki_append(lay, caches[0], rows, t.k, t.v, q=t.q, q_out=q_out, interleaved=interleaved, **t.rot)
    api.loki_append(lay, caches[1], rows, t.k, t.v, q=q, q_out=q, interleaved=interleaved, **t.rot)
    torch.cuda.synchronize()
    assert torch.equal(q, q_out)
    for x, y in zip(caches[0].tensors[:4], caches[1].tensors[:4]):
        assert x is None or torch.equal(x, y)


@pytest.mark.parametrize("bits", [0, 4])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 40])
def test_captured_with_other_rows_positions_and_pages_at_each_replay(n, dtype, bits):
    """Appends and reads of a graph that is replayed, on a stream of their own, give what the same calls give one by one."""
    B, Hq, H, S = 3, 8, 2, 200
    gen = torch.Generator(device="cuda").manual_seed(n)
    lay = api.make_layout(B, Hq, H, 128, 128, S, DT[dtype])
    table, n_pages = make_table(B, S, 16, gen)
    t = Tokens(B, n, Hq, H, dtype, 64, 3000)
    rows = torch.zeros((B, n), dtype=torch.int32, device="cuda")

    def state():
        cache = api.alloc_whole_cache(lay, bits == 4, table, 16, n_pages)
        return cache, torch.zeros_like(t.q), [torch.zeros((B, H, n, 128), dtype=DT[dtype], device="cuda") for _ in "kv"]

    def call(s, stream=None):
        api.loki_append(lay, s[0], rows, t.k, t.v, q=t.q, q_out=s[1], stream=stream, **t.rot)
        api.loki_read_rows(lay, s[0], rows, *s[2], stream=stream)

    mine, other = state(), state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(mine, side)
    torch.cuda.synchronize()
    for i in range(4):
        for b in range(B):
            rows[b] = torch.randperm(S, generator=gen, device="cuda")[:n].int()
        rows[i % B, n // 2:] = -1
        t.positions.copy_(torch.randint(0, 100000, (B, n), generator=gen, device="cuda", dtype=torch.int32))
        t.k.normal_(generator=gen)
        table.copy_(table.flatten()[torch.randperm(table.numel(), generator=gen, device="cuda")].view_as(table))
        graph.replay()
        torch.cuda.synchronize()
        call(other)
        torch.cuda.synchronize()
        assert torch.equal(mine[1], other[1])
        for x, y in zip((*mine[0].tensors[:4], *mine[2]), (*other[0].tensors[:4], *other[2])):
            assert x is None or torch.equal(x, y)


def test_codes_next_to_their_borders():
    """Values half-way between two codes, and the fp32 numbers next to those: the codes are those of 64 bits, whatever the lowest value is."""
    n, H = 512, 4
    gen = torch.Generator(device="cuda").manual_seed(3)
    lay = api.make_layout(1, H, H, 128, 128, n, torch.float32)
    rows = torch.arange(n, dtype=torch.int32, device="cuda")[None]
    k = torch.randn((1, n, H, 128), generator=gen, device="cuda") * torch.exp(3 * torch.randn((1, n, H, 1), generator=gen, device="cuda"))
    k += 20 * torch.randn((1, n, H, 1), generator=gen, device="cuda") * (torch.rand((1, n, H, 1), generator=gen, device="cuda") < 0.3)
    cache = api.alloc_whole_cache(lay, four_bits=True)
    api.loki_append(lay, cache, rows, k, k)
    torch.cuda.synchronize()
    scales = cache.tensors[2].double().transpose(1, 2)  # [1, n, H, 4, 2]
    step, low = scales[..., :1], scales[..., 1:]
    g = k.unflatten(-1, (4, 32)).clone()
    lo, hi = g.amin(-1, True), g.amax(-1, True)
    at = torch.randint(0, 15, g.shape, generator=gen, device="cuda") + 0.5
    near = (low + at * step).float()
    for _ in range(3):  # up to three fp32 numbers off, in either direction
        move = torch.randint(-1, 2, g.shape, generator=gen, device="cuda")
        near = torch.where(move == 0, near, torch.nextafter(near, torch.where(move > 0, 1e30, -1e30).float()))
    keep = (g == lo) | (g == hi)  # the group's lowest and largest stay, and with them its scales
    g = torch.where(keep, g, torch.minimum(torch.maximum(near, lo), hi))
    k2 = g.flatten(-2).contiguous()
    api.loki_append(lay, cache, rows, k2, k2)
    torch.cuda.synchronize()
    assert torch.equal(cache.tensors[2].double().transpose(1, 2), scales)
    want = torch.where(step > 0, torch.round((g.double() - low) / torch.where(step > 0, step, 1.0)), 0.0).clamp(0, 15).long().flatten(-2)
    for t in cache.tensors[:2]:
        assert torch.equal(unpack(t).transpose(1, 2), want)
