"""dense_decode_cache against attention in 64 bits: windows, sinks, pages, several tokens, both storage types and 4 bits."""
import pytest
import torch

from paper_2406_02542_amd import api
from tests.attention_bound import worst
from tests.whole_cache import Case, reference

pytestmark = pytest.mark.gpu
KINDS = [("bf16", 0), ("f32", 0), ("bf16", 4), ("f32", 4)]


def last_tokens(totals, m):
    """seq_lens of the last m tokens of sequences of so many rows."""
    t = torch.tensor(totals)[:, None] - (m - 1) + torch.arange(m)[None]
    return t.clamp(min=0).int().cuda()


def check(c, q, lens, S_max, window, sinks, dtype, out=None):
    out = c.attend(q, lens, S_max, window, sinks) if out is None else out
    torch.cuda.synchronize()
    ref, bound = reference(q, c.k, c.v, lens.cpu(), window, sinks, c.scales)
    assert bool(torch.isfinite(out).all())
    excess = worst(out, ref, bound, dtype)
    assert excess <= 0, excess
    return out


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("page_rows", [0, 16, 256])
@pytest.mark.parametrize("B,Hq,Hkv,S,window,sinks", [
    (1, 1, 1, 1, 0, 0), (1, 8, 8, 33, 0, 0), (2, 8, 4, 300, 0, 7), (3, 32, 8, 517, 100, 4), (2, 8, 1, 1031, 1, 0), (2, 4, 4, 700, 16, 1),
    (1, 16, 2, 2500, 333, 40), (5, 2, 2, 64, 4096, 3), (1, 4, 1, 5000, 2000, 1999)])
def test_one_token(B, Hq, Hkv, S, window, sinks, page_rows, dtype, bits):
    print("case", B, Hq, Hkv, S, window, sinks, page_rows, dtype, bits, flush=True)
    c = Case(B, Hq, Hkv, S, dtype, page_rows, bits)
    totals = [S, 0, max(1, S // 3), 1, S // 2][:B]
    check(c, c.queries(1), last_tokens(totals, 1), S, window, sinks, dtype)


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("B,m,Hq,Hkv,S,window,sinks,page_rows", [
    (2, 2, 8, 8, 100, 0, 0, 0), (3, 3, 8, 4, 450, 64, 4, 16), (2, 5, 32, 8, 300, 0, 0, 256), (1, 17, 8, 2, 900, 130, 1, 64), (2, 33, 8, 1, 257, 40, 9, 0),
    (1, 64, 4, 4, 64, 0, 0, 0), (2, 70, 16, 4, 600, 200, 64, 256), (1, 150, 8, 1, 1100, 300, 4, 16), (1, 300, 2, 2, 310, 33, 2, 0), (1, 1, 8, 1, 9000, 0, 0, 256)])
def test_several_tokens(B, m, Hq, Hkv, S, window, sinks, page_rows, dtype, bits):
    """The last tokens of every sequence, those of the first less than there are tokens (the front ones see nothing)."""
    print("case", B, m, Hq, Hkv, S, window, sinks, page_rows, dtype, bits, flush=True)
    c = Case(B, Hq, Hkv, S, dtype, page_rows, bits)
    check(c, c.queries(m), last_tokens([max(1, m - 2), S, S // 2][-B:], m), S, window, sinks, dtype)


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("m,G", [(1, 4), (3, 2), (40, 8), (130, 4)])
def test_padded_tokens_and_rows_that_no_token_sees(m, G, dtype, bits):
    """A sequence of which the last tokens are padding, one without any; rows before the window and behind the end hold NaN."""
    B, Hkv, S, window, sinks = 3, 2, 700, 90, 5
    for page_rows in (0, 32):
        c = Case(B, G * Hkv, Hkv, S, dtype, page_rows, bits, seed=m)
        lens = last_tokens([S - 20, 0, 400], m)
        lens[0, m - m // 3:] = 0
        q = c.queries(m)
        for b in range(B):
            there = lens[b][lens[b] > 0]
            lo, hi = (max(0, int(there.min()) - window), int(there.max())) if len(there) else (0, 0)
            c.spoil(b, [s for s in range(S) if s >= hi or (s >= sinks and s < lo)] if hi else range(S))
        out = c.attend(q, lens, S, window, sinks)
        k, v = c.k.double().clone(), c.v.double().clone()
        ref, bound = reference(q, k, v, lens.cpu(), window, sinks, c.scales)
        torch.cuda.synchronize()
        assert bool((out[lens == 0] == 0).all())
        assert worst(out, ref, bound, dtype) <= 0


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("page_rows", [16, 256])
def test_entries_of_pages_that_hold_no_seen_row_may_be_any(page_rows, dtype, bits):
    B, S, window, sinks, m = 2, 3000, 260, 4, 2
    c = Case(B, 8, 2, S, dtype, page_rows, bits)
    lens = last_tokens([S - 700, 1500], m)
    q = c.queries(m)
    whole = c.attend(q, lens, S, window, sinks)
    for b in range(B):
        lo, hi = int(lens[b].min()) - window, int(lens[b].max())
        for p in range(c.table.shape[1]):
            if p > (hi - 1) // page_rows or (p < lo // page_rows and p > (sinks - 1) // page_rows):
                c.table[b, p] = [-1, 2 ** 31 - 1, -2 ** 31, 0][p % 4]
    assert torch.equal(c.attend(q, lens, S, window, sinks), whole)
    check(c, q, lens, S, window, sinks, dtype, whole)


@pytest.mark.parametrize("dtype,bits", KINDS)
def test_lengths_are_clamped_and_default_to_the_longest(dtype, bits):
    c = Case(2, 8, 4, 200, dtype, 0, bits)
    for m in (1, 4):
        q = c.queries(m)
        out = c.attend(q, None, 150, 50, 2)
        assert torch.equal(out, c.attend(q, last_tokens([150, 150], m), 150, 50, 2))
        check(c, q, last_tokens([150, 150], m), 150, 50, 2, dtype, out)
    q = c.queries(1)
    wild = torch.tensor([[2 ** 31 - 1], [-2 ** 31]], dtype=torch.int32, device="cuda")
    out = c.attend(q, wild, 150, 2 ** 31 - 1, 2 ** 31 - 1)
    check(c, q, torch.tensor([[150], [0]]), 150, 0, 0, dtype, out)
    q = c.queries(6)
    out = c.attend(q, None, 3, 0, 0)  # fewer rows than tokens
    check(c, q, last_tokens([3, 3], 6), 3, 0, 0, dtype, out)


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("m", [2, 30, 200])
def test_tokens_that_do_not_lie_next_to_each_other(m, dtype, bits):
    """Lengths in no order and far apart: slower, since rows between the shortest's window and the longest's end are read, but right."""
    B, G, Hkv, S = 2, 4, 2, 1500
    c = Case(B, G * Hkv, Hkv, S, dtype, 16, bits, seed=m)
    gen = torch.Generator(device="cuda").manual_seed(m)
    lens = torch.randint(0, S + 1, (B, m), generator=gen, device="cuda", dtype=torch.int32)
    lens[0, 0], lens[0, 1], lens[1, m - 1] = 1, S, 0
    for window, sinks in ((40, 3), (1, 0), (0, 0)):
        check(c, c.queries(m), lens, S, window, sinks, dtype)


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("m", [1, 4, 40])
def test_weights_over_many_orders_of_magnitude(m, dtype, bits):
    """Logits that grow along the rows, so that the reference of the exponentials moves many times, and large ones throughout."""
    B, Hq, Hkv, S = 1, 4, 2, 900
    c = Case(B, Hq, Hkv, S, dtype, 0, bits)
    q = c.queries(m, scale=30.0)
    check(c, q, last_tokens([S], m), S, 0, 0, dtype)
    check(c, q, last_tokens([S], m), S, 64, 300, dtype)


@pytest.mark.parametrize("dtype,bits", KINDS)
def test_a_larger_workspace_and_other_streams(dtype, bits):
    """One sized for the longest rows serves shorter ones; calls on two streams with a workspace each; the same bits every time."""
    c = Case(3, 16, 4, 4000, dtype, 256, bits)
    q = c.queries(2)
    lens = {S: last_tokens([S, S // 2, S // 5], 2) for S in (4000, 777, 50)}
    ref = {S: c.attend(q, n, S) for S, n in lens.items()}
    ws = torch.empty(api.dense_cache_workspace_bytes(c.lay, c.cache, 4000, 2), dtype=torch.uint8, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    outs = []
    for i in range(6):
        S = (4000, 777, 50)[i % 3]
        with torch.cuda.stream(streams[i % 2]):
            outs.append((S, c.attend(q, lens[S], S, ws=ws if i % 2 else None)))
    torch.cuda.synchronize()
    for S, out in outs:
        assert torch.equal(out, ref[S])


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("m", [1, 48])
def test_in_a_graph_with_other_lengths_and_tables(m, dtype, bits):
    """Captured once, replayed with lengths, queries and pages that change in between; two graphs share a workspace, one after the other."""
    c = Case(2, 8, 2, 1500, dtype, 64, bits)
    q, lens = c.queries(m), last_tokens([1500, 600], m)
    need = max(api.dense_cache_workspace_bytes(c.lay, c.cache, 1500, m, w, s) for w, s in ((0, 0), (200, 4)))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(q) for _ in range(2)]
    call = lambda i: api.dense_decode_cache(c.lay, c.cache, q, 1500, ws, outs[i], seq_lens=lens, queries_per_seq=m, window=200 * i, sinks=4 * i)
    call(0), call(1)
    torch.cuda.synchronize()
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(i)
        graphs.append(g)
    for totals in ([1500, 600], [700, 1500], [m, 0], [1499, 333]):
        lens.copy_(last_tokens(totals, m))
        q.copy_(c.queries(m))
        for i in (0, 1, 0):
            outs[i].fill_(float("nan"))
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i], c.attend(q, lens, 1500, 200 * i, 4 * i)), (totals, i)
    check(c, q, lens, 1500, 200, 4, dtype, outs[1])


@pytest.mark.parametrize("dtype,bits,B,m,Hq,Hkv,S,window,sinks,page_rows", [
    ("bf16", 0, 12, 1, 32, 8, 2100, 0, 0, 0), ("bf16", 0, 9, 2, 16, 16, 4000, 1300, 5, 256), ("f32", 0, 6, 1, 16, 16, 1100, 0, 0, 64),
    ("f32", 0, 3, 6, 16, 4, 9000, 0, 0, 0), ("bf16", 4, 10, 1, 32, 8, 7100, 0, 0, 256), ("bf16", 4, 5, 1, 64, 8, 15000, 0, 0, 0),
    ("f32", 4, 10, 1, 16, 8, 7100, 0, 0, 16), ("f32", 4, 9, 1, 64, 8, 9000, 8000, 3, 0), ("bf16", 0, 2, 11, 32, 8, 4300, 0, 0, 64),
    ("bf16", 0, 3, 8, 64, 8, 9000, 3000, 4, 0), ("bf16", 4, 2, 20, 32, 8, 1500, 700, 4, 64), ("bf16", 4, 2, 70, 32, 8, 900, 0, 0, 0)])
def test_large_calls(dtype, bits, B, m, Hq, Hkv, S, window, sinks, page_rows):
    """Calls large enough for rows past the caches and for tiles of 64, 128 and 256 query rows; some units of them."""
    print("case", dtype, bits, B, m, Hq, Hkv, S, window, sinks, page_rows, flush=True)
    c = Case(B, Hq, Hkv, S, dtype, page_rows, bits)
    q, lens = c.queries(m), last_tokens([S, S // 2, S - 77, 300][:min(B, 4)] + [S] * (B - 4), m)
    out = c.attend(q, lens, S, window, sinks)
    units = {(0, 0), (1, Hkv - 1), (B - 1, Hkv // 2)}
    ref, bound = reference(q, c.k, c.v, lens.cpu(), window, sinks, c.scales, units)
    torch.cuda.synchronize()
    G = Hq // Hkv
    assert bool(torch.isfinite(out).all())
    for b, h in units:
        at = (b, slice(None), slice(h * G, h * G + G))
        assert worst(out[at], ref[at], bound[at], dtype) <= 0, (b, h)


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("m", [1, 90])
def test_the_control_words_at_the_start_of_a_workspace_are_left_alone(m, dtype, bits):
    ctl = (128 * 9 * 16 + 64) * 4  # as the calls that rely on them count them
    c = Case(2, 8, 2, 900, dtype, 0, bits)
    need = api.dense_cache_workspace_bytes(c.lay, c.cache, 900, m)
    assert need >= ctl
    ws = torch.zeros(need, dtype=torch.uint8, device="cuda")
    q, lens = c.queries(m), last_tokens([900, 500], m)
    check(c, q, lens, 900, 0, 0, dtype, c.attend(q, lens, 900, ws=ws))
    assert not bool(ws[:ctl].any())


@pytest.mark.parametrize("dtype,bits", [("bf16", 0), ("bf16", 4)])
def test_rows_past_32_bits(dtype, bits):
    """A cache whose rows begin more than 2^32 bytes in."""
    B, Hkv, S_cap = (3, 2, 3 << 20) if bits == 0 else (5, 4, 4 << 20)
    dt = torch.bfloat16
    lay = api.make_layout(B, 2 * Hkv, Hkv, 128, 128, S_cap, dt)
    cache = api.alloc_whole_cache(lay, four_bits=bits == 4)
    n, far = 40, S_cap - 50
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn((B, n, Hkv, 128), generator=gen, device="cuda").to(dt) for _ in "kv")
    rows = (far + torch.arange(n, device="cuda"))[None].repeat(B, 1).int()
    api.loki_append(lay, cache, rows, k, v)
    k_back, v_back = (torch.empty((B, Hkv, n, 128), dtype=dt, device="cuda") for _ in "kv")
    api.loki_read_rows(lay, cache, rows, k_back, v_back)
    if not bits:
        assert torch.equal(k_back, k.transpose(1, 2)) and torch.equal(v_back, v.transpose(1, 2))
    q = torch.randn((B, 1, 2 * Hkv, 128), generator=gen, device="cuda").to(dt)
    lens = torch.full((B, 1), far + n, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    ws = torch.empty(api.dense_cache_workspace_bytes(lay, cache, S_cap, 1, n, 0), dtype=torch.uint8, device="cuda")
    api.dense_decode_cache(lay, cache, q, S_cap, ws, out, seq_lens=lens, window=n)
    near = Case(B, 2 * Hkv, Hkv, n, dtype, 0, bits)
    if bits:
        near.held[0].copy_(cache.tensors[0][:, :, far:far + n]), near.held[1].copy_(cache.tensors[1][:, :, far:far + n])
        near.held[2].copy_(cache.tensors[2][:, :, far:far + n]), near.held[3].copy_(cache.tensors[3][:, :, far:far + n])
    else:
        near.held[0].copy_(k.transpose(1, 2)), near.held[1].copy_(v.transpose(1, 2))
    same = near.attend(q, torch.full((B, 1), n, dtype=torch.int32, device="cuda"), n)
    # (steps begin at multiples of 16 rows, so the sums' order differs: two results within a bound of the same 64 bits)
    assert float((out.float() - same.float()).abs().max()) <= 2.0 ** -7 * float(same.float().abs().max())
