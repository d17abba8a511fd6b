"""dense_decode_cache where the blocks deal the rows among themselves by the lengths: large calls, above all in 4 bits, with lengths of all kinds."""
import pytest
import torch

from paper_2406_02542_amd import api
from tests.attention_bound import worst
from tests.test_gpu_whole_cache import last_tokens
from tests.whole_cache import Case, reference

pytestmark = pytest.mark.gpu
# (dtype, bits, B, m, Hq, Hkv, S, page_rows): 4, 8, 16 and more query rows of a KV head, 64 tiles, tiles of more than 8 tokens
SHAPES = [("bf16", 4, 8, 1, 32, 8, 4200, 256), ("bf16", 4, 64, 1, 8, 2, 1700, 0), ("bf16", 4, 2, 4, 64, 8, 14000, 64), ("bf16", 4, 3, 9, 8, 2, 12000, 16),
          ("bf16", 4, 2, 30, 8, 4, 7000, 0), ("bf16", 4, 7, 1, 16, 2, 20000, 64), ("f32", 4, 8, 1, 8, 8, 4100, 0), ("f32", 4, 3, 5, 16, 4, 9000, 32), ("bf16", 0, 8, 1, 32, 8, 2900, 16),
          ("bf16", 0, 2, 3, 32, 8, 12000, 0)]


def totals_of(kind, B, S):
    if kind == "all lengths":
        return [S] + [max(0, (S * (37 * b % 101)) // 101) for b in range(1, B)]
    return {"one long": [1] * (B - 1) + [S], "one there": [0] * (B - 1) + [S // 2], "none": [0] * B, "equal": [S] * B, "few rows": [5 + b for b in range(B)]}[kind]


def units_of(c, totals):
    return {(0, 0), (len(totals) - 1, c.lay.Hkv - 1), (len(totals) // 2, 1)}


def check(c, q, out, lens, window, sinks, dtype, units):
    ref, bound = reference(q, c.k, c.v, lens.cpu(), window, sinks, c.scales, units)
    G = c.lay.Hq // c.lay.Hkv
    for b, h in units:
        at = (b, slice(None), slice(h * G, (h + 1) * G))
        assert worst(out[at], ref[at], bound[at], dtype) <= 0, (b, h)
    assert bool(torch.isfinite(out).all())
    assert bool((out[lens == 0] == 0).all())


@pytest.mark.parametrize("dtype,bits,B,m,Hq,Hkv,S,page_rows", SHAPES)
def test_lengths_of_all_kinds(dtype, bits, B, m, Hq, Hkv, S, page_rows):
    """One workspace for all, not a byte behind it written; the same call gives the same bits."""
    print("case", dtype, bits, B, m, Hq, Hkv, S, page_rows, flush=True)
    c = Case(B, Hq, Hkv, S, dtype, page_rows, bits, seed=m)
    q = c.queries(m)
    for window, sinks in ((0, 0), (S - S // 7, 70)):
        need = api.dense_cache_workspace_bytes(c.lay, c.cache, S, m, window, sinks)
        whole = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
        for kind in ("all lengths", "one long", "one there", "none", "equal", "few rows"):
            totals = totals_of(kind, B, S)
            lens = last_tokens(totals, m)
            out = c.attend(q, lens, S, window, sinks, ws=whole[:need])
            again = c.attend(q, lens, S, window, sinks, ws=whole[:need])
            torch.cuda.synchronize()
            print(kind, window, sinks, flush=True)
            assert torch.equal(out, again)
            check(c, q, out, lens, window, sinks, dtype, units_of(c, totals))
            assert bool((whole[need:] == 171).all())


@pytest.mark.parametrize("dtype,bits,B,m,Hq,Hkv,S,page_rows", SHAPES[:3] + SHAPES[6:9])
def test_tokens_that_do_not_lie_next_to_each_other(dtype, bits, B, m, Hq, Hkv, S, page_rows):
    """Runs are dealt by some of a tile's tokens: others may see more rows, or all of those none."""
    m = 14
    c = Case(B, Hq, Hkv, S, dtype, page_rows, bits, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(9)
    q = c.queries(m)
    for far in (False, True):
        lens = torch.randint(0, S + 1, (B, m), generator=gen, device="cuda", dtype=torch.int32)
        if far:  # only a token in the middle of each tile sees any
            lens[:, [i for i in range(m) if i % 7 != 3]] = 0
        for window, sinks in ((0, 0), (300, 4)):
            out = c.attend(q, lens, S, window, sinks)
            torch.cuda.synchronize()
            check(c, q, out, lens, window, sinks, dtype, {(0, 0), (B - 1, Hkv - 1)})


@pytest.mark.parametrize("dtype,bits,B,m,Hq,Hkv,S,page_rows", [SHAPES[0], SHAPES[3], SHAPES[6], SHAPES[8]])
def test_a_captured_call_deals_by_the_lengths_of_each_replay(dtype, bits, B, m, Hq, Hkv, S, page_rows):
    c = Case(B, Hq, Hkv, S, dtype, page_rows, bits, seed=5)
    q, out = c.queries(m), torch.empty((B, m, Hq, 128), dtype=c.dt, device="cuda")
    lens = last_tokens([S] * B, m)
    ws = torch.full((api.dense_cache_workspace_bytes(c.lay, c.cache, S, m),), 255, dtype=torch.uint8, device="cuda")
    call = lambda: api.dense_decode_cache(c.lay, c.cache, q, S, ws, out, seq_lens=lens, queries_per_seq=m)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for kind in ("all lengths", "one long", "few rows", "equal", "none"):
        lens.copy_(last_tokens(totals_of(kind, B, S), m))
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        eager = c.attend(q, lens, S)
        torch.cuda.synchronize()
        assert torch.equal(got, eager), kind


@pytest.mark.parametrize("bits", [0, 4])
@pytest.mark.parametrize("B,m,Hq,Hkv,S,window,page_rows", [
    (16, 70, 32, 8, 300, 0, 16), (17, 130, 16, 16, 400, 100, 0), (9, 300, 32, 8, 420, 130, 64), (3, 700, 64, 8, 900, 0, 256), (65, 40, 32, 4, 250, 50, 0), (4, 520, 32, 16, 520, 0, 64)])
def test_tiles_of_many_query_rows_in_whole_rounds_and_halves(B, m, Hq, Hkv, S, window, page_rows, bits):
    """Chunks of prompts, some of them padded, one empty, one whose first tokens see nothing: as many tiles with rows as leave a round half empty, or full."""
    print("case", B, m, Hq, Hkv, S, window, page_rows, bits, flush=True)
    c = Case(B, Hq, Hkv, S, "bf16", page_rows, bits, seed=m)
    q = c.queries(m)
    for padded in (0.0, 0.3, 0.6, 0.95):
        lens = last_tokens([S - (3 * b) % 40 for b in range(B)], m)
        for b in range(B):
            if padded:
                lens[b, max(1, int(m * (1 - padded * ((b % 4) + 1) / 4))):] = 0
        lens[1] = 0
        lens[2] = last_tokens([m // 2], m)[0]
        out = c.attend(q, lens, S, window, 3)
        again = c.attend(q, lens, S, window, 3)
        torch.cuda.synchronize()
        assert torch.equal(out, again)
        check(c, q, out, lens, window, 3, "bf16", {(0, 0), (2, Hkv - 1), (B - 1, Hkv // 2)})
