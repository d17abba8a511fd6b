"""dense_decode_cache where what a token does not see is not finite: rows of later tokens and rows before its window, queries of padded tokens."""
import pytest
import torch

from tests.attention_bound import worst
from tests.test_gpu_whole_cache import KINDS, last_tokens
from tests.whole_cache import Case, reference, seen

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")
# (B, m, Hq, Hkv, S): up to 4, 8, 16, 32, 64, 128 and 256 query rows of a KV head, and several tiles of them, 69 MB and more read, and whole rounds of tiles
SHAPES = [(2, 3, 2, 2, 300), (2, 2, 8, 2, 300), (1, 1, 8, 2, 2100), (2, 4, 8, 2, 2100), (2, 7, 8, 2, 700), (1, 16, 8, 2, 600), (1, 30, 8, 2, 500), (2, 60, 8, 2, 900), (1, 300, 4, 2, 700),
          (4, 16, 32, 8, 4200), (1, 64, 8, 2, 5000), (16, 70, 32, 8, 300), (2, 1, 32, 8, 16500)]


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("B,m,Hq,Hkv,S", SHAPES)
def test_padded_tokens_with_queries_that_are_not_finite(B, m, Hq, Hkv, S, dtype, bits):
    if m == 1:
        m = 2
    print("case", B, m, Hq, Hkv, S, dtype, bits, flush=True)
    c = Case(B, Hq, Hkv, S, dtype, 16, bits, seed=m)
    lens = last_tokens([S - 5 * b for b in range(B)], m)
    lens[0, m - (m + 2) // 3:] = 0
    q = c.queries(m)
    given = q.clone()
    for b in range(B):
        for i, j in enumerate(torch.nonzero(lens[b] == 0).flatten().tolist()):
            given[b, j] = (NAN, INF, -INF)[i % 3]
    units = {(0, 0), (B - 1, Hkv - 1)}
    for window, sinks in ((0, 0), (90, 5)):
        out = c.attend(given, lens, S, window, sinks)
        torch.cuda.synchronize()
        assert bool((out[lens == 0] == 0).all())
        assert bool(torch.isfinite(out).all())
        ref, bound = reference(q, c.k, c.v, lens.cpu(), window, sinks, c.scales, units)
        G = Hq // Hkv
        for b, h in units:
            at = (b, slice(None), slice(h * G, (h + 1) * G))
            assert worst(out[at], ref[at], bound[at], dtype) <= 0


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 5)])
@pytest.mark.parametrize("B,m,Hq,Hkv,S", SHAPES)
def test_rows_that_are_not_finite_reach_only_tokens_that_see_them(B, m, Hq, Hkv, S, window, sinks, dtype, bits):
    """Two rows, of the last token and of one before most windows, hold a few values that are not finite; a third, of a middle token, such keys."""
    print("case", B, m, Hq, Hkv, S, window, sinks, dtype, bits, flush=True)
    c = Case(B, Hq, Hkv, S, dtype, 16, bits, seed=m)
    lens = last_tokens([S] * B, m)
    first = max(0, S - m + 1 - window) if window else 0  # of the first token's window
    bad_values = {S - 1: (3, NAN), first: (77, INF)}     # row: a column and what it holds
    bad_key = S - 1 - m // 2
    G = Hq // Hkv
    for b in range(B):
        for s, (col, what) in bad_values.items():
            page = (int(c.table[b, s // 16]), slice(None), s % 16)
            if bits:
                c.held[3][page + (col // 32, s % 2)] = what  # the group's step or lowest
            else:
                c.held[1][page + (col,)] = what
        page = (int(c.table[b, bad_key // 16]), slice(None), bad_key % 16)
        if m > 2:
            if bits:
                c.held[2][page + (1, 1)] = NAN
            else:
                c.held[0][page + (100,)] = NAN
    q = c.queries(m)
    out = c.attend(q, lens, S, window, sinks)
    torch.cuda.synchronize()
    units = {(0, 0), (B - 1, Hkv - 1)}
    ref, bound = reference(q, c.k, c.v, lens.cpu(), window, sinks, c.scales, units)
    clean = 0
    for b, h in units:
        for j in range(m):
            rows = set(seen(int(lens[b, j]), window, sinks).tolist())
            at = (b, j, slice(h * G, (h + 1) * G))
            if m > 2 and bad_key in rows:
                assert not bool(torch.isfinite(out[at]).any())
                continue
            cols = torch.zeros(128, dtype=torch.bool, device="cuda")
            for s, (col, _) in bad_values.items():
                if s in rows:
                    cols[slice(col // 32 * 32, col // 32 * 32 + 32) if bits else col] = True
            assert not bool(torch.isfinite(out[at][:, cols]).any())
            assert bool(torch.isfinite(out[at][:, ~cols]).all())
            assert worst(out[at][:, ~cols], ref[at][:, ~cols], bound[at][:, ~cols], dtype) <= 0
            clean += 1
    assert clean > 0 or m <= 2
