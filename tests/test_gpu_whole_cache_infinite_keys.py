"""dense_decode_cache where a key that a token sees holds an infinity: a logit of minus infinity has weight 0, plus infinity or NaN makes all of the output NaN."""
import pytest
import torch

from tests.attention_bound import worst
from tests.test_gpu_whole_cache import KINDS, last_tokens
from tests.whole_cache import Case, reference, seen

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("what", [INF, -INF])
@pytest.mark.parametrize("B,m,Hq,Hkv,S,window,sinks", [
    (1, 1, 4, 4, 90, 0, 0), (2, 1, 8, 2, 2600, 0, 0), (2, 3, 8, 4, 400, 0, 0), (1, 6, 8, 4, 1700, 900, 3), (1, 40, 8, 2, 600, 0, 0), (1, 90, 4, 2, 700, 130, 2), (1, 150, 8, 2, 500, 0, 0)])
def test_keys_with_an_infinity(B, m, Hq, Hkv, S, window, sinks, what, dtype, bits):
    print("case", B, m, Hq, Hkv, S, window, sinks, what, dtype, bits, flush=True)
    c = Case(B, Hq, Hkv, S, dtype, 16, bits, seed=m)
    lens = last_tokens([S] * B, m)
    q, G = c.queries(m), Hq // Hkv
    # an early row, which tokens may see or not by their windows, and one that all see, in a column each (4 bits: a group's lowest value)
    rows, cols = (S - m - 60 if window == 0 else S - window, S - m - 20), (37, 100)
    for s, col in zip(rows, cols):
        for b in range(B):
            at = (int(c.table[b, s // 16]), slice(None), s % 16)
            if bits:
                c.held[2][at + (col // 32, 1)] = what
            else:
                c.held[0][at + (col,)] = what
    out = c.attend(q, lens, S, window, sinks)
    torch.cuda.synchronize()
    kept = [s for s in range(S) if s not in rows]
    none = weight_0 = 0
    for b in range(B):
        for h in {0, Hkv - 1}:
            for j in sorted({0, 1, m // 2, m - 2, m - 1} & set(range(m))):
                met = [i for i in range(2) if rows[i] in set(seen(int(lens[b, j]), window, sinks).tolist())]
                if window == 0:
                    there = [s for s in kept if s < int(lens[b, j])]
                else:
                    there = [s for s in kept if s < int(lens[b, j]) and (s < sinks or s >= int(lens[b, j]) - window)]
                at = torch.tensor(there, device="cuda")
                x = [t[b:b + 1, h:h + 1, at] for t in (c.k, c.v)]
                scales = [t[b:b + 1, h:h + 1, at] for t in c.scales] if bits else None
                heads = slice(h * G, (h + 1) * G)
                ref, bound = reference(q[b:b + 1, j:j + 1, heads], *x, torch.tensor([[len(there)]]), 0, 0, scales)
                for g in range(G):
                    got = out[b, j, h * G + g]
                    signs = [float(q[b, j, h * G + g, cols[i]]) * what for i in met]
                    if bits:  # (whether such a logit is NaN or infinite goes by the order of its sums)
                        if bool(torch.isnan(got).all()):
                            none += 1
                            continue
                    elif any(not x < 0 for x in signs):
                        assert bool(torch.isnan(got).all()), (b, j, h, g)
                        none += 1
                        continue
                    assert worst(got, ref[0, 0, g], bound[0, 0, g], dtype) <= 0, (b, j, h, g)
                    weight_0 += 1
    assert none > 0 or m * G == 1
    assert weight_0 > 0 or bits or m * G == 1
