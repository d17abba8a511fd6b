"""dense_decode_cache where padded tokens' queries hold anything: they get zeros, and no other token anything of them."""
import pytest
import torch

from tests.attention_bound import worst
from tests.test_gpu_whole_cache import KINDS, last_tokens
from tests.whole_cache import Case, reference

pytestmark = pytest.mark.gpu
INF = float("inf")
# (B, m, Hq, Hkv, S): up to 4, 8, 16, 32, 64, 128 and 256 query rows of a KV head; rows in one part, in up to four, in more; runs dealt by
# the lengths; whole rounds of tiles, and halves of them
SHAPES = [(2, 3, 2, 2, 100), (2, 3, 2, 2, 400), (2, 4, 2, 2, 2100), (2, 3, 8, 4, 120), (2, 4, 8, 4, 3000), (2, 7, 8, 4, 110), (2, 8, 8, 4, 2600), (2, 12, 8, 4, 90), (1, 30, 8, 2, 2500), (4, 16, 32, 8, 4200),
          (1, 100, 2, 2, 128), (1, 100, 2, 2, 2000), (1, 300, 4, 2, 2500), (16, 70, 32, 8, 300), (2, 2, 32, 8, 16500)]
# what columns 5 and 127 of such a query hold; the others are ordinary
QUERIES = [(INF, 1.0), (1.0, -INF), (0.0, 3e38), (-3e38, 1e38)]


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("B,m,Hq,Hkv,S", SHAPES)
def test_padded_tokens_with_infinite_logits(B, m, Hq, Hkv, S, dtype, bits):
    print("case", B, m, Hq, Hkv, S, dtype, bits, flush=True)
    c = Case(B, Hq, Hkv, S, dtype, 16, bits, seed=m)
    lens = last_tokens([S - 5 * b for b in range(B)], m)
    lens[0, m - (m + 2) // 3:] = 0
    lens[B - 1, m // 2] = 0
    q = c.queries(m)
    units = {(0, 0), (B - 1, Hkv - 1)}
    G = Hq // Hkv
    for window, sinks in ((0, 0), (S - 30, 5)):
        ref, bound = reference(q, c.k, c.v, lens.cpu(), window, sinks, c.scales, units)
        for low, high in QUERIES:
            given = q.clone()
            given[lens == 0, :, 5] = low
            given[lens == 0, :, 127] = high
            out = c.attend(given, lens, S, window, sinks)
            torch.cuda.synchronize()
            assert bool((out[lens == 0] == 0).all()), (window, low, high)
            assert bool(torch.isfinite(out).all())
            for b, h in units:
                at = (b, slice(None), slice(h * G, (h + 1) * G))
                assert worst(out[at], ref[at], bound[at], dtype) <= 0, (window, low, high)


@pytest.mark.parametrize("dtype,bits", KINDS)
@pytest.mark.parametrize("B,m,Hq,Hkv,S", SHAPES)
def test_padded_queries_change_no_bit_of_other_tokens(B, m, Hq, Hkv, S, dtype, bits):
    """Large logits of a padded token, or such that are no number, move no reference of the exponentials of the tokens beside it."""
    print("case", B, m, Hq, Hkv, S, dtype, bits, flush=True)
    c = Case(B, Hq, Hkv, S, dtype, 16, bits, seed=m)
    lens = last_tokens([S - 5 * b for b in range(B)], m)
    lens[0, m - (m + 2) // 3:] = 0
    lens[B - 1, m // 2] = 0
    q = c.queries(m)
    for window, sinks in ((0, 0), (S - 30, 5)):
        outs = []
        for what in (0.0, 40.0, -40.0, float("nan"), INF):
            given = q.clone()
            given[lens == 0] = what * q[lens == 0]
            outs.append(c.attend(given, lens, S, window, sinks))
        torch.cuda.synchronize()
        for out in outs[1:]:
            assert torch.equal(out, outs[0]), (window,)
