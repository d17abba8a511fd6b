"""dense_decode_weights against attention in 64 bits: outputs, weights, what is left alone."""
import pytest
import torch

from paper_2406_02542_amd import api
from tests.attention_bound import DT, attend64, worst

pytestmark = pytest.mark.gpu


def make(B, Hq, Hkv, cap, lens, dtype, seed=0, peak=0.0, used=None):
    """Caches whose rows behind every sequence hold NaN; `used`: rows that are filled at all."""
    gen = torch.Generator(device="cuda").manual_seed(seed * 7919 + B * 131 + cap % 100003)
    used = used or cap
    k, v = (torch.empty((B, Hkv, cap, 128), dtype=DT[dtype], device="cuda") for _ in "kv")
    for t in (k, v):
        t[:, :, :used] = torch.randn((B, Hkv, used, 128), generator=gen, device="cuda").to(DT[dtype])
    q = (torch.randn((B, Hq, 128), generator=gen, device="cuda") * (1.0 + peak)).to(DT[dtype])
    for b, n in enumerate(lens):
        k[b, :, n:used] = float("nan")
        v[b, :, n:used] = float("nan")
    return q, k, v


def check(B, Hq, Hkv, cap, S_max, lens, dtype, ragged=True, w_in="fresh", seed=0, peak=0.0, used=None):
    print("case", B, Hq, Hkv, cap, S_max, lens, dtype, ragged, w_in, flush=True)
    q, k, v = make(B, Hq, Hkv, cap, lens, dtype, seed, peak, used)
    used, G = used or cap, Hq // Hkv
    lay = api.make_layout(B, Hq, Hkv, 128, 128, cap, DT[dtype])
    ws = torch.full((api.dense_weights_workspace_bytes(lay, S_max),), 255, dtype=torch.uint8, device="cuda")  # NaN
    old = torch.rand((B, Hkv, cap), device="cuda")
    w_out = old if w_in == "same" else torch.full((B, Hkv, cap), -3.0, device="cuda")
    start = old.clone() if w_in != "none" else torch.zeros_like(old)
    behind = old.clone() if w_in == "same" else w_out.clone()
    out = torch.full((B, Hq, 128), 5.0, dtype=DT[dtype], device="cuda")
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda") if ragged else None
    api.dense_decode_weights(lay, q, k, v, S_max, sl, None if w_in == "none" else old, w_out, ws, out)
    torch.cuda.synchronize()
    for b in range(B):
        n = lens[b]
        for h in range(Hkv):
            ref, p, bound, rel = attend64(q[b, h * G:(h + 1) * G], k[b, h, :n], v[b, h, :n])
            assert worst(out[b, h * G:(h + 1) * G], ref, bound, dtype) <= 0, (b, h)
            total = start[b, h, :n].double() + p.sum(0)
            # G + 1 terms added in fp32
            off = (w_out[b, h, :n].double() - total).abs() - (p.sum(0) * rel + (G + 1) * 2.0 ** -24 * total)
            assert n == 0 or float(off.max()) <= 0, (b, h, float(off.max()))
            assert torch.equal(w_out[b, h, n:used], behind[b, h, n:used])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(3, 3), (4, 2), (8, 2), (8, 1)])
@pytest.mark.parametrize("lens", [[1], [0, 1, 2], [31, 32, 33], [63, 64, 65, 0], [127, 129, 255, 257], [300, 7, 1000]])
def test_lengths_and_groups(lens, Hq, Hkv, dtype):
    cap = max(lens) + 5
    check(len(lens), Hq, Hkv, cap, cap - 2, lens, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("w_in", ["none", "same", "fresh"])
def test_totals_fresh_in_place_and_from_nothing(w_in, dtype):
    check(2, 8, 2, 700, 700, [700, 411], dtype, w_in=w_in)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,S", [(8, 2, 1), (8, 8, 33), (8, 4, 2311), (8, 1, 5000)])
def test_equal_lengths_without_a_list(Hq, Hkv, S, dtype):
    check(2, Hq, Hkv, S, S, [S, S], dtype, ragged=False)


@pytest.mark.parametrize("Hq,Hkv,B,S", [(32, 8, 16, 4096), (8, 8, 40, 1500), (64, 8, 70, 600), (4, 1, 1, 60000)])
def test_large_batches_and_long_sequences(Hq, Hkv, B, S):
    lens = [max(1, S - (b * 977) % (S * 3 // 4)) for b in range(B)]
    check(B, Hq, Hkv, S, S, lens, "bf16")


@pytest.mark.parametrize("Hq,Hkv,B,S", [(32, 8, 16, 3500), (64, 8, 70, 600), (4, 1, 1, 60000), (8, 1, 1030, 90), (16, 4, 300, 77)])
def test_large_fp32_batches_of_groups(Hq, Hkv, B, S):
    """Rows through and past the caches, one run and many of a sequence, more units than blocks are resident."""
    lens = [max(0, S - (b * 977) % (S + 1)) for b in range(B)]
    check(B, Hq, Hkv, S, S, lens, "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_peaked_attention(dtype):
    """Logits of hundreds: one row takes all, the others' weights vanish without a NaN."""
    check(2, 8, 2, 900, 900, [900, 500], dtype, peak=30.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_past_32_bits(dtype):
    """16 units of a cache with more than 2^32 bytes of keys; lengths as they are there."""
    cap = 1200000 if dtype == "bf16" else 600000
    check(4, 16, 4, cap, 700, [700, 1, 333, 0], dtype, used=800)


def test_entries_outside_their_range_are_clamped():
    q, k, v = make(2, 4, 2, 64, [64, 0], "f32")
    lay = api.make_layout(2, 4, 2, 128, 128, 64, torch.float32)
    ws = torch.empty(api.dense_weights_workspace_bytes(lay, 64), dtype=torch.uint8, device="cuda")
    res = []
    for lens in ([64, 0], [1 << 30, -5]):
        out, w = torch.empty((2, 4, 128), device="cuda"), torch.zeros((2, 2, 64), device="cuda")
        api.dense_decode_weights(lay, q, k, v, 64, torch.tensor(lens, dtype=torch.int32, device="cuda"), None, w, ws, out)
        res.append((out, w))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])
    assert bool((res[0][0][1] == 0).all()) and bool((res[0][1][1] == 0).all())


def test_same_result_every_time_and_on_a_replayed_graph():
    B, S = 3, 2000
    q, k, v = make(B, 32, 8, S, [S] * B, "bf16")
    lay = api.make_layout(B, 32, 8, 128, 128, S, torch.bfloat16)
    ws = torch.empty(api.dense_weights_workspace_bytes(lay, S), dtype=torch.uint8, device="cuda")
    lens = torch.tensor([S, 700, 1], dtype=torch.int32, device="cuda")
    w0 = torch.rand((B, 8, S), device="cuda")

    def eager():
        out, w = torch.empty((B, 32, 128), dtype=q.dtype, device="cuda"), w0.clone()
        api.dense_decode_weights(lay, q, k, v, S, lens, w, w, ws, out)
        torch.cuda.synchronize()
        return out, w

    first = eager()
    for _ in range(3):
        again = eager()
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    out, w = torch.empty((B, 32, 128), dtype=q.dtype, device="cuda"), w0.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.dense_decode_weights(lay, q, k, v, S, lens, w, w, ws, out)
    for n in (S, 1300, 0):
        lens.copy_(torch.tensor([n, 700, n // 2], dtype=torch.int32))
        w.copy_(w0)
        graph.replay()
        torch.cuda.synchronize()
        ref = eager()
        assert torch.equal(out, ref[0]) and torch.equal(w, ref[1])
