"""dense_decode_shared against attention in 64 bits over the prefix and every sequence's own rows."""
import pytest
import torch

from paper_2406_02542_amd import api
from tests.attention_bound import DT, attend64, worst

pytestmark = pytest.mark.gpu
ONE_TERM = {"bf16": 2 * 2.0 ** -8, "f32": 0.0}  # the prefix's weights enter the matrix product as one bf16 each


def check(B, Hq, Hkv, P, cap_p, S_max, lens, dtype, ragged=True, peak=0.0, cap=None, used=None):
    print("case", B, Hq, Hkv, P, cap_p, S_max, lens[:4], dtype, ragged, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(B * 1009 + P * 31 + S_max)
    dt, G = DT[dtype], Hq // Hkv
    cap = cap or S_max + 3
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)
    q = (rand(B, Hq, 128).float() * (1.0 + peak)).to(dt)
    used_p = used or cap_p
    kp, vp = (torch.empty((Hkv, cap_p, 128), dtype=dt, device="cuda") for _ in "kv")
    k, v = rand(B, Hkv, cap, 128), rand(B, Hkv, cap, 128)
    for t in (kp, vp):
        t[:, :used_p] = rand(Hkv, used_p, 128)
        t[:, P:used_p] = float("nan")  # rows behind the prefix and behind every sequence
    for b, n in enumerate(lens):
        k[b, :, n:], v[b, :, n:] = float("nan"), float("nan")
    lay = api.make_layout(B, Hq, Hkv, 128, 128, cap, dt)
    ws = torch.full((max(256, api.dense_shared_workspace_bytes(lay, P, S_max)),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full((B, Hq, 128), 5.0, dtype=dt, device="cuda")
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda") if ragged else None
    api.dense_decode_shared(lay, q, kp if P else None, vp if P else None, P, k if S_max else None, v if S_max else None, S_max, sl, ws, out)
    torch.cuda.synchronize()
    for b in range(B):
        for h in range(Hkv):
            kk, vv = torch.cat([kp[h, :P], k[b, h, :lens[b]]]), torch.cat([vp[h, :P], v[b, h, :lens[b]]])
            ref, _, bound, _ = attend64(q[b, h * G:(h + 1) * G], kk, vv, ONE_TERM[dtype])
            assert worst(out[b, h * G:(h + 1) * G], ref, bound, dtype) <= 0, (b, h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(3, 3), (4, 2), (8, 2), (8, 1)])
@pytest.mark.parametrize("P,S_max", [(0, 40), (1, 1), (31, 2), (32, 33), (33, 100), (129, 64), (700, 1), (513, 0), (2047, 300)])
def test_lengths_and_groups(P, S_max, Hq, Hkv, dtype):
    for B in (1, 3):
        lens = [S_max, 0, S_max // 2][:B]
        check(B, Hq, Hkv, P, P + 7, S_max, lens, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows_at_all(dtype):
    check(2, 4, 2, 0, 7, 0, [0, 0], dtype, cap=8)
    check(2, 4, 2, 0, 7, 5, [0, 5], dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hq,Hkv,P,S_max", [(17, 8, 8, 1000, 50), (33, 8, 4, 4097, 17), (64, 64, 8, 2000, 130), (7, 32, 8, 9000, 600),
                                              (130, 8, 1, 515, 9), (16, 4, 1, 30000, 5), (5, 16, 2, 12345, 777), (40, 4, 1, 5000, 40)])
def test_batches(B, Hq, Hkv, P, S_max, dtype):
    lens = [max(0, S_max - (37 * b) % (S_max + 1)) for b in range(B)]
    check(B, Hq, Hkv, P, P, S_max, lens, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B", [2, 20])
def test_peaked_attention_and_no_list(B, dtype):
    check(B, 16, 4, 1500, 1500, 200, [200] * B, dtype, ragged=False, peak=30.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_past_32_bits(dtype):
    """A prefix cache of more than 2^32 bytes, of which the first rows are the prefix."""
    cap = 4300000 if dtype == "bf16" else 2200000
    check(20, 16, 4, 600, cap, 20, [20] * 20, dtype, used=700)


def test_same_result_every_time_and_on_a_replayed_graph():
    B, Hq, Hkv, P, S = 24, 32, 8, 3000, 100
    rand = lambda *s: torch.randn(s, device="cuda").bfloat16()
    q, kp, vp, k, v = rand(B, Hq, 128), rand(Hkv, P, 128), rand(Hkv, P, 128), rand(B, Hkv, S, 128), rand(B, Hkv, S, 128)
    lay = api.make_layout(B, Hq, Hkv, 128, 128, S, torch.bfloat16)
    ws = torch.empty(api.dense_shared_workspace_bytes(lay, P, S), dtype=torch.uint8, device="cuda")
    lens = torch.full((B,), S, dtype=torch.int32, device="cuda")

    def eager():
        out = torch.empty((B, Hq, 128), dtype=q.dtype, device="cuda")
        api.dense_decode_shared(lay, q, kp, vp, P, k, v, S, lens, ws, out)
        torch.cuda.synchronize()
        return out

    first = eager()
    assert all(torch.equal(first, eager()) for _ in range(3))
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.dense_decode_shared(lay, q, kp, vp, P, k, v, S, lens, ws, out)
    for n in (S, 3, 0):
        lens.fill_(n)
        q.copy_(rand(B, Hq, 128))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("B,Hq,Hkv", [(8, 32, 8), (40, 16, 2)])
def test_one_workspace_for_growing_prefixes_and_sequences(B, Hq, Hkv, dtype):
    """Sized once for the longest of both; nothing behind it is written."""
    P, S, G, dt = 9000, 700, Hq // Hkv, DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(9)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)
    q, kp, vp, k, v = rand(B, Hq, 128), rand(Hkv, P, 128), rand(Hkv, P, 128), rand(B, Hkv, S, 128), rand(B, Hkv, S, 128)
    lay = api.make_layout(B, Hq, Hkv, 128, 128, S, dt)
    need = api.dense_shared_workspace_bytes(lay, P, S)
    buf = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)
    for rows, own in ((P, S), (8193, 5), (8192, 300), (4097, S), (4096, 64), (4096, 0), (129, 33), (1, 1), (0, S)):
        print("case", B, Hq, Hkv, dtype, rows, own, flush=True)
        assert api.dense_shared_workspace_bytes(lay, rows, own) <= need
        api.dense_decode_shared(lay, q, kp, vp, rows, k, v, own, None, buf[:need], out)
        torch.cuda.synchronize()
        assert bool((buf[need:] == 255).all())
        for b in (0, B - 1):
            for h in (0, Hkv - 1):
                kk, vv = torch.cat([kp[h, :rows], k[b, h, :own]]), torch.cat([vp[h, :rows], v[b, h, :own]])
                ref, _, bound, _ = attend64(q[b, h * G:(h + 1) * G], kk, vv, {"bf16": 2.0 ** -16, "f32": 0.0}[dtype])
                assert worst(out[b, h * G:(h + 1) * G], ref, bound, dtype) <= 0, (b, h)
