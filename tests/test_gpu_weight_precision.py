"""Softmax weights enter the products with the values in 32 bits, or on the matrix cores in two bf16 terms: rows of large weights
whose values cancel show what a weight is off by, as the output's own rounding is then small beside it."""
import pytest
import torch

from paper_2406_02542_amd import api
from tests.attention_bound import DT, attend64, worst

pytestmark = pytest.mark.gpu
TERMS = {"bf16": 2.0 ** -16, "f32": 0.0}  # what a weight is off by, relative to itself, where it meets the values


def cancelling(lead, rows, gen, dt):
    """Keys and values [*lead, rows, 128]: rows come in pairs of nearly the same key along one direction and opposite values; the
    first pair outweighs the others."""
    n = rows // 2 + 1
    u = torch.linspace(-1.0, 1.0, 128, device="cuda")
    k = 0.2 * torch.randn((*lead, n, 128), generator=gen, device="cuda")
    k[..., 0, :] += 2.0 * u
    v = torch.randn((*lead, n, 128), generator=gen, device="cuda")
    k = torch.stack([k, k + 0.01 * torch.randn(k.shape, generator=gen, device="cuda")], dim=-2).flatten(-3, -2)[..., :rows, :]
    v = torch.stack([v, -v], dim=-2).flatten(-3, -2)[..., :rows, :]
    return k.to(dt).contiguous(), v.to(dt).contiguous()


def queries(B, Hq, gen, dt):
    u = torch.linspace(-1.0, 1.0, 128, device="cuda")
    return (u * torch.rand((B, Hq, 1), generator=gen, device="cuda") * 2.0 + 0.3 * torch.randn((B, Hq, 128), generator=gen, device="cuda")).to(dt)


def compare(out, q, rows_of, dtype, Hkv):
    G = q.shape[1] // Hkv
    for b in range(q.shape[0]):
        for h in range(Hkv):
            k, v = rows_of(b, h)
            ref, _, bound, _ = attend64(q[b, h * G:(h + 1) * G], k, v, TERMS[dtype])
            assert worst(out[b, h * G:(h + 1) * G], ref, bound, dtype) <= 0, (b, h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv", [(2, 2), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("B,P,S", [(1, 40, 0), (3, 1000, 31), (8, 300, 64), (15, 2100, 5), (33, 700, 40), (70, 515, 3), (5, 0, 200)])
def test_shared_prefix(B, P, S, Hq, Hkv, dtype):
    """From one block of query rows to several, waves with other keys and with other queries; and own rows alone."""
    print("case", B, P, S, Hq, Hkv, dtype, flush=True)
    gen, dt = torch.Generator(device="cuda").manual_seed(B * 1000 + P + Hq), DT[dtype]
    kp, vp = cancelling((Hkv,), P, gen, dt) if P else (None, None)
    k, v = cancelling((B, Hkv), max(S, 1), gen, dt)
    q, out = queries(B, Hq, gen, dt), torch.empty((B, Hq, 128), dtype=dt, device="cuda")
    lay = api.make_layout(B, Hq, Hkv, 128, 128, max(S, 1), dt)
    ws = torch.full((api.dense_shared_workspace_bytes(lay, P, S),), 255, dtype=torch.uint8, device="cuda")
    api.dense_decode_shared(lay, q, kp, vp, P, k if S else None, v if S else None, S, None, ws, out)
    torch.cuda.synchronize()
    join = lambda p, t: torch.cat([x for x in (p, t) if x is not None])
    compare(out, q, lambda b, h: (join(kp[h] if P else None, k[b, h, :S]), join(vp[h] if P else None, v[b, h, :S])), dtype, Hkv)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,B,S", [(2, 2, 2, 300), (4, 2, 3, 1000), (8, 2, 2, 700), (16, 2, 5, 2100)])
def test_whole_caches(Hq, Hkv, B, S, dtype):
    """dense_decode_step and dense_decode_weights over the same rows."""
    print("case", Hq, Hkv, B, S, dtype, flush=True)
    gen, dt = torch.Generator(device="cuda").manual_seed(B * 1000 + S + Hq), DT[dtype]
    k, v = cancelling((B, Hkv), S, gen, dt)
    q = queries(B, Hq, gen, dt)
    lay = api.make_layout(B, Hq, Hkv, 128, 128, S, dt)
    lens = torch.tensor([S - 13 * b for b in range(B)], dtype=torch.int32, device="cuda")
    ws = torch.full((max(api.dense_weights_workspace_bytes(lay, S), api.loki_workspace_bytes(lay, S, 0, 0, -1)),), 255, dtype=torch.uint8,
                    device="cuda")
    step, weighed, w = torch.empty_like(q), torch.empty_like(q), torch.zeros((B, Hkv, S), device="cuda")
    api.dense_decode_step(lay, q, k, v, S, lens, ws, step)
    torch.cuda.synchronize()
    api.dense_decode_weights(lay, q, k, v, S, lens, None, w, ws, weighed)
    torch.cuda.synchronize()
    rows = lambda b, h: (k[b, h, :S - 13 * b], v[b, h, :S - 13 * b])
    compare(step, q, rows, dtype, Hkv)
    compare(weighed, q, rows, dtype, Hkv)
