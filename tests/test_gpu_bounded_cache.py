"""The operators as a server runs them together: new tokens turned by their positions into a cache, attended over with
their weights added up, and the cache brought back under its bound; and a batch behind a shared prefix."""
import pytest
import torch

from paper_2406_02542_amd import api
from tests.attention_bound import DT, attend64, worst
from tests.test_gpu_evict import kept_rows
from tests.test_gpu_rotary import turned
from tests.test_gpu_shared_prefix import ONE_TERM

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_under_a_bound(dtype):
    B, Hq, Hkv, cap, budget, sinks, recent = 3, 8, 2, 96, 64, 2, 16
    dt, G = DT[dtype], Hq // Hkv
    lay = api.make_layout(B, Hq, Hkv, 128, 128, cap, dt)
    f, scale = api.loki_rotary_frequencies(128, 10000.0, api.ROTARY_RAMP, 4.0, 64.0, 1.0, 8.0)
    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)
    kc, vc = torch.zeros((B, Hkv, cap, 128), dtype=dt, device="cuda"), torch.zeros((B, Hkv, cap, 128), dtype=dt, device="cuda")
    w = torch.zeros((B, Hkv, cap), device="cuda")
    ws = torch.empty(max(api.dense_weights_workspace_bytes(lay, cap), api.loki_evict_workspace_bytes(lay, cap, budget)),
                     dtype=torch.uint8, device="cuda")
    lens, seen = torch.tensor([0, 40, 88], dtype=torch.int32, device="cuda"), torch.tensor([0, 40, 88], dtype=torch.int32, device="cuda")
    # what the sequences hold already
    n0 = 88
    pos = torch.arange(n0, dtype=torch.int32, device="cuda").repeat(B, 1)
    rows = torch.where(pos < lens[:, None], pos, -1).contiguous()
    k0, v0 = rand(B, n0, Hkv, 128), rand(B, n0, Hkv, 128)
    api.loki_rotary(lay, pos, f, k=k0, k_out=kc, v=v0, v_out=vc, rows=rows, scale=scale)
    assert bool((kc[0] == 0).all())
    evictions = 0
    for step in range(60):
        qkv = rand(B, 1, (Hq + 2 * Hkv) * 128)
        q, k, v = (qkv[..., a * 128:(a + h) * 128].unflatten(-1, (h, 128)) for a, h in ((0, Hq), (Hq, Hkv), (Hq + Hkv, Hkv)))
        q_out = torch.empty((B, 1, Hq, 128), dtype=dt, device="cuda")
        api.loki_rotary(lay, seen[:, None].contiguous(), f, q=q, q_out=q_out, k=k, k_out=kc, v=v, v_out=vc, rows=lens[:, None].contiguous(), scale=scale)
        ref, e = turned(k, seen[:, None], f, 128, False, False, scale)
        for b in range(B):
            n = int(lens[b])
            half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
            assert float(((kc[b, :, n].double() - ref[b, 0]).abs() - (e[b, 0] + half * (ref[b, 0].abs() + e[b, 0]))).max()) <= 0
            w[b, :, n] = 0  # a new row has no weight yet
        lens += 1
        seen += 1
        before, out = w.clone(), torch.empty((B, Hq, 128), dtype=dt, device="cuda")
        api.dense_decode_weights(lay, q_out, kc, vc, cap, lens, w, w, ws, out)
        torch.cuda.synchronize()
        for b in range(B):
            n = int(lens[b])
            for h in range(Hkv):
                r, p, bound, rel = attend64(q_out[b, 0, h * G:(h + 1) * G], kc[b, h, :n], vc[b, h, :n])
                assert worst(out[b, h * G:(h + 1) * G], r, bound, dtype) <= 0
                total = before[b, h, :n].double() + p.sum(0)
                assert float(((w[b, h, :n].double() - total).abs() - p.sum(0) * rel - (G + 1) * 2.0 ** -24 * total).max()) <= 0
        if int(lens.max()) == cap:
            evictions += 1
            ok, ov, ow, ol = kc.clone(), vc.clone(), w.cpu().numpy(), lens.tolist()
            api.loki_evict(lay, w, kc, None, vc, cap, budget, sinks, recent, ws, seq_lens=lens, lens_out=lens)
            torch.cuda.synchronize()
            assert lens.tolist() == [min(n, budget) for n in ol]
            for b in range(B):
                for h in range(Hkv):
                    at = torch.from_numpy(kept_rows(ow[b, h], ol[b], budget, sinks, recent)).cuda()
                    m = len(at)
                    assert torch.equal(kc[b, h, :m], ok[b, h][at]) and torch.equal(vc[b, h, :m], ov[b, h][at])
    assert evictions >= 2


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_batch_behind_a_prefix_is_the_dense_step_over_both(dtype):
    """Prompts turned at the positions behind the prefix; the shared call agrees with dense_decode_step over copies."""
    B, Hq, Hkv, P, S = 6, 16, 4, 300, 20
    dt = DT[dtype]
    gen = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)
    f, _ = api.loki_rotary_frequencies(64, 10000.0)
    kp, vp = (torch.empty((1, Hkv, P, 128), dtype=dt, device="cuda") for _ in "kv")
    lay1 = api.make_layout(1, Hq, Hkv, 128, 128, P, dt)
    api.loki_rotary(lay1, torch.arange(P, dtype=torch.int32, device="cuda")[None], f, k=rand(1, P, Hkv, 128), k_out=kp, v=rand(1, P, Hkv, 128), v_out=vp)
    lay = api.make_layout(B, Hq, Hkv, 128, 128, S, dt)
    k, v = (torch.empty((B, Hkv, S, 128), dtype=dt, device="cuda") for _ in "kv")
    q = torch.empty((B, S, Hq, 128), dtype=dt, device="cuda")
    pos = (P + torch.arange(S, dtype=torch.int32, device="cuda")).repeat(B, 1)
    api.loki_rotary(lay, pos, f, q=rand(B, S, Hq, 128), q_out=q, k=rand(B, S, Hkv, 128), k_out=k, v=rand(B, S, Hkv, 128), v_out=v)
    lens = torch.tensor([1, 2, 20, 7, 13, 19], dtype=torch.int32, device="cuda")
    last = q[torch.arange(B, device="cuda"), (lens - 1).long()].contiguous()
    ws = torch.empty(api.dense_shared_workspace_bytes(lay, P, S), dtype=torch.uint8, device="cuda")
    out, dense = torch.empty_like(last), torch.empty_like(last)
    api.dense_decode_shared(lay, last, kp[0], vp[0], P, k, v, S, lens, ws, out)
    whole = api.make_layout(B, Hq, Hkv, 128, 128, P + S, dt)
    kk, vv = (torch.cat([a.expand(B, -1, -1, -1), b], dim=2).contiguous() for a, b in ((kp, k), (vp, v)))
    api.dense_decode_step(whole, last, kk, vv, P + S, lens + P, api.alloc_workspace(whole, P + S, 0, 0, -1), dense)
    torch.cuda.synchronize()
    G = Hq // Hkv
    for b in range(B):
        for h in range(Hkv):
            n = P + int(lens[b])
            ref, _, bound, _ = attend64(last[b, h * G:(h + 1) * G], kk[b, h, :n], vv[b, h, :n], ONE_TERM[dtype])
            assert worst(out[b, h * G:(h + 1) * G], ref, bound, dtype) <= 0
            assert worst(dense[b, h * G:(h + 1) * G], ref, bound, dtype) <= 0


def test_two_graphs_on_one_workspace():
    """Captured weights and a captured shared step take turns on one workspace; neither leaves anything the other needs."""
    B, Hq, Hkv, S, P = 2, 8, 2, 700, 500
    rand = lambda *s: torch.randn(s, device="cuda").bfloat16()
    q, k, v, kp, vp = rand(B, Hq, 128), rand(B, Hkv, S, 128), rand(B, Hkv, S, 128), rand(Hkv, P, 128), rand(Hkv, P, 128)
    lay = api.make_layout(B, Hq, Hkv, 128, 128, S, torch.bfloat16)
    lens = torch.tensor([S, 33], dtype=torch.int32, device="cuda")
    ws = torch.full((max(api.dense_weights_workspace_bytes(lay, S), api.dense_shared_workspace_bytes(lay, P, S)),), 255, dtype=torch.uint8, device="cuda")
    out, w, both = torch.empty_like(q), torch.zeros((B, Hkv, S), device="cuda"), torch.empty_like(q)
    calls = [lambda: api.dense_decode_weights(lay, q, k, v, S, lens, None, w, ws, out),
             lambda: api.dense_decode_shared(lay, q, kp, vp, P, k, v, S, lens, ws, both)]
    graphs = []
    for call in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for step in range(4):
        q.copy_(rand(B, Hq, 128))
        lens.copy_(torch.tensor([S - 100 * step, 33 * step], dtype=torch.int32))
        w.zero_()
        for g in graphs if step % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (out, w, both)]
        w.zero_()
        for call in calls:
            call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, w, both)))


def test_two_streams_with_their_own_workspaces():
    B, Hq, Hkv, S, keep = 4, 16, 4, 3000, 500
    lay = api.make_layout(B, Hq, Hkv, 128, 128, S, torch.bfloat16)
    rand = lambda *s: torch.randn(s, device="cuda").bfloat16()
    sets = []
    for i in range(2):
        s = dict(q=rand(B, Hq, 128), k=rand(B, Hkv, S, 128), v=rand(B, Hkv, S, 128), w=torch.rand((B, Hkv, S), device="cuda"),
                 out=torch.empty((B, Hq, 128), dtype=torch.bfloat16, device="cuda"), idx=torch.empty((B, Hkv, keep), dtype=torch.int32, device="cuda"),
                 ws=torch.empty(api.dense_weights_workspace_bytes(lay, S), dtype=torch.uint8, device="cuda"),
                 we=torch.empty(api.loki_evict_workspace_bytes(lay, S, keep), dtype=torch.uint8, device="cuda"))
        s["total"] = torch.empty_like(s["w"])
        sets.append(s)

    def work(s, k, v):
        api.dense_decode_weights(lay, s["q"], k, v, S, None, s["w"], s["total"], s["ws"], s["out"])
        api.loki_evict(lay, s["total"], k, None, v, S, keep, 4, 100, s["we"], out_idx=s["idx"])

    alone = []
    for s in sets:
        k, v = s["k"].clone(), s["v"].clone()
        work(s, k, v)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in (s["out"], s["total"], s["idx"], k, v)])
    streams = [torch.cuda.Stream() for _ in sets]
    caches = [(s["k"].clone(), s["v"].clone()) for s in sets]
    torch.cuda.synchronize()
    for st, s, (k, v) in zip(streams, sets, caches):
        with torch.cuda.stream(st):
            work(s, k, v)
    torch.cuda.synchronize()
    for s, (k, v), ref in zip(sets, caches, alone):
        assert all(torch.equal(a, b) for a, b in zip((s["out"], s["total"], s["idx"], k, v), ref))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_totals_of_rows_appended_behind_an_eviction(dtype):
    """A new row's place holds the total of the row that was there; cleared with the append, on the device, a row has gathered
    what its own steps gave it, over several evictions; left alone it begins with the old total."""
    B, Hq, Hkv, cap, budget, sinks, recent = 2, 4, 2, 48, 32, 2, 8
    dt, G = DT[dtype], Hq // Hkv
    lay = api.make_layout(B, Hq, Hkv, 128, 128, cap, dt)
    gen = torch.Generator(device="cuda").manual_seed(17)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)
    k, v = rand(B, Hkv, cap, 128), rand(B, Hkv, cap, 128)
    w, total = torch.zeros((B, Hkv, cap), device="cuda"), torch.zeros((B, Hkv, cap), dtype=torch.float64, device="cuda")
    lens = torch.full((B,), 20, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(api.dense_weights_workspace_bytes(lay, cap), api.loki_evict_workspace_bytes(lay, cap, budget)), dtype=torch.uint8,
                     device="cuda")
    idx = torch.empty((B, Hkv, budget), dtype=torch.int32, device="cuda")
    out, off, evictions = torch.empty((B, Hq, 128), dtype=dt, device="cuda"), 0.0, 0
    for step in range(80):
        at = lens.long()[:, None, None].expand(-1, Hkv, 1)
        k.scatter_(2, at[..., None].expand(-1, -1, -1, 128), rand(B, Hkv, 1, 128))
        v.scatter_(2, at[..., None].expand(-1, -1, -1, 128), rand(B, Hkv, 1, 128))
        inherited = w.gather(2, at).clone()
        if step == 79:  # the last one keeps what it finds
            assert float(inherited.min()) > 0
        else:
            w.scatter_(2, at, 0.0)
            total.scatter_(2, at, 0.0)
        lens += 1
        q = rand(B, Hq, 128)
        api.dense_decode_weights(lay, q, k, v, cap, lens, w, w, ws, out)
        torch.cuda.synchronize()
        n = int(lens[0])
        if step == 79:
            total.scatter_(2, at, inherited.double())
        rels = []
        for b in range(B):
            for h in range(Hkv):
                _, p, _, rel = attend64(q[b, h * G:(h + 1) * G], k[b, h, :n], v[b, h, :n])
                total[b, h, :n] += p.sum(0)
                rels.append(rel)
        off += max(rels) + (G + 1) * 2.0 ** -24  # of each step, relative to a total that only grows
        assert bool(((w - total).abs()[:, :, :n] <= off * total[:, :, :n]).all()), step
        if n == cap:
            evictions += 1
            api.loki_evict(lay, w, k, None, v, cap, budget, sinks, recent, ws, seq_lens=lens, lens_out=lens, out_idx=idx)
            total[:, :, :budget] = total.gather(2, idx.long())
    assert evictions >= 3


def test_tensors_of_another_device_are_refused(monkeypatch):
    """The kernels would be launched on the current device with addresses of another."""
    lay = api.make_layout(1, 2, 2, 128, 128, 16, torch.float32)
    t, w, ws = torch.zeros((1, 2, 16, 128), device="cuda"), torch.zeros((1, 2, 16), device="cuda"), torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    q, out = torch.zeros((1, 2, 128), device="cuda"), torch.full((1, 2, 128), 7.0, device="cuda")
    pos, f = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros(64, dtype=torch.float64, device="cuda")
    stream = torch.cuda.current_stream()
    monkeypatch.setattr(api, "_current_device", lambda: t.get_device() + 1)
    for call in (lambda **kw: api.loki_rotary(lay, pos, f, q=q[:, None], q_out=out[:, None], **kw),
                 lambda **kw: api.dense_decode_weights(lay, q, t, t, 16, None, None, w, ws, out, **kw),
                 lambda **kw: api.loki_evict(lay, w, t, None, t, 16, 4, 0, 0, ws, **kw),
                 lambda **kw: api.dense_decode_shared(lay, q, None, None, 0, t, t, 16, None, ws, out, **kw)):
        for kw in ({}, dict(stream=stream)):
            with pytest.raises(ValueError, match="current device"):
                call(**kw)
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())
