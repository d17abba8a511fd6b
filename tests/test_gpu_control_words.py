"""A workspace that was filled with zeros once stays good for LOKI_WORKSPACE_ZEROED whatever calls of the library use it in
between: all of them leave the control words of the cooperating blocks, at its start, alone."""
import numpy as np
import pytest
import torch

from paper_2406_02542_amd import api, synth
from tests.parity import DeviceCase

CTL = (128 * 9 * 16 + 64) * 4  # a line for each of nine words of 128 units, and the error word's
DENSE = -1


def _others():
    """{name: (workspace bytes, call(workspace))} of every other entry point that takes a workspace, small: what a call keeps
    would lie where the control words are if they were not left out."""
    B, Hq, Hkv, S, P, keep = 2, 16, 4, 700, 500, 40
    dt = torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(11)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dt)
    q, k, v, kp, vp = rand(B, Hq, 128), rand(B, Hkv, S, 128), rand(B, Hkv, S, 128), rand(Hkv, P, 128), rand(Hkv, P, 128)
    w = torch.rand((B, Hkv, S), generator=gen, device="cuda")
    lens = torch.tensor([S, 333], dtype=torch.int32, device="cuda")
    lay = api.make_layout(B, Hq, Hkv, 128, 128, S, dt)
    out, w_out = torch.empty_like(q), torch.zeros_like(w)
    idx = torch.empty((B, Hkv, keep), dtype=torch.int32, device="cuda")
    ko, vo = (torch.empty((B, Hkv, keep, 128), dtype=dt, device="cuda") for _ in "kv")
    basis = torch.eye(128, device="cuda").repeat(Hkv, 1, 1)
    keys, eig, fit = rand(Hkv, 300, 128), torch.empty((Hkv, 128), device="cuda"), torch.empty((Hkv, 128, 128), device="cuda")
    one = api.make_layout(1, Hq, Hkv, 128, 128, S, dt)
    evict = lambda ws, **kw: api.loki_evict(lay, w, k, None, v, S, keep, 2, 10, ws, seq_lens=lens, klo_out=ko, v_out=vo, **kw)
    return {
        "weights": (api.dense_weights_workspace_bytes(lay, S),
                    lambda ws: api.dense_decode_weights(lay, q, k, v, S, lens, w, w_out, ws, out)),
        "evict": (api.loki_evict_workspace_bytes(lay, S, keep), evict),
        "evict_own_list": (api.loki_evict_workspace_bytes(lay, S, keep), lambda ws: evict(ws, out_idx=idx)),
        "shared": (api.dense_shared_workspace_bytes(lay, P, S),
                   lambda ws: api.dense_decode_shared(lay, q, kp, vp, P, k, v, S, lens, ws, out)),
        "shared_own_rows": (api.dense_shared_workspace_bytes(lay, 0, S),
                            lambda ws: api.dense_decode_shared(lay, q, None, None, 0, k, v, S, lens, ws, out)),
        "dense": (api.loki_workspace_bytes(lay, S, 0, 0, DENSE), lambda ws: api.dense_decode_step(lay, q, k, v, S, lens, ws, out)),
        "pca_attn": (api.loki_workspace_bytes(lay, S, 128, 0, -2), lambda ws: api.loki_pca_attn(lay, q, basis, k, v, S, 128, ws, out)),
        "pca_fit": (api.loki_pca_workspace_bytes(one, 300), lambda ws: api.loki_pca_fit(one, keys, 300, fit, eig, ws)),
    }


def test_every_workspace_has_room_for_them():
    """(no GPU) The smallest calls that keep anything in their workspace."""
    for dt in (torch.bfloat16, torch.float32):
        lay = api.make_layout(1, 1, 1, 128, 128, 1024, dt)
        assert api.dense_weights_workspace_bytes(lay, 1) > CTL
        assert api.loki_evict_workspace_bytes(lay, 1, 1) > CTL
        assert api.dense_shared_workspace_bytes(lay, 1, 0) > CTL and api.dense_shared_workspace_bytes(lay, 0, 1) > CTL
        assert api.loki_workspace_bytes(lay, 1024, 0, 0, DENSE) > CTL
        assert api.loki_workspace_bytes(lay, 1, 128, 0, -2) > CTL
        assert api.loki_pca_workspace_bytes(lay, 2) > CTL


def test_evict_workspace_grows_with_budget_and_length():
    """(no GPU) One of the largest S_max and budget serves all smaller ones; lists of the whole budget fit."""
    lay = api.make_layout(4, 8, 8, 128, 32, 16384, torch.bfloat16)
    lens, budgets = (1, 64, 700, 5000, 16384), (1, 63, 64, 1000, 16384, 100000)
    size = [[api.loki_evict_workspace_bytes(lay, S, n) for n in budgets] for S in lens]
    assert all(row == sorted(row) for row in size) and all(list(col) == sorted(col) for col in zip(*size))
    assert all(x >= 4 * 32 * n for row in size for x, n in zip(row, budgets))


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["weights", "evict", "evict_own_list", "shared", "shared_own_rows", "dense", "pca_attn", "pca_fit"])
def test_one_zeroed_workspace_for_all(name):
    print("case", name, flush=True)
    w = synth.Workload(name="control_words", B=1, Hq=8, Hkv=2, D=128, S=9000, dtype="bf16", d=32, k=900, seed=81)
    case = DeviceCase(w, synth.make_inputs(w))
    ref, ref_idx = case.run_loki(1, path=api.PATH_CLUSTER)
    need, call = _others()[name]
    ws = torch.zeros(max(need, api.loki_workspace_bytes(case.layout, w.S, w.d, w.k, 1)), dtype=torch.uint8, device="cuda")
    for turn in range(3):
        call(ws)
        torch.cuda.synchronize()
        # (before any block waits for what lies there)
        assert int(torch.count_nonzero(ws[:CTL])) == 0, turn
        out = torch.full((w.B, w.Hq, w.D), float("nan"), dtype=torch.bfloat16, device="cuda")
        idx = torch.full((w.B, w.Hkv, w.k), -7, dtype=torch.int32, device="cuda")
        api.loki_decode_attn(case.layout, case.q, case.P, case.klo, case.khi, case.v, w.S, w.d, w.k,
                             1 | api.PATH_CLUSTER | api.WORKSPACE_ZEROED, ws, out, idx)
        torch.cuda.synchronize()
        assert np.array_equal(out.float().cpu().numpy().astype(np.float64), ref) and np.array_equal(idx.cpu().numpy(), ref_idx)
        assert int(torch.count_nonzero(ws[:CTL])) == 0, turn


@pytest.mark.gpu
def test_a_graph_of_all_calls_around_a_step_on_one_zeroed_workspace():
    """Captured once: the other calls, then the step that vouches for the workspace; replayed, equal to eager every time."""
    w = synth.Workload(name="control_words", B=2, Hq=16, Hkv=4, D=128, S=5000, dtype="bf16", d=32, k=500, seed=82)
    case = DeviceCase(w, synth.make_inputs(w))
    ref, _ = case.run_loki(1, path=api.PATH_CLUSTER)
    others = {n: c for n, c in _others().items() if n != "pca_fit"}
    ws = torch.zeros(max([n for n, _ in others.values()] + [api.loki_workspace_bytes(case.layout, w.S, w.d, w.k, 1)]), dtype=torch.uint8,
                     device="cuda")
    out = torch.empty((w.B, w.Hq, w.D), dtype=torch.bfloat16, device="cuda")
    for _, call in others.values():
        call(ws)
    torch.cuda.synchronize()
    assert int(torch.count_nonzero(ws[:CTL])) == 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _, call in others.values():
            call(ws)
        api.loki_decode_attn(case.layout, case.q, case.P, case.klo, case.khi, case.v, w.S, w.d, w.k,
                             1 | api.PATH_CLUSTER | api.WORKSPACE_ZEROED, ws, out, None)
    for _ in range(3):
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out.float().cpu().numpy().astype(np.float64), ref)
        assert int(torch.count_nonzero(ws[:CTL])) == 0
