"""loki_evict against a plain selection and gather: equal, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2406_02542_amd import api
from tests.attention_bound import DT

pytestmark = pytest.mark.gpu


def kept_rows(w, n, budget, sinks, recent):
    """The rows that go on, of one unit's totals w[:n], ascending."""
    if n <= budget:
        return np.arange(n)
    middle = np.arange(sinks, n - recent)
    best = middle[np.lexsort((middle, -w[middle]))[:budget - sinks - recent]]
    return np.sort(np.concatenate([np.arange(sinks), best, np.arange(n - recent, n)]))


def weights(kind, B, H, cap, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    u = torch.rand((B, H, cap), generator=gen, device="cuda")
    if kind == "totals":  # as attention leaves them: few large, many small, some never looked at
        w = u.pow(8) * 16
        return torch.where(torch.rand((B, H, cap), generator=gen, device="cuda") < 0.3, 0.0, w)
    if kind == "equal":
        return torch.full((B, H, cap), 0.25, device="cuda")
    if kind == "zero":
        return torch.zeros((B, H, cap), device="cuda")
    if kind == "few":  # many ties at every level
        return (u * 5).floor()
    if kind == "signed":
        w = (u - 0.5) * 2.0 ** (torch.rand((B, H, cap), generator=gen, device="cuda") * 200 - 100)
        w[..., ::7] = float("inf")
        w[..., 3::11] = -float("inf")
        w[..., 5::13] = -0.0
        return w
    if kind == "close":  # the same leading bits, told apart by the last ones
        return 1.0 + (u * 1000).floor() * 2.0 ** -23
    raise ValueError(kind)


def check(B, H, cap, S_max, lens, budget, sinks, recent, dtype, d=128, kind="totals", into=None, page_rows=0, ragged=True, lens_in_place=False,
          seed=1):
    print("case", B, H, cap, S_max, lens[:4], budget, sinks, recent, dtype, d, kind, into, page_rows, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DT[dtype]
    w = weights(kind, B, H, cap, seed + 1)
    lay = api.make_layout(B, H, H, 128, d, cap, dt)
    if page_rows:
        per = -(-S_max // page_rows)
        n_pages = B * per + 2
        table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))[:B * per].to(torch.int32).reshape(B, per)
        lead = (n_pages, H, page_rows)
        paged = dict(page_table=table.cuda(), page_rows=page_rows, n_pages=n_pages)
    else:
        lead, paged = (B, H, cap), {}
    cache = [torch.randint(-30000, 30000, (*lead, x), generator=gen, device="cuda").to(dt) if x else None for x in (d, 128 - d, 128)]
    before, w_before = [t.clone() if t is not None else None for t in cache], w.clone()
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    lens_out = sl if lens_in_place else torch.full((B,), -9, dtype=torch.int32, device="cuda")
    idx = torch.full((B, H, budget), -9, dtype=torch.int32, device="cuda")
    ws = torch.full((api.loki_evict_workspace_bytes(lay, S_max, budget),), 255, dtype=torch.uint8, device="cuda")
    if into:
        outs = [torch.full((B, H, into, x), 3.0, dtype=dt, device="cuda") if x else None for x in (d, 128 - d, 128)]
        w_out = torch.full((B, H, into), -3.0, device="cuda")
        more = dict(klo_out=outs[0], khi_out=outs[1], v_out=outs[2], weights_out=w_out)
    else:
        more = {}
    api.loki_evict(lay, w, cache[0], cache[1], cache[2], S_max, budget, sinks, recent, ws, seq_lens=sl if ragged else None,
                   lens_out=lens_out, out_idx=idx, **more, **paged)
    torch.cuda.synchronize()
    assert lens_out.tolist() == [min(n, budget) for n in lens]

    def rows_of(t):  # [B, H, rows, x] in the sequences' order
        if not page_rows:
            return t
        return t[table.long().cuda().flatten()].reshape(B, per, H, page_rows, t.shape[-1]).transpose(1, 2).reshape(B, H, per * page_rows, -1)

    host = w_before.cpu().numpy()
    got = idx.cpu().numpy()
    for b in range(B):
        n = lens[b]
        for h in range(H):
            keep = kept_rows(host[b, h], n, budget, sinks, recent)
            m = len(keep)
            assert np.array_equal(got[b, h, :m], keep), (b, h)
            assert (got[b, h, m:] == -1).all()
            at = torch.from_numpy(keep).cuda()
            for i, t in enumerate(cache):
                if t is None:
                    continue
                src = rows_of(before[i])[b, h]
                if into:
                    assert torch.equal(outs[i][b, h, :m], src[at]) and bool((outs[i][b, h, m:] == 3.0).all())
                    assert torch.equal(t, before[i])
                else:
                    now = rows_of(t)[b, h]
                    assert torch.equal(now[:m], src[at]) and torch.equal(now[m:], src[m:])
            if into:
                assert torch.equal(w_out[b, h, :m], w_before[b, h][at]) and bool((w_out[b, h, m:] == -3.0).all())
            else:
                assert torch.equal(w[b, h, :m], w_before[b, h][at]) and torch.equal(w[b, h, m:], w_before[b, h, m:])
    if page_rows:  # pages of no sequence
        free = sorted(set(range(n_pages)) - set(table.flatten().tolist()))
        for i, t in enumerate(cache):
            assert t is None or torch.equal(t[free], before[i][free])


@pytest.mark.parametrize("into", [None, 200])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 24), ("f32", 128), ("f32", 32)])
@pytest.mark.parametrize("budget,sinks,recent", [(1, 0, 0), (1, 0, 1), (1, 1, 0), (64, 4, 16), (100, 0, 100), (100, 60, 40), (200, 3, 70)])
def test_budgets_and_caches(budget, sinks, recent, dtype, d, into):
    lens = [0, 1, budget, budget + 1, 333, 700]
    check(len(lens), 2, 710, 703, lens, budget, sinks, recent, dtype, d, into=into)


@pytest.mark.parametrize("kind", ["totals", "equal", "zero", "few", "signed", "close"])
@pytest.mark.parametrize("S,budget", [(257, 100), (5000, 1234), (40000, 7001), (70000, 9000)])  # keys in 4, 16, 48 and no registers a lane
def test_totals_of_every_kind(S, budget, kind):
    check(2, 2, S, S, [S, S - 13], budget, 4, 33, "bf16", 32, kind=kind, into=budget)


@pytest.mark.parametrize("S", [63, 64, 65, 1023, 1024, 1025, 4095, 4096, 4097, 16384, 16385, 49152, 49153])
def test_sizes_around_the_blocks(S):
    check(1, 1, S, S, [S], S - 1, 0, 1, "bf16", into=None)
    check(1, 2, S, S, [S], max(1, S // 3), 1, 2, "bf16", into=S, ragged=False)


@pytest.mark.parametrize("budget", [20, 511, 513, 1030, 2500])
def test_in_place_runs(budget):
    """Runs of 512 rows, the last one partial; sources in runs that have and have not been written yet."""
    check(3, 2, 3001, 3000, [3000, 2600, 514], budget, 2, 10, "bf16", 32)
    check(2, 2, 3001, 3000, [3000, 2600], budget, 2, 10, "f32", 128, kind="few")


@pytest.mark.parametrize("into", [None, 500])
@pytest.mark.parametrize("dtype,d", [("bf16", 32), ("f32", 128)])
def test_pages(dtype, d, into):
    check(3, 2, 1500, 1400, [1400, 257, 900], 300, 4, 50, dtype, d, into=into, page_rows=256)


@pytest.mark.parametrize("into", [None, 300])
@pytest.mark.parametrize("budget", [300, 301, 5000])
def test_nothing_has_to_go(budget, into):
    """A bound at or beyond the rows there can be: everything stays, a shorter cache takes S_max rows."""
    check(3, 2, 310, 300, [300, 17, 0], budget, 4, 50, "bf16", 32, into=into)


def test_lengths_written_where_they_are_read():
    check(4, 3, 900, 900, [900, 10, 300, 301], 300, 4, 50, "bf16", 32, lens_in_place=True)


def test_large_batch():
    check(64, 8, 1100, 1100, [1100 - 7 * b for b in range(64)], 256, 4, 64, "bf16", into=256)
    check(64, 8, 1100, 1100, [1100 - 7 * b for b in range(64)], 256, 4, 64, "bf16")


def test_offsets_past_32_bits():
    """More than 2^32 bytes of keys in front of the last unit."""
    B, H, cap, S, budget = 2, 8, 1200000, 600, 100
    lay = api.make_layout(B, H, H, 128, 128, cap, torch.bfloat16)
    k, v = (torch.empty((B, H, cap, 128), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    w = torch.zeros((B, H, cap), device="cuda")
    k[:, :, :S], v[:, :, :S] = (torch.randn((B, H, S, 128), device="cuda").bfloat16() for _ in "kv")
    w[:, :, :S] = torch.rand((B, H, S), device="cuda")
    old, ow = k[:, :, :S].clone(), w[:, :, :S].cpu().numpy()
    ws = torch.empty(api.loki_evict_workspace_bytes(lay, S, budget), dtype=torch.uint8, device="cuda")
    api.loki_evict(lay, w, k, None, v, S, budget, 4, 20, ws)
    torch.cuda.synchronize()
    for b in range(B):
        for h in range(H):
            at = torch.from_numpy(kept_rows(ow[b, h], S, budget, 4, 20)).cuda()
            assert torch.equal(k[b, h, :budget], old[b, h][at])


def test_replayed_graph():
    B, H, S, budget = 2, 4, 2000, 300
    lay = api.make_layout(B, H, H, 128, 128, S, torch.bfloat16)
    k0, v0 = (torch.randn((B, H, S, 128), device="cuda").bfloat16() for _ in "kv")
    k, v, w = k0.clone(), v0.clone(), torch.zeros((B, H, S), device="cuda")
    ws = torch.empty(api.loki_evict_workspace_bytes(lay, S, budget), dtype=torch.uint8, device="cuda")
    idx = torch.empty((B, H, budget), dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        api.loki_evict(lay, w, k, None, v, S, budget, 4, 20, ws, out_idx=idx)
    for step in range(3):
        k.copy_(k0), v.copy_(v0)
        w.copy_(torch.rand((B, H, S), device="cuda"))
        host = w.cpu().numpy()
        graph.replay()
        torch.cuda.synchronize()
        for b in range(B):
            for h in range(H):
                keep = kept_rows(host[b, h], S, budget, 4, 20)
                assert np.array_equal(idx[b, h].cpu().numpy(), keep)
                assert torch.equal(v[b, h, :budget], v0[b, h][torch.from_numpy(keep).cuda()])


@pytest.mark.parametrize("into", [None, 900])
@pytest.mark.parametrize("page_rows", [0, 256])
@pytest.mark.parametrize("budget", [1, 100, 899, 900, 901, 40000])
def test_lists_of_the_workspace(budget, page_rows, into):
    """Without out_idx the lists lie in the workspace, no longer than the rows there can be; nothing behind it is written."""
    B, H, S, cap, lens = 3, 2, 900, 910, [900, 0, 333]
    print("case", budget, page_rows, into, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(budget + page_rows)
    lay = api.make_layout(B, H, H, 128, 32, cap, torch.bfloat16)
    w = weights("few", B, H, cap, budget)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda").bfloat16()
    paged, lead = {}, (B, H, cap)
    if page_rows:
        table = torch.randperm(12, generator=torch.Generator().manual_seed(3)).to(torch.int32).reshape(B, 4)
        paged, lead = dict(page_table=table.cuda(), page_rows=page_rows, n_pages=12), (12, H, page_rows)
    cache = [rand(*lead, x) for x in (32, 96, 128)]

    def rows_of(t):
        return t[table.long().cuda().flatten()].reshape(B, 4, H, page_rows, -1).transpose(1, 2).reshape(B, H, 4 * page_rows, -1) if page_rows else t

    before, w0 = [rows_of(t).clone() for t in cache], w.cpu().numpy()
    outs = [torch.zeros((B, H, into, x), dtype=torch.bfloat16, device="cuda") for x in (32, 96, 128)] if into else [None] * 3
    need = api.loki_evict_workspace_bytes(lay, S, budget)
    buf = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    recent = min(20, budget)
    api.loki_evict(lay, w, *cache, S, budget, 0, recent, buf[:need], seq_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                   klo_out=outs[0], khi_out=outs[1], v_out=outs[2], **paged)
    torch.cuda.synchronize()
    assert bool((buf[need:] == 255).all())
    for b, n in enumerate(lens):
        for h in range(H):
            at = torch.from_numpy(kept_rows(w0[b, h], n, budget, 0, recent)).cuda()
            for t, old, new in zip(cache, before, outs):
                got = new[b, h] if into else rows_of(t)[b, h]
                assert torch.equal(got[:len(at)], old[b, h][at])
