"""Rows that begin more than 2^32 bytes (in 4 bits 2^31 words) into a cache: appended, read back and attended over as those of a small cache of the same tokens are."""
import pytest
import torch

from paper_2406_02542_amd import api
from tests.attention_bound import DT, worst
from tests.whole_cache import reference, unpack, values64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,bits,page_rows,B,Hkv,S_cap", [
    ("bf16", 4, 0, 9, 4, 4 << 20), ("bf16", 4, 256, 9, 4, 4 << 20), ("f32", 4, 0, 5, 4, 4 << 20), ("bf16", 0, 256, 3, 2, 3 << 20), ("f32", 0, 0, 3, 2, 2 << 20)])
def test_rows_past_32_bits(dtype, bits, page_rows, B, Hkv, S_cap):
    print("case", dtype, bits, page_rows, B, Hkv, S_cap, flush=True)
    dt, n, Hq = DT[dtype], 40, 2 * Hkv
    far = S_cap - 50
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.randn((B, n, Hkv, 128), generator=gen, device="cuda").to(dt) for _ in "kv")
    q = torch.randn((B, 1, Hq, 128), generator=gen, device="cuda").to(dt)

    def run(first, S, table=None, n_pages=0):
        """The tokens' rows first .. of a cache of S rows: as they are held, as they are read back, and the attention over them."""
        lay = api.make_layout(B, Hq, Hkv, 128, 128, S, dt)
        cache = api.alloc_whole_cache(lay, bits == 4, table, page_rows if n_pages else 0, n_pages)
        rows = (first + torch.arange(n, device="cuda"))[None].repeat(B, 1).int()
        api.loki_append(lay, cache, rows, k, v)
        back = [torch.full((B, Hkv, n, 128), 9.0, dtype=dt, device="cuda") for _ in "kv"]
        api.loki_read_rows(lay, cache, rows, *back)
        out, lens = torch.full_like(q, float("nan")), torch.full((B, 1), first + n, dtype=torch.int32, device="cuda")
        ws = torch.empty(api.dense_cache_workspace_bytes(lay, cache, S, 1, n, 0), dtype=torch.uint8, device="cuda")
        api.dense_decode_cache(lay, cache, q, S, ws, out, seq_lens=lens, window=n)
        torch.cuda.synchronize()
        at = torch.arange(first, first + n, device="cuda")
        if table is None:
            held = [None if t is None else t[:, :, at] for t in cache.tensors[:4]]
        else:
            pages = table[:, at // page_rows].long()
            held = [None if t is None else t[pages, :, at % page_rows].transpose(1, 2) for t in cache.tensors[:4]]
        return held, back, out

    table = n_pages = None
    if page_rows:  # the last pages of every sequence at the pool's end, sequence 0's last of all
        each = S_cap // page_rows
        n_pages = B * each
        table = torch.arange(n_pages, dtype=torch.int32, device="cuda").view(B, each).flip(0).contiguous()
    near = run(0, n)
    held, back, out = run(far, S_cap, table, n_pages or 0)
    for x, y in zip((*held, *back), (*near[0], *near[1])):
        assert x is None or torch.equal(x, y)
    if bits:
        keys, values = (values64(unpack(near[0][i]), near[0][2 + i]) for i in range(2))
    else:
        keys, values = near[1]
        assert torch.equal(keys, k.transpose(1, 2)) and torch.equal(values, v.transpose(1, 2))
    ref, bound = reference(q, keys, values, torch.full((B, 1), n), 0, 0, near[0][2:] if bits else None)
    assert worst(out, ref, bound, dtype) <= 0
    assert worst(near[2], ref, bound, dtype) <= 0
