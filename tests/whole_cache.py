"""Caches held whole for the tests: rows in 64 bits to and from the 4-bit form, and attention over what a token sees."""
import math

import torch

from paper_2406_02542_amd import api
from tests.attention_bound import DT, attend64


def columns(word):
    """The columns whose codes word `word` of a row holds, in the order of its 4-bit fields."""
    return [32 * g + 2 * word + i for i in range(2) for g in range(4)]


def pack(codes):
    """int32 words [.., 16] of codes [.., 128]."""
    words = torch.zeros(codes.shape[:-1] + (16,), dtype=torch.int64, device=codes.device)
    for m in range(16):
        for at, col in enumerate(columns(m)):
            words[..., m] |= codes[..., col].long() << (4 * at)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).int()


def unpack(words):
    codes = torch.empty(words.shape[:-1] + (128,), dtype=torch.int64, device=words.device)
    for m in range(16):
        for at, col in enumerate(columns(m)):
            codes[..., col] = words[..., m].long() >> (4 * at) & 15
    return codes


def quantise64(x):
    """(codes [.., 128], scales fp16 [.., 4, 2]) of x by the definition, in 64 bits."""
    g = x.double().unflatten(-1, (4, 32))
    lo, hi = g.amin(-1), g.amax(-1)
    scales = torch.stack([((hi - lo) / 15).half(), lo.half()], dim=-1)
    step, low = scales[..., 0].double()[..., None], scales[..., 1].double()[..., None]
    codes = torch.where(step > 0, torch.round((g - low) / torch.where(step > 0, step, 1.0)), 0.0).clamp(0, 15)
    return codes.flatten(-2).long(), scales


def values64(codes, scales):
    s = scales.double()[..., None, :]
    return (s[..., 1] + codes.unflatten(-1, (4, 32)).double() * s[..., 0]).flatten(-2)


def paged(x, table, n_pages, page_rows, fill):
    """x [B, H, S, ..] as a pool [n_pages, H, page_rows, ..]; what no row takes holds `fill`."""
    B, H, S = x.shape[:3]
    pool = torch.full((n_pages, H, page_rows) + x.shape[3:], fill, dtype=x.dtype, device=x.device)
    for b in range(B):
        for p in range((S + page_rows - 1) // page_rows):
            rows = x[b, :, p * page_rows:(p + 1) * page_rows]
            pool[int(table[b, p]), :, :rows.shape[1]] = rows
    return pool


def make_table(B, S_cap, page_rows, gen, spare=3):
    """A page table of pages in no order, with some that no sequence has: (table, n_pages)."""
    each = (S_cap + page_rows - 1) // page_rows + 1
    n = B * each + spare
    return torch.randperm(n, generator=gen, device="cuda")[:B * each].view(B, each).int(), n


def seen(L, window, sinks):
    """The rows that a token which sees L rows attends over."""
    s = torch.arange(L)
    return (s[(s < sinks) | (s >= L - window)] if window else s).cuda()


def reference(q, k, v, lens, window, sinks, scales=None, units=None):
    """(out, bound) [B, m, Hq, 128] in 64 bits; k, v [B, H, S, 128]; scales: (k's, v's) of caches in 4 bits; units: only those (b, KV head)."""
    B, m, Hq, _ = q.shape
    G = Hq // k.shape[1]
    out, bound = (torch.zeros(q.shape, dtype=torch.float64, device=q.device) for _ in range(2))
    for b in range(B):
        for j in range(m):
            rows = seen(int(lens[b, j]), window, sinks)
            for h in range(k.shape[1]):
                if units is not None and (b, h) not in units:
                    continue
                at = (b, j, slice(h * G, (h + 1) * G))
                if scales is None:
                    step = 2.0 ** -16 if q.dtype == torch.bfloat16 else 0.0
                    out[at], _, bound[at], _ = attend64(q[at], k[b, h, rows], v[b, h, rows], step)
                else:
                    out[at], bound[at] = attend_4bits(q[at], k[b, h, rows], v[b, h, rows], *(s[b, h, rows] for s in scales), q.dtype)
    return out, bound


def attend_4bits(q, k, v, ks, vs, dtype):
    """attend64 with what a kernel that multiplies codes may be off.  A logit is the sum over four groups of 16 step (a product of q with
    codes as 1 + n / 16, begun with minus the group's sum of q) and lowest times that sum: 33 roundings of at most 3 sum |q|, the
    sums' own 34, each product's one: together at most D + 2 of (64 step + 2 |lowest|) sum |q|.  An output is a sum of
    products of 16 p step with 1 + n / 16 less that of 16 p step, and p lowest: relative to 48 p step + |p lowest|.  The weights
    enter in two bf16 terms (2^-16), in 32 bits in three (2^-23)."""
    n, D = k.shape
    q = q.double()
    if n == 0:
        return torch.zeros_like(q), torch.zeros_like(q)
    p = torch.softmax(q @ k.t().contiguous() / math.sqrt(D), dim=-1)
    sums = q.abs().unflatten(-1, (4, 32)).sum(-1)
    ks, vs = ks.double(), vs.double()
    size = float((sums @ (64 * ks[..., 0] + 2 * ks[..., 1].abs()).t().contiguous()).max()) / math.sqrt(D)
    chain = (n / 4 + 64) * 2.0 ** -24
    rel = 2 * ((D + 2) * 2.0 ** -24 * size + 2.0 ** -22) + chain
    mass = (p @ (48 * vs[..., 0] + vs[..., 1].abs())).repeat_interleave(32, dim=-1)
    return p @ v, mass * (rel + chain + (2.0 ** -16 if dtype == torch.bfloat16 else 2.0 ** -23))


class Case:
    """A cache with rows in it, contiguous or paged, in the storage type or in 4 bits; what it stands for in 64 bits."""

    def __init__(self, B, Hq, Hkv, S_cap, dtype, page_rows=0, bits=0, seed=0, fill=float("nan")):
        self.gen = gen = torch.Generator(device="cuda").manual_seed(seed + 17 * S_cap + B)
        self.lay = api.make_layout(B, Hq, Hkv, 128, 128, S_cap, DT[dtype])
        self.dt, self.page_rows = DT[dtype], page_rows
        x = [torch.randn((B, Hkv, S_cap, 128), generator=gen, device="cuda") * torch.linspace(0.3, 3.0, 128, device="cuda") + 0.2 for _ in "kv"]
        self.table, n_pages = make_table(B, S_cap, page_rows, gen) if page_rows else (None, 0)
        self.scales = None
        if bits:
            parts = [quantise64(y) for y in x]
            self.k, self.v = (values64(*p) for p in parts)
            self.scales = [p[1] for p in parts]
            held = [pack(parts[0][0]), pack(parts[1][0]), *self.scales]
        else:
            self.k, self.v = (y.to(self.dt) for y in x)
            held = [self.k, self.v]
        if page_rows:  # what no row takes: bytes that are NaN as scales and as rows
            held = [paged(y, self.table, n_pages, page_rows, -1 if y.dtype == torch.int32 else fill) for y in held]
        else:
            held = [y.clone() for y in held]
        self.held = held
        self.cache = api.Cache(self.lay, *held, page_table=self.table)

    def queries(self, m, scale=2.0):
        return (scale * torch.randn((self.lay.B, m, self.lay.Hq, 128), generator=self.gen, device="cuda")).to(self.dt)

    def spoil(self, b, rows):
        """Rows that no call may read hold NaN from here on (and their pages' entries name none, where a page holds nothing else)."""
        rows = list(rows)
        for y in self.held:
            bad = -1 if y.dtype == torch.int32 else float("nan")
            if not self.page_rows:
                y[b, :, rows] = bad
                continue
            for s in rows:
                y[int(self.table[b, s // self.page_rows]), :, s % self.page_rows] = bad

    def attend(self, q, lens, S_max, window=0, sinks=0, ws=None):
        m = q.shape[1]
        need = api.dense_cache_workspace_bytes(self.lay, self.cache, S_max, m, window, sinks)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda") if ws is None else ws
        out = torch.full_like(q, float("nan"))
        api.dense_decode_cache(self.lay, self.cache, q, S_max, ws, out, seq_lens=lens, queries_per_seq=m, window=window, sinks=sinks)
        return out
