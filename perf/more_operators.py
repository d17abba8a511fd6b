"""Performance cases of the operators on whole caches, contiguous or paged, in the storage type or in 4 bits, and the operators
in their plain form.

A case is a dict of plain values.  Its "kind" says which operator it calls:

  append  loki_append: keys and values of new tokens into a paged cache, the keys (and the queries, which come out beside it)
          turned by their positions on the way.  Into a cache in 4 bits the pass also reads the rows back (loki_read_rows)
  window  dense_decode_cache: attention over the last rows of a cache and its first few, for one new token of every sequence, for
          several, or for chunks of prompts
  q4      dense_decode_cache over a cache held in 4 bits

`own` says how a pass is computed: False, by elementary torch operations in 32 bits; True, by the library.  Both take the same
inputs and give the same outputs.

A row in 4 bits is four groups of 32 columns with a step and a lowest value each, both fp16: a value is lowest + code * step.
"""
import math

import numpy as np
import torch

own = False

D = 128
NOISE = 0.01
PLANTED = 64  # rows of a unit that its queries look for


def listed():
    return [
        # One user chatting with a Llama-2-7B-shaped model: one token's key and value into its page. Launch and latency count.
        _append("append_b1", 1, 1, 32, 32, "bf16", 4096, far=4000),
        # A serving batch with grouped queries, sequences of all lengths, pairs side by side, frequencies scaled for far positions.
        _append("append_b64", 64, 1, 64, 8, "bf16", 16384, interleaved=True, scaled=True, far=120000),
        # A chunk of prompts out of one projection, some of them shorter than the chunk.
        _append("append_prefill", 8, 2048, 32, 8, "bf16", 4096, fused=True, padded=True),
        # Prompts into a cache in 4 bits, odd sizes, half of each head turned.
        _append("append_q4", 4, 1111, 32, 8, "bf16", 2048, R=64, bits=4, padded=True),
        # One sequence, grouped queries: the last 1024 rows and 4 sinks of a contiguous cache.
        _window("window_b1", 1, 1, 32, 8, 8192, 1024, 4, "bf16"),
        # A serving batch on pages, sequences of all lengths, most of them longer than the window.
        _window("window_b64", 64, 1, 64, 8, 16384, 4096, 4, "bf16", page=256, ragged=True),
        # Chunks of two prompts behind what is cached, one of them shorter.
        _window("window_prefill", 2, 2048, 32, 8, 8192, 4096, 4, "bf16", page=256, padded=True),
        # 32 bits, three drafted tokens each, one query head per KV head, odd sizes.
        _window("window_f32", 5, 3, 24, 24, 2311, 700, 1, "f32", ragged=True),
        # One sequence on a cache in 4 bits.
        _q4("q4_b1", 1, 1, 32, 8, 8192, "bf16"),
        # The grouped-query model's batch at its full length, on pages, sequences of all lengths.
        _q4("q4_gqa", 16, 1, 32, 8, 16384, "bf16", page=256, ragged=True),
        # Four drafted tokens of each sequence.
        _q4("q4_tokens", 8, 4, 64, 8, 8192, "bf16", page=64, ragged=True),
        # 32 bits beside the cache, one query head per KV head, odd sizes.
        _q4("q4_f32", 5, 1, 24, 24, 2311, "f32", ragged=True),
    ]


def _append(name, B, n, Hq, Hkv, dtype, S, R=128, page=256, bits=0, interleaved=False, scaled=False, far=0, fused=False, padded=False):
    return _named(name, {"kind": "append", "B": B, "n": n, "Hq": Hq, "Hkv": Hkv, "dtype": dtype, "S": S, "R": R, "page": page, "bits": bits,
                         "interleaved": interleaved, "scaled": scaled, "far": far, "fused": fused, "padded": padded})


def _window(name, B, m, Hq, Hkv, S, window, sinks, dtype, page=0, ragged=False, padded=False):
    return _named(name, {"kind": "window", "B": B, "m": m, "Hq": Hq, "Hkv": Hkv, "S": S, "window": window, "sinks": sinks, "dtype": dtype,
                         "page": page, "ragged": ragged, "padded": padded})


def _q4(name, B, m, Hq, Hkv, S, dtype, window=0, sinks=0, page=0, ragged=False):
    return _named(name, {"kind": "q4", "B": B, "m": m, "Hq": Hq, "Hkv": Hkv, "S": S, "window": window, "sinks": sinks, "dtype": dtype,
                         "page": page, "ragged": ragged, "padded": False})


def _named(name, c):
    return dict(c, name=name) if name else c


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges, at most the bytes, operations and logits of the largest listed ones."""
    while True:
        kind = rng.choice(["append", "window", "window", "q4"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        Hkv, G = rng.choice([(32, 1), (24, 1), (16, 2), (8, 4), (8, 4), (8, 8), (4, 8)])
        page = rng.choice([256, 256, 64, 16])
        if kind == "append":
            n = rng.choice([1, _log(rng, 2, 4096)])
            c = _append("", _log(rng, 1, 64), n, Hkv * G, Hkv, dtype, n + _log(rng, 1, 4096), R=rng.choice([128, 128, 96, 64, 32]), page=page,
                        bits=rng.choice([0, 4]), interleaved=rng.random() < 0.4, scaled=rng.random() < 0.4,
                        far=rng.choice([0, _log(rng, 1000, 1000000)]), fused=rng.random() < 0.5, padded=n > 1 and rng.random() < 0.5)
        elif kind == "window":
            m = rng.choice([1, 1, _log(rng, 2, 16), _log(rng, 16, 2048)])
            S = m + _log(rng, 32, 16384)
            c = _window("", _log(rng, 1, 64), m, Hkv * G, Hkv, S, rng.choice([S, _log(rng, 16, 8192)]), rng.choice([0, 1, 4, 64]), dtype,
                        page=rng.choice([0, page]), ragged=m <= 16 and rng.random() < 0.6, padded=m > 16 and rng.random() < 0.5)
        else:
            m = rng.choice([1, 1, rng.randrange(2, 9)])
            S = m + _log(rng, 100, 32768)
            c = _q4("", _log(rng, 1, 64), m, Hkv * G, Hkv, S, dtype, window=rng.choice([0, 0, _log(rng, 16, 8192)]), sinks=rng.choice([0, 4]),
                    page=rng.choice([0, page]), ragged=rng.random() < 0.6)
            if not c["window"]:
                c["sinks"] = 0
        w = work(c)
        if kind != "append" and (c["B"] * c["Hq"] * c["m"] * c["S"] > 1.1e9 or c["B"] * c["Hkv"] * c["S"] > 8.4e6):
            continue  # what the plain form holds at a time
        if w["bytes"] <= 1.0e9 and w["flops"] <= 2.0e11 / (8 if dtype == "f32" else 1):
            return c


# ---- inputs -------------------------------------------------------------------------------------
def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _gen(seed, tag):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + tag * 7919 + 41) & 0x7FFFFFFFFFFF)


def _normal(shape, seed, tag, dtype=torch.float32):
    return torch.randn(shape, generator=_gen(seed, tag), device="cuda", dtype=torch.float32).to(dtype)


def _uniform(shape, seed, tag):
    return torch.rand(shape, generator=_gen(seed, tag), device="cuda", dtype=torch.float32)


def _direction():
    sig = torch.exp(-torch.arange(D, dtype=torch.float64) / 20.0)
    return (sig / sig.norm()).float().cuda()


def _keys(shape, seed, tag):
    """Keys with the library's synthetic spectrum; PLANTED rows of every unit lie along one direction."""
    i = torch.arange(D, dtype=torch.float64)
    k = _normal((*shape, D), seed, tag)
    k.mul_(torch.sqrt(torch.exp(-i / 20.0) ** 2 + NOISE).float().cuda())
    flat = k.view(-1, shape[-1], D)
    pos = (_uniform((flat.shape[0], min(PLANTED, shape[-1])), seed, tag + 50) * shape[-1]).long()
    flat.scatter_add_(1, pos[..., None].expand(-1, -1, D), (4.0 * _direction()).expand(*pos.shape, D).contiguous())
    return k


def _queries(shape, seed, tag):
    """Queries that look along that direction, some more and some less."""
    return _normal((*shape, D), seed, tag) + 32.0 * _uniform((*shape, 1), seed, tag + 50) * _direction()


def _frequencies(R, scaled):
    """Radians per position of the R / 2 pairs; scaled: long wavelengths eightfold, short ones as they were."""
    base = 500000.0 if scaled else 10000.0
    f = base ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)
    if scaled:
        turns = 8192.0 * f / (2.0 * math.pi)
        mix = ((turns - 1.0) / 3.0).clamp(0.0, 1.0)
        f = f * mix + f / 8.0 * (1.0 - mix)
    return f.cuda()


def _table(c, seed):
    """The sequences' pages, in no order, and how many there are."""
    each = (c["S"] + c["page"] - 1) // c["page"]
    order = np.random.default_rng([int(seed), 33]).permutation(c["B"] * each).astype(np.int32)
    return torch.from_numpy(order.reshape(c["B"], each)).cuda(), c["B"] * each


def _split_words(x):
    """Codes and scales of x [.., D] in 4 bits: the code of column 32 g + 2 m + i in bits 16 i + 4 g of word m; (step, lowest) per group."""
    g = x.unflatten(-1, (4, 32))
    lo, hi = g.amin(dim=-1, keepdim=True), g.amax(dim=-1, keepdim=True)
    scales = torch.cat([(hi - lo) / 15.0, lo], dim=-1).half()
    step, low = scales[..., :1].float(), scales[..., 1:].float()
    codes = torch.where(step > 0, torch.round((g - low) / step), 0.0).clamp_(0, 15).to(torch.int32)
    pairs = codes.unflatten(-1, (16, 2))  # [.., g, m, i]
    shift = (4 * torch.arange(4, device="cuda")[:, None, None] + 16 * torch.arange(2, device="cuda")).int()
    return (pairs << shift).sum(dim=(-3, -1), dtype=torch.int64).to(torch.int32), scales


def _as_pool(x, table, pages, page):
    """x [B, H, S, ..] by pages [n_pages, H, page, ..]; rows behind S are zeros."""
    B, H, S = x.shape[:3]
    each = table.shape[1]
    pool = torch.zeros((pages, H, page, *x.shape[3:]), dtype=x.dtype, device="cuda")
    full = torch.zeros((B, H, each * page, *x.shape[3:]), dtype=x.dtype, device="cuda")
    full[:, :, :S] = x
    pool[table.long().flatten()] = full.unflatten(2, (each, page)).transpose(1, 2).flatten(0, 1)
    return pool


def _append_inputs(c, seed):
    B, n, Hq, H, dt = c["B"], c["n"], c["Hq"], c["Hkv"], _dtype(c)
    x = {"freqs": _frequencies(c["R"], c["scaled"])}
    if c["fused"]:  # one projection's output
        qkv = _normal((B, n, (Hq + 2 * H) * D), seed, 1, dt)
        parts = [(0, Hq), (Hq, H), (Hq + H, H)]
        x["q"], x["k"], x["v"] = (qkv[..., a * D:(a + h) * D].unflatten(-1, (h, D)) for a, h in parts)
    else:
        x["q"], x["k"], x["v"] = (_normal((B, n, h, D), seed, t, dt) for t, h in ((1, Hq), (2, H), (3, H)))
    rng = np.random.default_rng([int(seed), 34])
    held = rng.integers(0, c["S"] - n + 1, size=(B, 1))  # rows that the sequences hold already
    j = np.arange(n)[None]
    new = rng.integers(n // 2, n + 1, size=(B, 1)) if c["padded"] else np.full((B, 1), n)
    x["rows"] = torch.from_numpy(np.where(j < new, held + j, -1).astype(np.int32)).cuda()
    first = rng.integers(0, c["far"] + 1, size=(B, 1))
    x["positions"] = torch.from_numpy((first + held + j).astype(np.int32)).cuda()
    x["table"], pages = _table(c, seed)
    x["q_out"] = torch.empty((B, n, Hq, D), dtype=dt, device="cuda")
    if c["bits"]:
        for t in ("k", "v"):
            x[t + "_pool"] = torch.zeros((pages, H, c["page"], D // 8), dtype=torch.int32, device="cuda")
            x[t + "_scales"] = torch.zeros((pages, H, c["page"], 4, 2), dtype=torch.float16, device="cuda")
            x[t + "_back"] = torch.zeros((B, H, n, D), dtype=dt, device="cuda")
    else:
        for t in ("k", "v"):
            x[t + "_pool"] = torch.zeros((pages, H, c["page"], D), dtype=dt, device="cuda")
    return x


def _lens(c, seed):
    """Rows that every new token sees, itself among them: sequences of S rows, or of S / 4 to S; padded: the last tokens of some are none."""
    B, m, S = c["B"], c["m"], c["S"]
    rng = np.random.default_rng([int(seed), 35])
    total = np.full(B, S)
    if c["ragged"]:
        total = rng.integers(max(m, S // 4), S + 1, size=B)
        total[0] = S
    lens = total[:, None] - (m - 1) + np.arange(m)[None]
    if c["padded"]:
        lens = np.where(np.arange(m)[None] < rng.integers((m + 1) // 2, m + 1, size=(B, 1)), lens, 0)
    return torch.from_numpy(lens.astype(np.int32)).cuda()


def _window_inputs(c, seed):
    B, H, S, dt = c["B"], c["Hkv"], c["S"], _dtype(c)
    x = {"lens": _lens(c, seed), "q": _queries((B, c["m"], c["Hq"]), seed, 3).to(dt)}
    x["out"] = torch.empty((B, c["m"], c["Hq"], D), dtype=dt, device="cuda")
    k, v = _keys((B, H, S), seed, 1), _normal((B, H, S, D), seed, 2, dt)
    parts = {"k": k.to(dt), "v": v}
    if c["kind"] == "q4":
        parts["k"], parts["k_scales"] = _split_words(k)
        parts["v"], parts["v_scales"] = _split_words(v.float())
    del k, v
    x["table"] = None
    if c["page"]:
        x["table"], pages = _table(c, seed)
        parts = {t: _as_pool(p, x["table"], pages, c["page"]) for t, p in parts.items()}
    return {**x, **parts}


_INPUTS = {"append": _append_inputs, "window": _window_inputs, "q4": _window_inputs}


def prepare(case, seed):
    return {"c": case, **_INPUTS[case["kind"]](case, seed)}


# ---- the library's calls ------------------------------------------------------------------------
def _plan(s):
    """The layout, the cache and the workspace, which a program makes once."""
    from paper_2406_02542_amd import api
    c = s["c"]
    lay = api.make_layout(c["B"], c["Hq"], c["Hkv"], D, D, c["S"], _dtype(c))
    k, v = ("k_pool", "v_pool") if c["kind"] == "append" else ("k", "v")
    cache = api.Cache(lay, s[k], s[v], k_scales=s.get("k_scales"), v_scales=s.get("v_scales"), page_table=s["table"])
    need = 0
    if c["kind"] != "append":
        need = api.dense_cache_workspace_bytes(lay, cache, c["S"], queries_per_seq=c["m"], window=c["window"], sinks=c["sinks"])
    return api, lay, cache, torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")


def _run_own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    api, lay, cache, ws = s["plan"]
    c = s["c"]
    if c["kind"] == "append":
        api.loki_append(lay, cache, s["rows"], k=s["k"], v=s["v"], positions=s["positions"], frequencies=s["freqs"], q=s["q"],
                        q_out=s["q_out"], interleaved=c["interleaved"])
        if c["bits"]:
            api.loki_read_rows(lay, cache, s["rows"], s["k_back"], s["v_back"])
            return {"q": s["q_out"], "k": s["k_back"], "v": s["v_back"]}
        return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}
    api.dense_decode_cache(lay, cache, s["q"], c["S"], ws, s["out"], seq_lens=s["lens"], queries_per_seq=c["m"], window=c["window"],
                           sinks=c["sinks"])
    return {"out": s["out"]}


# ---- the plain forms ----------------------------------------------------------------------------
def _turn(x, cos, sin, R, interleaved):
    """x [B, n, H, D] with the first R columns of every head turned, in 32 bits."""
    x = x.float()
    if interleaved:
        a, b = x[..., 0:R:2], x[..., 1:R:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = x[..., :R // 2], x[..., R // 2:R]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, x[..., R:]], dim=-1)


def _in_4_bits(x, dtype):
    """What x [.., D] is in a cache in 4 bits; the codes in 64 bits, because of values next to a border."""
    g = x.unflatten(-1, (4, 32))
    lo, hi = g.amin(dim=-1, keepdim=True), g.amax(dim=-1, keepdim=True)
    step, low = ((hi - lo) / 15.0).half().double(), lo.half().double()
    codes = torch.where(step > 0, torch.round((g.double() - low) / step), 0.0).clamp_(0, 15)
    return (low + codes * step).flatten(-2).to(dtype)


def _plain_append(s):
    c, R = s["c"], s["c"]["R"]
    angle = s["positions"].double()[..., None, None] * s["freqs"]  # far positions need 64 bits
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    q = _turn(s["q"], cos, sin, R, c["interleaved"]).to(s["q"].dtype)
    k = _turn(s["k"], cos, sin, R, c["interleaved"])
    there = (s["rows"] >= 0)[:, None, :, None]
    if c["bits"]:
        back = {t: torch.where(there, _in_4_bits(x, s["q"].dtype).transpose(1, 2), s[t + "_back"]) for t, x in (("k", k), ("v", s["v"].float()))}
        return {"q": q, **back}
    b, j = torch.nonzero(s["rows"] >= 0, as_tuple=True)
    row = s["rows"][b, j].long()
    page = s["table"][b, row // c["page"]].long()
    s["k_pool"][page, :, row % c["page"]] = k[b, j].to(s["q"].dtype)
    s["v_pool"][page, :, row % c["page"]] = s["v"][b, j]
    return {"q": q, "k": s["k_pool"], "v": s["v_pool"]}


def _unpaged(pool, table, S):
    """[B, H, S, ..] out of a pool [n_pages, H, page, ..]."""
    if table is None:
        return pool
    return pool[table.long()].transpose(1, 2).flatten(2, 3)[:, :, :S]


def _values(words, scales):
    """fp32 values [.., D] of a cache in 4 bits."""
    shift = (4 * torch.arange(4, device="cuda")[:, None, None] + 16 * torch.arange(2, device="cuda")).int()
    codes = ((words[..., None, :, None] >> shift) & 15).flatten(-2).float()
    return (codes * scales[..., :1].float() + scales[..., 1:].float()).flatten(-2)


def _plain_attention(s):
    c = s["c"]
    B, m, H, S, G = c["B"], c["m"], c["Hkv"], c["S"], c["Hq"] // c["Hkv"]
    k, v = _unpaged(s["k"], s["table"], S), _unpaged(s["v"], s["table"], S)
    if c["kind"] == "q4":
        k = _values(k, _unpaged(s["k_scales"], s["table"], S))
        v = _values(v, _unpaged(s["v_scales"], s["table"], S))
    q = s["q"].float().view(B, m, H, G, D).permute(0, 2, 1, 3, 4).reshape(B, H, m * G, D)
    a = torch.matmul(q, k.float().transpose(2, 3).contiguous()).view(B, H, m, G, S).mul_(1.0 / math.sqrt(D))
    pos, n = torch.arange(S, device="cuda"), s["lens"][..., None]
    seen = pos < n
    if c["window"]:
        seen = seen & ((pos < c["sinks"]) | (pos >= n - c["window"]))
    a.masked_fill_(~seen[:, None, :, None], -math.inf)
    a = a.sub_(a.amax(dim=-1, keepdim=True).clamp_(min=-1e30)).exp_()
    total = a.sum(dim=-1, keepdim=True)
    o = torch.matmul(a.view(B, H, m * G, S), v.float()).view(B, H, m, G, D) / torch.where(total > 0, total, 1.0)
    return {"out": o.permute(0, 2, 1, 3, 4).reshape(B, m, c["Hq"], D).to(s["q"].dtype)}


def run(s):
    if own:
        return _run_own(s)
    return _plain_append(s) if s["c"]["kind"] == "append" else _plain_attention(s)


# ---- what a pass cannot do without --------------------------------------------------------------
def _seen(c):
    """(rows that a KV head reads, pairs of a query head and a row) of a batch, on average over the lengths."""
    B, m, S = c["B"], c["m"], c["S"]
    W = c["window"] + c["sinks"] if c["window"] else S
    totals = np.linspace(max(m, S // 4), S, 65) if c["ragged"] else np.asarray([float(S)])
    real = 0.75 * m if c["padded"] else m
    rows = np.minimum(totals - (m - real), W + real - 1).mean()
    ends = totals[:, None] - (m - 1) + np.linspace(0.0, real - 1.0, 65)[None]
    return B * rows, B * real * np.minimum(ends, W).mean()


def work(case):
    c, e = case, 4 if case["dtype"] == "f32" else 2
    B, H = c["B"], c["Hkv"]
    if c["kind"] == "append":
        tokens = B * c["n"]
        kept = tokens * (0.75 if c["padded"] else 1.0)
        cached = kept * 2 * H * (80 if c["bits"] else D * e)
        return {"bytes": 2 * tokens * c["Hq"] * D * e + kept * 2 * H * D * e * (2 if c["bits"] else 1) + cached * (2 if c["bits"] else 1) + tokens * 8,
                "flops": 3 * tokens * (c["Hq"] + H) * c["R"]}
    rows, pairs = _seen(c)
    row_bytes = 160 if c["kind"] == "q4" else 2 * D * e
    return {"bytes": rows * H * row_bytes + 2 * B * c["m"] * c["Hq"] * D * e + 4 * B * c["m"], "flops": 4.0 * pairs * c["Hq"] * D}


# ---- the same in 64 bits ------------------------------------------------------------------------
def _grid_of_16(x):
    """x [.., D] in 64 bits on each group's 16 values."""
    parts = []
    for g in range(4):
        y = x[..., 32 * g:32 * g + 32]
        low = y.min(dim=-1, keepdim=True).values
        step = ((y.max(dim=-1, keepdim=True).values - low) / 15).to(torch.float16).double()
        low = low.to(torch.float16).double()
        n = torch.round((y - low) / torch.where(step == 0, 1.0, step)).clamp(0, 15)
        parts.append(torch.where(step == 0, low.expand_as(y), low + n * step))
    return torch.cat(parts, dim=-1)


def _exact_append(c, x):
    """Each pair as a complex number times exp(i position frequency); rows one sequence at a time."""
    R = c["R"]
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), x["positions"].double()[:, :, None] * x["freqs"][None, None])
    turned = {}
    for name in ("q", "k"):
        t = x[name].double().clone()
        first, second = (slice(0, R, 2), slice(1, R, 2)) if c["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
        z = torch.complex(t[..., first].contiguous(), t[..., second].contiguous()) * turn[:, :, None, :]
        t[..., first], t[..., second] = z.real, z.imag
        turned[name] = t
    outs = {"q": turned["q"]}
    for name, new in (("k", turned["k"]), ("v", x["v"].double())):
        full = x[name + ("_back" if c["bits"] else "_pool")].double()
        for b in range(c["B"]):
            rows = x["rows"][b].cpu().numpy()
            n = int((rows >= 0).sum())
            if c["bits"]:
                full[b, :, :n] = _grid_of_16(new[b, :n]).transpose(0, 1)
                continue
            for p in range(rows[0] // c["page"], (rows[n - 1] // c["page"] if n else -1) + 1):
                a, z = max(rows[0], p * c["page"]), min(rows[0] + n, (p + 1) * c["page"])
                full[int(x["table"][b, p]), :, a - p * c["page"]:z - p * c["page"]] = new[b, a - rows[0]:z - rows[0]].transpose(0, 1)
        outs[name] = full
    return outs


def _exact_rows(c, x, name, b, h):
    """Rows 0 .. S of one head in 64 bits."""
    def rows(t):
        return t[b, h] if x["table"] is None else t[x["table"][b].long(), h].flatten(0, 1)[:c["S"]]
    y = rows(x[name])
    if c["kind"] != "q4":
        return y.double()
    out = torch.empty((c["S"], D), dtype=torch.float64, device="cuda")
    scales = rows(x[name + "_scales"]).double()
    for g in range(4):
        for i in range(2):
            out[:, 32 * g + i:32 * g + 32:2] = scales[:, g, 1:] + ((y >> (4 * g + 16 * i)) & 15).double() * scales[:, g, :1]
    return out


def _exact_attention(c, x):
    G, m = c["Hq"] // c["Hkv"], c["m"]
    out = torch.zeros((c["B"], m, c["Hq"], D), dtype=torch.float64, device="cuda")
    lens = x["lens"].cpu().numpy()
    pos = torch.arange(c["S"], device="cuda")
    for b in range(c["B"]):
        real = int((lens[b] > 0).sum())  # (the padded tokens are the last)
        top = int(lens[b].max())
        ends = x["lens"][b, :real, None]
        hidden = pos[:top] >= ends
        if c["window"]:
            hidden = hidden | ((pos[:top] >= c["sinks"]) & (pos[:top] < ends - c["window"]))
        for h in range(c["Hkv"]):
            k, v = (_exact_rows(c, x, t, b, h)[:top] for t in ("k", "v"))
            kt = k.t().contiguous()
            for g in range(h * G, h * G + G):
                a = (x["q"][b, :real, g].double() @ kt / math.sqrt(D)).masked_fill(hidden, -math.inf)
                out[b, :real, g] = torch.softmax(a, dim=-1) @ v
    return {"out": out}


def exact(case, seed):
    x = _INPUTS[case["kind"]](case, seed)
    return _exact_append(case, x) if case["kind"] == "append" else _exact_attention(case, x)
