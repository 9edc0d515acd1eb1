"""The compressed-step operators as cases that can be timed and checked: a K/V cache held in 4 bits and the
attention that reads it, the attention weight its rows accumulate and the eviction of rows by it, and linear maps
in 8-bit integers.

A case is one pass through one operator (``op``):

* ``rows``     rows of K or V written into a 4-bit cache and read back as the values it holds.
* ``attend``   queries against a whole 4-bit cache: the attention rows and their log-sum-exp.
* ``weigh``    the attention weight every cached position gets from a set of queries, added to what it had.
* ``evict``    the positions that stay under a budget, and the caches compacted to them.
* ``linear``   activations to 8-bit integers with a scale per token, times weights in 8 bits with a scale per channel.

Formats: ``f32`` and ``bf16`` caches are [rows, H_kv, d_h].  A 4-bit cache tensor is a byte buffer: codes [H_kv, rows,
d_h / 2] (element 2t in the low half of byte t), and from the next multiple of 256 bytes on scale bytes [H_kv, rows,
d_h / 32].  A scale byte s stands for 2^(s - 127), 255 for a block of NaN; a code for sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6.
8-bit rows are padded with zeros to a multiple of 128 bytes.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# n_q_heads, n_kv_heads, head_dim of the framework's models
HEADS = {"toy": (4, 4, 64), "mini_dream": (7, 1, 128), "mini_llada": (8, 8, 128), "dream7b": (28, 4, 128),
         "llada8b": (32, 32, 128)}
# (N, K) of the linear maps of those models: Q or O, Q | K of grouped heads, gate or up, down
MAPS = [(256, 256), (1024, 1024), (4096, 4096), (8192, 4096), (12288, 4096), (4096, 12288), (3584, 3584), (4096, 3584),
        (18944, 3584), (3584, 18944)]
PAGE = 64


def _attend(heads, Mq, n, B=1, dtype="bf16", ragged=False, paged=False):
    return {"op": "attend", "heads": heads, "dtype": dtype, "B": B, "Mq": Mq, "n": n, "ragged": ragged, "paged": paged}


def _rows(heads, M, cache_rows, dtype="bf16"):
    return {"op": "rows", "heads": heads, "dtype": dtype, "M": M, "cache_rows": cache_rows}


def _weigh(heads, Mq, n, B=1, dtype="bf16", cache="bf16", ragged=False, paged=False):
    return {"op": "weigh", "heads": heads, "dtype": dtype, "cache": cache, "B": B, "Mq": Mq, "n": n, "ragged": ragged,
            "paged": paged}


def _evict(heads, n, keep, first, last, B=1, cache="bf16", ragged=False, paged=False):
    return {"op": "evict", "heads": heads, "cache": cache, "B": B, "n": n, "keep": keep, "first": first, "last": last,
            "ragged": ragged, "paged": paged}


def _linear(M, N, K, dtype="bf16"):
    return {"op": "linear", "dtype": dtype, "M": M, "N": N, "K": K}


def listed():
    cases = [
        # a float32 model of two narrow layers, one query: latency is all
        ("attend_toy_f32", _attend("toy", 1, 96, dtype="f32")),
        # an adaptive step over a long prompt: floor(0.1 * 512) rows against 4608 cached ones
        ("attend_adaptive_long", _attend("llada8b", 51, 4608)),
        # one query per sequence, grouped heads, sequences of different lengths in pages: a served batch
        ("attend_grouped_batch", _attend("dream7b", 1, 4099, B=16, ragged=True, paged=True)),
        # the first step of a long document, every row a query
        ("attend_refresh_long", _attend("llada8b", 4608, 4608)),
        # an adaptive step's selected rows scattered into the cache
        ("rows_adaptive", _rows("llada8b", 64, 768)),
        # the prompt and response of sixteen sequences
        ("rows_batch", _rows("llada8b", 12288, 12288)),
        # what the selected rows of an adaptive step look at
        ("weigh_adaptive", _weigh("llada8b", 64, 768)),
        # a response refresh over a long prompt, cache in 4 bits
        ("weigh_refresh_long", _weigh("llada8b", 512, 4608, cache="kv4")),
        # a float32 model's cache halved, the response kept
        ("evict_toy_f32", _evict("toy", 96, 64, 4, 32, cache="f32")),
        # sixteen long prompts halved, their responses kept
        ("evict_batch_long", _evict("llada8b", 4608, 2304, 4, 512, B=16, ragged=True)),
        # gate projection of an adaptive step's rows: the weight stream
        ("linear_adaptive", _linear(64, 12288, 4096)),
        # the same map of sixteen whole sequences
        ("linear_batch", _linear(12288, 12288, 4096)),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm; odd ones as likely as even ones."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(("rows", "attend", "weigh", "evict", "linear"))
    heads = rng.choice(sorted(HEADS))
    H_q, H_kv, d_h = HEADS[heads]
    dtype = "f32" if heads == "toy" or rng.random() < 0.15 else "bf16"
    ragged, paged = rng.random() < 0.5, rng.random() < 0.3
    if op == "rows":
        cache_rows = _log(rng, 1, 16384)
        return _rows(heads, _log(rng, 1, min(cache_rows, 12288)), cache_rows, dtype)
    if op == "linear":
        N, K = rng.choice(MAPS)
        if rng.random() < 0.3:
            N, K = N - rng.randrange(1, 64), K - rng.randrange(1, 64)
        M = _log(rng, 1, min(12288, 12288 * 12288 * 4096 // (N * K)))
        return _linear(M, N, K, dtype)
    B = _log(rng, 1, 16)
    if op == "evict":
        n = _log(rng, 16, min(32768, 16 * 4608 * 4096 // (B * H_kv * d_h)))
        keep = rng.randrange(1, n + 1)
        last = rng.randrange(0, keep + 1) // 2
        first = min(4, keep - last)
        cache = dtype if rng.random() < 0.6 else "kv4"
        return _evict(heads, n, keep, first, last, B, cache, ragged, paged)
    n = _log(rng, 1, 32768)
    B = min(B, max(1, 16 * 4608 // n))
    most = (4608 if dtype == "bf16" else 576) * 4608 * 32   # queries x keys x heads
    Mq = _log(rng, 1, max(1, min(4608, most // (B * n * H_q))))
    if op == "attend":
        return _attend(heads, Mq, n, B, dtype, ragged, paged)
    return _weigh(heads, Mq, n, B, dtype, rng.choice((dtype, "kv4")), ragged, paged)


# ---- inputs ------------------------------------------------------------------------------------------
def _align256(v):
    return (v + 255) // 256 * 256


def _kv4_pack(x, H_kv, d_h):
    """float32 [rows, H_kv * d_h] -> the byte buffer of a 4-bit cache tensor."""
    rows = x.shape[0]
    x = x.view(rows, H_kv, d_h // 32, 32).permute(1, 0, 2, 3)
    amax = x.abs().amax(-1)
    f, e = torch.frexp(amax)
    e = torch.where(f <= 0.75, e - 3, e - 2)
    e = torch.where(amax > 0, e, -125).clamp(-125, 125)
    m = torch.ldexp(x.abs(), -e[..., None].to(torch.int32))
    code = ((m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5)).to(torch.uint8)
    code = code + 8 * torch.signbit(x).to(torch.uint8)
    code = code.reshape(H_kv, rows, d_h)
    codes = (code[..., 0::2] + 16 * code[..., 1::2]).reshape(-1)
    scales = (e + 127).to(torch.uint8).reshape(-1)
    buf = torch.zeros(_align256(codes.numel()) + scales.numel(), dtype=torch.uint8, device=x.device)
    buf[:codes.numel()] = codes
    buf[_align256(codes.numel()):] = scales
    return buf


def _kv4_unpack(buf, rows, H_kv, d_h):
    """The values of a 4-bit cache tensor, float32 [rows, H_kv, d_h]."""
    count = H_kv * rows * d_h // 2
    codes = buf[:count].view(H_kv, rows, d_h // 2)
    scales = buf[_align256(count):_align256(count) + H_kv * rows * d_h // 32].view(H_kv, rows, d_h // 32)
    code = torch.stack((codes & 15, codes >> 4), -1).view(H_kv, rows, d_h // 32, 32)
    mag = (code & 7).float()
    mag = torch.where(mag < 4, mag * 0.5, torch.where(mag < 6, mag - 2, 2 * mag - 8))
    val = torch.where(code >= 8, -mag, mag)
    scale = torch.exp2(scales.float() - 127)
    val = torch.where(scales[..., None] == 255, torch.nan, val * scale[..., None])
    return val.view(H_kv, rows, d_h).permute(1, 0, 2)


def _pad128(k):
    return (k + 127) // 128 * 128


def _to_int8(x):
    """Rows of float32 x as 8-bit integers, padded, and their scales."""
    amax = x.abs().amax(1)
    r = torch.where(amax > 0, 127.0 / amax, torch.zeros_like(amax))
    q = torch.zeros(x.shape[0], _pad128(x.shape[1]), dtype=torch.int8, device=x.device)
    q[:, :x.shape[1]] = torch.round(x * r[:, None]).to(torch.int8)
    return q, amax / 127.0


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _features(g, rows, H, d_h):
    """Keys or values as projections give them: a few channels of a head are larger than the rest."""
    x = _randn(g, rows, H, d_h)
    return (x * torch.exp(0.6 * _randn(g, H, d_h))).view(rows, H * d_h)


def _places(case, g):
    """(cache rows, row_map or None, lens or None) of a batch of cached sequences."""
    B, n = case["B"], case["n"]
    rows, row_map, lens = B * n, None, None
    if case["paged"]:
        pages = (n + PAGE - 1) // PAGE
        pool = B * pages + 3
        table = torch.randperm(pool, generator=g, device="cuda")[:B * pages].view(B, pages)
        row_map = (table[:, :, None] * PAGE + torch.arange(PAGE, device="cuda")).view(B, pages * PAGE)[:, :n]
        row_map = row_map.to(torch.int32).contiguous()
        rows = pool * PAGE
    if case["ragged"]:
        lens = torch.randint((n + 1) // 2, n + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    return rows, row_map, lens


def _cache(fmt, x, H_kv, d_h):
    return _kv4_pack(x, H_kv, d_h) if fmt == "kv4" else x.to(DTYPES[fmt])


def prepare(case, seed):
    g = _gen(seed)
    st = {"case": case}
    if case["op"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        x = _randn(g, M, K) * torch.exp(0.5 * _randn(g, K))
        st["x"] = x.to(DTYPES[case["dtype"]])
        st["w"], st["w_scale"] = _to_int8((0.02 * _randn(g, N, K)).to(torch.bfloat16).float())
        return st
    H_q, H_kv, d_h = HEADS[case["heads"]]
    if case["op"] == "rows":
        M, R = case["M"], case["cache_rows"]
        st["x"] = _features(g, M, H_kv, d_h).to(DTYPES[case["dtype"]])
        st["rows"] = torch.randperm(R, generator=g, device="cuda")[:M].to(torch.int32)
        st["cache"] = torch.zeros(_align256(H_kv * R * d_h // 2) + H_kv * R * d_h // 32, dtype=torch.uint8, device="cuda")
        return st
    B, n = case["B"], case["n"]
    st["cache_rows"], st["row_map"], st["lens"] = _places(case, g)
    R = st["cache_rows"]
    if case["op"] == "evict":
        for name in ("k", "v"):
            st[name] = _cache(case["cache"], _features(g, R, H_kv, d_h), H_kv, d_h)
            shape = (_align256(H_kv * B * case["keep"] * d_h // 2) + H_kv * B * case["keep"] * d_h // 32,) \
                if case["cache"] == "kv4" else (B * case["keep"], H_kv * d_h)
            st[name + "_out"] = torch.zeros(shape, dtype=st[name].dtype, device="cuda")
        u = torch.rand(B, n, generator=g, device="cuda")
        st["acc"] = torch.exp(1.5 * _randn(g, B, n)) * (u > 0.05)   # a few positions nobody looked at
        return st
    q = _randn(g, B, case["Mq"], H_q, d_h) * (1.0 + torch.rand(H_q, 1, generator=g, device="cuda"))
    st["q"] = q.view(B, case["Mq"], H_q * d_h).to(DTYPES[case["dtype"]])
    fmt = "kv4" if case["op"] == "attend" else case["cache"]
    st["k"] = _cache(fmt, _features(g, R, H_kv, d_h), H_kv, d_h)
    if case["op"] == "attend":
        st["v"] = _cache(fmt, _features(g, R, H_kv, d_h), H_kv, d_h)
    else:
        st["acc"] = torch.rand(B, n, generator=g, device="cuda")
    return st


# ---- one pass ------------------------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(st):
    from paper_2506_06295_amd import binding as L
    c = st["case"]
    if c["op"] == "linear":
        a, a_scale = L.op_quant8(c["dtype"], st["x"])
        return L.op_linear_i8(c["dtype"], a, a_scale, st["w"], st["w_scale"], c["K"])
    H_q, H_kv, d_h = HEADS[c["heads"]]
    if c["op"] == "rows":
        L.op_kv4_store(c["dtype"], st["x"], st["cache"], c["cache_rows"], H_kv, d_h, rows=st["rows"])
        return L.op_kv4_load(c["dtype"], st["cache"], c["cache_rows"], H_kv, d_h, rows=st["rows"])
    where = {"lens": st["lens"], "row_map": st["row_map"]}
    if c["op"] == "attend":
        return L.op_attention_kv4(c["dtype"], st["q"], st["k"], st["v"], st["cache_rows"], c["n"], H_q, H_kv, d_h,
                                  with_lse=True, **where)
    if c["op"] == "weigh":
        return L.op_attention_weights(c["dtype"], c["cache"], st["q"], st["k"], st["cache_rows"], c["n"], H_q, H_kv, d_h,
                                      acc=st["acc"], **where)
    kept, kept_rows, lens, acc = L.op_evict(st["acc"], c["keep"], st["cache_rows"], first=c["first"], last=c["last"], **where)
    L.op_compact(c["cache"], kept_rows, st["cache_rows"], H_kv, d_h, st["k"], st["k_out"], st["v"], st["v_out"])
    k, v = st["k_out"], st["v_out"]
    if c["cache"] == "kv4":
        k, v = (L.op_kv4_load("f32", t, c["B"] * c["keep"], H_kv, d_h) for t in (k, v))
    return kept, lens, acc, k, v


def _values(fmt, t, rows, H_kv, d_h):
    return _kv4_unpack(t, rows, H_kv, d_h) if fmt == "kv4" else t.float().view(rows, H_kv, d_h)


def _sequence(st, b):
    """Cache rows of sequence b's positions, and how many of them there are."""
    c = st["case"]
    n = c["n"]
    idx = st["row_map"][b].long() if st["row_map"] is not None else torch.arange(b * n, (b + 1) * n, device="cuda")
    there = torch.arange(n, device="cuda") < (st["lens"][b] if st["lens"] is not None else n)
    return idx, there


def _scores(q, k, there):
    """[H_q, Mq, n] scaled scores of float32 q [Mq, H_q, d_h] against k [n, H_kv, d_h], -inf where there is no key."""
    G = q.shape[1] // k.shape[1]
    k = k.permute(1, 2, 0).repeat_interleave(G, 0)
    s = torch.matmul(q.permute(1, 0, 2), k) / math.sqrt(q.shape[2])
    return torch.where(there, s, -torch.inf)


def _run_plain(st):
    c = st["case"]
    if c["op"] == "linear":
        K = c["K"]
        q, a_scale = _to_int8(st["x"].float())
        out = torch.matmul(q[:, :K].float(), st["w"][:, :K].float().t())
        return (out * a_scale[:, None] * st["w_scale"]).to(DTYPES[c["dtype"]])
    H_q, H_kv, d_h = HEADS[c["heads"]]
    if c["op"] == "rows":
        M = c["M"]
        buf = _kv4_pack(st["x"].float(), H_kv, d_h)
        return _kv4_unpack(buf, M, H_kv, d_h).reshape(M, H_kv * d_h).to(DTYPES[c["dtype"]])
    B, n = c["B"], c["n"]
    if c["op"] == "evict":
        return _evict_plain(st)
    R = st["cache_rows"]
    k = _values("kv4" if c["op"] == "attend" else c["cache"], st["k"], R, H_kv, d_h)
    q = st["q"].float().view(B, c["Mq"], H_q, d_h)
    if c["op"] == "weigh":
        acc = st["acc"].clone()
        for b in range(B):
            idx, there = _sequence(st, b)
            s = _scores(q[b], k[idx], there)
            p = torch.exp(s - s.amax(-1, keepdim=True))
            acc[b] += (p / p.sum(-1, keepdim=True)).sum((0, 1))
        return acc
    v = _values("kv4", st["v"], R, H_kv, d_h)
    out, lse = [], []
    for b in range(B):
        idx, there = _sequence(st, b)
        s = _scores(q[b], k[idx], there)
        m = s.amax(-1, keepdim=True)
        p = torch.exp(s - m)
        l = p.sum(-1, keepdim=True)
        o = torch.matmul(p, v[idx].permute(1, 0, 2).repeat_interleave(H_q // H_kv, 0)) / l
        out.append(o.permute(1, 0, 2).reshape(c["Mq"], H_q * d_h))
        lse.append((m + torch.log(l))[..., 0].t())
    return torch.stack(out).to(DTYPES[c["dtype"]]), torch.stack(lse).contiguous()


def _evict_plain(st):
    c = st["case"]
    B, n, keep = c["B"], c["n"], c["keep"]
    H_q, H_kv, d_h = HEADS[c["heads"]]
    kept = torch.full((B, keep), -1, dtype=torch.int32, device="cuda")
    acc = torch.zeros(B, keep, device="cuda")
    new_lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    src = [_values(c["cache"], st[t], st["cache_rows"], H_kv, d_h) for t in ("k", "v")] if c["cache"] == "kv4" else \
        [st[t].view(-1, H_kv, d_h) for t in ("k", "v")]
    dst = [torch.zeros(B * keep, H_kv, d_h, dtype=s.dtype, device="cuda") for s in src]
    pos = torch.arange(n, device="cuda")
    for b in range(B):
        idx, there = _sequence(st, b)
        length = int(there.sum())
        rank = torch.where((pos < c["first"]) | (pos >= length - c["last"]), torch.inf, st["acc"][b])
        rank = torch.where(there, rank, -torch.inf)
        order = torch.sort(rank, descending=True, stable=True).indices[:min(keep, length)]
        order = torch.sort(order).values
        m = order.numel()
        kept[b, :m] = order.to(torch.int32)
        acc[b, :m] = st["acc"][b, order]
        new_lens[b] = m
        for s, d in zip(src, dst):
            d[b * keep:b * keep + m] = s[idx[order]]
    return kept, new_lens, acc, *(d.view(B * keep, H_kv * d_h) for d in dst)


# ---- what a pass cannot do without -----------------------------------------------------------------------
def work(case):
    c = case
    esz = 2 if c.get("dtype", c.get("cache")) == "bf16" else 4
    if c["op"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        return {"bytes": float(M * K * esz + N * K + 4 * N + M * N * esz), "flops": 2.0 * M * N * K}
    H_q, H_kv, d_h = HEADS[c["heads"]]
    width = H_kv * d_h
    if c["op"] == "rows":  # in, the 4-bit rows, out
        return {"bytes": c["M"] * width * (2.0 * esz + 17 / 32), "flops": 0.0}
    B, n = c["B"], c["n"]
    there = B * n * (0.75 if c["ragged"] else 1.0)
    fmt = "kv4" if c["op"] == "attend" else c["cache"]
    row = width * {"kv4": 17 / 32, "bf16": 2.0, "f32": 4.0}[fmt]
    maps = there * 4.0 if c["paged"] else 0.0
    if c["op"] == "evict":
        kept = min(there, B * c["keep"])
        return {"bytes": there * 4.0 + maps + kept * (4 * row + 8), "flops": 0.0}
    rows = B * c["Mq"] * H_q
    flops = 2.0 * rows * there / B * d_h
    if c["op"] == "attend":
        return {"bytes": 2 * there * row + maps + 2 * rows * d_h * esz + rows * 4.0, "flops": 2 * flops}
    return {"bytes": there * row + maps + rows * d_h * esz + B * n * 8.0, "flops": flops}


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_nearest(x, H_kv, d_h):
    """Every block of 32 rounded to the nearest level times the smallest power of two that holds the block."""
    y = x.double().view(-1, 32)
    top = y.abs().amax(1, keepdim=True)
    step = torch.full_like(top, 2.0 ** -125)
    for e in range(-124, 126):
        step = torch.where(top > 6.0 * step, torch.full_like(top, 2.0 ** e), step)
    levels = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    u = (y.abs() / step).clamp(max=6.0)
    hi = torch.bucketize(u, levels).clamp(max=7)
    lo = (hi - 1).clamp(min=0)
    down, up = u - levels[lo], levels[hi] - u
    pick = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return torch.where(y < 0, -levels[pick], levels[pick]).mul(step).view(x.shape)


def _exact_values(fmt, t, rows, H_kv, d_h):
    if fmt != "kv4":
        return t.double().view(rows, H_kv, d_h)
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float64, device=t.device)
    half = d_h // 2
    raw = t[:H_kv * rows * half].long().view(H_kv, rows, half)
    val = torch.empty(H_kv, rows, d_h, dtype=torch.float64, device=t.device)
    val[:, :, 0::2] = table[raw % 16]
    val[:, :, 1::2] = table[raw // 16]
    start = -(-H_kv * rows * half // 256) * 256
    e = t[start:start + H_kv * rows * (d_h // 32)].double().view(H_kv, rows, d_h // 32) - 127
    return (val * torch.pow(2.0, e).repeat_interleave(32, 2)).transpose(0, 1)


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    if c["op"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        x = st["x"].double()
        top = x.abs().amax(1, keepdim=True)
        r = (127 / torch.where(top > 0, top, torch.ones_like(top))).float().double()
        q = torch.round((x * r).float().double())   # the product is a float32 number by definition
        w = st["w"][:, :K].double()
        out = torch.empty(M, N, dtype=torch.float64, device="cuda")
        for i in range(0, M, 2048):
            out[i:i + 2048] = (q[i:i + 2048] @ w.t()) * (top[i:i + 2048] / 127) * st["w_scale"].double()
        return out
    H_q, H_kv, d_h = HEADS[c["heads"]]
    if c["op"] == "rows":
        return _exact_nearest(st["x"], H_kv, d_h)
    B, n = c["B"], c["n"]
    R = st["cache_rows"]
    row_map = st["row_map"].cpu().numpy() if st["row_map"] is not None else np.arange(B * n).reshape(B, n)
    lens = st["lens"].cpu().numpy() if st["lens"] is not None else np.full(B, n)
    if c["op"] == "evict":
        keep = c["keep"]
        weight = st["acc"].double().cpu().numpy()
        kept = np.full((B, keep), -1, np.int32)
        acc = np.zeros((B, keep))
        k, v = (_exact_values(c["cache"], st[t], R, H_kv, d_h).reshape(R, -1) for t in ("k", "v"))
        k_out, v_out = (torch.zeros(B * keep, H_kv * d_h, dtype=torch.float64, device="cuda") for _ in range(2))
        left = np.minimum(lens, keep).astype(np.int32)
        for b in range(B):
            L = int(lens[b])
            j = np.arange(L)
            safe = (j < c["first"]) | (j >= L - c["last"])
            order = np.lexsort((j, -weight[b, :L], ~safe))[:keep]
            order.sort()
            kept[b, :len(order)] = order
            acc[b, :len(order)] = weight[b, order]
            rows = torch.from_numpy(row_map[b, order].astype(np.int64)).cuda()
            k_out[b * keep:b * keep + len(order)] = k[rows]
            v_out[b * keep:b * keep + len(order)] = v[rows]
        return (torch.from_numpy(kept).cuda(), torch.from_numpy(left).cuda(), torch.from_numpy(acc).cuda(), k_out, v_out)
    fmt = "kv4" if c["op"] == "attend" else c["cache"]
    q = st["q"].double().view(B, c["Mq"], H_q, d_h)
    out = torch.zeros(B, c["Mq"], H_q, d_h, dtype=torch.float64, device="cuda")
    lse = torch.full((B, c["Mq"], H_q), -math.inf, dtype=torch.float64, device="cuda")
    acc = st["acc"].double() if c["op"] == "weigh" else None
    k = _exact_values(fmt, st["k"], R, H_kv, d_h)
    v = _exact_values(fmt, st["v"], R, H_kv, d_h) if c["op"] == "attend" else None
    for b in range(B):
        L = int(lens[b])
        rows = torch.from_numpy(row_map[b, :L].astype(np.int64)).cuda()
        kb = k[rows]
        vb = v[rows] if v is not None else None
        for a in range(H_q):
            h = a // (H_q // H_kv)
            s = q[b, :, a] @ kb[:, h].t().contiguous() / math.sqrt(d_h)
            z = torch.logsumexp(s, 1)
            p = torch.exp(s - z[:, None])
            if acc is not None:
                acc[b, :L] += p.sum(0)
            else:
                out[b, :, a] = p @ vb[:, h].contiguous()
                lse[b, :, a] = z
    return acc if acc is not None else (out.view(B, c["Mq"], H_q * d_h), lse)
