"""From the residual stream to token log probabilities in few bits, as cases that can be timed and checked: a norm with the residual's
addition whose rows leave in 8 or 4 bits, linear maps on 4-bit blocks, and what a row of logits says about tokens.

A case is one pass through one operator (``op``):

* ``norm``     a sublayer's output added to the residual stream, the sum's RMS norm in few bits: ``i8`` (8-bit integers, a
  scale per row) or ``mx4`` (4-bit floating point, a power of two per block of 32).  Returns the values the rows hold, and the sums.
* ``linear``   activations to 4-bit blocks, times weights held in 4-bit blocks.
* ``tokens``   log probabilities of given tokens, the entropy, and the likeliest tokens with theirs (equal logits: lower id first).

A 4-bit tensor is a byte buffer.  Codes [rows, Kp / 2], Kp = K rounded up to 256, zeros behind the K-th (element 2t in the low half of
byte t; a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6).  From the next multiple of 256 bytes on one scale byte s for 32 elements, which stands
for 2^(s - 127): [ceil(rows / 32), Kp / 256, 2, 32, 4], that of block 8 c + 2 j + b of row 32 g + r at [g, c, b, r, j].
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 9.999999747378752e-06   # 1e-5 as float32 has it
# widths and vocabularies of the framework's models; (N, K) of their linear maps: Q or O, Q | K of grouped heads, gate or up, down, head
WIDTHS = [256, 1024, 3584, 4096]
VOCABS = [1024, 126464, 152064]
MAPS = [(256, 256), (704, 256), (1024, 1024), (4096, 4096), (8192, 4096), (12288, 4096), (4096, 12288), (3584, 3584), (4096, 3584),
        (18944, 3584), (3584, 18944), (126464, 4096)]


def _norm(form, M, d, dtype="bf16", stream="bf16", rows=None):
    """M rows; rows: how many the stream has of which they are some, or None: all of them."""
    return {"op": "norm", "form": form, "M": M, "d": d, "dtype": dtype, "stream": stream, "rows": 0 if rows is None else rows}


def _linear(M, N, K, dtype="bf16"):
    return {"op": "linear", "M": M, "N": N, "K": K, "dtype": dtype}


def _tokens(M, vocab, given=1, top=8, dtype="f32", pad=0, banned=0):
    """pad: logits behind a row's last one; banned: tokens of a row at minus infinity."""
    return {"op": "tokens", "M": M, "vocab": vocab, "given": given, "top": top, "dtype": dtype, "pad": pad, "banned": banned}


def listed():
    cases = [
        # a float32 model's response of a few positions: latency is all
        ("norm_toy_f32", _norm("mx4", 8, 256, "f32", "f32")),
        # an adaptive step's selected rows, the stream in float32 as it is inside a step
        ("norm_adaptive", _norm("i8", 64, 4096, "bf16", "f32", rows=768)),
        # prompt and response of a model of odd width, for 4-bit maps
        ("norm_refresh", _norm("mx4", 1280, 3584)),
        # sixteen whole sequences
        ("norm_batch", _norm("i8", 12288, 4096)),
        # the smallest map of a float32 model
        ("linear_toy_f32", _linear(8, 256, 256, "f32")),
        # gate projection of an adaptive step's rows: the weight stream
        ("linear_adaptive", _linear(64, 12288, 4096)),
        # up projection of a prompt and its response
        ("linear_refresh", _linear(1280, 18944, 3584)),
        # gate projection of sixteen whole sequences
        ("linear_batch", _linear(12288, 12288, 4096)),
        # a small vocabulary: latency
        ("tokens_toy_f32", _tokens(32, 1024, given=1, top=4)),
        # one position, its twenty likeliest tokens, [MASK] and the like banned
        ("tokens_one", _tokens(1, 126464, given=1, top=20, banned=3)),
        # confidences, margins and entropies of a step's masked positions
        ("tokens_step", _tokens(64, 126464, given=1, top=2)),
        # scoring of whole documents, logits in bf16
        ("tokens_score", _tokens(4096, 152064, given=1, top=8, dtype="bf16")),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm; odd ones as likely as even ones."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(("norm", "linear", "tokens"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if op == "norm":
        d = rng.choice(WIDTHS)
        if rng.random() < 0.3:
            d -= rng.randrange(1, 64)
        M = _log(rng, 1, 12288)
        stream = "f32" if dtype == "f32" or rng.random() < 0.4 else "bf16"
        rows = _log(rng, M, 12288) if rng.random() < 0.4 else None
        return _norm(rng.choice(("i8", "mx4")), M, d, dtype, stream, rows)
    if op == "linear":
        N, K = rng.choice(MAPS)
        if rng.random() < 0.3:
            N, K = N - rng.randrange(1, 64), K - rng.randrange(1, 64)
        M = _log(rng, 1, min(12288, 12288 * 12288 * 4096 // (N * K)))
        return _linear(M, N, K, dtype)
    vocab = rng.choice(VOCABS) - (rng.randrange(1, 64) if rng.random() < 0.4 else 0)
    M = _log(rng, 1, min(16384, 4096 * 152064 // (vocab * (2 if dtype == "f32" else 1))))
    return _tokens(M, vocab, _log(rng, 1, 16), _log(rng, 1, 64), dtype, rng.choice((0, 0, 7, 64)), rng.choice((0, 0, 1, 300)))


# ---- inputs ------------------------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _align256(v):
    return (v + 255) // 256 * 256


def _mx4_parts(x):
    """Of float32 x [rows, 32 k] the exponent of every block and the index of every element's level."""
    y = x.view(x.shape[0], -1, 32)
    amax = y.abs().amax(-1)
    f, e = torch.frexp(amax)
    e = torch.where(f <= 0.75, e - 3, e - 2)
    e = torch.where(amax > 0, e, -125).clamp(-125, 125)
    m = torch.ldexp(y.abs(), -e[..., None].to(torch.int32))
    level = (m > 0.25).to(torch.uint8) + (m >= 0.75) + (m > 1.25) + (m >= 1.75) + (m > 2.5) + (m >= 3.5) + (m > 5)
    return e, level, torch.signbit(y)


def _mx4_magnitude(level):
    v = level.float()
    return torch.where(v < 4, v * 0.5, torch.where(v < 6, v - 2, 2 * v - 8))


def _mx4_round(x):
    """float32 x [rows, K] as the values that its 4-bit blocks hold."""
    K = x.shape[1]
    e, level, minus = _mx4_parts(torch.nn.functional.pad(x, (0, -K % 32)))
    v = torch.ldexp(_mx4_magnitude(level), e[..., None].to(torch.int32))
    return torch.where(minus, -v, v).flatten(1)[:, :K]


def _mx4_pack(x):
    """float32 x [rows, K] -> the byte buffer of a 4-bit tensor."""
    rows, K = x.shape
    e, level, minus = _mx4_parts(torch.nn.functional.pad(x, (0, -K % 256)))
    code = (level + 8 * minus.to(torch.uint8)).flatten(1)
    codes = (code[:, 0::2] + 16 * code[:, 1::2]).flatten()
    s = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, 0, 0, -rows % 32))
    s = s.view(s.shape[0] // 32, 32, s.shape[1] // 8, 4, 2).permute(0, 2, 4, 1, 3).flatten()   # [g, r, c, j, b] -> [g, c, b, r, j]
    buf = torch.zeros(_align256(codes.numel()) + s.numel(), dtype=torch.uint8, device=x.device)
    buf[:codes.numel()] = codes
    buf[_align256(codes.numel()):] = s
    return buf


def _mx4_unpack(buf, rows, K):
    """The values of a 4-bit tensor, float32 [rows, K]."""
    Kp = _align256(K)
    codes = buf[:rows * Kp // 2].view(rows, Kp // 2)
    code = torch.stack((codes & 15, codes >> 4), -1).view(rows, Kp // 32, 32)
    v = _mx4_magnitude(code & 7)
    v = torch.where(code >= 8, -v, v)
    s = buf[_align256(rows * Kp // 2):].view(-1, Kp // 256, 2, 32, 4).permute(0, 3, 1, 4, 2).reshape(-1, Kp // 32)[:rows]
    return torch.ldexp(v, s[..., None].to(torch.int32) - 127).view(rows, Kp)[:, :K]


def prepare(case, seed):
    g = _gen(seed)
    c, st = case, {"case": case}
    t = DTYPES[c["dtype"]]
    M = c["M"]
    if c["op"] == "linear":
        st["x"] = (_randn(g, M, c["K"]) * torch.exp(0.5 * _randn(g, c["K"]))).to(t)
        st["w"] = _mx4_pack((0.02 * _randn(g, c["N"], c["K"])).to(torch.bfloat16).float())
        return st
    if c["op"] == "norm":
        d, rows = c["d"], c["rows"] or M
        st["x"] = (0.3 * _randn(g, M, d)).to(t)
        st["stream"] = (_randn(g, rows, d) * torch.exp(0.6 * _randn(g, d))).to(DTYPES[c["stream"]])   # a few channels stand out
        st["gain"] = (1 + 0.1 * _randn(g, d)).to(t)
        pick = torch.randperm(rows, generator=g, device="cuda")[:M].sort().values
        st["row_idx"] = pick.to(torch.int32) if c["rows"] else None
        return st
    vocab, ld = c["vocab"], c["vocab"] + c["pad"]
    l = _randn(g, M, ld)
    l.mul_(2.0)
    peak = torch.randint(0, vocab, (M, 24), generator=g, device="cuda")
    l.scatter_add_(1, peak, 10 * torch.rand(M, 24, generator=g, device="cuda"))       # a few likely tokens
    if c["banned"]:
        l.scatter_(1, torch.randint(0, vocab, (M, c["banned"]), generator=g, device="cuda"), -math.inf)
    st["logits"] = l.to(t)[:, :vocab]
    given = torch.randint(0, vocab, (M, c["given"]), generator=g, device="cuda")
    given[:, 0] = peak[:, 0]
    st["given"] = given.to(torch.int32)
    return st


# ---- one pass ------------------------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(st):
    from paper_2506_06295_amd import binding as L
    c = st["case"]
    if c["op"] == "linear":
        a = L.op_quant_mx4(c["dtype"], st["x"])
        return L.op_linear_mx4(c["dtype"], a, c["M"], st["w"], c["N"], c["K"])
    if c["op"] == "norm":
        call = L.op_norm_quant8 if c["form"] == "i8" else L.op_norm_mx4
        *held, total = call(c["dtype"], st["stream"], st["gain"], EPS, x=st["x"], row_idx=st["row_idx"], stream_dtype=c["stream"])
        if c["form"] == "i8":
            return L.op_load8(c["dtype"], *held, c["d"]), total
        return L.op_mx4_load(c["dtype"], *held, c["M"], c["d"]), total
    logp, entropy, ids, top = L.op_logprobs(c["dtype"], st["logits"], tokens=st["given"], top_k=c["top"])
    return logp, entropy, ids, top


def _run_plain(st):
    c = st["case"]
    if c["op"] == "linear":
        w = _mx4_unpack(st["w"], c["N"], c["K"])
        return torch.matmul(_mx4_round(st["x"].float()), w.t()).to(DTYPES[c["dtype"]])
    if c["op"] == "norm":
        stream = st["stream"] if st["row_idx"] is None else st["stream"][st["row_idx"].long()]
        total = (stream.float() + st["x"].float()).to(stream.dtype)
        s = total.float()
        mean = s.double().square().mean(1, keepdim=True)   # in 64 bits: the codes behind it do not hang on the order of a sum
        h = s * torch.rsqrt(mean + EPS).float() * st["gain"].float()
        if c["form"] == "mx4":
            return _mx4_round(h).to(DTYPES[c["dtype"]]), total
        amax = h.abs().amax(1, keepdim=True)
        q = torch.round(h * (127.0 / amax))
        return (q * (amax / 127.0)).to(DTYPES[c["dtype"]]), total
    l = st["logits"].float()
    m = l.amax(1, keepdim=True)
    p = torch.exp(l - m)
    z = p.sum(1, keepdim=True)
    lse = m + torch.log(z)
    entropy = torch.log(z[:, 0]) - torch.where(p > 0, p * (l - m), 0).sum(1) / z[:, 0]
    logp = l.gather(1, st["given"].long()) - lse
    # one whole number per token that orders by logit, then by lower id
    bits = l.view(torch.int32).long()
    key = torch.where(bits < 0, -2 ** 31 - bits, bits) * 2 ** 20 + (2 ** 20 - 1 - torch.arange(l.shape[1], device="cuda"))
    ids = torch.topk(key, c["top"], dim=1).indices
    return logp, entropy, ids.to(torch.int32), l.gather(1, ids) - lse


# ---- what a pass cannot do without -----------------------------------------------------------------------
def work(case):
    c = case
    esz = 2 if c["dtype"] == "bf16" else 4
    M = c["M"]
    if c["op"] == "linear":
        N, K = c["N"], c["K"]
        return {"bytes": float(M * K * esz + N * K * 17 / 32 + M * N * esz), "flops": 2.0 * M * N * K}
    if c["op"] == "norm":  # in, stream in and out, the rows in few bits, their values
        held = 1.0 if c["form"] == "i8" else 17 / 32
        return {"bytes": M * c["d"] * (2.0 * esz + 2 * (2 if c["stream"] == "bf16" else 4) + held) + c["d"] * esz,
                "flops": 8.0 * M * c["d"]}
    return {"bytes": float(M * c["vocab"] * esz + M * (8 * c["given"] + 8 * c["top"] + 4)), "flops": 6.0 * M * c["vocab"]}


# ---- from the definitions, in 64 bits ----------------------------------------------------------------------
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_blocks(x):
    """Every block of 32 of x [rows, K] rounded to the nearest level times the smallest power of two that holds the block."""
    rows, K = x.shape
    full = torch.zeros(rows, -(-K // 32) * 32, dtype=torch.float64, device=x.device)
    full[:, :K] = x
    y = full.view(-1, 32)
    top = y.abs().amax(1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 6.0)) - 1    # (one too small at least: log2 is not exact)
    step = torch.pow(2.0, torch.where(top > 0, e, -125.0).clamp(-125, 125))
    step = torch.where(top > 6 * step, 2 * step, step)
    step = torch.where(top > 6 * step, 2 * step, step)
    levels = torch.tensor(LEVELS, dtype=torch.float64, device=x.device)
    u = (y.abs() / step).clamp(max=6.0)
    hi = torch.bucketize(u, levels).clamp(max=7)
    lo = (hi - 1).clamp(min=0)
    down, up = u - levels[lo], levels[hi] - u
    pick = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return (torch.sign(y) * levels[pick] * step).view(rows, -1)[:, :K]


def exact(case, seed):
    c = case
    st = prepare(c, seed)
    if c["op"] == "linear":
        N, K = c["N"], c["K"]
        half = -(-K // 256) * 128
        table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), dtype=torch.float64, device="cuda")
        w = torch.empty(N, 2 * half, dtype=torch.float64, device="cuda")
        raw = st["w"][:N * half].view(N, half)
        w[:, 0::2] = table[(raw % 16).long()]
        w[:, 1::2] = table[(raw // 16).long()]
        block = torch.arange(half // 16, device="cuda")
        row = torch.arange(N, device="cuda")[:, None]
        at = (((row // 32 * (half // 128) + block // 8) * 2 + block % 2) * 32 + row % 32) * 4 + block % 8 // 2
        s = st["w"][-(-N * half // 256) * 256:][at].double()
        w *= torch.pow(2.0, s - 127).repeat_interleave(32, 1)
        return _exact_blocks(st["x"].double()) @ w[:, :K].t()
    if c["op"] == "norm":
        pick = torch.arange(c["M"], device="cuda") if st["row_idx"] is None else st["row_idx"].long()
        total = (st["stream"][pick].double() + st["x"].double()).float().to(DTYPES[c["stream"]])   # the sums that are kept
        s = total.double()
        h = s / torch.sqrt((s * s).sum(1, keepdim=True) / c["d"] + EPS) * st["gain"].double()
        if c["form"] == "mx4":
            return _exact_blocks(h), s
        step = h.abs().amax(1, keepdim=True) / 127
        return torch.round(h / step) * step, s
    l = st["logits"].double()
    logp = torch.log_softmax(l, 1)
    entropy = -(torch.where(torch.isinf(logp), 0.0, logp) * logp.exp()).sum(1)
    ids = torch.sort(l, dim=1, descending=True, stable=True).indices[:, :c["top"]]
    return logp.gather(1, st["given"].long()), entropy, ids.to(torch.int32), logp.gather(1, ids)
