"""Plain 64-bit forms of the operators in fewer bits (numpy), and inputs for their tests.  Written from the definitions in
include/dllmc.h; nothing of the library is used."""
import numpy as np
import torch

from paper_2506_06295_amd.inputs import to_bf16_grid

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def grid(a, dtype):
    """float32 values that the dtype holds."""
    a = np.asarray(a, np.float32)
    return to_bf16_grid(a) if dtype == "bf16" else a


def dev(a, dtype="f32"):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def ints(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


# ---- 4-bit rows
def _block_exponents(y):
    """For blocks [count, 32] the smallest e in -125 .. 125 with max |y| <= 6 * 2^e (125 where there is none)."""
    top = np.abs(y).max(1)
    e = np.full(len(y), -125)
    for t in range(-124, 126):
        e[top > 6.0 * 2.0 ** (t - 1)] = t
    return e


def _level_index(y, e):
    """Index of the level nearest to |y| / 2^e, of two equally near ones the even one."""
    u = np.minimum(np.abs(y) / 2.0 ** e[:, None].astype(np.float64), 6.0)
    hi = np.searchsorted(LEVELS, u)
    lo = np.maximum(hi - 1, 0)
    down, up = u - LEVELS[lo], LEVELS[hi] - u
    return np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)


def _blocks(x):
    y = np.asarray(x, np.float64).reshape(-1, 32)
    bad = ~np.isfinite(y).all(1)
    y = np.where(bad[:, None], 0.0, y)
    e = _block_exponents(y)
    return y, bad, e, _level_index(y, e)


def kv4_values(x):
    """What a 4-bit row holds of x [..., 32 k]: float64."""
    y, bad, e, idx = _blocks(x)
    out = np.copysign(LEVELS[idx], y) * 2.0 ** e[:, None].astype(np.float64)
    out[bad] = np.nan
    return out.reshape(np.shape(x))


def kv4_pack(x, H, d_h):
    """Byte buffer of a 4-bit tensor that holds x [rows, H * d_h]."""
    rows = x.shape[0]
    y, bad, e, idx = _blocks(np.asarray(x, np.float64).reshape(rows, H, d_h).transpose(1, 0, 2))
    codes = np.where(bad[:, None], 0, idx + 8 * np.signbit(y)).astype(np.uint8).reshape(H, rows, d_h)
    scales = np.where(bad, 255, e + 127).astype(np.uint8)
    packed = (codes[..., 0::2] | (codes[..., 1::2] << 4)).reshape(-1)
    start = -(-packed.size // 256) * 256
    buf = np.zeros(start + scales.size, np.uint8)
    buf[:packed.size] = packed
    buf[start:] = scales
    return buf


# ---- attention
def present(B, n, cache_rows, lens, row_map):
    """For every sequence the positions that are there and their cache rows."""
    out = []
    for b in range(B):
        L = n if lens is None else int(np.clip(lens[b], 0, n))
        j = np.arange(L)
        r = b * n + j if row_map is None else np.asarray(row_map[b][:L], np.int64)
        ok = (r >= 0) & (r < cache_rows)
        out.append((j[ok], r[ok]))
    return out


def attend(q, k, v, where, H_q, H_kv, d_h):
    """q [B, Mq, H_q, d_h], k, v [rows, H_kv, d_h] float64.  Returns out, lse, the probabilities [b][a] -> [Mq, keys], and the bound
    pieces: sum of p |v| (like out) and the largest sum of |q||k| / sqrt(d_h) per query and head."""
    B, Mq = q.shape[:2]
    out = np.zeros((B, Mq, H_q, d_h))
    mass = np.zeros_like(out)
    lse = np.full((B, Mq, H_q), -np.inf)
    reach = np.zeros((B, Mq, H_q))
    probs = []
    for b, (_, rows) in enumerate(where):
        heads = []
        for a in range(H_q):
            h = a // (H_q // H_kv)
            if len(rows) == 0:
                heads.append(np.zeros((Mq, 0)))
                continue
            s = q[b, :, a] @ k[rows, h].T / np.sqrt(d_h)
            m = s.max(1, keepdims=True)
            p = np.exp(s - m)
            l = p.sum(1, keepdims=True)
            p /= l
            lse[b, :, a] = (m + np.log(l))[:, 0]
            reach[b, :, a] = (np.abs(q[b, :, a]) @ np.abs(k[rows, h]).T / np.sqrt(d_h)).max(1)
            if v is not None:
                out[b, :, a] = p @ v[rows, h]
                mass[b, :, a] = p @ np.abs(v[rows, h])
            heads.append(p)
        probs.append(heads)
    return out, lse, probs, mass, reach


def score_error(reach, lse, d_h):
    """Bound on the error of a scaled score in float32: 4 d_h additions of products (float32 queries go through the matrix cores in
    three parts), the scale, and the exponent's argument, each a rounding of something no larger than `reach`."""
    lse = np.where(np.isfinite(lse), np.abs(lse), 0.0)
    return reach * (4 * d_h + 16) * 2.0 ** -24 + (reach + lse) * 2.0 ** -22


# ---- eviction
def evict(acc, keep, where, lens, n, first, last):
    B = len(where)
    kept = np.full((B, keep), -1, np.int32)
    rows_out = np.full((B, keep), -1, np.int32)
    left = np.zeros((B, keep), np.float32)
    new = np.zeros(B, np.int32)
    for b, (pos, rows) in enumerate(where):
        L = n if lens is None else int(np.clip(lens[b], 0, n))
        w = acc[b, pos].astype(np.float64)
        safe = (pos < first) | (pos >= L - last)
        bad = np.isnan(w)
        order = sorted(range(len(pos)), key=lambda t: (not safe[t], bool(bad[t]), 0.0 if bad[t] else -w[t], pos[t]))[:keep]
        order = sorted(order, key=lambda t: pos[t])
        new[b] = len(order)
        for i, t in enumerate(order):
            kept[b, i], rows_out[b, i], left[b, i] = pos[t], rows[t], acc[b, pos[t]]
    return kept, rows_out, new, left


# ---- 8-bit rows
def quant8(x):
    """x float32 [M, K] -> int64 values, float32 scales."""
    x = np.asarray(x, np.float32)
    q = np.zeros(x.shape, np.int64)
    scale = np.zeros(x.shape[0], np.float32)
    for i, row in enumerate(x):
        if not np.isfinite(row).all():
            scale[i] = np.nan
            continue
        top = np.abs(row).max()
        if top < 2.0 ** -118:
            continue
        scale[i] = np.float32(top / np.float32(127))
        q[i] = np.rint(row * np.float32(np.float32(127) * np.float32(np.float32(1) / top))).astype(np.int64)
    return q, scale


def attend_device(q, k, v, where, H_q, H_kv, d_h):
    """As attend, in float64 on the GPU for larger shapes.  q, k, v: float64 CUDA tensors of attend's shapes.  Returns out, lse, mass,
    reach (numpy) and columns(rel [B, Mq, H_q]) -> (sum of p, sum of p * rel) per sequence's keys."""
    B, Mq = q.shape[:2]
    out = torch.zeros(B, Mq, H_q, d_h, dtype=torch.float64, device="cuda")
    mass = torch.zeros_like(out)
    lse = torch.full((B, Mq, H_q), -torch.inf, dtype=torch.float64, device="cuda")
    reach = torch.zeros(B, Mq, H_q, dtype=torch.float64, device="cuda")

    def probs(b, a):
        rows = torch.from_numpy(where[b][1]).cuda()
        kh = k[rows, a // (H_q // H_kv)]
        s = q[b, :, a] @ kh.t().contiguous() / d_h ** 0.5
        return s, kh, rows

    for b in range(B):
        if len(where[b][1]) == 0:
            continue
        for a in range(H_q):
            s, kh, rows = probs(b, a)
            lse[b, :, a] = torch.logsumexp(s, 1)
            reach[b, :, a] = (q[b, :, a].abs() @ kh.abs().t().contiguous() / d_h ** 0.5).amax(1)
            if v is not None:
                p = torch.exp(s - lse[b, :, a, None])
                vh = v[rows, a // (H_q // H_kv)].contiguous()
                out[b, :, a] = p @ vh
                mass[b, :, a] = p @ vh.abs()

    def columns(rel):
        rel = torch.from_numpy(rel).cuda()
        want, tol = [], []
        for b in range(B):
            n = len(where[b][1])
            w, t = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
            for a in range(H_q if n else 0):
                p = torch.exp(probs(b, a)[0] - lse[b, :, a, None])
                w += p.sum(0)
                t += (p * rel[b, :, a, None]).sum(0)
            want.append(w.cpu().numpy())
            tol.append(t.cpu().numpy())
        return want, tol

    return out.cpu().numpy(), lse.cpu().numpy(), mass.cpu().numpy(), reach.cpu().numpy(), columns
