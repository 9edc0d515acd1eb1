"""Plain 64-bit forms of the norm in few bits, the 4-bit blocks and the token log probabilities (numpy).  Written from the definitions in
include/dllmc.h; nothing of the library is used."""
import numpy as np

from tests import lowbit_ref as R

U = 2.0 ** -24   # half a step of float32


# ---- 4-bit blocks of rows
def mx4_values(x):
    """What 4-bit blocks hold of x [rows, K]: float64."""
    rows, K = x.shape
    full = np.zeros((rows, -(-K // 32) * 32))
    full[:, :K] = x
    return R.kv4_values(full)[:, :K]


def mx4_pack(x):
    """(byte buffer, which of its bytes are stated) of x [rows, K] in 4-bit blocks."""
    rows, K = x.shape
    Kp = -(-K // 256) * 256
    full = np.zeros((rows, Kp))
    full[:, :K] = x
    y, bad, e, idx = R._blocks(full)
    codes = np.where(bad[:, None], 0, idx + 8 * np.signbit(y)).astype(np.uint8).reshape(rows, Kp)
    packed = (codes[:, 0::2] | (codes[:, 1::2] << 4)).reshape(-1)
    scales = np.where(bad, 255, e + 127).astype(np.uint8).reshape(rows, Kp // 32)
    start = -(-packed.size // 256) * 256
    groups = -(-rows // 32)
    buf = np.zeros(start + groups * 32 * (Kp // 32), np.uint8)
    told = np.zeros(buf.shape, bool)
    buf[:packed.size], told[:packed.size] = packed, True
    for r in range(rows):
        for k in range(Kp // 32):
            at = start + ((((r // 32) * (Kp // 256) + k // 8) * 2 + k % 2) * 32 + r % 32) * 4 + k % 8 // 2
            buf[at], told[at] = scales[r, k], True
    return buf, told


def product_error(a, w, slices=8):
    """How far the product of 4-bit values a [M, K], w [N, K] may be from float64's: a rounding of at most 2^-22 of the running mass for every 64
    elements that are taken at once (their own alignment and the addition), as many again for parts that are added."""
    steps = -(-a.shape[1] // 64) + 2 * slices + 8
    return steps * 4 * U * (np.abs(a) @ np.abs(w).T)


# ---- the norm
def norm(stream, x, gain, eps, stream_dtype):
    """(sums in the stream's type, float64 norm) of float32 arrays [M, d]."""
    s = np.asarray(stream, np.float32)
    if x is not None:
        s = R.grid(s + np.asarray(x, np.float32), stream_dtype)
    t = s.astype(np.float64)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        h = t / np.sqrt((t * t).mean(1, keepdims=True) + float(np.float32(eps))) * gain
    h[~np.isfinite(t).all(1)] = np.nan
    return s, h


# ---- token log probabilities
def logprobs(l, tokens, top_k):
    """(logp, entropy, ids, top logp, tolerances of the first, second and fourth) of float64 l [M, vocab]."""
    M, V = l.shape
    n = 0 if tokens is None else tokens.shape[1]
    logp, top = np.full((M, n), -np.inf), np.full((M, top_k), -np.inf)
    ids = np.full((M, top_k), -1, np.int32)
    entropy = np.zeros(M)
    tol_p, tol_h, tol_t = np.zeros((M, n)), np.zeros(M), np.zeros((M, top_k))
    chain = -(-V // 256) + 40   # additions that a term goes through: a thread's own, then trees
    for i in range(M):
        if not (l[i] < np.inf).all():
            logp[i], entropy[i], top[i] = np.nan, np.nan, np.nan
            continue
        if not (l[i] > -np.inf).any():
            continue
        v = l[i] - l[i].max()
        p = np.exp(v)
        z = p.sum()
        p /= z
        fin = p > 0
        lz = np.log(z)
        entropy[i] = lz - (p[fin] * v[fin]).sum()
        e1, e2 = (p[fin] * -v[fin]).sum(), (p[fin] * v[fin] ** 2).sum()
        # an exponential: its argument's roundings (of the difference, of a factor log2 e and of what is left: 4 half steps of v) and 4 of its own
        dz = U * (chain + 4 + 4 * e1)
        tol_h[i] = dz * (1 + e1) + U * ((chain + 8) * e1 + 4 * e2 + 4 * abs(lz)) + 2 * U * abs(entropy[i]) + 1e-30

        def of(t):
            lp = v[t] - lz
            return lp, dz + U * (2 * abs(v[t]) + 4 * abs(lz) + 2 * abs(lp)) + 1e-30
        for k in range(n):
            t = int(tokens[i, k])
            if 0 <= t < V and l[i, t] > -np.inf:
                logp[i, k], tol_p[i, k] = of(t)
        order = np.lexsort((np.arange(V), -l[i]))[:top_k]
        order = order[l[i][order] > -np.inf]
        ids[i, :len(order)] = order
        for k, t in enumerate(order):
            top[i, k], tol_t[i, k] = of(t)
    for lp in (logp, top):
        lp[lp <= -(2.0 - 2.0 ** -24) * 2.0 ** 127] = -np.inf   # (rounds to an infinity in float32)
    return logp, entropy, ids, top, tol_p, tol_h, tol_t
