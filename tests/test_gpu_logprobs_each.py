"""Token log probabilities: every logit counts, once.  Rows of equal low logits hold 60 high ones at chosen places, whose sums are known in 64 bits: a
high logit that is left out or counted twice moves every result by some percent, tolerances are some 1e-5.  What lies between rows is NaN.

Places: the first and last ids, both sides of every chunk's edge (8192 logits counted from the 128-byte line that a row starts in; slices
of rows are whole chunks), and every id of a row; rows start at every element of a line."""
import numpy as np
import pytest
import torch

from paper_2506_06295_amd import binding as L
from tests import lowbit_ref as R
from tests import stream_ref as S

CHUNK, HIGH = 8192, 60
LOW = -12.0
VALUES = 2 + np.arange(HIGH) / 64.0   # (bf16 has them all)


def logprobs_of(V, values=VALUES):
    """(log probabilities of `values`, of a low logit, entropy) of V logits, `values` and low ones."""
    n = len(values)
    v = np.append(values, LOW) - values.max()
    count = np.append(np.ones(n), V - n)
    e = count * np.exp(v)
    lz = np.log(e.sum())
    return v[:-1] - lz, v[-1] - lz, lz - (e * v).sum() / e.sum()


def tolerances(V):
    """Of log probabilities and of the entropy.  A term of z goes through 32 additions in its block, then for every chunk at most one more and, where the maximum
    rises, a factor (an exponential of 2 half steps and a product); the ends of slice and row are a factor and 8 additions in trees each.  An exponential's
    own roundings: 4 half steps, and 4 of its argument in all, over however many rising maxima.  A term of y: a rounding or two more at each place."""
    chunks = min(33, -(-(V + 63) // CHUNK))   # (of a slice at most)
    chain_z, chain_y = 32 + 4 * chunks + 24, 32 + 6 * chunks + 30
    logp, low, h = logprobs_of(V)
    v = np.append(VALUES, LOW) - VALUES.max()
    p = np.append(np.exp(logp), (V - HIGH) * np.exp(low))
    lz = -logp[-1]
    e1, e2 = (p * -v).sum(), (p * v * v).sum()
    dz = S.U * (chain_z + 4 + 4 * e1)
    tol_p = dz + S.U * (2 * abs(v).max() + 4 * abs(lz) + 2 * abs(low))
    tol_h = dz * (1 + e1) + S.U * ((chain_y + 8) * e1 + 5 * e2 + 4 * abs(lz) + 2 * abs(h))
    return tol_p, tol_h


@pytest.mark.parametrize("V", [61, 1985, 20013, 1 << 24])
def test_the_check_sees_one_logit(V):
    """On the 64-bit form: the least high logit missing or there twice."""
    logp, _, h = logprobs_of(V)
    tol_p, tol_h = tolerances(V)
    for wrong in (VALUES[1:], np.append(VALUES, VALUES[0])):
        other, _, other_h = logprobs_of(V, wrong)
        assert abs(other[-1 if len(wrong) < HIGH else -2] - logp[-1]) > 20 * tol_p and abs(other_h - h) > 20 * tol_h


def deal(ids, seed):
    """Rows of HIGH of the ids; the last is filled with ids of the first."""
    ids = np.random.default_rng(seed).permutation(ids)
    rows = -(-len(ids) // HIGH)
    return np.resize(ids, (rows, HIGH))


def rows_like(M, V, dtype):
    """([M, V] of low logits whose rows start one element further in their line each, NaN between them; where in its line each starts)"""
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    line = 128 // t.itemsize
    ld = -(-V // line) * line + 1
    flat = torch.full((M * ld + line,), float("nan"), dtype=t, device="cuda")
    l = flat.as_strided((M, V), (ld, 1))
    l.fill_(LOW)
    return l, (flat.data_ptr() // t.itemsize + np.arange(M) * ld) % line


def check(dtype, l, places, k, seed=0):
    """places [M, HIGH]: ids of the high logits."""
    M, V = l.shape
    r = np.random.default_rng(seed)
    order = r.permuted(np.tile(np.arange(HIGH), (M, 1)), axis=1)   # which value stands at which place
    at = torch.from_numpy(places.astype(np.int64)).cuda()
    l.scatter_(1, at, torch.from_numpy(VALUES[order]).to(l.dtype).cuda())
    low = [next(t for t in range(V) if t not in s) if V > HIGH else 0 for s in map(set, places.tolist())]
    given = np.concatenate([places, np.array(low)[:, None]], 1)
    logp, h, ids, top = L.op_logprobs(dtype, l, R.ints(given), k)
    want, of_low, want_h = logprobs_of(V)
    tol_p, tol_h = tolerances(V)
    logp, h, ids, top = (x.cpu().numpy().astype(np.float64) for x in (logp, h, ids, top))
    assert (np.abs(logp[:, :HIGH] - want[order]) <= tol_p).all()
    if V > HIGH:
        assert (np.abs(logp[:, HIGH] - of_low) <= tol_p).all()
    assert (np.abs(h - want_h) <= tol_h).all()
    by_value = np.take_along_axis(places, np.argsort(-order, axis=1), 1)[:, :k]
    assert np.array_equal(ids, by_value)
    assert (np.abs(top - want[::-1][:k]) <= tol_p).all()


gpu = pytest.mark.gpu
# rows of a wavefront each, one chunk, some, many; fewer rows than a slice takes alone, and one slice a row
VOCABS = [61, 200, 1985, 2017, 2049, 8129, 8193, 20013, 100003]
ROWS = [70, 256]


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("M", ROWS)
@pytest.mark.parametrize("k", [8, 60])
def test_first_and_last_logits(dtype, V, M, k):
    """At every place of a line that a row starts at, so that its partial first and last 16 bytes hold any number of logits."""
    l, _ = rows_like(M, V, dtype)
    half = HIGH // 2
    check(dtype, l, np.tile(np.append(np.arange(half), np.arange(V - half, V)), (M, 1)), k)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,M", [(20013, 70), (20013, 256), (100003, 20), (100003, 200), (100003, 256), (270001, 70), (270001, 256)])
def test_both_sides_of_chunks(dtype, V, M):
    l, start = rows_like(M, V, dtype)
    places = np.empty((M, HIGH), np.int64)
    for i in range(M):
        edges = np.arange(CHUNK, V + start[i], CHUNK) - start[i]
        near = np.concatenate([edges + o for o in range(-16, 17)])
        near = near[(near >= 0) & (near < V)]
        first = np.unique(np.concatenate([edges - 1, edges]))
        first = first[:HIGH] if i % 2 else first[-HIGH:]   # (33 chunks have 64 of these)
        rest = np.random.default_rng(i).permutation(np.setdiff1d(near, first))
        places[i] = np.append(first, rest)[:HIGH]
    check(dtype, l, places, 8)
    check(dtype, l.fill_(LOW), places, 60)


@gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", VOCABS)
def test_every_logit(dtype, V):
    """Every id high in one row, among rows of one slice each and among fewer."""
    places = deal(np.arange(V), V)
    for most in (len(places), 100):
        for a in range(0, len(places), most):
            some = places[a:a + most]
            if most == len(places) and len(some) < 256:
                some = np.resize(some, (256, HIGH))
            l, _ = rows_like(len(some), V, dtype)
            check(dtype, l, some, 8, seed=a)


@gpu
def test_every_edge_of_the_longest_rows():
    """2^24 logits: a row is sliced whatever the number of rows."""
    V = 1 << 24
    line = 64
    edges = np.arange(1, V // CHUNK)
    rows = -(-2 * len(edges) // HIGH)
    l, start = rows_like(rows, V, "bf16")
    places = deal(np.concatenate([edges * CHUNK, -edges * CHUNK]), 1)   # (negative: the logit before the edge)
    places = np.where(places > 0, places - start[:, None], -places - start[:, None] - 1)
    assert line > start.max() and places.min() >= 0 and places.max() < V
    check("bf16", l, places, 8)
