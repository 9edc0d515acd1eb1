"""Infinities and NaN in queries and keys that are there, by every kernel that sums a row: few keys and many, ranges that are joined,
a given log-sum-exp.  What a bad value spoils is known exactly; what it does not touch has to be what it is without it."""
import numpy as np
import pytest
import torch

from paper_2506_06295_amd import binding as L
from tests import lowbit_ref as R
from tests.test_gpu_lowbit import Case

pytestmark = pytest.mark.gpu

FORMATS = [("bf16", "bf16"), ("bf16", "kv4"), ("f32", "f32"), ("f32", "kv4")]
# Mq, n, H_q, H_kv, d_h: all keys in registers; row sums in ranges that are joined; row sums by one workgroup
WEIGHTS = [(3, 90, 4, 2, 128), (9, 1500, 4, 2, 64), (20, 3000, 2, 2, 128), (600, 1100, 8, 4, 128), (5, 700, 2, 1, 256)]


def weights(c, fmt, q, k, **more):
    return L.op_attention_weights(c.dtype, fmt, q, k, c.rows, c.n, c.H_q, c.H_kv, c.d_h, **more)


def test_the_shapes_take_the_kernels_they_are_for():
    ranges = [L.plan_attention_weights("bf16", "bf16", 2, *s)[1] for s in WEIGHTS]
    assert ranges[0] == 0 and ranges[1] > 1 and ranges[2] > 1 and ranges[3] == 1 and ranges[4] > 1


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("Mq,n,H_q,H_kv,d_h", WEIGHTS)
@pytest.mark.parametrize("what", ["query", "key", "infinite key"])
def test_weights_of_a_sequence_with_nan(dtype, fmt, Mq, n, H_q, H_kv, d_h, what):
    """A NaN score makes its row's sum NaN, and so the weight of every key of the sequence; other sequences are as they were."""
    c = Case(17, dtype, 2, Mq, n, H_q, H_kv, d_h)
    good_k = c.k.copy()
    if what != "query":
        # (an infinite element of one key meets queries of both signs: rows whose score is infinity have a NaN sum)
        c.k[n + n // 2, 5] = np.nan if what == "key" else np.inf
    q, k, _, _ = c.device(fmt)
    if what == "query":
        q[1, Mq // 2, 3] = float("nan")
    got = weights(c, fmt, q, k)
    c.k = good_k
    q, k, _, _ = c.device(fmt)
    want = weights(c, fmt, q, k)
    assert torch.equal(got[0], want[0]) and got[0].isfinite().all()
    assert got[1].isnan().all()


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("Mq,n,H_q,H_kv,d_h", WEIGHTS)
def test_weights_of_rows_that_look_at_nothing(dtype, fmt, Mq, n, H_q, H_kv, d_h):
    """Rows whose every score is minus infinity add nothing, as their log-sum-exp of minus infinity says."""
    c = Case(18, dtype, 2, Mq, n, H_q, H_kv, d_h)
    huge = 2.0 ** 120
    c.k = R.grid(c.r.uniform(1.0, 2.0, c.k.shape) * huge, dtype)  # (level 4 at least in 4 bits: no product is zero)
    c.q[:] = 0.0
    c.q[:, :, :, 1] = R.grid(c.r.uniform(-1.0, 1.0, c.q.shape[:3]) / huge, dtype)
    lost = (1, Mq // 2, H_q - 1)
    c.q[lost] = 0.0
    c.q[lost + (0,)] = -2.0 ** 100                                # -2^100 * 2^120 is beyond float32
    q, k, v, _ = c.device(fmt)
    got = weights(c, fmt, q, k)
    assert got.isfinite().all()
    c.q[lost] = 0.0                                              # a row of equal scores: a weight of 1 / n each
    q, k, _, _ = c.device(fmt)
    even = weights(c, fmt, q, k)
    # sums of Mq * H_q weights of at most 1, each off by a few roundings, their sum by one for each
    tol = float(even.max()) * Mq * H_q * 2.0 ** -22
    assert torch.equal(got[0], even[0])
    assert float((got[1] + 1.0 / n - even[1]).abs().max()) <= tol


@pytest.mark.parametrize("Mq,n", [(3, 90), (20, 3000), (600, 1100)])
def test_given_sums_of_minus_infinity(Mq, n):
    """A row whose log-sum-exp is minus infinity adds nothing where it is given either, and NaN stays in its sequence."""
    c = Case(19, "bf16", 2, Mq, n, 4, 2, 128)
    huge = 2.0 ** 120
    c.k = R.grid(c.r.uniform(1.0, 2.0, c.k.shape) * huge, "bf16")
    c.v = R.grid(c.r.standard_normal(c.v.shape), "bf16")
    c.q = R.grid(c.q / (16 * huge), "bf16")
    c.q[1, Mq // 2, 3] = 0.0
    c.q[1, Mq // 2, 3, 0] = -2.0 ** 100
    q, k, v, _ = c.device("kv4")
    out, lse = L.op_attention_kv4("bf16", q, k, v, c.rows, c.n, 4, 2, 128, with_lse=True)
    assert torch.isneginf(lse[1, Mq // 2, 3]) and int(torch.isneginf(lse).sum()) == 1
    assert (out[1, Mq // 2, 3 * 128:] == 0).all() and out.isfinite().all()
    alone, given = weights(c, "kv4", q, k), weights(c, "kv4", q, k, lse=lse)
    assert alone.isfinite().all() and given.isfinite().all()
    # scores of at most 128 * 2 * 4 / 16 / sqrt(128) < 6: both exponents are right to 6 * 2^-22 and the rounding of the logarithm
    assert float((alone - given).abs().max()) <= float(alone.max()) * (n * 2.0 ** -23 + Mq * 4 * 2.0 ** -23 + 2.0 ** -17)
    lse[0, 0, 0] = float("nan")
    if n > 1024:   # (fewer keys: the sums are worked out anyway)
        spoilt = weights(c, "kv4", q, k, lse=lse)
        assert spoilt[0].isnan().all() and torch.equal(spoilt[1], given[1])


# Mq, n, H_q, H_kv, d_h: 16 rows by four and eight wavefronts, 32 rows, tiles of 128 and 256, float32's and heads of 256; in ranges and not
ATTENTION = [(2, 2000, 2, 1, 64), (3, 2255, 2, 1, 128), (51, 4608, 2, 2, 128), (5, 3607, 56, 8, 128), (529, 4136, 2, 2, 128),
             (598, 919, 14, 2, 128), (20, 1416, 1, 1, 256), (90, 70, 2, 2, 128), (1320, 6304, 8, 4, 64), (1320, 6304, 8, 4, 128)]


def test_the_attention_shapes_take_every_kernel():
    plans = {(s[4], *L.plan_attention_kv4("bf16", 2, *s)[:2]) for s in ATTENTION}
    assert plans >= {(64, 16, 8), (64, 128, 4), (128, 16, 4), (128, 16, 8), (128, 32, 8), (128, 128, 4), (128, 256, 8), (256, 16, 4)}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Mq,n,H_q,H_kv,d_h", ATTENTION)
@pytest.mark.parametrize("what", ["query", "key", "value"])
def test_attention_with_nan(dtype, Mq, n, H_q, H_kv, d_h, what):
    """A NaN query spoils its row, a NaN key every row of its head, a NaN value every row of its head and block of 32 elements; whatever
    range of keys it lies in."""
    c = Case(20, dtype, 2, Mq, n, H_q, H_kv, d_h)
    args = (c.rows, c.n, H_q, H_kv, d_h)
    q, k, v, _ = c.device("kv4")
    want, want_lse = L.op_attention_kv4(dtype, q, k, v, *args, with_lse=True)
    G = H_q // H_kv
    for at in (0, n // 3, n - 1):
        spoilt = torch.zeros(2, Mq, H_q, d_h // 32, dtype=torch.bool, device="cuda")
        q, k, v, _ = c.device("kv4")
        h = H_kv - 1
        if what == "query":
            q.view(2, Mq, H_q, d_h)[1, at % Mq, H_q - 1, 7] = float("nan")
            spoilt[1, at % Mq, H_q - 1] = True
        else:
            bad = L.op_kv4_load("f32", k if what == "key" else v, c.rows, H_kv, d_h, rows=R.ints([n + at]))
            bad[0, h * d_h + 40] = float("nan")
            L.op_kv4_store("f32", bad, k if what == "key" else v, c.rows, H_kv, d_h, rows=R.ints([n + at]))
            if what == "key":
                spoilt[1, :, h * G:] = True
            else:
                spoilt[1, :, h * G:, 1] = True
        got, lse = L.op_attention_kv4(dtype, q, k, v, *args, with_lse=True)
        wide = spoilt.repeat_interleave(32, 3).view_as(got)
        assert got[wide].isnan().all()
        assert torch.equal(got[~wide], want[~wide])
        if what == "value":
            assert torch.equal(lse, want_lse)
        else:
            assert lse[spoilt[..., 0]].isnan().all() and torch.equal(lse[~spoilt[..., 0]], want_lse[~spoilt[..., 0]])


@pytest.mark.parametrize("Mq,n", [(3, 90), (20, 3000)])
@pytest.mark.parametrize("value", [float("-inf"), float("inf"), 3.4028234e38, 3.3961e38])
def test_float32_queries_at_the_end_of_the_range(Mq, n, value):
    """Over 4 bits: what bf16 has as an infinity makes its row NaN; other rows are as they were, whatever the score (2^107 here, far
    beyond what the header allows)."""
    c = Case(21, "f32", 1, Mq, n, 2, 1, 128)
    c.k = (np.sign(c.k) * 2.0 ** -20).astype(np.float32)
    q, k, v, _ = c.device("kv4")
    args = (c.rows, n, 2, 1, 128)
    want, want_lse = L.op_attention_kv4("f32", q, k, v, *args, with_lse=True)
    row, rest = (0, Mq // 2, 1), torch.ones(1, Mq, 2, dtype=torch.bool, device="cuda")
    rest[row] = False
    q[0, Mq // 2, 128:] = 0.0
    q[0, Mq // 2, 130] = value
    got, lse = L.op_attention_kv4("f32", q, k, v, *args, with_lse=True)
    assert torch.equal(got.view(1, Mq, 2, 128)[rest], want.view(1, Mq, 2, 128)[rest]) and torch.equal(lse[rest], want_lse[rest])
    if value != 3.3961e38:
        assert got.view(1, Mq, 2, 128)[row].isnan().all() and lse[row].isnan()
        assert weights(c, "kv4", q, k).isnan().all()


@pytest.mark.parametrize("Mq,n", [(3, 90), (20, 3000)])
def test_float32_queries_below_the_end_of_the_range(Mq, n):
    """The largest element that bf16 does not have as an infinity, over keys that make scores of +-22.6 of it: the keys of its sign share the
    row, the others have e^-45 of their weight."""
    c = Case(22, "f32", 1, Mq, n, 2, 1, 128)
    c.k = (np.sign(c.k) * 2.0 ** -120).astype(np.float32)
    c.q[0, Mq // 2, 1] = 0.0
    c.q[0, Mq // 2, 1, 2] = 3.3961e38
    check = c.values("kv4", c.k)
    assert np.array_equal(check.reshape(c.k.shape), c.k)          # a power of two is held exactly
    q, k, v, _ = c.device("kv4")
    got, lse = L.op_attention_kv4("f32", q, k, v, c.rows, n, 2, 1, 128, with_lse=True)
    up = c.k[:, 2] > 0
    score = 3.3961e38 * 2.0 ** -120 / np.sqrt(128)
    # scores off by 3 * 2^-24 of themselves, the same for all; sums of n terms
    assert abs(float(lse[0, Mq // 2, 1]) - (score + np.log(up.sum()))) <= (score + np.log(n)) * 2.0 ** -21 + n * 2.0 ** -24
    values = c.values("kv4", c.v)[:, 0]
    err = np.abs(got.view(1, Mq, 2, 128)[0, Mq // 2, 1].double().cpu().numpy() - values[up].mean(0))
    assert (err <= np.abs(values).max() * (n * 2.0 ** -22 + 2.0 ** -20)).all()
    w = weights(c, "kv4", q, k).double().cpu().numpy()[0]
    rest = torch.arange(Mq, device="cuda") != Mq // 2
    assert np.isfinite(w).all() and abs(w.sum() - 2 * Mq) <= 2 * Mq * n * 2.0 ** -22 and bool(got[0, rest].isfinite().all())


@pytest.mark.parametrize("dtype,fmt", FORMATS)
@pytest.mark.parametrize("Mq,n,d_h", [(3, 90, 128), (20, 3000, 128), (200, 1100, 64), (5, 700, 256)])
def test_the_largest_scores(dtype, fmt, Mq, n, d_h):
    """Scores of both signs to just below 2^30: everything finite, every row's weights sum to one, its log-sum-exp is its largest score."""
    c = Case(23, dtype, 1, Mq, n, 2, 1, d_h)
    c.q[:] = 0.0
    c.q[..., 3] = R.grid(c.r.uniform(0.25, 1.0, c.q.shape[:3]) * c.r.choice([-1.0, 1.0], c.q.shape[:3]) * 2.0 ** 20 * np.sqrt(d_h), dtype)
    c.k = R.grid(c.r.uniform(-1.0, 1.0, c.k.shape) * 2.0 ** 9.98, dtype)
    q, k, v, _ = c.device(fmt)
    held = c.values(fmt, c.k)[:, 0, 3]
    scores = c.q[0, :, :, 3, None].astype(np.float64) * held / np.sqrt(d_h)      # [Mq, H_q, n]
    assert 2.0 ** 29 < np.abs(scores).max() < 2.0 ** 30
    w = weights(c, fmt, q, k).double().cpu().numpy()[0]
    assert np.isfinite(w).all() and (w >= 0).all()
    assert abs(w.sum() - 2 * Mq) <= 2 * Mq * (n + 2 * Mq) * 2.0 ** -22
    if fmt == "kv4":
        out, lse = L.op_attention_kv4(dtype, q, k, v, c.rows, n, 2, 1, d_h, with_lse=True)
        assert out.isfinite().all()
        top = scores.max(2)
        assert (np.abs(lse[0].double().cpu().numpy() - top) <= np.abs(top) * 2.0 ** -20 + np.log(n)).all()
