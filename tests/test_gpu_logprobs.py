"""GPU tests of token log probabilities, entropy and alternatives against their plain 64-bit form (tests/stream_ref.py)."""
import numpy as np
import pytest
import torch

from paper_2506_06295_amd import binding as L
from tests import lowbit_ref as R
from tests import stream_ref as S
from tests.test_gpu_lowbit import host

pytestmark = pytest.mark.gpu


def close(got, want, tol):
    got = host(got)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        return bool((same | (np.abs(got - want) <= tol)).all())


def check(dtype, l, tokens=None, top_k=0, pad=0):
    """l: float32 values of the type [M, vocab]."""
    M, V = l.shape
    wide = np.full((M, V + pad), np.nan, np.float32)   # (what lies between the rows has no say)
    wide[:, :V] = l
    logp, entropy, ids, top = L.op_logprobs(dtype, R.dev(wide, dtype)[:, :V], None if tokens is None else R.ints(tokens), top_k)
    want = S.logprobs(l.astype(np.float64), tokens, top_k)
    if tokens is not None:
        assert close(logp, want[0], want[4])
    else:
        assert logp is None
    assert close(entropy, want[1], want[5])
    if top_k:
        assert np.array_equal(ids.cpu().numpy(), want[2])
        assert close(top, want[3], want[6])
    else:
        assert ids is None and top is None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,n,k,pad", [(1, 1, 1, 1, 0), (2, 2, 1, 3, 0), (3, 7, 2, 7, 0), (5, 63, 1, 64, 1), (4, 64, 3, 5, 0),
                                         (33, 1024, 1, 4, 0), (7, 1023, 9, 64, 5), (2, 4096, 1, 20, 64), (3, 8192, 1, 1, 0), (3, 8193, 1, 33, 7),
                                         (2, 16500, 2, 64, 0), (1, 126464, 1, 20, 0), (3, 152064, 1, 8, 0), (2, 152031, 16, 64, 3)])
def test_rows(dtype, M, V, n, k, pad):
    r = np.random.default_rng(M + V + k)
    l = 2 * r.standard_normal((M, V))
    l[np.arange(M), r.integers(0, V, M)] += 9
    l = R.grid(l, dtype)
    check(dtype, l, r.integers(0, V, (M, n)), k, pad)


@pytest.mark.parametrize("M", [300, 1100])
def test_many_rows(M):
    r = np.random.default_rng(M)
    check("bf16", R.grid(3 * r.standard_normal((M, 2500)), "bf16"), r.integers(0, 2500, (M, 2)), 6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_parts_alone(dtype):
    r = np.random.default_rng(1)
    l = R.grid(r.standard_normal((4, 5000)), dtype)
    check(dtype, l)
    check(dtype, l, r.integers(0, 5000, (4, 3)))
    check(dtype, l, None, 9)


@pytest.mark.parametrize("V", [40, 1024, 20000, 126464])
@pytest.mark.parametrize("k", [1, 7, 64])
def test_ties(V, k):
    """Equal logits: the lower id first.  All alike, few different values, a plateau at the top longer than the list, zeros of both signs."""
    r = np.random.default_rng(V + k)
    l = np.zeros((5, V), np.float32)
    l[1] = r.integers(0, 3, V)
    l[2] = -5
    l[2, r.permutation(V)[:min(V, 200)]] = 4
    l[3] = np.where(r.random(V) < 0.5, -0.0, 0.0)
    l[4] = -3.5
    check("f32", l, r.integers(0, V, (5, 1)), k)
    check("bf16", l, r.integers(0, V, (5, 1)), k)


@pytest.mark.parametrize("V", [300, 9000, 126464])
def test_sorted_rows(V):
    """The likeliest tokens all next to each other, at either end, and every 256 or 1024 tokens."""
    up = np.linspace(-20, 20, V).astype(np.float32)
    rows = [up, up[::-1]]
    for step in (4, 64, 256, 1024):
        s = np.full(V, -8.0, np.float32)
        s[::step] = np.linspace(0, 5, len(s[::step]))
        rows.append(s)
    l = np.stack(rows)
    check("f32", l, np.array([[0], [V - 1], [0], [1], [2], [3]]), 64)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [100, 5000, 126464])
def test_tokens_that_cannot_be(dtype, V):
    r = np.random.default_rng(V)
    l = R.grid(2 * r.standard_normal((6, V)), dtype)
    l[0, r.random(V) < 0.9] = -np.inf
    l[1] = -np.inf                    # nothing is left
    l[2] = -np.inf
    l[2, V // 3] = 2.5                # one token
    l[3, :] = -np.inf
    l[3, [5, V - 1, 50]] = [1, 1, 3]  # fewer than are asked for
    lowest = -3.38953139e38 if dtype == "bf16" else np.finfo(np.float32).min
    l[4] = lowest                     # the type's lowest value is a logit as any other
    l[5, :] = lowest
    l[5, V // 2] = 0
    tokens = np.tile(np.array([0, V // 3, V // 2, V - 1, -1, V, 2 ** 31 - 1, -2 ** 31]), (6, 1))
    check(dtype, l, tokens, 12)


@pytest.mark.parametrize("V", [100, 5000, 126464])
def test_bad_rows_are_nan_and_others_are_not(V):
    r = np.random.default_rng(V + 1)
    l = R.grid(r.standard_normal((5, V)), "f32")
    l[1, V - 1], l[3, 0] = np.nan, np.inf
    l[4] = -np.inf
    l[4, 7] = np.nan
    check("f32", l, np.tile(np.array([0, 7, -1, V]), (5, 1)), 5)


@pytest.mark.parametrize("V", [2000, 126464])
def test_logits_of_any_size(V):
    """Far from zero and far apart: the maximum is taken off first."""
    r = np.random.default_rng(V)
    l = np.stack([1e4 + r.standard_normal(V), -3e37 + 1e30 * r.standard_normal(V), 3e38 * r.uniform(-1, 1, V), 1e-38 * r.standard_normal(V),
                  100 * r.standard_normal(V)]).astype(np.float32)
    check("f32", l, r.integers(0, V, (5, 3)), 10)
