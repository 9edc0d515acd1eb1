"""GPU tests of the norm in few bits, the 4-bit maps and the token log probabilities at the largest sizes that they take, and of operands that
are the same tensor.  Expected values are exact, or those of tests/stream_ref.py."""
import numpy as np
import pytest
import torch

from paper_2506_06295_amd import binding as L
from tests import lowbit_ref as R
from tests import stream_ref as S
from tests.test_gpu_logprobs import check
from tests.test_gpu_lowbit import host
from tests.test_gpu_norm8 import EPS, TYPES, check_rows4, check_rows8, inputs

pytestmark = pytest.mark.gpu
WIDEST = 131072


def levels(seed, rows, K, most):
    """Float32 numbers that 4-bit blocks hold exactly, of magnitudes up to LEVELS[most]."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    of = torch.tensor([-v for v in R.LEVELS[:most + 1]] + list(R.LEVELS[:most + 1]), dtype=torch.float32, device="cuda")
    return of[torch.randint(0, len(of), (rows, K), generator=g, device="cuda")]


def product(a, w, K, dtype="f32"):
    return L.op_linear_mx4(dtype, L.op_quant_mx4("f32", a), a.shape[0], L.op_quant_mx4("f32", w), w.shape[0], K)


@pytest.mark.parametrize("dtype,stream_dtype", TYPES)
def test_widest_norm(dtype, stream_dtype):
    for d in (WIDEST, WIDEST - 1):
        stream, x, gain, _ = inputs(d, 2, d, dtype, stream_dtype)
        s, h = S.norm(stream, x, gain, EPS, stream_dtype)
        args = (dtype, R.dev(stream, stream_dtype), R.dev(gain, dtype), EPS)
        kw = dict(x=R.dev(x, dtype), stream_dtype=stream_dtype)
        q, scale, total = L.op_norm_quant8(*args, **kw)
        check_rows8(q, scale, h, d)
        assert np.array_equal(host(total), s.astype(np.float64))
        check_rows4(host(L.op_mx4_load("f32", L.op_norm_mx4(*args, **kw)[0], 2, d)), h)


def test_most_rows_of_a_norm():
    """Powers of two in rows of one element, eps 0: the norm is the sign, exactly."""
    M = (1 << 23) - 1
    sign = torch.randint(0, 2, (M, 1), device="cuda", dtype=torch.float32) * 2 - 1
    stream = sign * torch.exp2(torch.randint(-20, 20, (M, 1), device="cuda").float())
    gain = torch.ones(1, device="cuda")
    q, scale, _ = L.op_norm_quant8("f32", stream, gain, 0.0)
    assert torch.equal(q[:, :1].float(), 127 * sign) and not q[:, 1:].any()
    assert ((scale.double() * 127 - 1).abs() <= 5 * S.U).all()
    del q
    assert torch.equal(L.op_mx4_load("f32", L.op_norm_mx4("f32", stream, gain, 0.0)[0], M, 1), sign)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [300, 4096, 20000])
def test_stream_added_to_itself(dtype, d):
    stream, _, gain, _ = inputs(d, 5, d, dtype, dtype)
    s, h = S.norm(stream, stream, gain, EPS, dtype)
    for over in (False, True):
        t = R.dev(stream, dtype)
        q, scale, total = L.op_norm_quant8(dtype, t, R.dev(gain, dtype), EPS, x=t, sum_out=t if over else None)
        check_rows8(q, scale, h, d)
        assert np.array_equal(host(total), s.astype(np.float64)) and (total is t) == over
        t = R.dev(stream, dtype)
        mx, total = L.op_norm_mx4(dtype, t, R.dev(gain, dtype), EPS, x=t, sum_out=t if over else None)
        check_rows4(host(L.op_mx4_load("f32", mx, 5, d)), h)
        assert np.array_equal(host(total), s.astype(np.float64))


@pytest.mark.parametrize("M,N,whole", [(1, 40, False), (200, 130, False), (1300, 1300, True)])
def test_widest_product(M, N, whole):
    """Quarters that stay below 2^22 (6 * 3 * 131072 = 2359296 < 2^22): every partial sum is a float32 number, in any order."""
    assert L.plan_linear_mx4(M, N, WIDEST)[2] == whole
    a, w = levels(M, M, WIDEST, 7), levels(N + 1, N, WIDEST, 5)
    assert torch.equal(product(a, w, WIDEST), a @ w.T)


@pytest.mark.parametrize("M,N", [(1, (1 << 24) - 1), (1 << 22, 3)])
def test_most_rows_of_a_product(M, N):
    a, w = levels(1, M, 2, 7), levels(2, N, 2, 7)
    assert torch.equal(product(a, w, 2), a[:, :1] * w[:, 0] + a[:, 1:] * w[:, 1])


@pytest.mark.parametrize("M,K", [(1, 300), (70, 512), (1500, 1024)])
def test_a_matrix_by_itself(M, K):
    a = levels(M, M, K, 7)
    m = L.op_quant_mx4("f32", a)
    assert torch.equal(L.op_linear_mx4("f32", m, M, m, M, K), a @ a.T)   # (36 * 4 * 1024 < 2^24)


@pytest.mark.parametrize("V", [1000, 20000])
def test_most_given_tokens(V):
    r = np.random.default_rng(V)
    l = R.grid(3 * r.standard_normal((2, V)), "f32")
    check("f32", l, r.integers(-2, V + 2, (2, 65536)), 3)   # (most of them more than once, some outside)


def test_most_rows_of_logits():
    """Of rows with one token it is certain."""
    M = (1 << 23) - 1
    l = torch.randn(M, 1, device="cuda", dtype=torch.bfloat16)
    logp, entropy, ids, top = L.op_logprobs("bf16", l, torch.zeros(M, 1, device="cuda", dtype=torch.int32), 2)
    assert not logp.any() and not entropy.any()
    assert not ids[:, 0].any() and (ids[:, 1] == -1).all() and not top[:, 0].any() and (top[:, 1] == -float("inf")).all()
