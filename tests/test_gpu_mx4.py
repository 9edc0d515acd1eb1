"""GPU tests of 4-bit blocks and their product against plain 64-bit forms (tests/stream_ref.py)."""
import numpy as np
import pytest
import torch

from paper_2506_06295_amd import binding as L
from tests import lowbit_ref as R
from tests import stream_ref as S
from tests.test_gpu_lowbit import host, special_rows

pytestmark = pytest.mark.gpu


def put(x):
    return torch.from_numpy(S.mx4_pack(x)[0]).cuda()


# ------------------------------------------------------------------ rows in and out
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 32), (5, 100), (7, 256), (33, 300), (64, 704), (40, 2048), (6, 4104), (3, 18944), (9, 4095)])
def test_rows_in_and_out(dtype, rows, K):
    r = np.random.default_rng(rows * 1000 + K)
    wide = special_rows(r, rows, -(-K // 32) * 32, dtype)
    x = np.ascontiguousarray(wide[:, :K])
    mx = L.op_quant_mx4(dtype, R.dev(x, dtype))
    want, told = S.mx4_pack(x)
    assert mx.numel() == want.size
    assert np.array_equal(mx.cpu().numpy()[told], want[told])
    values = S.mx4_values(x)
    for out in ("f32", "bf16"):
        assert np.array_equal(host(L.op_mx4_load(out, mx, rows, K)), values, equal_nan=True)


@pytest.mark.parametrize("K", [64, 300])
def test_listed_rows(K):
    r = np.random.default_rng(K)
    x = R.grid(r.standard_normal((9, K)), "bf16")
    at = np.array([8, 0, 3, 3, -1, 9, -2 ** 31, 2 ** 31 - 1, 5])
    ok = (at >= 0) & (at < 9)
    want = np.where(ok[:, None], x[np.where(ok, at, 0)], 0)
    mx = L.op_quant_mx4("bf16", R.dev(x, "bf16"), row_idx=R.ints(at))
    assert np.array_equal(host(L.op_mx4_load("bf16", mx, 9, K)), S.mx4_values(want))
    whole = L.op_quant_mx4("bf16", R.dev(x, "bf16"))
    assert np.array_equal(host(L.op_mx4_load("f32", whole, 9, K, row_idx=R.ints(at))), S.mx4_values(want))


def test_rows_at_odd_addresses():
    """Rows that start between 16-byte boundaries: a slice of a longer buffer."""
    r = np.random.default_rng(3)
    x = R.grid(r.standard_normal((5, 264)), "bf16")
    flat = torch.zeros(5 * 264 + 8, dtype=torch.bfloat16, device="cuda")
    for off in (1, 3):
        view = flat[off:off + 5 * 264].view(5, 264)
        view.copy_(R.dev(x, "bf16"))
        assert torch.equal(L.op_mx4_load("bf16", L.op_quant_mx4("bf16", view), 5, 264), R.dev(S.mx4_values(x), "bf16"))


# ------------------------------------------------------------------ the product
def check_product(dtype, a, w, out):
    """out = a w^T for float64 values a and w, to the bound of its float32 sums and its own rounding."""
    want = a @ w.T
    err = np.abs(host(out) - want)
    tol = S.product_error(a, w) + np.abs(want) * R.HALF_STEP[dtype]
    assert (err <= tol).all(), float((err - tol).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 5, 32), (3, 33, 70), (16, 64, 256), (17, 100, 300), (32, 32, 512), (33, 129, 640),
                                   (64, 160, 1000), (70, 257, 768), (128, 128, 256), (130, 300, 1024), (200, 64, 2048), (257, 513, 513),
                                   (300, 704, 256), (5, 1024, 4096), (64, 96, 18944)])
def test_product(dtype, M, N, K):
    r = np.random.default_rng(M * 7 + N * 3 + K)
    x = R.grid(r.standard_normal((M, K)) * np.exp(0.7 * r.standard_normal(K)), dtype)
    w = R.grid(0.02 * r.standard_normal((N, K)) * np.exp(0.7 * r.standard_normal((N, 1))), "bf16")
    out = L.op_linear_mx4(dtype, L.op_quant_mx4(dtype, R.dev(x, dtype)), M, L.op_quant_mx4("bf16", R.dev(w, "bf16")), N, K)
    check_product(dtype, S.mx4_values(x), S.mx4_values(w), out)


@pytest.mark.parametrize("M,N,K", [(1, 40, 512), (33, 65, 300), (64, 200, 4096), (200, 130, 1024), (300, 270, 768)])
def test_product_of_small_numbers_is_exact(M, N, K):
    """Levels times one power of two each: every partial sum is a float32 number, so the order cannot matter."""
    r = np.random.default_rng(M + N + K)
    a, w = (R.LEVELS[r.integers(0, 8, (n, K))] * r.choice([-1, 1], (n, K)) for n in (M, N))
    a[:, 0], w[:, 0] = 6, 6    # (most blocks hold a 6, and those that do not have a smaller power of two)
    out = L.op_linear_mx4("f32", put(a * 2.0 ** -7), M, put(w * 2.0 ** 5), N, K)
    assert np.array_equal(host(out), a @ w.T / 4)


def test_each_element_meets_its_own():
    """One element of a row at a time against one of a weight row, each block with its own power of two."""
    K = 1024
    a = np.zeros((K, K))
    a[np.arange(K), np.arange(K)] = 2.0 ** (np.arange(K) // 32 % 20 - 9)
    r = np.random.default_rng(0)
    w = S.mx4_values(R.grid(r.standard_normal((96, K)) * np.exp(r.uniform(-3, 3, (96, K // 32))).repeat(32, 1), "f32"))
    out = L.op_linear_mx4("f32", put(a), K, put(w), 96, K)
    assert np.array_equal(host(out), a @ w.T)


@pytest.mark.parametrize("M,N,K", [(3, 40, 700), (70, 100, 300), (300, 260, 512)])
def test_nan_blocks_reach_their_row_and_column_only(M, N, K):
    r = np.random.default_rng(M)
    x, w = (R.grid(r.standard_normal((n, K)), "f32") for n in (M, N))
    x[M // 2, K - 1], w[N - 1, 3] = np.inf, np.nan
    out = host(L.op_linear_mx4("f32", L.op_quant_mx4("f32", R.dev(x)), M, L.op_quant_mx4("f32", R.dev(w)), N, K))
    bad = np.zeros((M, N), bool)
    bad[M // 2], bad[:, N - 1] = True, True
    assert np.array_equal(np.isnan(out), bad)
    a, b = np.nan_to_num(S.mx4_values(x)), np.nan_to_num(S.mx4_values(w))
    assert (np.abs(out - a @ b.T)[~bad] <= (S.product_error(a, b) + np.abs(a @ b.T) * S.U)[~bad]).all()


def test_extreme_scales():
    """Powers of two at both ends: what a float32 sum holds comes out, what it does not is zero or infinite."""
    K = 64
    a, w = np.zeros((4, K)), np.zeros((4, K))
    a[0, 0], a[1, 0], a[2, 0], a[3, 40] = 6 * 2.0 ** 120, 2.0 ** -125, -1.5, 4 * 2.0 ** -20
    w[0, 0], w[1, 0], w[2, 40], w[3, 0] = 2.0 ** -124, 6 * 2.0 ** 119, 3 * 2.0 ** 30, 0
    out = host(L.op_linear_mx4("f32", put(a), 4, put(w), 4, K))
    want = np.zeros((4, 4))
    want[0] = [6 * 2.0 ** -4, np.inf, 0, 0]
    want[1] = [0, 6 * 2.0 ** -6, 0, 0]
    want[2] = [-1.5 * 2.0 ** -124, -9 * 2.0 ** 119, 0, 0]
    want[3, 2] = 12 * 2.0 ** 10
    assert np.array_equal(out, want)


def test_rows_that_are_not_there_have_no_say():
    """Scale bytes behind the last row, whatever they hold, and codes behind K."""
    r = np.random.default_rng(9)
    for M, N, K in ((5, 37, 300), (65, 33, 256), (257, 300, 512)):
        x, w = (R.grid(r.standard_normal((n, K)), "f32") for n in (M, N))
        out = []
        for fill in (0, 255, 0x7f):
            bufs = []
            for t in (x, w):
                buf, told = S.mx4_pack(t)
                buf[~told] = fill
                bufs.append(torch.from_numpy(buf).cuda())
            out.append(L.op_linear_mx4("f32", bufs[0], M, bufs[1], N, K))
        assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])
        check_product("f32", S.mx4_values(x), S.mx4_values(w), out[0])
