"""GPU tests of the norm in few bits with rows at both ends of float32 and eps = 0: reciprocal roots past float32 (rows of subnormals) and below its
normal numbers (rows near its largest) against the plain 64-bit form.  h has the three roundings that it has elsewhere (tests/test_gpu_norm8.py)."""
import numpy as np
import pytest

from paper_2506_06295_amd import binding as L
from tests import lowbit_ref as R
from tests import stream_ref as S
from tests.test_gpu_lowbit import host
from tests.test_gpu_norm8 import TYPES, check_rows4, check_rows8

pytestmark = pytest.mark.gpu

# a width for every kernel: a wavefront a row, 256 and 512 threads with the row in registers, rows that are read again
WIDTHS = [96, 1000, 1500, 4096, 4101, 8000, 12288, 25000]


def rows_at_the_ends(d, stream_dtype):
    r = np.random.default_rng(d)
    rows = [r.standard_normal(d) * 2.0 ** p for p in (-146, -135, -131, -128.5, -127.5, -126.5, -125, 124)]
    rows += [r.choice([-1, 1], d) * r.uniform(1, 1.9, d) * 2.0 ** p for p in (125, 126)]   # doubled: a root mean square up to 2^127.5
    smallest, largest = np.zeros(d), np.ones(d)
    smallest[d // 2], largest[d // 3] = 2.0 ** (-133 if stream_dtype == "bf16" else -149), -1.9 * 2.0 ** 126
    return R.grid(np.stack(rows + [smallest, largest, np.zeros(d)]), stream_dtype)


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype,stream_dtype", TYPES)
@pytest.mark.parametrize("add", [False, True])
def test_rows_at_both_ends(dtype, stream_dtype, d, add):
    stream = rows_at_the_ends(d, stream_dtype)
    M = len(stream)
    x = R.grid(stream, dtype) if add else None
    gain = R.grid(1 + 0.1 * np.random.default_rng(1).standard_normal(d), dtype)
    s, h = S.norm(stream, x, gain, 0.0, stream_dtype)
    assert np.isfinite(h[s.any(1)]).all() and np.isnan(h[-1]).all()
    args = (dtype, R.dev(stream, stream_dtype), R.dev(gain, dtype), 0.0)
    kw = dict(x=None if x is None else R.dev(x, dtype), stream_dtype=stream_dtype)
    q, scale, total = L.op_norm_quant8(*args, **kw)
    if add:
        assert np.array_equal(host(total), s.astype(np.float64))
    check_rows8(q, scale, h, d)
    check_rows4(host(L.op_mx4_load("f32", L.op_norm_mx4(*args, **kw)[0], M, d)), h)
