"""Attention weights with the rows' log-sum-exp given, over caches of every format and by every kernel that reads it, against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2506_06295_amd import binding as L
from tests import lowbit_ref as R
from tests.test_gpu_lowbit import Case, host

pytestmark = pytest.mark.gpu

# Mq, n, H_q, H_kv, d_h: beyond the keys that one workgroup's registers hold, and one shape within them (given or not: the same)
SHAPES = [(1, 1100, 4, 4, 64), (9, 1500, 4, 2, 64), (20, 2100, 2, 2, 128), (33, 1031, 7, 1, 128), (5, 1300, 2, 1, 256), (6, 200, 4, 2, 128)]


@pytest.mark.parametrize("dtype,fmt", [("bf16", "bf16"), ("bf16", "kv4"), ("f32", "f32"), ("f32", "kv4")])
@pytest.mark.parametrize("Mq,n,H_q,H_kv,d_h", SHAPES)
@pytest.mark.parametrize("mode", ["flat", "holes"])
def test_given_log_sum_exp(dtype, fmt, Mq, n, H_q, H_kv, d_h, mode):
    B = 3
    c = Case(n + Mq, dtype, B, Mq, n, H_q, H_kv, d_h, None if mode == "flat" else np.array([n, 0, n - 3]), mode)
    q, k, _, where = c.device(fmt)
    _, lse, probs, _, reach = c.reference(fmt)
    acc = R.grid(c.r.random((B, n)), "f32")
    args = (dtype, fmt, q, k, c.rows, n, H_q, H_kv, d_h)
    got = L.op_attention_weights(*args, lse=R.dev(lse), acc=R.dev(acc), **where)
    # a score is off by ds, and with it the exponential; the given logarithm is rounded to float32, and so is its product with
    # log2 e: both are in ds; then the exponential's own error and the sum over queries and heads.  What is below 2^-126 may be zero.
    ds, rows = R.score_error(reach, lse, d_h), Mq * H_q
    want, tol = acc.astype(np.float64), np.full((B, n), rows * 2.0 ** -126)
    for b, (pos, _) in enumerate(c.where):
        for a in range(H_q):
            want[b, pos] += probs[b][a].sum(0)
            tol[b, pos] += (probs[b][a] * (2 * ds[b, :, a] + rows * 2.0 ** -23 + 2.0 ** -20)[:, None]).sum(0)
    if n <= 1024:   # (the sums are worked out: n additions of each row)
        tol += n * 2.0 ** -23 * want
        assert torch.equal(got, L.op_attention_weights(*args, acc=R.dev(acc), **where))
    assert (np.abs(host(got) - want) <= tol + want * 2.0 ** -23).all()
    # and in place, where it was
    again = R.dev(acc)
    L.op_attention_weights(*args, lse=R.dev(lse), acc=again, out=again, **where)
    assert torch.equal(again, got)


@pytest.mark.parametrize("Mq,n,H_q,H_kv,d_h", SHAPES)
def test_the_sums_of_an_attention_over_the_same_cache(Mq, n, H_q, H_kv, d_h):
    """A captured attention and the weights from its sums, replayed with other queries between, as they come eagerly."""
    c, other = (Case(s, "bf16", 2, Mq, n, H_q, H_kv, d_h) for s in (31, 32))
    q, k, v, _ = c.device("kv4")
    first, second = q.clone(), other.device("kv4")[0]
    args = (c.rows, n, H_q, H_kv, d_h)

    def both():
        o, lse = L.op_attention_kv4("bf16", q, k, v, *args, with_lse=True)
        return o, lse, L.op_attention_weights("bf16", "kv4", q, k, *args, lse=lse)

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both()
    torch.cuda.current_stream().wait_stream(stream)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        res = both()
    for x in (first, second, first, second):
        q.copy_(x)
        want = [t.clone() for t in both()]
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, res))


def test_the_same_bits_with_other_work_between():
    """Kernels whose ranges are joined, and one that walks all keys, again and again on the same operands with other operands' calls
    behind and before them."""
    for B, Mq, n, H_q, H_kv, dtype, cut in ((1, 51, 4608, 32, 32, "bf16", 1), (16, 1, 1099, 28, 4, "bf16", 0), (16, 1, 4099, 28, 4, "bf16", 1),
                                            (1, 9, 2000, 4, 4, "f32", 1)):
        one, two = (Case(s, dtype, B, Mq, n, H_q, H_kv, 128).device("kv4") for s in (41, 42))
        args = (B * n, n, H_q, H_kv, 128)
        assert (L.plan_attention_kv4(dtype, B, Mq, n, H_q, H_kv, 128)[2] > 1) == cut
        first = L.op_attention_kv4(dtype, *one[:3], *args, with_lse=True)
        for _ in range(10):
            L.op_attention_kv4(dtype, *two[:3], *args, with_lse=True)
            again = L.op_attention_kv4(dtype, *one[:3], *args, with_lse=True)
            assert all(torch.equal(a, b) for a, b in zip(first, again))
