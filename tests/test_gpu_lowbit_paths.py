"""The kernels among which the operators in fewer bits choose, each named by its plan, against 64 bits; the operators together, on
other streams, captured and replayed; offsets past 32 bits; refusals of the binding.  Tolerances as in test_gpu_lowbit."""
import numpy as np
import pytest
import torch

from paper_2506_06295_amd import binding as L
from tests import lowbit_ref as R
from tests.test_gpu_lowbit import Case, host

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ kernels by name
def tiles_of(plan, B, Mq, H_q, H_kv):
    return -(-Mq * (H_q // H_kv) // plan[0]) * B * H_kv


ATTEND = [  # dtype, B, Mq, n, H_q, H_kv, d_h -> rows, wavefronts, what becomes of the tiles
    ("bf16", 16, 1, 3679, 8, 8, 64, 16, 4, "cut"), ("bf16", 1, 5, 90, 2, 1, 64, 16, 4, "whole"), ("bf16", 1, 9, 1385, 1, 1, 64, 16, 8, "cut"),
    ("bf16", 1, 1, 141, 1, 1, 64, 16, 8, "whole"), ("bf16", 1, 84, 7413, 8, 8, 64, 32, 8, "cut"), ("bf16", 4, 37, 919, 28, 4, 64, 32, 8, "whole"),
    ("bf16", 1, 1320, 6304, 8, 4, 64, 128, 4, "cut"), ("bf16", 1, 1030, 62, 16, 8, 64, 128, 4, "whole"),
    ("bf16", 1, 3, 2255, 2, 1, 128, 16, 4, "cut"), ("bf16", 2, 5, 93, 7, 1, 128, 16, 4, "whole"), ("bf16", 1, 7, 1085, 1, 1, 128, 16, 8, "cut"),
    ("bf16", 1, 2, 131, 1, 1, 128, 16, 8, "whole"), ("bf16", 1, 5, 3607, 224, 32, 128, 32, 8, "cut"), ("bf16", 1, 528, 665, 8, 8, 128, 32, 8, "whole"),
    ("bf16", 4, 529, 4136, 2, 2, 128, 128, 4, "cut"), ("bf16", 4, 592, 299, 28, 4, 128, 128, 4, "mixed"), ("bf16", 16, 70, 33, 32, 32, 128, 128, 4, "whole"),
    ("bf16", 2, 598, 919, 14, 2, 128, 256, 8, "cut"), ("bf16", 16, 612, 326, 7, 1, 128, 256, 8, "mixed"), ("bf16", 1, 1025, 65, 32, 32, 128, 256, 8, "whole"),
    ("bf16", 1, 20, 416, 1, 1, 256, 16, 4, "cut"), ("bf16", 2, 30, 70, 3, 3, 256, 16, 4, "whole"), ("f32", 1, 20, 1238, 1, 1, 64, 16, 4, "cut"),
    ("f32", 1, 33, 404, 1, 1, 128, 16, 4, "cut"), ("f32", 1, 18, 316, 1, 1, 256, 16, 4, "cut"), ("f32", 2, 40, 50, 4, 2, 256, 16, 4, "whole"),
]


@pytest.mark.parametrize("dtype,B,Mq,n,H_q,H_kv,d_h,rows,waves,kind", ATTEND)
@pytest.mark.parametrize("where", ["flat", "holes"])
def test_attention_kernels(dtype, B, Mq, n, H_q, H_kv, d_h, rows, waves, kind, where):
    plan = L.plan_attention_kv4(dtype, B, Mq, n, H_q, H_kv, d_h)
    whole = {"whole": tiles_of(plan, B, Mq, H_q, H_kv), "cut": 0, "mixed": plan[3]}[kind]
    assert plan[:2] == (rows, waves) and plan[3] == whole and (kind == "whole") == (plan[2] == 1)
    assert kind != "mixed" or 0 < plan[3] < tiles_of(plan, B, Mq, H_q, H_kv)
    lens = None if where == "flat" else np.random.default_rng(n).choice([n, n - 1, n // 2, 1, 0], B)
    c = Case(n + Mq, dtype, B, Mq, n, H_q, H_kv, d_h, lens, where)
    q, k, v, at = c.device("kv4")
    out, lse = L.op_attention_kv4(dtype, q, k, v, c.rows, n, H_q, H_kv, d_h, with_lse=True, **at)
    dev = [torch.from_numpy(x).cuda() for x in (c.q.astype(np.float64), c.values("kv4", c.k), c.values("kv4", c.v))]
    want, want_lse, mass, reach, _ = R.attend_device(*dev, c.where, H_q, H_kv, d_h)
    got, got_lse = host(out).reshape(want.shape), lse.cpu().numpy().astype(np.float64)
    ds, some = R.score_error(reach, want_lse, d_h), np.isfinite(want_lse)
    assert np.array_equal(np.isneginf(got_lse), ~some)
    assert (np.abs(got_lse[some] - want_lse[some]) <= (ds + n * 2.0 ** -24)[some] + np.abs(want_lse[some]) * 2.0 ** -22).all()
    rel = 2 * ds + n * 2.0 ** -23 + 2.0 ** -21 + (2.0 ** -16 if dtype == "bf16" else 0.0)
    lost = n * 2.0 ** -125 * np.abs(c.values("kv4", c.v)).max()
    assert (np.abs(got - want) <= mass * rel[..., None] + np.abs(want) * R.HALF_STEP[dtype] + lost).all()
    assert (got[~some] == 0).all()


WEIGH = [  # dtype, format, B, Mq, n, H_q, H_kv, d_h -> keys of a wavefront, ranges (0: one launch; 2: several), rows, several shares
    ("bf16", "bf16", 1, 40, 200, 2, 2, 64, 32, 0, 16, 1), ("bf16", "bf16", 1, 24, 306, 1, 1, 64, 64, 0, 16, 1),
    ("bf16", "bf16", 1, 9, 538, 1, 1, 64, 96, 0, 16, 0), ("bf16", "bf16", 1, 5, 1377, 1, 1, 64, 64, 2, 16, 0),
    ("bf16", "bf16", 1, 39, 1351, 1, 1, 64, 64, 2, 64, 0), ("bf16", "bf16", 1, 1056, 1029, 8, 4, 64, 64, 1, 64, 1),
    ("bf16", "bf16", 1, 18, 601, 1, 1, 128, 96, 0, 16, 1), ("bf16", "bf16", 1, 1, 1038, 1, 1, 128, 64, 2, 16, 0),
    ("bf16", "bf16", 1, 3, 1040, 7, 1, 128, 64, 2, 32, 0), ("bf16", "bf16", 1, 22, 1081, 2, 1, 128, 64, 2, 64, 1),
    ("bf16", "bf16", 4, 529, 1059, 4, 4, 128, 64, 1, 64, 1), ("bf16", "bf16", 1, 19, 265, 1, 1, 256, 64, 0, 16, 1),
    ("bf16", "bf16", 1, 3, 525, 7, 1, 256, 32, 2, 16, 1), ("bf16", "bf16", 4, 37, 523, 14, 2, 256, 32, 1, 16, 1),
    ("bf16", "kv4", 1, 17, 621, 1, 1, 64, 96, 0, 16, 1), ("bf16", "kv4", 1, 26, 1185, 1, 1, 64, 64, 2, 32, 0),
    ("bf16", "kv4", 2, 264, 1042, 16, 8, 64, 64, 1, 64, 1), ("bf16", "kv4", 1, 17, 526, 1, 1, 128, 96, 0, 16, 1),
    ("bf16", "kv4", 1, 17, 1083, 2, 1, 128, 64, 2, 64, 1), ("bf16", "kv4", 1, 627, 1027, 14, 2, 128, 64, 1, 64, 1),
    ("bf16", "kv4", 1, 12, 557, 2, 1, 256, 32, 2, 16, 1), ("f32", "f32", 1, 19, 933, 1, 1, 64, 128, 0, 16, 1),
    ("f32", "f32", 1, 22, 1376, 2, 1, 64, 32, 2, 16, 1), ("f32", "f32", 1, 10, 279, 2, 1, 128, 64, 0, 16, 1),
    ("f32", "f32", 1, 1050, 533, 2, 2, 128, 32, 1, 16, 1), ("f32", "f32", 1, 25, 305, 1, 1, 256, 32, 1, 16, 1),
    ("f32", "f32", 1, 3, 604, 7, 1, 256, 32, 2, 16, 1), ("f32", "kv4", 1, 4, 572, 7, 1, 64, 96, 0, 16, 1),
    ("f32", "kv4", 1, 34, 1081, 1, 1, 64, 64, 2, 16, 1), ("f32", "kv4", 1, 9, 308, 2, 1, 128, 64, 0, 16, 1),
    ("f32", "kv4", 1, 12, 576, 2, 1, 128, 64, 2, 16, 1), ("f32", "kv4", 1, 18, 363, 1, 1, 256, 32, 1, 16, 1),
    ("bf16", "bf16", 1, 9, 857, 1, 1, 64, 128, 0, 16, 0), ("bf16", "bf16", 1, 18, 902, 1, 1, 128, 128, 0, 16, 1), ("bf16", "kv4", 1, 17, 1001, 1, 1, 64, 128, 0, 16, 1),
    ("bf16", "kv4", 1, 17, 771, 1, 1, 128, 128, 0, 16, 1), ("f32", "kv4", 1, 4, 969, 7, 1, 64, 128, 0, 16, 1), ("f32", "f32", 1, 21, 767, 1, 1, 64, 96, 0, 16, 1),
]


@pytest.mark.parametrize("dtype,fmt,B,Mq,n,H_q,H_kv,d_h,keys,ranges,rows,shares", WEIGH)
@pytest.mark.parametrize("where", ["flat", "holes"])
def test_weight_kernels(dtype, fmt, B, Mq, n, H_q, H_kv, d_h, keys, ranges, rows, shares, where):
    plan = L.plan_attention_weights(dtype, fmt, B, Mq, n, H_q, H_kv, d_h)
    assert (plan[0], min(plan[1], 2), plan[2], int(plan[3] > 1)) == (keys, ranges, rows, shares)
    lens = None if where == "flat" else np.random.default_rng(n).choice([n, n - 1, n // 2, 1, 0], B)
    c = Case(n + Mq, dtype, B, Mq, n, H_q, H_kv, d_h, lens, where)
    q, k, v, at = c.device(fmt)
    acc = R.grid(c.r.random((B, n)), "f32")
    got = host(L.op_attention_weights(dtype, fmt, q, k, c.rows, n, H_q, H_kv, d_h, acc=R.dev(acc), **at))
    dev = [torch.from_numpy(x).cuda() for x in (c.q.astype(np.float64), c.values(fmt, c.k))]
    _, lse, _, reach, columns = R.attend_device(*dev, None, c.where, H_q, H_kv, d_h)
    ds = R.score_error(reach, lse, d_h)
    sums, err = columns(3 * ds + (n + Mq * H_q) * 2.0 ** -23 + 2.0 ** -20)
    want, tol = acc.astype(np.float64), np.full((B, n), Mq * H_q * 2.0 ** -126)
    for b, (pos, _) in enumerate(c.where):
        want[b, pos] += sums[b]
        tol[b, pos] += err[b]
    assert (np.abs(got - want) <= tol + want * 2.0 ** -23).all()


LINEAR = [  # M, N, K -> rows, columns, several slices, tile kernel
    (3, 3, 603, 16, 16, 0, 0), (3, 3, 5632, 16, 16, 1, 0), (3, 4217, 695, 16, 48, 0, 0), (3, 1673, 10471, 16, 48, 1, 0),
    (3, 12494, 675, 16, 80, 0, 0), (3, 2121, 11110, 16, 80, 1, 0), (3, 7996, 2022, 32, 32, 0, 0), (17, 794, 8817, 32, 32, 1, 0),
    (17, 8199, 616, 32, 48, 0, 0), (3, 1385, 9268, 32, 48, 1, 0), (3, 16369, 787, 32, 64, 0, 0), (3, 5250, 13219, 32, 64, 1, 0),
    (20, 16549, 622, 32, 80, 0, 0), (4326, 3, 634, 48, 16, 0, 0), (710, 3, 6786, 48, 16, 1, 0), (4266, 37, 627, 64, 16, 0, 0),
    (2026, 3, 9829, 64, 16, 1, 0), (8347, 17, 735, 64, 32, 0, 0), (2158, 17, 6265, 64, 32, 1, 0), (66, 5477, 804, 64, 48, 0, 0),
    (1463, 34, 7095, 64, 48, 1, 0), (33, 8692, 729, 64, 64, 0, 0), (3, 2579, 12887, 64, 64, 1, 0), (18, 18773, 727, 64, 80, 0, 0),
    (3, 6763, 16791, 64, 80, 1, 0), (8532, 35, 702, 128, 16, 0, 0), (4328, 3, 5699, 128, 16, 1, 0), (8847, 17, 9216, 128, 64, 1, 0),
    (66, 16435, 1052, 128, 80, 0, 0), (66, 2084, 13149, 128, 80, 1, 0),
]


def check_linear(dtype, M, N, K):
    g = torch.Generator(device="cuda")
    g.manual_seed(M + 3 * N + 7 * K)
    kp = L.i8_row_bytes(K)
    a, w = (torch.zeros(m, kp, dtype=torch.int8, device="cuda") for m in (M, N))
    for t in (a, w):
        t[:, :K] = torch.randint(-127, 128, (t.shape[0], K), generator=g, device="cuda", dtype=torch.int8)
    sa, sw = (torch.rand(m, generator=g, device="cuda") + 0.01 for m in (M, N))
    got = L.op_linear_i8(dtype, a, sa, w, sw, K)
    for i in range(0, M, 4096):
        s = slice(i, i + 4096)
        want = (a[s].double() @ w.double().t()) * sa[s].double()[:, None] * sw.double()
        # the sum as float32, two products, the result's rounding
        tol = want.abs() * (3 * 2.0 ** -24 + (R.HALF_STEP["bf16"] if dtype == "bf16" else 0.0)) * 1.0001
        assert ((got[s].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K,rows,cols,slices,whole", LINEAR)
def test_linear_ring(dtype, M, N, K, rows, cols, slices, whole):
    shape, S, w = L.plan_linear_i8(M, N, K)
    assert shape == (rows, cols) and (S > 1) == bool(slices) and w == bool(whole)
    check_linear(dtype, M, N, K)


STEPS = (1, 129, 300, 500, 640, 700, 1000)  # one to eight 128-byte steps
TILES = [(128, 64, 512, 2141, STEPS), (128, 128, 131, 8242, STEPS), (128, 256, 257, 16851, STEPS), (192, 128, 132, 17136, STEPS),
         (192, 256, 395, 16573, STEPS), (256, 128, 50146, 65, STEPS[:2]), (256, 128, 194, 17888, STEPS[2:]), (256, 256, 797, 14214, STEPS)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,M,N,lengths", TILES)
def test_linear_tiles(dtype, rows, cols, M, N, lengths):
    """Every shape at fewer and more steps than its rings are deep."""
    for K in lengths:
        assert L.plan_linear_i8(M, N, K) == ((rows, cols), 1, True)
        check_linear(dtype, M, N, K)


def test_linear_tile_step_counts():
    """One to nine steps of whatever tile kernel takes them."""
    for K in range(64, 1200, 128):
        for M, N in ((260, 4100), (700, 2052), (1500, 3000), (2100, 4096), (4000, 4100)):
            check_linear("bf16", M, N, K)


@pytest.mark.parametrize("n", [255, 256, 257, 1023, 1024, 1025, 4095, 4096, 4097, 8191, 8192, 8193, 16384, 16385, 32768, 32769])
def test_evict_register_classes(n):
    r = np.random.default_rng(n)
    acc = R.grid(r.integers(0, 1 << 20, (2, n)) / 64.0, "f32")
    acc[1] = R.grid(r.exponential(1.0, n), "f32")
    for keep in (1, n // 3, n - 1):
        got = L.op_evict(R.dev(acc), keep, 2 * n, 0, min(keep, 5))
        want = R.evict(acc, keep, R.present(2, n, 2 * n, None, None), None, n, 0, min(keep, 5))
        for g, w in zip(got, want):
            assert np.array_equal(g.cpu().numpy(), w)


@pytest.mark.parametrize("n", [700, 17000, 40000])
def test_evict_pages_and_holes(n):
    """Lengths, rows from pages, entries that are no row, NaN and infinite weights: keys in registers and loaded again."""
    r = np.random.default_rng(n)
    B, rows = 3, 2 * n
    acc = R.grid(r.exponential(1.0, (B, n)), "f32")
    acc[1, r.integers(0, n, 50)] = np.nan
    acc[2, r.integers(0, n, 50)] = np.inf
    m = r.integers(0, rows, (B, n)).astype(np.int32)
    m[r.random((B, n)) < 0.3] = -1
    m[0, :20] = rows
    lens = np.array([n - 7, n, 0], np.int32)
    for keep in (5, n // 2, n):
        got = L.op_evict(R.dev(acc), keep, rows, 2, 3, lens=R.ints(lens), row_map=R.ints(m))
        want = R.evict(acc, keep, R.present(B, n, rows, lens, m), lens, n, 2, 3)
        for g, w in zip(got, want):
            assert np.array_equal(g.cpu().numpy(), w, equal_nan=g.dtype == torch.float32)


# ------------------------------------------------------------------ together
class Layer:
    """Projections in 8 bits fill a 4-bit cache, rows attend, positions accumulate weight, the cache is halved, the rest attends again."""

    def __init__(self, seed, dtype="bf16", B=2, n=150, Mq=20, H_q=8, H_kv=2, d_h=128, d=512):
        self.dtype, self.B, self.n, self.Mq, self.H_q, self.H_kv, self.d_h, self.d = dtype, B, n, Mq, H_q, H_kv, d_h, d
        r = np.random.default_rng(seed)
        dkv, dq = H_kv * d_h, H_q * d_h
        self.w = [L.op_quant8(dtype, R.dev(R.grid(0.05 * r.standard_normal(s), dtype), dtype)) for s in ((dkv, d), (dkv, d), (dq, d), (d, dq))]
        self.keep = n // 2
        self.cache = [torch.zeros(L.kv4_bytes(B * n, H_kv, d_h), dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.small = [torch.zeros(L.kv4_bytes(B * self.keep, H_kv, d_h), dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.acc = torch.zeros(B, n, device="cuda")
        self.sel = R.ints(np.stack([b * n + np.sort(r.permutation(n)[:Mq]) for b in range(B)]).reshape(-1))

    def step(self, h):
        """h [B * n, d]: all rows' keys and values, the selected rows' attention."""
        dt, B, n, Mq, H_q, H_kv, d_h = self.dtype, self.B, self.n, self.Mq, self.H_q, self.H_kv, self.d_h
        a, sa = L.op_quant8(dt, h)
        for c, (w, sw) in zip(self.cache, self.w):
            L.op_kv4_store(dt, L.op_linear_i8(dt, a, sa, w, sw, self.d), c, B * n, H_kv, d_h)
        a, sa = L.op_quant8(dt, h, row_idx=self.sel)
        q = L.op_linear_i8(dt, a, sa, *self.w[2], self.d).view(B, Mq, H_q * d_h)
        o, lse = L.op_attention_kv4(dt, q, *self.cache, B * n, n, H_q, H_kv, d_h, with_lse=True)
        L.op_attention_weights(dt, "kv4", q, self.cache[0], B * n, n, H_q, H_kv, d_h, lse=lse, acc=self.acc, out=self.acc)
        kept, rows, lens, acc = L.op_evict(self.acc, self.keep, B * n, 2, 10)
        L.op_compact("kv4", rows, B * n, H_kv, d_h, self.cache[0], self.small[0], self.cache[1], self.small[1])
        o2 = L.op_attention_kv4(dt, q, *self.small, B * self.keep, self.keep, H_q, H_kv, d_h, lens=lens)
        a, sa = L.op_quant8(dt, o2.view(B * Mq, H_q * d_h))
        return L.op_linear_i8(dt, a, sa, *self.w[3], H_q * d_h), o, o2, kept, lens, acc, self.acc


def hidden(layer, seed):
    r = np.random.default_rng(seed)
    return R.dev(R.grid(r.standard_normal((layer.B * layer.n, layer.d)), layer.dtype), layer.dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_layer_in_fewer_bits(dtype):
    """The chain against the same chain of plain 64-bit forms, each fed with what the device's step before it gave."""
    y = Layer(1, dtype)
    h = hidden(y, 2)
    out, o, o2, kept, lens, acc, total = [t.clone() for t in y.step(h)]
    B, n, Mq, H_q, H_kv, d_h = y.B, y.n, y.Mq, y.H_q, y.H_kv, y.d_h

    def project(x, w):
        q, s = R.quant8(x.float().cpu().numpy())
        return (q.astype(np.float64) @ w[0][:, :x.shape[1]].double().cpu().numpy().T) * s.astype(np.float64)[:, None] * host(w[1])

    half = R.HALF_STEP[dtype]
    kv = [host(L.op_kv4_load("f32", c, B * n, H_kv, d_h)) for c in y.cache]
    for got, w in zip(kv, y.w):
        x = project(h, w)
        # the projection is off by half a step (and three float32 roundings), the row by a level's width: a third of the value, at least
        # an eighth of the block's maximum's power of two
        block = np.abs(x).reshape(-1, 32).max(1).repeat(32).reshape(x.shape)
        assert (np.abs(got - x) <= np.maximum(np.abs(x) / 3, block / 4) * (1 + 4 * half)).all()
    sel = y.sel.cpu().numpy()
    q = project(h[y.sel.long()], y.w[2])
    q = R.grid(q, dtype).astype(np.float64).reshape(B, Mq, H_q, d_h)
    k, v = (t.reshape(B * n, H_kv, d_h) for t in kv)
    where = R.present(B, n, B * n, None, None)
    want, lse, probs, mass, reach = R.attend(q, k, v, where, H_q, H_kv, d_h)
    # a query element may be the neighbour of the one here (a projection next to a border): one step, 2 * half
    ds = R.score_error(reach, lse, d_h) + reach * 2 * half
    rel = 2 * ds + n * 2.0 ** -23 + 2.0 ** -15
    assert (np.abs(host(o).reshape(want.shape) - want) <= mass * rel[..., None] + np.abs(want) * half).all()
    cols = np.stack([sum(probs[b][a].sum(0) for a in range(H_q)) for b in range(B)])
    tol = np.stack([sum((probs[b][a] * (3 * ds[b, :, a] + 2.0 ** -14)[:, None]).sum(0) for a in range(H_q)) for b in range(B)])
    assert (np.abs(host(total) - cols) <= tol).all()
    ref = R.evict(total.cpu().numpy(), y.keep, where, None, n, 2, 10)
    assert np.array_equal(kept.cpu().numpy(), ref[0]) and np.array_equal(lens.cpu().numpy(), ref[2]) and np.array_equal(acc.cpu().numpy(), ref[3])
    small = [host(L.op_kv4_load("f32", c, B * y.keep, H_kv, d_h)) for c in y.small]
    for got, full in zip(small, kv):
        assert np.array_equal(got, full[ref[1].reshape(-1)])
    want, lse, _, mass, reach = R.attend(q, *(t.reshape(-1, H_kv, d_h) for t in small), R.present(B, y.keep, B * y.keep, ref[2], None), H_q, H_kv, d_h)
    rel = 2 * (R.score_error(reach, lse, d_h) + reach * 2 * half) + n * 2.0 ** -23 + 2.0 ** -15
    assert (np.abs(host(o2).reshape(want.shape) - want) <= mass * rel[..., None] + np.abs(want) * half).all()
    want = project(o2.view(B * Mq, H_q * d_h), y.w[3])
    assert (np.abs(host(out) - want) <= np.abs(want) * (half + 2.0 ** -21)).all()


def test_captured_and_replayed():
    """A captured step gives what the eager one gives, replay after replay, with other inputs and eager work between."""
    eager, graphed = Layer(3), Layer(3)
    h = hidden(eager, 10)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        graphed.step(h)   # warm up
    torch.cuda.current_stream().wait_stream(stream)
    graphed.acc.zero_()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        res = graphed.step(h)
    graphed.acc.zero_()
    for i in range(4):
        h.copy_(hidden(eager, 10 + i))
        want = [t.clone() for t in eager.step(h)]
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, res):
            assert torch.equal(a, b), i
        L.op_attention_weights("bf16", "kv4", torch.zeros_like(want[1]), eager.cache[0], 300, 150, 8, 2, 128)


def test_two_streams_at_once():
    """Two layers that share nothing, each on a stream of its own, against themselves one after the other."""
    one = [Layer(s) for s in (5, 6)]
    two = [Layer(s) for s in (5, 6)]
    hs = [hidden(y, 20 + i) for i, y in enumerate(one)]
    want = [[[t.clone() for t in y.step(h)] for _ in range(3)] for y, h in zip(one, hs)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in two]
    got = [[], []]
    for _ in range(3):
        for i, (s, y, h) in enumerate(zip(streams, two, hs)):
            with torch.cuda.stream(s):
                got[i].append([t.clone() for t in y.step(h)])
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        for x, z in zip(a, b):
            assert all(torch.equal(p, q) for p, q in zip(x, z))


def test_same_bits_every_time():
    c = Case(9, "bf16", 2, 64, 1500, 8, 2, 128)
    q, k, v, _ = c.device("kv4")
    first = None
    for _ in range(5):
        o, lse = L.op_attention_kv4("bf16", q, k, v, c.rows, c.n, 8, 2, 128, with_lse=True)
        w = L.op_attention_weights("bf16", "kv4", q, k, c.rows, c.n, 8, 2, 128)
        if first is None:
            first = (o, lse, w)
        assert all(torch.equal(a, b) for a, b in zip(first, (o, lse, w)))


def test_a_cache_row_listed_twice():
    """Two positions may share a cache row: the key counts twice; rows may be read and moved twice."""
    c = Case(12, "bf16", 1, 9, 60, 2, 1, 128)
    q, k, v, _ = c.device("kv4")
    row_map = np.concatenate([np.arange(60), [5, 5, 17]])[None]
    out = L.op_attention_kv4("bf16", q, k, v, 60, 63, 2, 1, 128, row_map=R.ints(row_map))
    where = R.present(1, 63, 60, None, row_map)
    want, lse, _, mass, reach = R.attend(c.q.astype(np.float64), c.values("kv4", c.k), c.values("kv4", c.v), where, 2, 1, 128)
    rel = 2 * R.score_error(reach, lse, 128) + 2.0 ** -15
    assert (np.abs(host(out).reshape(want.shape) - want) <= mass * rel[..., None] + np.abs(want) * 2.0 ** -8).all()
    got = host(L.op_kv4_load("f32", k, 60, 1, 128, rows=R.ints([7, 7, 0, 7])))
    assert np.array_equal(got, c.values("kv4", c.k).reshape(60, 128)[[7, 7, 0, 7]])


# ------------------------------------------------------------------ offsets past 32 bits
def test_a_cache_of_more_than_4_gib():
    rows, H, d_h, n = 2_200_000, 32, 128, 70
    k, v = (torch.zeros(L.kv4_bytes(rows, H, d_h), dtype=torch.uint8, device="cuda") for _ in range(2))
    assert k.numel() > 1 << 32
    r = np.random.default_rng(1)
    at = rows - 1 - np.arange(n) * 3
    x = [R.grid(r.standard_normal((n, H * d_h)), "bf16") for _ in range(2)]
    for c, t in zip((k, v), x):
        L.op_kv4_store("bf16", R.dev(t, "bf16"), c, rows, H, d_h, rows=R.ints(at))
    want = [R.kv4_values(t) for t in x]
    for c, t in zip((k, v), want):
        assert np.array_equal(host(L.op_kv4_load("f32", c, rows, H, d_h, rows=R.ints(at))), t)
    for Mq in (2, 150):
        q = R.grid(r.standard_normal((1, Mq, H, d_h)), "bf16")
        qd, m = R.dev(q.reshape(1, Mq, -1), "bf16"), R.ints(at[None])
        out = L.op_attention_kv4("bf16", qd, k, v, rows, n, H, H, d_h, row_map=m)
        kk, vv = (t.reshape(n, H, d_h) for t in want)
        ref, lse, probs, mass, reach = R.attend(q.astype(np.float64), kk, vv, [(np.arange(n), np.arange(n))], H, H, d_h)
        ds = R.score_error(reach, lse, d_h)
        assert (np.abs(host(out).reshape(ref.shape) - ref) <= mass * (2 * ds + 2.0 ** -15)[..., None] + np.abs(ref) * 2.0 ** -8).all()
        got = host(L.op_attention_weights("bf16", "kv4", qd, k, rows, n, H, H, d_h, row_map=m))
        cols = sum(probs[0][a].sum(0) for a in range(H))
        tol = sum((probs[0][a] * (3 * ds[0, :, a] + 2.0 ** -14)[:, None]).sum(0) for a in range(H))
        assert (np.abs(got[0] - cols) <= tol).all()
    dst = [torch.zeros(L.kv4_bytes(n, H, d_h), dtype=torch.uint8, device="cuda") for _ in range(2)]
    L.op_compact("kv4", R.ints(at), rows, H, d_h, k, dst[0], v, dst[1])
    for c, t in zip(dst, want):
        assert np.array_equal(host(L.op_kv4_load("f32", c, n, H, d_h)), t)


def test_plain_rows_past_4_gib():
    src, H, d_h = 700_000, 32, 128
    x = torch.zeros(src, H * d_h, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([src - 1, 3, src - 2, 600_001], dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x[rows.long()] = torch.randn(4, H * d_h, generator=g, device="cuda").to(torch.bfloat16)
    out = torch.zeros(4, H * d_h, dtype=torch.bfloat16, device="cuda")
    L.op_compact("bf16", rows, src, H, d_h, x, out)
    assert torch.equal(out, x[rows.long()])
    # the keys of a sequence at the end of it
    q = torch.randn(1, 5, H * d_h, generator=g, device="cuda").to(torch.bfloat16)
    a = L.op_attention_weights("bf16", "bf16", q, x, src, 4, H, H, d_h, row_map=rows[None].contiguous())
    b = L.op_attention_weights("bf16", "bf16", q, out, 4, 4, H, H, d_h)
    assert torch.equal(a, b)
    big, scale = L.op_quant8("bf16", x)
    few, few_scale = L.op_quant8("bf16", x[rows.long()])
    assert torch.equal(big[rows.long()], few) and torch.equal(scale[rows.long()], few_scale)
    w, sw = L.op_quant8("bf16", out)
    assert torch.equal(L.op_linear_i8("f32", big, scale, w, sw, H * d_h)[rows.long()], L.op_linear_i8("f32", few, few_scale, w, sw, H * d_h))


def test_largest_batch():
    """65535 sequences of 128 heads, one workgroup each: as many as a launch takes.  With one key in two there all is exact."""
    B, H, d_h, R_ = 65535, 128, 64, 96
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    k, v = (torch.zeros(L.kv4_bytes(R_, H, d_h), dtype=torch.uint8, device="cuda") for _ in range(2))
    for c in (k, v):
        L.op_kv4_store("bf16", torch.randn(R_, H * d_h, generator=g, device="cuda").to(torch.bfloat16), c, R_, H, d_h)
    q = torch.randn(B, 1, H * d_h, generator=g, device="cuda", dtype=torch.bfloat16)
    m = torch.randint(0, R_, (B, 2), generator=g, device="cuda", dtype=torch.int32)
    m[torch.arange(B, device="cuda"), m[:, 0] % 2] = -1
    at = m.amax(1).long()
    out = L.op_attention_kv4("bf16", q, k, v, R_, 2, H, H, d_h, row_map=m)
    values = L.op_kv4_load("bf16", v, R_, H, d_h)
    for i in range(0, B, 8192):
        assert torch.equal(out[i:i + 8192, 0], values[at[i:i + 8192]])
    del out
    assert torch.equal(L.op_attention_weights("bf16", "kv4", q, k, R_, 2, H, H, d_h, row_map=m), H * (m >= 0).float())


# ------------------------------------------------------------------ refusals of the binding
def test_binding_refuses():
    f = torch.zeros
    cache = f(L.kv4_bytes(8, 2, 64), dtype=torch.uint8, device="cuda")
    x, q = f(4, 128, device="cuda"), f(1, 3, 128, device="cuda")
    bad = [
        lambda: L.op_kv4_store("f32", f(4, 128), cache, 8, 2, 64),                                   # not on the device
        lambda: L.op_kv4_store("bf16", x, cache, 8, 2, 64),                                          # other dtype
        lambda: L.op_kv4_store("f32", f(128, 4, device="cuda").t(), cache, 8, 2, 64),                # not contiguous
        lambda: L.op_kv4_store("f32", x, cache[:-1], 8, 2, 64),                                      # cache too small
        lambda: L.op_kv4_store("f32", x, cache, 8, 2, 64, rows=f(4, dtype=torch.int64, device="cuda")),
        lambda: L.op_kv4_store("f32", x, cache, 8, 2, 64, rows=f(5, dtype=torch.int32, device="cuda")),
        lambda: L.op_kv4_store("f32", f(9, 128, device="cuda"), cache, 8, 2, 64),                    # more rows than the cache has
        lambda: L.op_kv4_store("f32", f(0, 128, device="cuda"), cache, 8, 2, 64),
        lambda: L.op_attention_kv4("f32", q, cache, cache, 8, 9, 2, 2, 64),                          # n beyond the cache
        lambda: L.op_attention_kv4("f32", q, cache, cache, 8, 8, 2, 2, 64, lens=f(2, dtype=torch.int32, device="cuda")),
        lambda: L.op_attention_kv4("f32", q, cache, cache, 8, 8, 2, 2, 64, row_map=f(1, 7, dtype=torch.int32, device="cuda")),
        lambda: L.op_attention_kv4("f32", q, cache, cache, 8, 8, 3, 2, 64),
        lambda: L.op_attention_weights("f32", "bf16", q, cache, 8, 8, 2, 2, 64),
        lambda: L.op_attention_weights("f32", "f32", q, x, 4, 4, 2, 2, 64, acc=f(1, 5, device="cuda")),
        lambda: L.op_evict(f(1, 8, device="cuda"), 9, 8),
        lambda: L.op_evict(f(1, 8, device="cuda"), 0, 8),
        lambda: L.op_evict(f(1, 8, device="cuda"), 4, 8, first=3, last=2),
        lambda: L.op_evict(f(1, 8, device="cuda"), 4, 7),
        lambda: L.op_compact("f32", f(3, dtype=torch.int32, device="cuda"), 4, 2, 64, x, x),         # in place
        lambda: L.op_compact("f32", f(3, dtype=torch.int32, device="cuda"), 4, 2, 64, x, f(2, 128, device="cuda"), dst_rows=2),
        lambda: L.op_linear_i8("f32", f(2, 100, dtype=torch.int8, device="cuda"), f(2, device="cuda"),
                               f(2, 128, dtype=torch.int8, device="cuda"), f(2, device="cuda"), 100),  # rows not padded
    ]
    for i, call in enumerate(bad):
        with pytest.raises(L.DllmcError):
            call()
            pytest.fail(f"call {i} was taken")
