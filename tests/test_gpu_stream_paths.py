"""The kernels among which the 4-bit maps, the norm and the log probabilities choose, against 64 bits; the operators together, on other
streams, captured and replayed; offsets past 32 bits; refusals of the binding.  Tolerances as in test_gpu_mx4 and its neighbours."""
import numpy as np
import pytest
import torch

from paper_2506_06295_amd import binding as L
from tests import lowbit_ref as R
from tests import stream_ref as S
from tests.test_gpu_lowbit import host
from tests.test_gpu_norm8 import check_rows8

pytestmark = pytest.mark.gpu


def randn(seed, *shape, dtype="bf16"):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def product_ok(dtype, a, w, M, N, K, out):
    """out against the float64 product of the values that a and w hold (op_mx4_load, whose own tests are test_gpu_mx4's)."""
    x, y = L.op_mx4_load("f32", a, M, K).double(), L.op_mx4_load("f32", w, N, K).double()
    want, mass = x @ y.t(), x.abs() @ y.abs().t()
    tol = (-(-K // 64) + 24) * 4 * S.U * mass + want.abs() * R.HALF_STEP[dtype]
    return bool(((out.double() - want).abs() <= tol).all())


# ------------------------------------------------------------------ kernels by name
# M, N, K -> tile, and whether the contraction is sliced.  Tiles of 64 rows and more have one to seven steps of 256 elements, fewer than their rings hold and
# more; columns that fill whole 16 bytes and columns that do not.
PRODUCTS = [
    (183, 160, 1, 128, 64, 0), (1366, 161, 263, 128, 64, 0), (4359, 98, 525, 128, 64, 0), (4332, 96, 514, 128, 64, 0),
    (105, 4198, 801, 128, 64, 0), (2788, 136, 1106, 128, 64, 0), (5663, 136, 1581, 128, 64, 0), (347, 5768, 1, 128, 128, 0),
    (2503, 781, 267, 128, 128, 0), (389, 4207, 571, 128, 128, 0), (284, 5752, 577, 128, 128, 0), (264, 5594, 857, 128, 128, 0),
    (286, 5688, 1080, 128, 128, 0), (279, 5584, 1619, 128, 128, 0), (686, 5528, 2, 192, 128, 0), (698, 5772, 270, 192, 128, 0),
    (3669, 1063, 519, 192, 128, 0), (1041, 3704, 525, 192, 128, 0), (3239, 1162, 778, 192, 128, 0),
    (5569, 680, 1064, 192, 128, 0), (1107, 3608, 1576, 192, 128, 0), (3814, 2200, 1, 192, 256, 0),
    (2321, 3274, 281, 192, 256, 0), (1300, 5396, 522, 192, 256, 0), (2318, 3280, 536, 192, 256, 0),
    (1544, 4609, 825, 192, 256, 0), (1285, 5744, 1062, 192, 256, 0), (1600, 4744, 1567, 192, 256, 0),
    (2148, 3416, 14, 256, 128, 0), (3149, 1955, 276, 256, 128, 0), (1368, 4451, 530, 256, 128, 0),
    (1059, 5384, 534, 256, 128, 0), (1200, 4866, 792, 256, 128, 0), (1025, 5520, 1054, 256, 128, 0),
    (986, 5536, 1607, 256, 128, 0), (5491, 4416, 49, 256, 192, 0), (2557, 4702, 263, 256, 192, 0),
    (2522, 4795, 566, 256, 192, 0), (4506, 2632, 734, 256, 192, 0), (4425, 2686, 813, 256, 192, 0),
    (3775, 3088, 1084, 256, 192, 0), (3713, 3224, 1674, 256, 192, 0), (5469, 2400, 2, 256, 256, 0),
    (4020, 3180, 275, 256, 256, 0), (2446, 4938, 544, 256, 256, 0), (3437, 3632, 559, 256, 256, 0),
    (3353, 3785, 813, 256, 256, 0), (5559, 2264, 1048, 256, 256, 0), (2158, 5408, 1610, 256, 256, 0), (1, 1, 774, 16, 16, 0),
    (1, 4, 809, 16, 16, 0), (1, 1, 16561, 16, 16, 1), (1, 4, 17855, 16, 16, 1), (1, 1, 32, 16, 48, 0), (1, 4, 32, 16, 48, 0),
    (1, 1, 8536, 16, 48, 1), (1, 4, 8898, 16, 48, 1), (113, 2121, 279, 16, 80, 0), (311, 764, 276, 16, 80, 0),
    (1, 2173, 10755, 16, 80, 1), (1, 2288, 14122, 16, 80, 1), (161, 1102, 262, 32, 32, 0), (116, 1540, 276, 32, 32, 0),
    (1, 955, 12400, 32, 32, 1), (1, 836, 14613, 32, 32, 1), (508, 642, 520, 32, 64, 0), (250, 1308, 539, 32, 64, 0),
    (20, 2097, 8757, 32, 64, 1), (3, 2048, 14072, 32, 64, 1), (165, 2701, 1424, 64, 64, 0), (300, 1760, 1521, 64, 64, 0),
    (34, 1373, 13558, 64, 64, 1), (34, 1520, 19399, 64, 64, 1), (388, 2659, 6363, 64, 80, 0), (435, 2540, 8630, 64, 80, 0),
    (33, 2809, 22302, 64, 80, 1), (43, 2692, 23212, 64, 80, 1),
]


@pytest.mark.parametrize("M,N,K,bm,bn,sliced", PRODUCTS)
def test_product_kernels(M, N, K, bm, bn, sliced):
    tile, slices, _ = L.plan_linear_mx4(M, N, K)
    assert tile == (bm, bn) and (slices > 1) == bool(sliced)
    a, w = L.op_quant_mx4("bf16", randn(M, M, K)), L.op_quant_mx4("bf16", randn(N + 1, N, K))
    for dtype in ("bf16", "f32"):
        out = L.op_linear_mx4(dtype, a, M, w, N, K)
        assert product_ok(dtype, a, w, M, N, K, out)
        assert torch.equal(out, L.op_linear_mx4(dtype, a, M, w, N, K))   # the same bits again


def test_scratch_and_free_memory_have_no_say():
    """Whatever scratch and results held before."""
    M, N, K = 34, 1373, 13558
    lib, st = L.lib(), torch.cuda.current_stream().cuda_stream
    a, w = L.op_quant_mx4("bf16", randn(1, M, K)), L.op_quant_mx4("bf16", randn(2, N, K))
    need = lib.dllmc_op_linear_mx4_scratch_bytes(M, N, K)
    assert need > 0
    got = []
    for fill in (0, 255):
        scratch = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        out = torch.full((M, N), float("nan"), device="cuda")
        assert lib.dllmc_op_linear_mx4(0, a.data_ptr(), M, w.data_ptr(), N, K, out.data_ptr(), scratch.data_ptr(), need, st) == 0
        got.append(out)
    assert torch.equal(*got)
    l = randn(3, 5, 50000)
    need = lib.dllmc_op_logprobs_scratch_bytes(1, 5, 50000, 20)
    assert need > 0
    got = []
    for fill in (0, 255):
        scratch = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        h, ids, top = torch.empty(5, device="cuda"), torch.empty(5, 20, dtype=torch.int32, device="cuda"), torch.empty(5, 20, device="cuda")
        assert lib.dllmc_op_logprobs(1, l.data_ptr(), 50000, 5, 50000, None, 0, 20, None, h.data_ptr(), ids.data_ptr(), top.data_ptr(),
                                     scratch.data_ptr(), need, st) == 0
        got.append((h, ids, top))
    assert all(torch.equal(x, y) for x, y in zip(*got))


# ------------------------------------------------------------------ logits: slices, chunks, alignments
def tokens_ok(dtype, l, top_k):
    """Against float64 on the device; ids exactly, values to the bound of tests/stream_ref.py with the sums' chain at its longest."""
    logp, h, ids, top = L.op_logprobs(dtype, l, l[:, :3].argsort(1).int().contiguous() * (l.shape[1] // 3), top_k)
    d = l.double()
    lse = torch.logsumexp(d, 1, keepdim=True)
    lp = d - lse
    p = lp.exp()
    e1 = (p * (d.amax(1, keepdim=True) - d)).sum(1, keepdim=True)
    tol = S.U * (l.shape[1] / 256 + 60 + 4 * e1) + 8 * S.U * (lp.abs() + 1)
    want = torch.sort(d, dim=1, descending=True, stable=True).indices[:, :top_k]
    given = (l[:, :3].argsort(1) * (l.shape[1] // 3))
    assert torch.equal(ids.long(), want)
    for got, at in ((top, want), (logp, given)):
        assert ((got.double() - lp.gather(1, at)).abs() <= tol.gather(1, at)).all()
    # the entropy's sum of p log p: the same chain, times its terms
    assert ((h.double() + (p * lp).sum(1)).abs() <= S.U * (l.shape[1] / 256 + 80 + 8 * e1[:, 0]) * (2 + e1[:, 0])).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,k", [(1, 8192, 5), (1, 8193, 5), (1, 262144, 64), (2, 270000, 64), (1500, 270001, 3), (1024, 8200, 7), (1023, 8200, 7), (256, 20000, 7), (255, 20000, 7),
                                   (1100, 40001, 20), (1, 1 << 24, 10), (3, (1 << 24) - 5, 2)])
def test_slices_and_chunks(dtype, M, V, k):
    if M * V > 1 << 28 and dtype == "f32":
        M = 1030   # (memory of the reference)
    tokens_ok(dtype, randn(V + k, M, V, dtype=dtype) * 3, k)


@pytest.mark.parametrize("dtype,per", [("f32", 4), ("bf16", 8)])
def test_every_alignment_of_rows(dtype, per):
    """Rows that start anywhere in their 16 bytes and end anywhere in them."""
    flat = randn(9, 3 * 20020 + 64, dtype=dtype) * 3
    for off in range(per):
        for V in (9, 8191, 20000 + off, 20013):
            l = flat[off:off + 3 * 20015].view(3, 20015)[:, :V]
            same = l.contiguous()
            got, want = L.op_logprobs(dtype, l, None, 6), L.op_logprobs(dtype, same, None, 6)
            assert torch.equal(got[2], want[2])
            assert torch.allclose(got[1], want[1], rtol=1e-4, atol=1e-5) and torch.allclose(got[3], want[3], rtol=1e-4, atol=1e-5)
            tokens_ok(dtype, l, 6)


def test_tokens_and_ties_do_not_depend_on_the_cut():
    """The same row alone (slices) and among many (one workgroup a row): the same tokens, whatever is equal."""
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    l = torch.randint(0, 40, (1200, 30000), generator=g, device="cuda").to(torch.bfloat16)
    many = L.op_logprobs("bf16", l, None, 64)
    for i in (0, 7, 1199):
        assert torch.equal(L.op_logprobs("bf16", l[i:i + 1], None, 64)[2], many[2][i:i + 1])


def test_no_given_tokens():
    l = randn(1, 3, 500)
    for none in (torch.zeros(3, 0, dtype=torch.int32, device="cuda"), torch.zeros(3, 4, dtype=torch.int32, device="cuda")[:, 4:]):
        logp, h, ids, top = L.op_logprobs("bf16", l, none, 2)
        assert logp.shape == (3, 0) and torch.equal(h, L.op_logprobs("bf16", l)[1]) and ids.shape == (3, 2)


# ------------------------------------------------------------------ the operators together
def chain(stream, x, gain, w8, w4, head, d, vocab, given):
    """The end of a model in few bits: a sublayer's output joins the stream, its norm goes through an 8-bit map, the next one's through a 4-bit map to
    logits, of which tokens' log probabilities are taken."""
    q, scale, s = L.op_norm_quant8("bf16", stream, gain, 1e-5, x=x)
    y = L.op_linear_i8("bf16", q, scale, *w8, d)
    h4, s2 = L.op_norm_mx4("bf16", s, gain, 1e-5, x=y)
    z = L.op_linear_mx4("bf16", h4, x.shape[0], w4, d, d)
    h5, s3 = L.op_norm_mx4("bf16", s2, gain, 1e-5, x=z)
    logits = L.op_linear_mx4("f32", h5, x.shape[0], head, vocab, d)
    return (s, y, s2, z, s3, logits, *L.op_logprobs("f32", logits, given, 5)), (q, scale, h4, h5)


def chain_inputs(M=40, d=512, vocab=1000):
    stream, x = randn(1, M, d) * 2, randn(2, M, d)
    gain = (1 + 0.1 * randn(3, d).float()).to(torch.bfloat16)
    w8 = L.op_quant8("bf16", randn(4, d, d) * 0.05)
    w4 = L.op_quant_mx4("bf16", randn(5, d, d) * 0.05)
    head = L.op_quant_mx4("bf16", randn(6, vocab, d) * 0.05)
    given = torch.randint(0, vocab, (M, 2), device="cuda", dtype=torch.int32)
    return stream, x, gain, w8, w4, head, d, vocab, given


def test_chain():
    """Every link against its plain form on what the link before it gave."""
    a = chain_inputs()
    stream, x, gain, w8, w4, head, d, vocab, given = a
    (s, y, s2, z, s3, logits, logp, ent, ids, top), (q, scale, h4, h5) = chain(*a)
    want, h = S.norm(host(stream), host(x), host(gain), 1e-5, "bf16")
    assert np.array_equal(host(s), want.astype(np.float64))
    check_rows8(q, scale, h, d)
    ref = host(q)[:, :d] @ host(w8[0])[:, :d].T * host(scale)[:, None] * host(w8[1])   # (whole numbers first: float64 has them exactly)
    assert (np.abs(host(y) - ref) <= np.abs(ref) * (2.0 ** -8 + 4 * S.U) + 1e-30).all()
    for total, add, held, w, n, out in ((s2, y, h4, w4, d, z), (s3, z, h5, head, vocab, logits)):
        before = s if total is s2 else s2
        want, h = S.norm(host(before), host(add), host(gain), 1e-5, "bf16")
        assert np.array_equal(host(total), want.astype(np.float64))
        v = host(L.op_mx4_load("f32", held, 40, d))
        lo, hi = S.mx4_values(h * (1 - 4 * S.U)), S.mx4_values(h * (1 + 4 * S.U))
        assert ((v == lo) | (v == hi)).all()
        assert product_ok("f32" if out is logits else "bf16", held, w, 40, n, d, out)
    want = S.logprobs(host(logits), given.cpu().numpy(), 5)
    assert np.array_equal(ids.cpu().numpy(), want[2])
    for got, at, tol in ((logp, 0, 4), (ent, 1, 5), (top, 3, 6)):
        assert (np.abs(host(got) - want[at]) <= want[tol]).all()


def test_chain_captured_and_replayed():
    a = list(chain_inputs())
    eager = [t.clone() for t in chain(*a)[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        chain(*a)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = chain(*a)[0]
    for replay in range(4):
        if replay == 2:   # other inputs in the same places
            a[1].copy_(randn(77, *a[1].shape))
            eager = [t.clone() for t in chain(*a)[0]]
        for t in held:
            t.zero_()
        graph.replay()
        other = torch.randn(512, 512, device="cuda").softmax(1).sum()   # eager work between replays
        torch.cuda.synchronize()
        assert torch.isfinite(other)
        assert all(torch.equal(x, y) for x, y in zip(held, eager)), replay


def test_slices_captured():
    """Calls with scratch and two launches, replayed."""
    a, w = L.op_quant_mx4("bf16", randn(1, 1, 16561)), L.op_quant_mx4("bf16", randn(2, 1, 16561))
    l = randn(3, 2, 100000)

    def both():
        return (L.op_linear_mx4("f32", a, 1, w, 1, 16561), *L.op_logprobs("bf16", l, None, 9)[1:])
    eager = [t.clone() for t in both()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for _ in range(3):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, eager))


def test_other_streams():
    a = chain_inputs()
    want = chain(*a)[0]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for s in streams:
        with torch.cuda.stream(s):
            got.append(chain(*a)[0])
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(x, y) for x, y in zip(g, want))


# ------------------------------------------------------------------ offsets past 32 bits
def test_blocks_of_more_than_4_gib():
    rows, K, n = 2_200_000, 4096, 70
    w = torch.zeros(L.mx4_bytes(rows, K), dtype=torch.uint8, device="cuda")
    assert w.numel() > 1 << 32
    x = randn(1, n, K)
    few = L.op_quant_mx4("bf16", x)
    # the last rows' blocks put where they lie among all of them
    first = rows - n
    src, told = S.mx4_pack(host(x))
    assert np.array_equal(src[told], few.cpu().numpy()[told])
    half, start = K // 2, -(-rows * K // 2 // 256) * 256
    w[first * half:rows * half] = few[:n * half]
    s = few[n * half:].view(-1, K // 256, 2, 32, 4).permute(0, 3, 1, 2, 4).reshape(-1, K // 32)[:n]      # [row, (c, b, j)]
    groups = w[start:].view(-1, K // 256, 2, 32, 4)
    at = torch.arange(first, rows, device="cuda")
    groups[at // 32, :, :, at % 32] = s.view(n, K // 256, 2, 4)
    values = L.op_mx4_load("f32", few, n, K)
    assert torch.equal(L.op_mx4_load("f32", w, rows, K, row_idx=at.int()), values)
    for M in (3, 300):
        a = L.op_quant_mx4("bf16", randn(2, M, K))
        out = L.op_linear_mx4("bf16", a, M, w, rows, K)
        assert torch.equal(out[:, first:], L.op_linear_mx4("bf16", a, M, few, n, K)) or product_ok("bf16", a, few, M, n, K, out[:, first:])
        assert (out[:, :first] == 0).all()
        del out


def test_streams_and_logits_past_4_gib():
    d, rows = 4096, 700_000
    stream = torch.zeros(rows, d, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([rows - 1, 5, rows - 7, 600_001], device="cuda")
    part = randn(1, 4, d)
    stream[at] = part
    gain = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    for got, want in zip(L.op_norm_quant8("bf16", stream, gain, 1e-5, row_idx=at.int())[:2], L.op_norm_quant8("bf16", part, gain, 1e-5)[:2]):
        assert torch.equal(got, want)
    whole = L.op_norm_mx4("bf16", stream, gain, 1e-5, x=torch.zeros_like(stream))
    assert torch.equal(whole[1], stream)
    few = L.op_norm_mx4("bf16", part, gain, 1e-5)[0]
    assert torch.equal(L.op_mx4_load("bf16", whole[0], rows, d, row_idx=at.int()), L.op_mx4_load("bf16", few, 4, d))
    q, scale = L.op_quant8("bf16", stream)
    assert torch.equal(L.op_load8("bf16", q, scale, d)[at], L.op_load8("bf16", *L.op_quant8("bf16", part), d))
    del whole, q, scale
    logits = stream.view(-1)[:22_000 * 126_464].view(22_000, 126_464)
    logits[-3:] = randn(2, 3, 126_464)
    got, want = L.op_logprobs("bf16", logits, None, 4), L.op_logprobs("bf16", logits[-3:].clone(), None, 4)
    assert torch.equal(got[2][-3:], want[2]) and torch.allclose(got[1][-3:], want[1], rtol=1e-5)


# ------------------------------------------------------------------ refusals of the binding
def test_binding_refuses():
    f = torch.zeros
    x, g = f(4, 96, device="cuda"), f(96, device="cuda")
    ids = f(4, dtype=torch.int32, device="cuda")
    mx, q, sc = L.op_quant_mx4("f32", x), *L.op_quant8("f32", x)
    l = f(3, 50, device="cuda")
    bad = [
        lambda: L.op_norm_quant8("bf16", x, g, 1e-5),                                      # other dtype
        lambda: L.op_norm_quant8("f32", x, g, 1e-5, stream_dtype="bf16"),
        lambda: L.op_norm_quant8("f32", x.to(torch.bfloat16), g, 1e-5, stream_dtype="bf16"),  # a stream of fewer bits than what joins it
        lambda: L.op_norm_quant8("f32", x, g[:-1], 1e-5),
        lambda: L.op_norm_quant8("f32", x, g, 1e-5, x=x[:3]),
        lambda: L.op_norm_quant8("f32", x, g, 1e-5, x=x[:3], row_idx=ids),
        lambda: L.op_norm_quant8("f32", x, g, 1e-5, row_idx=ids.long()),
        lambda: L.op_norm_quant8("f32", x, g, 1e-5, x=x.clone(), row_idx=ids, sum_out=x),  # in place of listed rows
        lambda: L.op_norm_quant8("f32", x, g, -1.0),
        lambda: L.op_norm_quant8("f32", x, g, float("inf")),
        lambda: L.op_norm_quant8("f32", f(0, 96, device="cuda"), g, 1e-5),
        lambda: L.op_norm_mx4("f32", x.t(), g, 1e-5),                                      # not contiguous
        lambda: L.op_norm_mx4("f32", x, g.cpu(), 1e-5),
        lambda: L.op_load8("f32", q, sc, 300), lambda: L.op_load8("f32", q, sc[:3], 96), lambda: L.op_load8("f32", x, sc, 96),
        lambda: L.op_quant_mx4("bf16", x), lambda: L.op_quant_mx4("f32", x.t()), lambda: L.op_quant_mx4("f32", x, row_idx=ids.long()),
        lambda: L.op_mx4_load("f32", mx, 33, 96), lambda: L.op_mx4_load("f32", mx[:-1], 4, 96), lambda: L.op_mx4_load("f32", mx, 4, 300),
        lambda: L.op_linear_mx4("f32", mx, 4, mx, 33, 96), lambda: L.op_linear_mx4("f32", mx, 33, mx, 4, 96),
        lambda: L.op_linear_mx4("f32", mx, 4, mx, 4, 300), lambda: L.op_linear_mx4("f32", mx, 0, mx, 4, 96),
        lambda: L.op_logprobs("bf16", l, None, 3), lambda: L.op_logprobs("f32", l.t(), None, 3), lambda: L.op_logprobs("f32", l, None, 65),
        lambda: L.op_logprobs("f32", l, None, -1), lambda: L.op_logprobs("f32", l, f(3, 2, device="cuda"), 3),
        lambda: L.op_logprobs("f32", l, f(2, 2, dtype=torch.int32, device="cuda"), 3),
        lambda: L.op_logprobs("f32", l, f(3, dtype=torch.int32, device="cuda"), 3),
        lambda: L.op_logprobs("f32", l[:1].expand(3, 50), None, 3),                        # rows over each other
        lambda: L.op_logprobs("f32", f(0, 50, device="cuda"), None, 3),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(L.DllmcError):
            call()
            pytest.fail(f"call {i} was taken")
