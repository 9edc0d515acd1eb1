"""Calls with scratch and two launches, different inputs on several streams at once: slices of a 4-bit map and of rows of logits."""
import pytest
import torch

from paper_2506_06295_amd import binding as L
from tests.test_gpu_stream_paths import randn

pytestmark = pytest.mark.gpu


def test_scratch_on_several_streams():
    M, N, K = 34, 1373, 13558
    assert L.lib().dllmc_op_linear_mx4_scratch_bytes(M, N, K) > 0 and L.lib().dllmc_op_logprobs_scratch_bytes(1, 2, 100000, 9) > 0
    inputs = [(L.op_quant_mx4("bf16", randn(i, M, K)), L.op_quant_mx4("bf16", randn(10 + i, N, K)), 3 * randn(20 + i, 2, 100000)) for i in range(4)]

    def both(a, w, l):
        return (L.op_linear_mx4("f32", a, M, w, N, K), *L.op_logprobs("bf16", l, None, 9)[1:])
    want = [both(*x) for x in inputs]
    assert not torch.equal(want[0][0], want[1][0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in inputs]
    got = [[] for _ in inputs]
    for _ in range(8):
        for s, x, g in zip(streams, inputs, got):
            with torch.cuda.stream(s):
                g.append(both(*x))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for one in g:
            assert all(torch.equal(a, b) for a, b in zip(one, w))


def test_scratch_in_graphs_on_several_streams():
    """A graph a stream, replayed together; each has scratch of its own."""
    M, N, K = 34, 1373, 13558
    inputs = [(L.op_quant_mx4("bf16", randn(i, M, K)), L.op_quant_mx4("bf16", randn(10 + i, N, K)), 3 * randn(20 + i, 2, 100000)) for i in range(2)]

    def both(a, w, l):
        return (L.op_linear_mx4("f32", a, M, w, N, K), *L.op_logprobs("bf16", l, None, 9)[1:])
    want = [both(*x) for x in inputs]
    graphs, held = [torch.cuda.CUDAGraph() for _ in inputs], []
    for g, x in zip(graphs, inputs):
        with torch.cuda.graph(g):
            held.append(both(*x))
    streams = [torch.cuda.Stream() for _ in inputs]
    for _ in range(4):
        for h in held:
            for t in h:
                t.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for h, w in zip(held, want):
            assert all(torch.equal(a, b) for a, b in zip(h, w))
