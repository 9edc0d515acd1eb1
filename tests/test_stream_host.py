"""Refusals of the norm in few bits, the 4-bit blocks and the token log probabilities, and the sizes they state: no GPU needed, nothing is
launched."""
import ctypes
import os

import pytest
import torch

from paper_2506_06295_amd import binding
from tests.test_lowbit_host import near, p

if not os.path.exists(binding.LIB_PATH):
    pytest.skip("libdllmc.so not built in this tree", allow_module_level=True)

L = binding.lib()
EINVAL, ENOMEM = -1, -4
F32, BF16 = 0, 1
INF = float("inf")


def f(v):
    return ctypes.c_float(v)


def test_sizes():
    assert L.dllmc_mx4_bytes(100, 4096) == 100 * 2048 + 128 * 128   # 2048 bytes of codes a row, scales for 128 rows
    assert L.dllmc_mx4_bytes(1, 1) == 256 + 32 * 8                  # scales start at a multiple of 256
    assert L.dllmc_mx4_bytes(33, 257) == 33 * 256 + 64 * 16
    assert L.dllmc_mx4_bytes(1 << 24, 131072) == (1 << 24) * (65536 + 4096)   # past 32 bits
    for bad in ((0, 1), (1, 0), (-1, 5), ((1 << 24) + 1, 5), (1, 131073)):
        assert L.dllmc_mx4_bytes(*bad) == 0
        with pytest.raises(binding.DllmcError):
            binding.mx4_bytes(*bad)
    with pytest.raises(binding.DllmcError):
        binding.mx4_bytes(1 << 40, 32)
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), ((1 << 22) + 1, 1, 1), (1, 1, 131073), (1 << 18, (1 << 17) + 1, 64)):
        assert L.dllmc_op_linear_mx4_scratch_bytes(*bad) == 0
    for bad in ((2, 1, 1, 1), (F32, 0, 1, 1), (F32, 1 << 23, 1, 1), (F32, 1 << 22, 1 << 19, 1), (F32, 1, 0, 1), (F32, 1, 1 << 25, 1), (F32, 1, 1, 65), (F32, 1, 1, -1)):
        assert L.dllmc_op_logprobs_scratch_bytes(*bad) == 0


NORM = dict(dtype=BF16, stream_dtype=F32, x=p(0), stream=p(1), rows=9, row_idx=p(2), M=4, d=100, gain=p(3), eps=f(1e-5), sum_out=p(4))
NORM8 = dict(NORM, q=p(5), scale=p(6), hip=None)
NORM4 = dict(NORM, out=p(5), hip=None)
LOAD8 = dict(dtype=BF16, q=p(0), scale=p(1), q_rows=9, K=100, row_idx=p(2), M=4, out=p(3), hip=None)
QUANT = dict(dtype=BF16, x=p(0), x_rows=9, row_idx=p(1), M=4, K=100, out=p(2), hip=None)
LOAD4 = dict(dtype=BF16, mx=p(0), rows=9, K=100, row_idx=p(1), M=4, out=p(2), hip=None)
LINEAR = dict(dtype=BF16, a=p(0), M=4, w=p(1), N=8, K=100, out=p(2), scratch=p(3), nbytes=1 << 36, hip=None)
LOGPROBS = dict(dtype=BF16, logits=p(0), ld=120, M=4, vocab=100, tokens=p(1), n=2, k=3, logp=p(2), entropy=p(3), ids=p(4), top=p(5),
                scratch=p(6), nbytes=1 << 36, hip=None)
CALLS = {"dllmc_op_norm_quant8": NORM8, "dllmc_op_norm_mx4": NORM4, "dllmc_op_load8": LOAD8, "dllmc_op_quant_mx4": QUANT,
         "dllmc_op_mx4_load": LOAD4, "dllmc_op_linear_mx4": LINEAR, "dllmc_op_logprobs": LOGPROBS}

BAD_NORM = [dict(dtype=2), dict(dtype=F32, stream_dtype=BF16), dict(stream_dtype=2), dict(stream=None), dict(gain=None), dict(M=0), dict(M=-1),
            dict(M=1 << 23), dict(M=1 << 24), dict(d=0), dict(d=131073), dict(rows=0), dict(row_idx=None, M=10), dict(eps=f(-1e-6)), dict(eps=f(INF)),
            dict(eps=f(float("nan"))), dict(x=near(p(0), 1)), dict(stream=near(p(1), 2)), dict(gain=near(p(3), 1)), dict(row_idx=near(p(2), 2)),
            dict(sum_out=near(p(4), 2)),
            dict(sum_out=p(1)),                                  # the stream's place, but rows are listed
            dict(sum_out=near(p(1), 400), row_idx=None),         # over the stream, but not row for row
            dict(sum_out=p(0)),                                  # x is of another type
            dict(sum_out=near(p(0), 4), stream_dtype=BF16), dict(sum_out=p(2)), dict(sum_out=p(3)), dict(sum_out=p(5)),
            dict(sum_out=near(p(5), -400 * 4 + 16))]
BAD = {
    "dllmc_op_norm_quant8": BAD_NORM + [dict(q=None), dict(scale=None), dict(q=near(p(5), 8)), dict(scale=near(p(6), 2)), dict(q=p(0)), dict(q=p(1)),
                                        dict(q=p(2)), dict(q=p(3)), dict(scale=p(0)), dict(scale=p(5)), dict(scale=p(1)), dict(scale=p(4))],
    "dllmc_op_norm_mx4": BAD_NORM + [dict(out=None), dict(out=near(p(5), 8)), dict(out=p(0)), dict(out=near(p(1), 9 * 400 - 16)), dict(out=p(2)),
                                     dict(out=p(3)), dict(out=p(4))],
    "dllmc_op_load8": [dict(dtype=2), dict(q=None), dict(scale=None), dict(out=None), dict(q_rows=0), dict(K=0), dict(K=131073), dict(M=0),
                       dict(M=1 << 24), dict(row_idx=None, M=10), dict(q=near(p(0), 4)), dict(out=near(p(3), 1)), dict(scale=near(p(1), 2)),
                       dict(out=p(0)), dict(out=p(1)), dict(out=p(2))],
    "dllmc_op_quant_mx4": [dict(dtype=2), dict(x=None), dict(out=None), dict(x_rows=0), dict(K=0), dict(K=131073), dict(M=0), dict(M=1 << 24),
                           dict(row_idx=None, M=10), dict(out=near(p(2), 8)), dict(x=near(p(0), 1)), dict(row_idx=near(p(1), 2)), dict(out=p(0)),
                           dict(out=p(1))],
    "dllmc_op_mx4_load": [dict(dtype=2), dict(mx=None), dict(out=None), dict(rows=0), dict(K=0), dict(M=0), dict(M=1 << 24),
                          dict(row_idx=None, M=10), dict(mx=near(p(0), 8)), dict(out=near(p(2), 1)), dict(out=p(0)), dict(out=p(1))],
    "dllmc_op_linear_mx4": [dict(dtype=2), dict(a=None), dict(w=None), dict(out=None), dict(M=0), dict(N=0), dict(K=0), dict(K=131073),
                            dict(M=(1 << 22) + 1), dict(N=(1 << 24) + 1), dict(M=1 << 18, N=(1 << 17) + 1), dict(a=near(p(0), 8)),
                            dict(w=near(p(1), 4)), dict(out=near(p(2), 8)), dict(scratch=near(p(3), 8)), dict(out=p(0)), dict(out=p(1))],
    "dllmc_op_logprobs": [dict(dtype=2), dict(logits=None), dict(ld=99), dict(M=0), dict(M=1 << 23), dict(M=1 << 22, vocab=1 << 19, ld=1 << 19), dict(vocab=0), dict(vocab=(1 << 24) + 1, ld=1 << 25),
                          dict(n=-1), dict(n=0), dict(n=65537), dict(k=-1), dict(k=0), dict(k=65), dict(tokens=None), dict(logp=None),
                          dict(ids=None), dict(top=None), dict(n=0, tokens=None, logp=None, k=0, ids=None, top=None, entropy=None),
                          dict(logits=near(p(0), 1)), dict(tokens=near(p(1), 2)), dict(logp=near(p(2), 2)), dict(entropy=near(p(3), 2)),
                          dict(ids=near(p(4), 1)), dict(top=near(p(5), 2)), dict(scratch=near(p(6), 8)), dict(logp=p(0)), dict(entropy=p(0)),
                          dict(ids=p(0)), dict(top=p(0)), dict(logp=p(1)), dict(top=p(1)), dict(logp=p(3)), dict(top=p(4)), dict(entropy=p(5))],
}


@pytest.mark.parametrize("name,change", [(n, c) for n in CALLS for c in BAD[n]], ids=lambda v: v if isinstance(v, str) else "-".join(v))
def test_refused(name, change):
    assert getattr(L, name)(*dict(CALLS[name], **change).values()) == EINVAL


def test_binding_refuses_host_tensors():
    x, g = torch.zeros(2, 64), torch.zeros(64)
    for call in (lambda: binding.op_norm_quant8("f32", x, g, 1e-5), lambda: binding.op_norm_mx4("f32", x, g, 1e-5),
                 lambda: binding.op_load8("f32", torch.zeros(2, 128, dtype=torch.int8), torch.zeros(2), 64),
                 lambda: binding.op_quant_mx4("f32", x), lambda: binding.op_mx4_load("f32", torch.zeros(512, dtype=torch.uint8), 1, 64),
                 lambda: binding.op_linear_mx4("f32", torch.zeros(512, dtype=torch.uint8), 1, torch.zeros(512, dtype=torch.uint8), 1, 64),
                 lambda: binding.op_logprobs("f32", x)):
        with pytest.raises(binding.DllmcError):
            call()
