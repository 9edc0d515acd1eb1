"""Refusals of the operators in fewer bits, and the sizes they state: no GPU needed, nothing is launched."""
import ctypes
import os
import random

import pytest

from paper_2506_06295_amd import binding

if not os.path.exists(binding.LIB_PATH):
    pytest.skip("libdllmc.so not built in this tree", allow_module_level=True)

L = binding.lib()
EINVAL, ENOMEM = -1, -4
F32, BF16, KV4 = 0, 1, 2


def p(k):
    """Addresses 2^40 bytes apart: never read, nothing overlaps."""
    return ctypes.c_void_p((k + 1) << 40)


def test_sizes():
    # 100 rows, 4 heads of 128: 64 bytes of codes and 4 scales per row and head
    assert L.dllmc_kv4_bytes(100, 4, 128) == 100 * 4 * 64 + 100 * 4 * 4
    assert L.dllmc_kv4_bytes(3, 1, 32) == 256 + 3          # scales start at a multiple of 256
    assert L.dllmc_kv4_bytes(1 << 24, 32, 128) == (1 << 24) * 32 * 68   # past 32 bits
    for bad in ((0, 1, 32), (1, 0, 32), (1, 1, 0), (1, 1, 33), (1, 1, 16), (-1, 1, 32), (1 << 25, 1, 32), (1, 4096, 32)):
        assert L.dllmc_kv4_bytes(*bad) == 0
    assert [L.dllmc_i8_row_bytes(k) for k in (1, 127, 128, 129, 131072)] == [128, 128, 128, 256, 131072]
    assert L.dllmc_i8_row_bytes(0) == L.dllmc_i8_row_bytes(-5) == L.dllmc_i8_row_bytes(131073) == 0
    assert L.dllmc_op_attention_kv4_scratch_bytes(BF16, 1, 1, 1, 4, 3, 128) == 0
    assert L.dllmc_op_attention_weights_scratch_bytes(BF16, F32, 1, 1, 1, 4, 4, 128) == 0
    assert L.dllmc_op_linear_i8_scratch_bytes(0, 1, 1) == 0


STORE = dict(dtype=BF16, x=p(0), M=4, rows=p(1), cache=p(2), cache_rows=9, H=2, d_h=64, stream=None)
LOAD = dict(dtype=BF16, cache=p(2), cache_rows=9, H=2, d_h=64, rows=p(1), M=4, out=p(0), stream=None)
ATTEND = dict(dtype=BF16, q=p(0), B=2, Mq=3, k=p(1), v=p(2), cache_rows=100, row_map=p(3), lens=p(4), n=50, H_q=4, H_kv=2, d_h=128,
              out=p(5), lse=p(6), scratch=p(7), nbytes=1 << 36, stream=None)
WEIGH = dict(dtype=BF16, fmt=BF16, q=p(0), B=2, Mq=3, k=p(1), cache_rows=100, row_map=p(3), lens=p(4), n=50, H_q=4, H_kv=2, d_h=128,
             lse=p(5), acc_in=p(6), acc_out=p(7), scratch=p(8), nbytes=1 << 36, stream=None)
EVICT = dict(acc=p(0), B=2, n=50, lens=p(1), row_map=p(2), cache_rows=100, keep=20, first=4, last=8, kept=p(3), kept_rows=p(4),
             new_lens=p(5), acc_out=p(6), stream=None)
COMPACT = dict(fmt=BF16, rows=p(0), M=5, src_rows=9, dst_rows=7, H=2, d_h=64, k_src=p(1), k_dst=p(2), v_src=p(3), v_dst=p(4),
               stream=None)
QUANT = dict(dtype=BF16, x=p(0), x_rows=9, rows=p(1), M=4, K=100, q=p(2), scale=p(3), stream=None)
LINEAR = dict(dtype=BF16, a=p(0), sa=p(1), M=4, w=p(2), sw=p(3), N=8, K=100, out=p(4), scratch=p(5), nbytes=1 << 36, stream=None)


def near(ptr, by):
    return ctypes.c_void_p(ptr.value + by)


CALLS = {"dllmc_op_kv4_store": STORE, "dllmc_op_kv4_load": LOAD, "dllmc_op_attention_kv4": ATTEND,
         "dllmc_op_attention_weights": WEIGH, "dllmc_op_evict": EVICT, "dllmc_op_compact": COMPACT, "dllmc_op_quant8": QUANT,
         "dllmc_op_linear_i8": LINEAR}

BAD = {
    "dllmc_op_kv4_store": [dict(dtype=2), dict(x=None), dict(cache=None), dict(M=0), dict(M=-1), dict(cache_rows=0), dict(H=0),
                           dict(d_h=48), dict(d_h=0), dict(rows=None, M=10), dict(x=near(p(0), 8)), dict(cache=near(p(2), 4)),
                           dict(rows=near(p(1), 2)), dict(x=near(p(2), 16)), dict(rows=near(p(2), 64))],
    "dllmc_op_kv4_load": [dict(dtype=-1), dict(out=None), dict(cache=None), dict(M=0), dict(cache_rows=1 << 25), dict(H=2000),
                          dict(rows=None, M=10), dict(out=near(p(0), 2)), dict(out=p(2)), dict(rows=p(0))],
    "dllmc_op_attention_kv4": [dict(dtype=3), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(B=0), dict(Mq=0), dict(n=0),
                               dict(H_q=5), dict(H_kv=0), dict(H_q=1), dict(d_h=96), dict(d_h=32), dict(cache_rows=0),
                               dict(row_map=None, cache_rows=99), dict(B=1 << 20, n=1 << 20), dict(Mq=1 << 30),
                               dict(q=near(p(0), 2)), dict(out=near(p(5), 8)), dict(lens=near(p(4), 1)), dict(row_map=near(p(3), 2)),
                               dict(lse=near(p(6), 2)), dict(scratch=near(p(7), 4)), dict(out=p(0)), dict(out=p(1)), dict(out=p(2)),
                               dict(lse=p(0)), dict(lse=p(5)), dict(lse=p(4)), dict(out=p(3))],
    "dllmc_op_attention_weights": [dict(dtype=2), dict(fmt=F32), dict(fmt=3), dict(q=None), dict(k=None), dict(acc_out=None),
                                   dict(B=0), dict(n=-1), dict(H_q=3), dict(d_h=80), dict(row_map=None, cache_rows=99),
                                   dict(acc_out=p(0)), dict(acc_out=p(1)), dict(acc_out=near(p(6), 4)), dict(acc_out=p(5)),
                                   dict(acc_out=near(p(7), 2)), dict(acc_in=near(p(6), 1))],
    "dllmc_op_evict": [dict(acc=None), dict(kept=None), dict(kept_rows=None), dict(new_lens=None), dict(B=0), dict(n=0), dict(keep=0),
                       dict(keep=51), dict(first=-1), dict(last=-1), dict(first=13), dict(last=17), dict(first=21, last=0),
                       dict(row_map=None, cache_rows=99), dict(cache_rows=0), dict(kept=p(0)), dict(acc_out=p(0)),
                       dict(kept_rows=p(3)), dict(new_lens=p(1)), dict(acc=near(p(0), 2)), dict(first=2 ** 31 - 1, last=2 ** 31 - 1)],
    "dllmc_op_compact": [dict(fmt=3), dict(rows=None), dict(k_src=None), dict(k_dst=None), dict(v_src=None), dict(v_dst=None), dict(M=0),
                         dict(M=8), dict(src_rows=0), dict(H=0), dict(d_h=0), dict(fmt=KV4, d_h=40), dict(k_dst=p(1)), dict(v_dst=p(2)),
                         dict(v_dst=p(1)), dict(k_dst=p(0)), dict(k_src=near(p(1), 1)), dict(fmt=KV4, k_src=near(p(1), 8))],
    "dllmc_op_quant8": [dict(dtype=2), dict(x=None), dict(x_rows=0), dict(rows=None, M=10), dict(q=near(p(0), 16 * 100)), dict(q=None), dict(scale=None), dict(M=0), dict(K=0), dict(K=131073),
                        dict(q=near(p(2), 8)), dict(x=near(p(0), 1)), dict(q=p(0)), dict(scale=p(2)), dict(scale=p(0)), dict(q=p(1))],
    "dllmc_op_linear_i8": [dict(dtype=2), dict(a=None), dict(sa=None), dict(w=None), dict(sw=None), dict(out=None), dict(M=0), dict(N=0),
                           dict(K=0), dict(K=131073), dict(a=near(p(0), 8)), dict(w=near(p(2), 4)), dict(out=near(p(4), 1)),
                           dict(out=near(p(4), 8)), dict(out=p(0)), dict(out=p(2)), dict(out=p(1)), dict(out=p(3))],
}


@pytest.mark.parametrize("name,change", [(n, c) for n in CALLS for c in BAD[n]], ids=lambda v: v if isinstance(v, str) else "-".join(v))
def test_refused(name, change):
    args = dict(CALLS[name], **change)
    assert getattr(L, name)(*args.values()) == EINVAL


def test_largest_shapes():
    """A launch has fewer than 2^32 work-items: the next larger batch is refused."""
    for B, ok in ((65535, True), (65536, False)):
        for n in (1, 128, 200):
            rows = (BF16, B, 1, n, 128, 128, 64)
            assert (L.dllmc_plan_attention_kv4(*rows, None, None, None) > 0) == ok
            fits = ok and B * n * 128 <= 1 << 30
            assert (L.dllmc_plan_attention_weights(BF16, KV4, *rows[1:], None, None, None) > 0) == fits
            assert (L.dllmc_op_attention_weights_scratch_bytes(BF16, KV4, *rows[1:]) > 0) == fits
    assert L.dllmc_plan_attention_weights(BF16, KV4, 1, 1, 1 << 24, 64, 64, 64, None, None, None) > 0
    assert L.dllmc_plan_attention_weights(BF16, KV4, 1, 1, 1 << 24, 65, 65, 64, None, None, None) == EINVAL
    r = random.Random(1)
    for _ in range(4000):
        M, N, K = min(1 << 22, int(2 ** r.uniform(0, 22.1))), int(2 ** r.uniform(0, 24)), int(2 ** r.uniform(0, 17))
        (rows, _), _, _ = binding.plan_linear_i8(M, N, K)
        assert -(-M // rows) <= 65535


def test_scratch_too_small():
    for name, size, args in (
            ("dllmc_op_attention_kv4", L.dllmc_op_attention_kv4_scratch_bytes, dict(ATTEND, B=1, Mq=1, n=50000, cache_rows=60000)),
            ("dllmc_op_attention_weights", None, dict(WEIGH, lse=None))):
        need = size(args["dtype"], args["B"], args["Mq"], args["n"], args["H_q"], args["H_kv"], args["d_h"]) if size else \
            L.dllmc_op_attention_weights_scratch_bytes(args["dtype"], args["fmt"], args["B"], args["Mq"], args["n"], args["H_q"],
                                                       args["H_kv"], args["d_h"])
        if need:
            assert getattr(L, name)(*dict(args, nbytes=need - 1).values()) == ENOMEM
            assert getattr(L, name)(*dict(args, scratch=None).values()) == ENOMEM
    need = L.dllmc_op_linear_i8_scratch_bytes(1, 4096, 4096)
    if need:
        args = dict(LINEAR, M=1, N=4096, K=4096)
        assert L.dllmc_op_linear_i8(*dict(args, nbytes=need - 1).values()) == ENOMEM


def test_binding_refuses_what_it_can_see():
    with pytest.raises(binding.DllmcError):
        binding.kv4_bytes(4, 1, 40)
    with pytest.raises(binding.DllmcError):
        binding.i8_row_bytes(0)
