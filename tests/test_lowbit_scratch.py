"""Scratch of the operators in fewer bits: too small, missing, or over an operand or a result.  No GPU needed, nothing is launched."""
import ctypes
import os

import pytest

from paper_2506_06295_amd import binding
from tests.test_lowbit_host import ATTEND, BF16, EINVAL, ENOMEM, F32, KV4, LINEAR, WEIGH, near

if not os.path.exists(binding.LIB_PATH):
    pytest.skip("libdllmc.so not built in this tree", allow_module_level=True)

L = binding.lib()


def attention(**change):
    c = dict(ATTEND, B=1, Mq=1, n=5000, cache_rows=6000, **change)
    return "dllmc_op_attention_kv4", c, L.dllmc_op_attention_kv4_scratch_bytes(c["dtype"], 1, 1, 5000, c["H_q"], c["H_kv"], c["d_h"])


def weights(**change):
    c = dict(WEIGH, B=1, n=2000, cache_rows=6000, **change)
    return "dllmc_op_attention_weights", c, L.dllmc_op_attention_weights_scratch_bytes(c["dtype"], c["fmt"], 1, c["Mq"], c["n"], c["H_q"],
                                                                                     c["H_kv"], c["d_h"])


def linear(**change):
    c = dict(LINEAR, M=3, N=3, K=5632, **change)
    assert binding.plan_linear_i8(3, 3, 5632)[1] > 1   # slices, which are added from scratch
    return "dllmc_op_linear_i8", c, L.dllmc_op_linear_i8_scratch_bytes(3, 3, 5632)


CALLS = {"attention": attention(), "attention f32": attention(dtype=F32), "weights": weights(), "weights kv4": weights(fmt=KV4),
         "weights, few keys": ("dllmc_op_attention_weights", dict(WEIGH), L.dllmc_op_attention_weights_scratch_bytes(
             BF16, BF16, *(WEIGH[k] for k in ("B", "Mq", "n", "H_q", "H_kv", "d_h")))),
         "linear": linear()}
OVER = {"dllmc_op_attention_kv4": ("q", "k", "v", "row_map", "lens", "out", "lse"),
        "dllmc_op_attention_weights": ("q", "k", "row_map", "lens", "lse", "acc_in", "acc_out"),
        "dllmc_op_linear_i8": ("a", "sa", "w", "sw", "out")}


@pytest.mark.parametrize("which", CALLS)
def test_too_small_or_missing(which):
    name, args, need = CALLS[which]
    assert need > 0
    assert getattr(L, name)(*dict(args, nbytes=need - 1).values()) == ENOMEM
    assert getattr(L, name)(*dict(args, scratch=None).values()) == ENOMEM


@pytest.mark.parametrize("which,operand", [(w, o) for w in CALLS for o in OVER[CALLS[w][0]]])
def test_over_an_operand_or_result(which, operand):
    name, args, need = CALLS[which]
    at = args[operand]
    for by in (0, 16 - need):   # the operand's first byte under scratch's first one, under its last ones
        by = -(-by // 16) * 16
        assert getattr(L, name)(*dict(args, scratch=near(at, by)).values()) == EINVAL, by


@pytest.mark.parametrize("which", CALLS)
def test_in_place_weights_over_scratch(which):
    name, args, _ = CALLS[which]
    if "acc_in" in args:
        args = dict(args, acc_in=args["acc_out"])
        assert getattr(L, name)(*dict(args, scratch=near(args["acc_out"], 16)).values()) == EINVAL
