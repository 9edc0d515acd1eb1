"""Sizes at the ends of what the norm in few bits, the 4-bit maps and the log probabilities take, scratch over operands, and numbers that do not fit
the calls' 32 bits.  No GPU needed, nothing is launched."""
import os
import random

import pytest
import torch

from paper_2506_06295_amd import binding
from tests.test_lowbit_host import near
from tests.test_stream_host import BF16, EINVAL, ENOMEM, F32, LINEAR, LOGPROBS

if not os.path.exists(binding.LIB_PATH):
    pytest.skip("libdllmc.so not built in this tree", allow_module_level=True)

L = binding.lib()


def test_launches_fit():
    """Tiles in a grid's second dimension, and work-items of a launch, of every product that is taken."""
    r = random.Random(1)
    shapes = [(1 << 22, 1 << 13, 64), (1 << 11, 1 << 24, 64), (1, 1 << 24, 131072), (1 << 22, 1, 131072), (1 << 22, 1, 1), (16, 1 << 24, 1)]
    shapes += [(min(1 << 22, int(2 ** r.uniform(0, 22.1))), int(2 ** r.uniform(0, 24)), int(2 ** r.uniform(0, 17))) for _ in range(4000)]
    for M, N, K in shapes:
        if M * N > 1 << 35:
            with pytest.raises(binding.DllmcError):
                binding.plan_linear_mx4(M, N, K)
            continue
        (bm, bn), slices, whole = binding.plan_linear_mx4(M, N, K)
        tiles = -(-M // bm) * -(-N // bn) * slices
        assert -(-M // bm) <= 65535 and tiles * (256 if whole else 512) < 1 << 32, (M, N, K)
        assert L.dllmc_op_linear_mx4_scratch_bytes(M, N, K) == (slices * M * N * 4 if slices > 1 else 0)


def test_logits_scratch():
    """A sum of 12 bytes and top_k keys of 8 for every slice of a row, where there are several."""
    assert L.dllmc_op_logprobs_scratch_bytes(BF16, 4096, 152064, 64) == 0
    assert L.dllmc_op_logprobs_scratch_bytes(F32, 1, 1000, 64) == 0
    one = L.dllmc_op_logprobs_scratch_bytes(F32, 1, 126464, 20)
    assert one > 0 and one == L.dllmc_op_logprobs_scratch_bytes(BF16, 1, 126464, 20)
    for M, V in ((1, 1 << 24), (1000, 1 << 24), (1 << 16, 1 << 24), (1 << 22, 1 << 18), ((1 << 23) - 1, 1 << 17)):
        for k in (0, 64):
            need = L.dllmc_op_logprobs_scratch_bytes(F32, M, V, k)
            slices = need // (M * (12 + 8 * k))   # (rounded up to 16 bytes in between)
            assert slices <= 64 and M * max(1, slices) < 1 << 24, (M, V)


def linear(**change):
    need = L.dllmc_op_linear_mx4_scratch_bytes(1, 1, 16561)
    assert need > 0
    return "dllmc_op_linear_mx4", dict(LINEAR, M=1, N=1, K=16561, **change), need


def logprobs(**change):
    return "dllmc_op_logprobs", dict(LOGPROBS, M=2, vocab=100000, ld=100000, **change), L.dllmc_op_logprobs_scratch_bytes(BF16, 2, 100000, 3)


CALLS = {"linear": linear(), "logprobs": logprobs()}
OVER = {"linear": ("a", "w", "out"), "logprobs": ("logits", "tokens", "logp", "entropy", "ids", "top")}


@pytest.mark.parametrize("which", CALLS)
def test_scratch_too_small_or_missing(which):
    name, args, need = CALLS[which]
    assert need > 0
    assert getattr(L, name)(*dict(args, nbytes=need - 1).values()) == ENOMEM
    assert getattr(L, name)(*dict(args, scratch=None).values()) == ENOMEM


@pytest.mark.parametrize("which,operand", [(w, o) for w in CALLS for o in OVER[w]])
def test_scratch_over_an_operand_or_result(which, operand):
    name, args, need = CALLS[which]
    for by in (0, -(-(16 - need) // 16) * 16):   # the operand's first byte under scratch's first one, under its last ones
        assert getattr(L, name)(*dict(args, scratch=near(args[operand], by)).values()) == EINVAL, by


def test_numbers_past_32_bits():
    for bad in ((1 << 32, 32), (32, 1 << 32), ((1 << 32) + 5, 32), (5, (1 << 32) + 32)):
        with pytest.raises(binding.DllmcError):
            binding.mx4_bytes(*bad)
    for bad in ((1 << 32, 8, 8), (8, (1 << 32) + 8, 8), (8, 8, 1 << 33)):
        with pytest.raises(binding.DllmcError):   # (ctypes takes 32 bits of a number)
            binding.plan_linear_mx4(*bad)
    meta = torch.empty(1 << 10, device="meta")
    with pytest.raises(binding.DllmcError):
        binding.op_linear_mx4("f32", meta, 1 << 40, meta, 4, 32)
