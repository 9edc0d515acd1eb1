"""Sizes beyond 32 bits are refused by the binding, not cut to the 32 bits that the C calls take.  No GPU needed."""
import os

import pytest
import torch

from paper_2506_06295_amd import binding

if not os.path.exists(binding.LIB_PATH):
    pytest.skip("libdllmc.so not built in this tree", allow_module_level=True)


@pytest.mark.parametrize("args", [((1 << 32) + 8, 1, 32), (8, (1 << 32) + 1, 32), (8, 1, (1 << 32) + 32), (-(1 << 32) + 8, 1, 32)])
def test_cache_sizes(args):
    with pytest.raises(binding.DllmcError):
        binding.kv4_bytes(*args)


@pytest.mark.parametrize("K", [(1 << 32) + 128, -(1 << 32) + 128])
def test_row_lengths(K):
    with pytest.raises(binding.DllmcError):
        binding.i8_row_bytes(K)


@pytest.mark.parametrize("change", [dict(keep=(1 << 32) + 3), dict(keep=0), dict(keep=-1), dict(keep=6), dict(keep=1 << 40), dict(first=1 << 32),
                                    dict(last=1 << 32), dict(first=-1), dict(first=2, last=2), dict(cache_rows=(1 << 32) + 100),
                                    dict(cache_rows=0)])
def test_evict_budgets(change, monkeypatch):
    """Refused before anything of the size that was asked for is allocated, and before the library is called."""
    monkeypatch.setattr(binding, "_device", lambda name, t: -1)   # (as if host memory were the current device)
    monkeypatch.setattr(binding, "lib", lambda: pytest.fail("the library was called"))
    with pytest.raises(binding.DllmcError):
        binding.op_evict(torch.zeros(1, 5), **dict(dict(keep=3, cache_rows=100, first=0, last=0), **change))


@pytest.mark.parametrize("n", [(1 << 32) + 50, 0, -5, -(1 << 32) + 50])
def test_positions(n, monkeypatch):
    monkeypatch.setattr(binding, "_device", lambda name, t: -1)
    monkeypatch.setattr(binding, "lib", lambda: pytest.fail("the library was called"))
    q, cache = torch.zeros(1, 1, 64), torch.zeros(100 * 34, dtype=torch.uint8)
    with pytest.raises(binding.DllmcError):
        binding.op_attention_kv4("f32", q, cache, cache, 100, n, 1, 1, 64)
    with pytest.raises(binding.DllmcError):
        binding.op_attention_weights("f32", "f32", q, torch.zeros(100, 64), 100, n, 1, 1, 64)
