"""op_attention refuses tensors that are smaller than the sizes it passes on: the library would read past their ends; and host memory.
No GPU needed."""
import pytest
import torch

from paper_2506_06295_amd import binding


def call(q=(1, 3, 256), k=(1, 7, 128), v=(1, 7, 128), heads=(4, 2, 64), dtype="f32", cast=torch.float32):
    return binding.op_attention(dtype, torch.zeros(q, dtype=cast), torch.zeros(k), torch.zeros(v), *heads)


@pytest.mark.parametrize("change", [dict(heads=(4, 2, 128)), dict(heads=(4608, 2, 64)), dict(q=(1, 3, 192)), dict(k=(1, 8, 128)), dict(k=(2, 7, 128)),
                                    dict(v=(1, 6, 128)), dict(v=(1, 7, 64)), dict(k=(7, 128), v=(7, 128)), dict(cast=torch.bfloat16),
                                    dict(dtype="bf16")])
def test_refused(change, monkeypatch):
    monkeypatch.setattr(binding, "lib", lambda: pytest.fail("the library was called"))
    with pytest.raises(binding.DllmcError, match="elements"):
        call(**change)


def test_not_contiguous(monkeypatch):
    monkeypatch.setattr(binding, "lib", lambda: pytest.fail("the library was called"))
    q, kv = torch.zeros(1, 256, 3).transpose(1, 2), torch.zeros(1, 7, 128)
    with pytest.raises(binding.DllmcError):
        binding.op_attention("f32", q, kv, kv, 4, 2, 64)


def test_what_fits_in_host_memory(monkeypatch):
    monkeypatch.setattr(binding, "lib", lambda: pytest.fail("the library was called"))
    with pytest.raises(binding.DllmcError, match="on the device"):
        call()
