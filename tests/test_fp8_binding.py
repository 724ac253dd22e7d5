"""The Python side of the block-scaled calls, against stand-ins for the library and the devices (no GPU needed)."""
import contextlib
import types

import pytest
import torch

from paper_2510_26771_b200 import binding


class Weights:
    """A matrix on the second of two devices."""
    shape, dtype, device, is_cuda = torch.Size((64, 256)), torch.bfloat16, torch.device("cuda:1"), True

    def dim(self):
        return 2

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096


def test_weights_are_quantized_on_their_own_device(monkeypatch):
    current, launches, outputs = [0], [], []

    @contextlib.contextmanager
    def device(d):
        before, current[0] = current[0], torch.device(d).index
        yield
        current[0] = before

    def empty(shape, dtype, device):
        outputs.append((tuple(shape), dtype, device))
        return Weights()

    def launch(*args):
        launches.append((current[0], args[-1].value))
        return 0

    monkeypatch.setattr(binding.torch.cuda, "device", device)
    monkeypatch.setattr(binding.torch.cuda, "current_stream", lambda *a: types.SimpleNamespace(cuda_stream=(7, 8)[current[0]]))
    monkeypatch.setattr(binding.torch, "empty", empty)
    monkeypatch.setattr(binding, "lib", lambda: types.SimpleNamespace(stamp_fp8_quantize_weights=launch))
    binding.stamp_fp8_quantize_weights(Weights())
    assert launches == [(1, 8)] and current == [0]
    assert [o[2] for o in outputs] == [Weights.device] * 2 and [o[0] for o in outputs] == [(64, 256), (1, 2)]


def test_weights_off_the_devices_are_refused():
    with pytest.raises(ValueError):
        binding.stamp_fp8_quantize_weights(torch.zeros(64, 256))
    with pytest.raises(ValueError):
        binding.stamp_fp8_quantize_weights(torch.zeros(256))


@pytest.mark.parametrize("shape", [(16, 1 << 32), (1 << 32, 16), (1 << 31, 2, 16)])
def test_sizes_past_32_bits_are_refused(monkeypatch, shape):
    class Large(Weights):
        def dim(self):
            return len(self.shape)
    Large.shape = torch.Size(shape)
    monkeypatch.setattr(binding, "lib", lambda: pytest.fail("the library was called"))
    monkeypatch.setattr(binding.torch, "empty", lambda *a, **k: pytest.fail("outputs were allocated"))
    with pytest.raises(ValueError):
        binding.stamp_fp8_quantize_weights(Large())
