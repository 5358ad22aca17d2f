"""What op_attend hands to the library, without a GPU: tensors are stand-ins, the library takes notes."""
import struct

import pytest
import torch

from paper_2502_01277_amd import binding


class Tensor:
    """Looks like a device tensor (or like one on the host) at a made-up address."""

    def __init__(self, shape, dtype, at, device=True, dense=True):
        self.shape, self.dtype, self.at, self.is_cuda, self.dense, self.device = torch.Size(shape), dtype, at, device, dense, "cuda"

    def stride(self):
        s, n = [], 1
        for x in reversed(self.shape):
            s.insert(0, n)
            n *= x
        return tuple(s)

    def data_ptr(self):
        return self.at

    def is_contiguous(self):
        return self.dense

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()


class Library:
    def __init__(self, need):
        self.need, self.calls = need, []

    def octo_op_attend_workspace_bytes(self, op):
        return self.need

    def octo_op_attend(self, op, stream, kid):
        self.calls.append(struct.unpack_from("PN", op, len(op) - 16))
        return binding.OK


@pytest.fixture
def call(monkeypatch):
    bf16 = torch.bfloat16
    q, out = Tensor((4, 2, 64), bf16, 4096), Tensor((4, 2, 64), bf16, 8192)
    held = (Tensor((9000, 1, 64), bf16, 1 << 20), Tensor((9000, 1, 64), bf16, 1 << 24))
    dev = [Tensor((2,), torch.int32, 64), Tensor((1,), torch.int64, 128), Tensor((1,), torch.int32, 192)]
    monkeypatch.setattr(binding, "_stream_ptr", lambda stream: 0)

    def run(workspace, need=4096):
        library = Library(need)
        monkeypatch.setattr(binding, "lib", lambda: library)
        binding.op_attend(q, held, out, *dev, workspace=workspace)
        return library.calls
    return run


@pytest.mark.parametrize("need", [0, 4096])
@pytest.mark.parametrize("workspace", [Tensor((8192,), torch.uint8, 256, device=False), Tensor((8192,), torch.uint8, 256, dense=False), Tensor((8192,), torch.float32, 256),
                                       Tensor((8192,), torch.int8, 256)], ids=["host", "strided", "fp32", "int8"])
def test_a_workspace_is_dense_bytes_on_the_device(call, workspace, need):
    with pytest.raises(binding.OctoError):
        call(workspace, need)


def test_a_workspace_goes_to_the_library_with_its_size(call):
    assert call(Tensor((8192,), torch.uint8, 256)) == [(256, 8192)]
    assert call(Tensor((64,), torch.uint8, 256)) == [(256, 64)]             # the library refuses one that is too small
    assert call(None, 0) == [(0, 0)]
