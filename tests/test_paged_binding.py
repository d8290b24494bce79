"""LtriPaged's host logic, with a torch and a library of the test's own in place of a GPU's."""
import contextlib
import sys
import types

import pytest

from paper_2412_04757_b200 import binding


class Tensor:
    def __init__(self, shape, dtype, strides=None, ptr=4096):
        self.shape, self.dtype, self.device, self._ptr = tuple(shape), dtype, types.SimpleNamespace(type="cuda", index=0), ptr
        dense, n = [], 1
        for x in reversed(shape):
            dense.insert(0, n)
            n *= x
        self._stride = tuple(strides or dense)
        self._dense = tuple(dense)

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        return self._stride if i is None else self._stride[i]

    def is_contiguous(self):
        return all(a == b or n == 1 for a, b, n in zip(self._stride, self._dense, self.shape))

    def data_ptr(self):
        return self._ptr


class Torch(types.SimpleNamespace):
    """What LtriPaged uses of torch; `events` tells under which stream things happened."""

    def __init__(self):
        super().__init__(bfloat16="bf16", float16="fp16", float8_e4m3fn="e4m3", float32="f32", int32="i32", uint8="u8", Size=tuple)
        self.events, self.current = [], 11
        self._C = types.SimpleNamespace(_cuda_getCurrentRawStream=lambda index: self.current)
        self.cuda = types.SimpleNamespace(device=lambda d: contextlib.nullcontext(), stream=self.on)

    @contextlib.contextmanager
    def on(self, stream):
        before = self.current
        self.current = before if stream is None else stream.cuda_stream
        yield
        self.current = before

    def empty(self, n, dtype, device):
        self.events.append(("empty", self.current))
        return Tensor([n], dtype, ptr=1 << 20)


@pytest.fixture
def fake(monkeypatch):
    torch = Torch()

    def create(params, stream, out):
        torch.events.append(("create", stream))
        torch.params = params._obj
        return binding.LTRI_OK

    real = binding.load()
    lib = types.SimpleNamespace(ltri_paged_workspace_bytes=real.ltri_paged_workspace_bytes, ltri_paged_create=create,
                                ltri_paged_destroy=lambda h: 0)
    monkeypatch.setitem(sys.modules, "torch", torch)
    monkeypatch.setattr(binding, "load", lambda: lib)
    return torch


@pytest.mark.parametrize("stream", [None, 22])
def test_the_workspace_is_allocated_on_the_stream_that_zeroes_it(fake, stream):
    k, v = Tensor([2, 5, 1, 16, 64], "bf16"), Tensor([2, 5, 1, 16, 64], "bf16", ptr=1 << 16)
    binding.LtriPaged(k, v, 2, stream=None if stream is None else types.SimpleNamespace(cuda_stream=stream))
    assert fake.events == [("empty", stream or 11), ("create", stream or 11)] and fake.current == 11


def test_strides_of_axes_of_one_entry_do_not_matter(fake):
    shape = [1, 5, 1, 16, 64]
    k, v = Tensor(shape, "bf16", [1, 1024, 3, 64, 1]), Tensor(shape, "bf16", [5120, 1024, 1024, 64, 1], ptr=1 << 16)
    binding.LtriPaged(k, v, 2)
    assert fake.events[-1][0] == "create" and fake.params.page_stride == 1024
    for strides in ([5120, 2048, 1024, 64, 1], [5120, 1024, 1024, 128, 1]):
        with pytest.raises(ValueError):
            binding.LtriPaged(k, Tensor(shape, "bf16", strides, ptr=1 << 16), 2)
