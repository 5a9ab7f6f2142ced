"""Sizes beyond what the C entry points take as int are refused by the binding, before anything is allocated or called: ctypes
would take 2^32 + 5 classes for 5."""
import pytest
import torch

import paper_1412_7580_amd as pkg

BIG = (1 << 32) + 5


class NoCalls:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


class Fake(torch.Tensor):
    """A tensor without memory that says it lies on the handle's device."""
    is_cuda = True

    def get_device(self):
        return 0

    def data_ptr(self):
        return 4096


def fake(*shape, dtype=torch.float32):
    return torch.empty(*shape, dtype=dtype, device="meta").as_subclass(Fake)


@pytest.fixture()
def hd():
    pkg.load_library()
    h = pkg.Handle.__new__(pkg.Handle)
    h._lib, h._h, h.device, h._stream = NoCalls(), None, 0, 0
    h._device_stream = lambda: None
    return h


@pytest.mark.parametrize("size", [BIG, 1 << 31, (1 << 30) + 1])
def test_sizes_that_the_library_does_not_take(hd, size):
    t, one = fake(3, dtype=torch.int64), fake(1, dtype=torch.int64)
    for call in (lambda: hd.embedding_fprop(fake(size, 1), t), lambda: hd.embedding_fprop(fake(1, size), t),
                 lambda: hd.embedding_fprop(fake(5, 1), fake(size, dtype=torch.int64)),
                 lambda: hd.embedding_fprop(fake(5, 1), fake(0, size, dtype=torch.int64), planes=True),
                 lambda: hd.embedding_accgrad(fake(3, 1), t, size), lambda: hd.embedding_accgrad(fake(1, size), one, 5),
                 lambda: hd.xent_fprop(fake(3, 2), fake(size, 2), t), lambda: hd.xent_fprop(fake(1, size), fake(2, size), one),
                 lambda: hd.xent_backward(fake(3, 2), fake(size, 2), t, fake(3))):
        with pytest.raises(pkg.FFTConvError, match="2\\^30"):
            call()
    # and their workspaces are of no bytes, as the library's own size functions say
    assert hd.embedding_workspace_bytes(torch.float32, 3, 1, size) == 0 and hd.embedding_workspace_bytes(torch.float32, 3, size, 5) == 0
    assert hd.xent_workspace_bytes(pkg.FPROP, torch.float32, 3, size, 5) == 0 and hd.xent_workspace_bytes(pkg.BPROP, torch.float32, 3, 2, size) == 0


def test_a_negative_number_of_classes(hd):
    with pytest.raises(pkg.FFTConvError, match="2\\^30"):
        hd.embedding_accgrad(fake(3, 1), fake(3, dtype=torch.int64), -5)
