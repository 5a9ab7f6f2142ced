"""Sizes whose grids one launch does not take are refused before anything else happens: a launch has fewer than 2^32 threads.
The handle here is a block of zeros and the tensors' addresses mean nothing, so a call that is not refused ends at the missing
device (FFTCONV_HIP_ERROR): for machines without one only."""
import ctypes

import pytest
import torch

import paper_1412_7580_amd as pkg

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are not refused would be launched")
UNSUPPORTED, HIP_ERROR = 2, 4
F32, BF16 = 0, 1
M24, M28, M30 = 1 << 24, 1 << 28, 1 << 30


@pytest.fixture()
def call():
    lib = pkg.load_library()
    handle, tensor = ctypes.create_string_buffer(1 << 16), ctypes.create_string_buffer(1 << 12)
    h, t = ctypes.addressof(handle), (ctypes.addressof(tensor) + 15) & ~15

    def run(name, dtype, N, D, V, T):
        if name == "fprop":
            return lib.fftconv_embedding_fprop(h, dtype, t, t, 64, t, N, D, V, T, 1.0)
        if name == "accgrad":
            return lib.fftconv_embedding_accgrad(h, dtype, t, t, 64, t, N, D, V, T, 1.0, 0, t, 1 << 62)
        if name == "xent_fprop":
            return lib.fftconv_xent_fprop(h, dtype, t, t, t, 64, t, t, N, D, V, T, t, 1 << 62)
        return lib.fftconv_xent_backward(h, dtype, t, t, t, 64, t, None, t, t, N, D, V, T, 1.0, 0, 0, t, 1 << 62)

    yield run
    del handle, tensor


# the first size of a kind that is refused, and the last that is not
@pytest.mark.parametrize("name,dtype,D,V,T,refused,taken", [
    ("fprop", BF16, 8, 4, 1, M24, M24 - 1),                     # a tile of planes for each sample, 256 threads
    ("fprop", BF16, 65, 4, 1, M24 // 2, M24 // 2 - 1),          # two
    ("fprop", BF16, 8, 4, 65, 65 * (M24 // 2), 65 * (M24 // 2 - 1)),
    ("fprop", F32, 8192, 4, 0, M24, M24 - 1),                   # a block a row
    ("accgrad", BF16, 8, 4, 1, M24, M24 - 1),
    ("accgrad", F32, 64, 4, 0, M30, M30 - 64),                  # a block for each 64 of the sorted rows joins them
    ("xent_fprop", BF16, 8, 2, 0, M28, M28 - 256),              # 1024 threads for each 64 rows
    ("xent_fprop", BF16, 4096, 2, 16, M24, M24 - 256),          # a tile for each 64 rows and 64 features
    ("xent_backward", BF16, 8, 2, 1, M24, M24 - 1),
])
def test_grids_of_too_many_threads(call, name, dtype, D, V, T, refused, taken):
    assert call(name, dtype, refused, D, V, T) == UNSUPPORTED
    assert call(name, dtype, taken, D, V, T) == HIP_ERROR


def test_tables_whose_clearing_takes_too_many_threads(call):
    """64 KB a block of 1024 threads, in one launch where few tokens are sorted."""
    assert call("accgrad", BF16, 4, 1 << 9, 1 << 29, 0) == UNSUPPORTED
    assert call("accgrad", BF16, 4, 1 << 8, 1 << 28, 0) == HIP_ERROR


@pytest.mark.parametrize("name", ["fprop", "accgrad", "xent_fprop", "xent_backward"])
@pytest.mark.parametrize("N,D,V,T", [(1, 1, 1, 0), (1, 1, 1, 1), (65536, 1024, 65536, 0), (65536, 512, 65536, 4), (1 << 20, 64, 1 << 21, 0), (5000, 4096, 1 << 20, 0)])
def test_ordinary_sizes_are_not_refused(call, name, N, D, V, T):
    assert call(name, F32, N, D, V, T) == HIP_ERROR


def test_no_workspace_for_grids_that_are_refused():
    lib = pkg.load_library()
    assert lib.fftconv_embedding_workspace_bytes(BF16, M24, 8, 4, 1) == 0 and lib.fftconv_embedding_workspace_bytes(BF16, M24 - 1, 8, 4, 1) > 0
    assert lib.fftconv_xent_workspace_bytes(pkg.FPROP, BF16, M28, 8, 2) == 0 and lib.fftconv_xent_workspace_bytes(pkg.FPROP, BF16, M28 - 256, 8, 2) > 0
