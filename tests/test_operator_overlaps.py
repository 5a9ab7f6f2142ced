"""Outputs of the clipping that overlap are refused before anything else happens.  The handle here is a block of zeros and the
addresses mean nothing, so a call that is not refused ends at the missing device (FFTCONV_HIP_ERROR): for machines without one
only."""
import ctypes

import pytest
import torch

import paper_1412_7580_amd as pkg

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are not refused would be launched")
INVALID_ARG, HIP_ERROR = 1, 4
A, B, N = 1 << 20, 1 << 21, 1 << 22       # addresses of two tensors of 64 floats and of the norm


def clip(grads, out, norm):
    lib = pkg.load_library()
    handle = ctypes.create_string_buffer(1 << 16)
    n = len(grads)
    pointers = [(ctypes.c_void_p * n)(*p) for p in (grads, out)]
    return lib.fftconv_grad_clip(ctypes.addressof(handle), n, pointers[0], (ctypes.c_long * n)(*[64] * n), (ctypes.c_int * n)(*[0] * n), pointers[1],
                                 1.0, norm, None, 0)


@pytest.mark.parametrize("norm", [A, A + 4, A + 252, B, B + 100, A - 2])
def test_a_norm_inside_a_tensor(norm):
    assert clip([A], [A], norm if norm < B else A) == INVALID_ARG
    assert clip([A, B], [A, B], norm) == INVALID_ARG
    assert clip([A], [B], norm) == INVALID_ARG                # an input, or an output


@pytest.mark.parametrize("norm", [N, A - 4, A + 256, B + 256])
def test_a_norm_beside_the_tensors(norm):
    assert clip([A, B], [A, B], norm) == HIP_ERROR
    assert clip([A], [B], norm) == HIP_ERROR
    assert clip([], [], norm) == HIP_ERROR


def test_tensors_that_overlap():
    assert clip([A, A], [A, A], N) == INVALID_ARG
    assert clip([A, B], [B, A], N) == INVALID_ARG             # each the other's output
    assert clip([A, A], [B, B + 255], N) == INVALID_ARG
    assert clip([A, A], [B, B + 256], N) == HIP_ERROR         # read twice, written apart
    assert clip([A], [A + 4], N) == INVALID_ARG
