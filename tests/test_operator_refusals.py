"""Refusals of the embedding, the linear cross entropy and the gradient norm that need no device: size functions,
null handles, and the Python binding's own checks (no library call is made for an argument it refuses)."""
import pytest
import torch

import paper_1412_7580_amd as pkg

MOST = 1 << 30


class NoCalls:
    def __getattr__(self, name):
        raise AssertionError(f"{name} was called")


@pytest.fixture()
def hd():
    pkg.load_library()
    h = pkg.Handle.__new__(pkg.Handle)
    h._lib, h._h, h.device, h._stream = NoCalls(), None, 0, 0
    return h


def test_a_null_handle_is_an_invalid_argument():
    lib = pkg.load_library()
    assert lib.fftconv_embedding_fprop(None, 0, None, None, 64, None, 1, 1, 1, 0, 1.0) == 1
    assert lib.fftconv_embedding_accgrad(None, 0, None, None, 64, None, 1, 1, 1, 0, 1.0, 0, None, 0) == 1
    assert lib.fftconv_xent_fprop(None, 0, None, None, None, 64, None, None, 1, 1, 1, 0, None, 0) == 1
    assert lib.fftconv_xent_backward(None, 0, None, None, None, 64, None, None, None, None, 1, 1, 1, 0, 1.0, 0, 0, None, 0) == 1
    assert lib.fftconv_grad_norm(None, 0, None, None, None, None, None, 0) == 1
    assert lib.fftconv_grad_clip(None, 0, None, None, None, None, 1.0, None, None, 0) == 1


@pytest.mark.parametrize("dtype,N,D,V,T", [(3, 4, 4, 4, 0), (-1, 4, 4, 4, 0), (0, -1, 4, 4, 0), (0, 4, 0, 4, 0), (0, 4, 4, 0, 0),
                                           (0, 4, 4, 4, -1), (0, 5, 4, 4, 2), (0, MOST + 1, 4, 4, 0), (0, 4, MOST + 1, 4, 0),
                                           (0, 4, 4, MOST + 1, 0), (0, 0, 4, 4, 0)])
def test_no_workspace_for_sizes_that_are_refused(dtype, N, D, V, T):
    lib = pkg.load_library()
    assert lib.fftconv_embedding_workspace_bytes(dtype, N, D, V, T) == 0
    if T == 0:
        assert lib.fftconv_xent_workspace_bytes(pkg.FPROP, dtype, N, D, V) == 0
        assert lib.fftconv_xent_workspace_bytes(pkg.BPROP, dtype, N, D, V) == 0


def test_workspaces_hold_what_the_calls_keep():
    """Lower bounds: two lists of keys and positions; the packed rows, and in fp32 the terms of both
    operands, two for the scores and three more for the gradients."""
    lib = pkg.load_library()
    assert lib.fftconv_embedding_workspace_bytes(1, 1000, 64, 5000, 0) >= 1000 * 16
    assert lib.fftconv_xent_workspace_bytes(pkg.FPROP, 1, 1000, 64, 5000) >= 1000 * 64 * 2
    assert lib.fftconv_xent_workspace_bytes(pkg.FPROP, 0, 1000, 64, 5000) >= (1000 + 5000) * 64 * 4
    assert lib.fftconv_xent_workspace_bytes(pkg.BPROP, 0, 1000, 64, 5000) >= (1000 + 5000) * 64 * 10 + 1000 * 64 * 4
    assert lib.fftconv_xent_workspace_bytes(pkg.ACCGRAD, 0, 1000, 64, 5000) == 0
    # without the scores: a piece of them stays far below all of them
    assert lib.fftconv_xent_workspace_bytes(pkg.BPROP, 1, 16384, 64, 1 << 20) < 16384 * 2 * (1 << 20) // 8


def test_tensors_that_are_not_on_the_device_are_refused(hd):
    x, w, t = torch.zeros(4, 8), torch.zeros(5, 8), torch.zeros(4, dtype=torch.long)
    for call in (lambda: hd.embedding_fprop(w, t), lambda: hd.embedding_accgrad(x, t, 5), lambda: hd.xent_fprop(x, w, t),
                 lambda: hd.xent_backward(x, w, t, torch.zeros(4)), lambda: hd.grad_norm([x]), lambda: hd.grad_clip([x], 1.0)):
        with pytest.raises(pkg.FFTConvError, match="device memory"):
            call()


class Fake(torch.Tensor):
    """A CPU tensor that says it lies on a device of this number."""
    at = 0
    is_cuda = True

    def get_device(self):
        return self.at


def fake(*shape, dtype=torch.float32, at=0):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(Fake)
    t.at = at
    return t


def test_another_device_is_refused(hd):
    with pytest.raises(pkg.FFTConvError, match="device 1, the handle on 0"):
        hd.embedding_fprop(fake(4, 8, at=1), fake(3, dtype=torch.int64))
    with pytest.raises(pkg.FFTConvError, match="device 1, the handle on 0"):
        hd.grad_norm([fake(4), fake(4, at=1)])


def test_strided_tensors_are_refused(hd):
    t = fake(3, dtype=torch.int64)
    with pytest.raises(pkg.FFTConvError, match="contiguous"):
        hd.embedding_fprop(fake(8, 4).t(), t)
    with pytest.raises(pkg.FFTConvError, match="contiguous"):
        hd.xent_fprop(fake(3, 8), fake(5, 16)[:, ::2], t)
    with pytest.raises(pkg.FFTConvError, match="contiguous"):
        hd.grad_clip([fake(8)[::2]], 1.0)


def test_types_and_shapes_that_disagree_are_refused(hd):
    x, w, t = fake(4, 8), fake(5, 8), fake(4, dtype=torch.int64)
    E = pkg.FFTConvError
    with pytest.raises(E, match="float32, bfloat16 or float16"):
        hd.embedding_fprop(fake(5, 8, dtype=torch.float64), t)
    with pytest.raises(E, match="int32 or int64"):
        hd.embedding_fprop(w, fake(4, dtype=torch.int16))
    with pytest.raises(E, match="V, D"):
        hd.embedding_fprop(fake(5), t)
    with pytest.raises(E, match="sample dimension"):
        hd.embedding_fprop(w, t, planes=True)
    with pytest.raises(E, match="y must be"):
        hd.embedding_fprop(w, t, y=fake(4, 7))
    with pytest.raises(E, match="disagree"):
        hd.embedding_accgrad(fake(5, 8), t, 5)
    with pytest.raises(E, match="existing gtable"):
        hd.embedding_accgrad(x, t, 5, accumulate=True)
    with pytest.raises(E, match="gtable must be"):
        hd.embedding_accgrad(x, t, 5, gtable=fake(6, 8))
    with pytest.raises(E, match="x's type"):
        hd.xent_fprop(x, fake(5, 8, dtype=torch.bfloat16), t)
    with pytest.raises(E, match="disagree"):
        hd.xent_fprop(x, fake(5, 9), t)
    with pytest.raises(E, match="disagree"):
        hd.xent_fprop(fake(2, 8, 3), w, fake(2, 4, dtype=torch.int64), planes=True)
    with pytest.raises(E, match="loss must be"):
        hd.xent_fprop(x, w, t, loss=fake(4, dtype=torch.float16))
    with pytest.raises(E, match="lse must be"):
        hd.xent_backward(x, w, t, fake(5))
    with pytest.raises(E, match="gloss must be"):
        hd.xent_backward(x, w, t, fake(4), gloss=fake(5))
    with pytest.raises(E, match="existing gw"):
        hd.xent_backward(x, w, t, fake(4), accumulate=True)
    with pytest.raises(E, match="gw must be"):
        hd.xent_backward(x, w, t, fake(4), gw=fake(5, 8, dtype=torch.bfloat16))
    with pytest.raises(E, match="out must be"):
        hd.grad_clip([x], 1.0, out=[fake(4, 9)])
    with pytest.raises(E, match="disagree"):
        hd.grad_clip([x], 1.0, out=[])
    with pytest.raises(E, match="norm must be"):
        hd.grad_norm([x], norm=fake(1))
