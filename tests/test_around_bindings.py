"""The binding's checks of the calls around the layer, without a GPU: tensors
that stand for device memory, whose addresses are never followed, show what a
call would have been given."""
import pytest
import torch

import paper_2511_21431_amd as mf

bf, u8 = torch.bfloat16, torch.uint8


class Device:
    """A contiguous device tensor, as far as the binding looks."""
    is_cuda, device = True, "cpu"

    def __init__(self, *shape, dtype=u8):
        self.shape, self.dtype = torch.Size(shape), dtype

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 4096

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()


def weights(E, N, K):
    return (Device(E, mf.memfine_mxw_code_bytes(N, K)), Device(E, mf.memfine_mxw_scale_bytes(N, K)))


@pytest.mark.parametrize("missing", (0, 1))
def test_weights_are_required(missing):
    """Weights are read, never made: None is refused, whatever else is right."""
    T, N, K, E, F, k = 3, 64, 64, 4, 64, 2
    X, Y = Device(T, K, dtype=bf), Device(T, N, dtype=bf)
    w = list(weights(1, N, K))
    w[missing] = None
    name = ("codes", "scales")[missing]
    with pytest.raises(ValueError, match=f"^{name} is required"):
        mf.memfine_linear_mxw(N, K, X, *w, Y, stream=0)
    with pytest.raises(ValueError, match=f"^{name} is required"):
        mf.memfine_mxw_unpack(*w, Device(1, N, K, dtype=bf), stream=0)
    for at in (0, 2):
        w = [*weights(E, 2 * F, K), *weights(E, K, F)]
        w[at + missing] = None
        name = ("W1_codes", "W1_scales", "W2_codes", "W2_scales")[at + missing]
        with pytest.raises(ValueError, match=f"^{name} is required"):
            mf.memfine_moe_fwd_mxw(mf.make_shape(T, K, F, E, k, mf.BF16), 1, X,
                                   Device(T, k, dtype=torch.int32),
                                   Device(T, k, dtype=torch.float32), *w, Device(T, K, dtype=bf),
                                   stream=0)


def test_outputs_are_required():
    w = weights(1, 64, 64)
    with pytest.raises(ValueError, match="^Y is required"):
        mf.memfine_linear_mxw(64, 64, Device(3, 64, dtype=bf), *w, None, stream=0)
    with pytest.raises(ValueError, match="^out is required"):
        mf.memfine_mx_values(Device(3, 64), Device(3, 2), None, stream=0)


def test_linear_working_memory():
    """Partial results of a split reduction, none where it is not split."""
    f = mf.memfine_linear_mxw_workspace_bytes
    assert f(0, 64, 8192) == f(1, 64, 8192) == f(16, 64, 4096) == f(16, 64, 4096, True) == 0
    assert f(16, 64, 4128) == f(16, 64, 8192, True) == 2 * 16 * 64 * 4
    assert f(64, 528, 12320) == 4 * 64 * 528 * 4
    assert f(5000, 8192, 8192) == 0
    for bad in ((-1, 64, 64), (1, 8, 64), (1, 64, 48), (2**31, 64, 64)):
        with pytest.raises(mf.MemfineError):
            f(*bad)


def test_experts_rows_of_a_chunk():
    """2^31 - 256 slots in one chunk: row blocks would end past an int."""
    import ctypes
    T, k, P = 2**23 - 1, 256, ctypes.c_void_p(4096)
    shape = mf.make_shape(T, 64, 64, 1024, k, mf.BF16)
    f, b = mf.lib().memfine_moe_fwd_mxw, mf.lib().memfine_moe_mxw_workspace_bytes
    args = [P, None, P, P, P, P, P, P, P]
    for xs in (None, P):
        args[1] = xs
        assert f(ctypes.byref(shape), 1, *args, None, None) == -2
        assert b(ctypes.byref(shape), 1, int(xs is not None)) == -2
        assert b(ctypes.byref(shape), 2, int(xs is not None)) > 0
