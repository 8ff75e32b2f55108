"""Calls of the loss, the norms around a block and the kept activations that end on the host, without a GPU: nothing to do, and refusals."""
import ctypes

from paper_2503_19050_amd import mist

r = ctypes.byref
A = [k << 22 for k in range(1, 32)]  # addresses of tensors that do not overlap


def test_no_sequences_have_no_gates():
    """Without sequences there are no rows of gates' gradients: nothing is launched, so no device is missed."""
    L = mist.load()
    d = mist.BlockDesc(0, 3, 16, 16, 16, 16, 16, 16, 0, 1, 0, 1, 1e-5, 1.0, 1.0)
    g = mist.BlockGrads(None, None, None, None, None, None, None, None, A[8], 16, 16, 16, 16, 16, 0)
    need = ctypes.c_size_t()
    assert L.mist_block_workspace(r(d), r(g), r(need)) == 0
    assert L.mist_block_backward(r(d), None, None, None, None, None, None, A[9], r(g), A[10], need.value, None) == 0
