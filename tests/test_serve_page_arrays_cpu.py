"""The list of a pool's arrays that the binding hands over is, byte by byte, one
of wedlm_page_array (include/wedlm_serve.h), and what it refuses."""
import ctypes

import pytest
import torch

from paper_2512_22737_amd import wedlm


class OnDevice:
    """A host tensor that says it is on a device."""
    is_cuda = True

    def __init__(self, x):
        self.x = x

    def __getattr__(self, name):
        return getattr(self.x, name)


def test_the_lists_layout():
    P, L = 5, 3
    xs = [torch.zeros(L, P, 2, 16, 8, dtype=torch.bfloat16),
          torch.zeros(L, P, 7, dtype=torch.uint8), torch.zeros(L, P)]
    made, n, layers = wedlm._page_arrays([OnDevice(x) for x in xs], P)
    assert (n, layers) == (3, L)
    want = (wedlm.PageArray * n)(*(
        wedlm.PageArray(x.data_ptr(), x[0, 0].nbytes) for x in xs))
    assert bytes(made) == bytes(want)
    # the C structure: a pointer and 64 bits
    assert ctypes.sizeof(wedlm.PageArray) == 16
    assert wedlm.PageArray.page_bytes.offset == 8
    assert wedlm._page_arrays([], P) == (None, 0, 1)


def test_refusals():
    x = OnDevice(torch.zeros(3, 5, 2))
    for bad in ([x, OnDevice(torch.zeros(2, 5, 2))],
                [x, OnDevice(torch.zeros(3, 6, 2))],
                [x, OnDevice(torch.zeros(3))],
                [x, OnDevice(torch.zeros(3, 2, 5).transpose(1, 2))],
                [OnDevice(torch.zeros(()))], [torch.zeros(3, 5, 2)]):
        with pytest.raises(wedlm.WedlmError, match="arrays"):
            wedlm._page_arrays(bad, 5)
