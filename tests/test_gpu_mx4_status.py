"""Products without a status word of their own: the device's word takes their bits, and a call reads and clears it."""
import ctypes as C

import pytest
import torch

from paper_2511_12934_b200 import binding as B

pytestmark = pytest.mark.gpu


def word():
    """The device's word as a tensor."""
    at = C.c_void_p()
    assert B.load_library().aif_mx4_status_word(C.byref(at)) == B.OK and at.value

    class View:
        __cuda_array_interface__ = {"shape": (1,), "typestr": "<i4", "data": (at.value, False), "version": 3}

    return torch.as_tensor(View(), device="cuda")


def test_products_leave_the_word_clear():
    B.mx4_poll_status()
    for m, n, k in ((300, 96, 160), (5, 300, 512), (40000, 256, 128)):   # the general kernel, and the one that quantises
        x = torch.randn(m, k, device="cuda").bfloat16()
        B.mx4_linear(x, B.mx4_quantize(torch.randn(n, k, device="cuda")), torch.empty(m, n, dtype=torch.bfloat16, device="cuda"))
    assert B.mx4_poll_status() == 0 and word().item() == 0


def test_bits_are_reported_once():
    w = word()
    w.fill_(B.STATUS_TIMEOUT)   # as a product whose wait runs out does
    assert B.mx4_poll_status() == B.STATUS_TIMEOUT
    assert w.item() == 0 and B.mx4_poll_status(stream=torch.cuda.Stream()) == 0
