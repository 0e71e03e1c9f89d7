"""The status word of the 4-bit products: refusals, which need no GPU."""
import ctypes as C

import torch

from paper_2511_12934_b200 import binding as B
from paper_2511_12934_b200 import build as libbuild


def test_refusals():
    libbuild.build()
    lib = B.load_library()
    assert lib.aif_mx4_poll(None, None) == B.ERR_ARG and lib.aif_mx4_status_word(None) == B.ERR_ARG
    if not torch.cuda.is_available():
        bits, at = C.c_uint32(7), C.c_void_p(9)
        assert lib.aif_mx4_poll(C.byref(bits), None) == B.ERR_CUDA and bits.value == 7
        assert lib.aif_mx4_status_word(C.byref(at)) == B.ERR_CUDA and at.value == 9 and b"aif_mx4_status_word" in lib.aif_last_error()
