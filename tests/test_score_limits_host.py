"""Caps that fp32 cannot work with are refused before any launch: the kernels multiply by sm_scale / softcap and by softcap log2(e)."""
import ctypes as C

import pytest

import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd
from paper_2604_21335_b200 import build as B


@pytest.fixture(scope="module")
def lib():
    B.build()
    return P.load_library()


# 2^128 / log2(e) = 2.3586e38 is the first cap whose product is infinite; the least normal fp32 is 1.1755e-38
@pytest.mark.parametrize("cap,scale,fits", [(3.4028e38, 10.0, False), (2.36e38, 10.0, False), (2.35e38, 10.0, True), (2.35e38, 0.1, False),
                                            (8.6e36, 0.1, False), (8.4e36, 0.1, True), (8.6e36, -0.1, False), (8.4e36, -0.1, True),
                                            (2.35e38, 0.0, True), (3.4e38, 0.0, False), (1e30, 0.1, True), (50.0, 0.1, True)])
def test_caps_near_the_largest_number(lib, cap, scale, fits):
    cs, fake = P.Shape(1, 8, 8, 8, 4096).c(), C.c_void_p(0x1000)
    cc, score = Bd._Cache(fake, fake, fake, fake, fake, fake, 100), Bd._Score(cap, 0)
    want = 3 if fits else 1                      # as far as the workspace check, or an invalid argument
    assert lib.stc_decode_attn_scored(C.byref(cs), C.byref(cc), fake, fake, fake, 64, scale, C.byref(score), fake, None, fake, 16, None) == want
    assert lib.stc_prefix_attn(C.byref(cs), C.byref(cc), 4, fake, fake, scale, C.byref(score), None, None, fake, None, fake, 16, None) == want
