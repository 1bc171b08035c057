"""max_new is an upper bound: one as large as an int goes with any sequence that fits the cache."""
import ctypes as C

import pytest
import torch

import operators_ref as R
import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_new", [64, 1000, 1 << 20, 2**31 - 4, 2**31 - 1])
@pytest.mark.parametrize("new", [0, 1, 64])
def test_bounds_beyond_the_cache(max_new, new):
    T, heads = 64, 4
    x = torch.randn(1, max(new, 1), heads, 128, device="cuda").to(torch.bfloat16)
    k = torch.full((1, heads, T, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    old, length = (torch.tensor([n], dtype=torch.int32, device="cuda") for n in (T - new, T))
    f, _ = P.rope_frequencies(128)
    freq, status = f.cuda(), torch.full((1,), -7, dtype=torch.int32, device="cuda")
    shape, rope = P.Shape(1, heads, heads, 8, T, length).c(), Bd._Rope(freq.data_ptr(), 128, 0, 1.0, 0)
    rc = P.load_library().stc_rope_write(C.byref(shape), C.byref(rope), old.data_ptr(), max_new, None, None, 0, x.data_ptr(), heads * 128,
                                         None, 0, None, k.data_ptr(), None, status.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert rc == 0 and status.tolist() == [0]
    y, tol = R.rope_ref(x[0, :new].cpu(), torch.arange(T - new, T), f, False, 1.0)
    assert ((k[0, :, T - new:].double().cpu() - y.transpose(0, 1)).abs() <= tol.transpose(0, 1)).all() and (k[0, :, :T - new] == 7).all()
