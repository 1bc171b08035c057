"""Capped scores by themselves: a sequence of one token has lse = its score.

q and k have one channel each, so the product is exact.  The cap's chain: sm_scale / cap, its product with x (2^-24 each; tanh does
not enlarge a relative error), tanh (below 0.55 the polynomial: 2^-23; above up to five units at 0.5, 5 * 2^-23), cap log2(e)
and its product (2^-24 each), ln 2 and its product (2^-24 each): 8 * 2^-23 of the score."""
import pytest
import torch

import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["one head", "two heads", "prefix"])
@pytest.mark.parametrize("cap", [1.0, 30.0])
def test_capped_scores(call, cap):
    """Both signs, from far below the cap to far beyond it, with both borders of the polynomials between."""
    z = torch.logspace(-4, 1.2, 4000, dtype=torch.float64)
    x = torch.cat([z, -z]).mul(cap).to(torch.bfloat16).unique()
    n, hq = x.numel(), 2 if call == "two heads" else 1
    k = torch.zeros(n, 1, 16, 128, dtype=torch.bfloat16, device="cuda")
    k[:, 0, 0, 5] = x.cuda()
    q = torch.zeros(n, hq, 128, dtype=torch.bfloat16, device="cuda")
    q[:, :, 5] = 1.0
    shape = P.Shape(n, hq, 1, 8, 16, torch.ones(n, dtype=torch.int32, device="cuda"))
    cache = P.Cache(k=k, v_packed=torch.zeros(n, 1, 1, 16, dtype=torch.bfloat16, device="cuda"),
                    v_mask=torch.zeros(n, 1, 16, dtype=torch.int16, device="cuda"),
                    v_offs=torch.zeros(n, 1, 17, dtype=torch.int32, device="cuda"), cap_groups=1)
    out, lse = torch.empty(n, hq, 128, device="cuda"), torch.empty(n, hq, device="cuda")
    if call == "prefix":
        start = torch.arange(n + 1, dtype=torch.int32, device="cuda")
        P.prefix_attn(shape, cache, q, start, 1.0, out, Bd.new_workspace(shape, Bd.OP_PREFIX_ATTN, n), lse=lse, score=P.Score(cap))
    else:
        P.decode_attn(shape, cache, q, None, None, 1.0, out, Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, 1), lse=lse, score=P.Score(cap))
    want = cap * torch.tanh(x.double() / cap)
    assert ((lse.double().cpu() - want[:, None]).abs() <= 8 * 2.0 ** -23 * want.abs()[:, None] + 1e-30).all() and (out == 0).all()
