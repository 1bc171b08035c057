"""Lists of no pages: an empty tensor has no address, and no address means every page; with or without options on the scores."""
import math

import pytest
import torch

import operators_ref as R
import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd

pytestmark = pytest.mark.gpu


def setup(heads):
    c = R.make_cache(8, 2, heads[1], 64, 8, 4, [64, 30])
    shape = P.Shape(2, *heads, 8, 64, torch.tensor([64, 30], dtype=torch.int32, device="cuda"))
    cache = P.Cache(**{k: c[k].cuda() for k in ("k", "v_packed", "v_mask", "v_offs")}, cap_groups=c["cap"])
    q = torch.randn(2, heads[0], 128, device="cuda").to(torch.bfloat16)
    return shape, cache, q, torch.empty(2, heads[0], 128, device="cuda"), torch.empty(2, heads[0], device="cuda")


@pytest.mark.parametrize("heads", [(8, 8), (8, 2), (1, 1)])
@pytest.mark.parametrize("score", [None, P.Score(), P.Score(softcap=5.0), P.Score(window=7)], ids=["none", "off", "cap", "window"])
@pytest.mark.parametrize("pages_of_workspace", [0, 4])
def test_a_list_of_no_pages_attends_nothing(heads, score, pages_of_workspace):
    shape, cache, q, out, lse = setup(heads)
    ids = torch.zeros(2, heads[1], 0, dtype=torch.int32, device="cuda")
    n = torch.zeros(2, heads[1], dtype=torch.int32, device="cuda")
    ws = Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, pages_of_workspace)
    P.decode_attn(shape, cache, q, ids, n, 0.1, out.fill_(1), ws, lse=lse.fill_(1), score=score)
    assert (out == 0).all() and (lse == -math.inf).all() and int(ws[:4].view(torch.int32)[0]) == 0


@pytest.mark.parametrize("pages", [0, 3])
@pytest.mark.parametrize("score", [None, P.Score(softcap=5.0)], ids=["none", "cap"])
def test_a_list_without_its_counts_is_refused(pages, score):
    shape, cache, q, out, lse = setup((8, 2))
    ids = torch.zeros(2, 2, pages, dtype=torch.int32, device="cuda")
    with pytest.raises(P.StcError):
        P.decode_attn(shape, cache, q, ids, None, 0.1, out, Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, 4), score=score)
