"""What stands in keys that nobody sees does not reach a bit of the results: finite values, small once and large once, behind the
sequences' ends, in the next KV head (which the last tile of a head reaches into), outside windows, in other documents."""
import math

import pytest
import torch

import operators_ref as R
import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)
T, HQ, HKV = 900, 8, 4


def results(c, k, lens, q, starts, score):
    shape = P.Shape(2, HQ, HKV, 8, T, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    cache = P.Cache(k=k.cuda(), v_packed=c["v_packed"].cuda(), v_mask=c["v_mask"].cuda(), v_offs=c["v_offs"].cuda(), cap_groups=c["cap"])
    n = q.shape[0]
    out, lse = torch.empty(n, HQ, 128, device="cuda"), torch.empty(n, HQ, device="cuda")
    if starts is None:
        P.decode_attn(shape, cache, q.cuda(), None, None, SCALE, out, Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, shape.n_pages), lse=lse, score=score)
    else:
        P.prefix_attn(shape, cache, q.cuda(), torch.tensor(starts, dtype=torch.int32, device="cuda"), SCALE, out,
                      Bd.new_workspace(shape, Bd.OP_PREFIX_ATTN, n), lse=lse, score=score)
    return out.cpu(), lse.cpu()


@pytest.mark.parametrize("where", ["behind the end", "next head", "window", "documents"])
@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("rows", [0, 9, 40, 150])               # none: scored decode attention; else rows of the first of two prefixes
def test_finite_keys_that_nobody_sees(where, slopes, rows):
    lens = [T, T] if where == "next head" else [870, 301]
    c = R.make_cache(3, 2, HKV, T, 8, 4, lens, poison=False)
    n = rows + 10 if rows else 2
    owner = torch.tensor([0] * rows + [1] * 10 if rows else [0, 1])
    q = torch.randn(n, HQ, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    window, tok_doc, q_doc = 0, None, None
    if where == "window":
        window = 200
    if where == "documents":
        tok_doc = (torch.arange(T) // 7 % 2).to(torch.int32).expand(2, T).contiguous()
        q_doc = torch.zeros(n, dtype=torch.int32)
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    score = P.Score(30.0, torch.full((HQ,), 0.02, device="cuda") if slopes else None,
                    (torch.tensor(lens)[owner] - (0 if rows else 1)).to(torch.int32).cuda(), window, cu(tok_doc), cu(q_doc))
    got = []
    for size in (0.01, 1e4, 3e38):
        k = c["k"].clone()
        for b, m in enumerate(lens):
            k[b, :, m:] = size
            if window:
                k[b, :, :m - window + (1 if rows else 0)] = size
        if where == "documents":
            k[:, :, tok_doc[0] == 1] = size
        if where == "next head":
            k[:, 1::2] = size
        got.append(results(c, k, lens, q, [0, rows, n] if rows else None, score))
    heads = [h for h in range(HQ) if where != "next head" or (h // (HQ // HKV)) % 2 == 0]
    assert torch.isfinite(got[0][0]).all()
    for o, l in got[1:]:
        assert torch.equal(o[:, heads], got[0][0][:, heads]) and torch.equal(l[:, heads], got[0][1][:, heads])
