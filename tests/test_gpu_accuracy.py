"""Accuracy of the attention operators as a whole: the norm of the difference from the 64-bit form against the norm of the result.

The bounds of operators_ref are worst cases of every element and leave room for errors that add up in one direction.  Here the
bound is on what unbiased rounding leaves.  A sum that takes n terms of like size one after the other, each addition rounded to
nearest, is off by about sqrt(n / 3) * 2^-24 / sqrt(3) of itself (an error uniform within half a step, on a sum that grows), for
n = 512: 4.5e-7.  That happens twice, in the sum of the weighted values and in the sum of the weights (6.4e-7 together).  Weights and
products add constants: 2^-23 of the scores' own size (below one here), 2^-22 for the exponential and up to three truncations of 2^-23,
partly the same above and below the line: 5e-7 together."""
import math

import pytest
import torch

import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)
BOUND = 2.0 ** -19                               # 1.9e-6: the sum of the above, and as much again


def long_cache(seed, B, Hkv, T, live, positive):
    """A cache of which the sequences `live` have T tokens and the others none; one of four value groups is kept per token.
    Returns shape arguments, cache and the dense f64 values of a problem."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    k = torch.empty(B, Hkv, T, 128, dtype=torch.bfloat16, device="cuda")
    packed = torch.empty(B, Hkv, T, 32, dtype=torch.bfloat16, device="cuda")
    for b in live:
        k[b].normal_(generator=g)
        packed[b].uniform_(0.5, 1.5, generator=g) if positive else packed[b].normal_(generator=g)
    mask = (1 << (torch.arange(T, device="cuda") % 4)).to(torch.int16).expand(B, Hkv, T).contiguous()
    offs = torch.arange(T + 1, dtype=torch.int32, device="cuda").expand(B, Hkv, T + 1).contiguous()
    length = torch.zeros(B, dtype=torch.int32, device="cuda")
    length[live] = T

    def dense(b, h):
        d = torch.zeros(T, 4, 32, dtype=torch.float64, device="cuda")
        at = torch.arange(T, device="cuda")
        d[at, at % 4] = packed[b, h].double()
        return d.view(T, 128)

    return length, P.Cache(k=k, v_packed=packed, v_mask=mask, v_offs=offs, cap_groups=T), dense


def error(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("positive", [True, False])
@pytest.mark.parametrize("B,heads,T", [(444, (4, 1), 16384), (130, (8, 1), 30011), (2, (16, 2), 16384), (444, (1, 1), 16384)])
def test_scored_attention_over_whole_caches(B, heads, T, positive):
    """Hundreds of pages per warp; values of one sign show a sum that loses a share of itself at every step."""
    Hq, Hkv = heads
    live = [0, B - 1]
    length, cache, dense = long_cache(B, B, Hkv, T, live, positive)
    shape = P.Shape(B, Hq, Hkv, 4, T, length)
    q = (torch.randn(B, Hq, 128, generator=torch.Generator().manual_seed(B)) * 0.1).to(torch.bfloat16).cuda()
    out, lse = torch.empty(B, Hq, 128, device="cuda"), torch.empty(B, Hq, device="cuda")
    P.decode_attn(shape, cache, q, None, None, SCALE, out, Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, shape.n_pages), lse=lse,
                  score=P.Score(softcap=50.0))
    gq = Hq // Hkv
    for b in live:
        for h in range(Hkv):
            hs = slice(h * gq, (h + 1) * gq)
            x = 50.0 * torch.tanh(q[b, hs].double() @ cache.k[b, h].double().T * SCALE / 50.0)
            assert error(out[b, hs], torch.softmax(x, 1) @ dense(b, h)) <= BOUND
            want = torch.logsumexp(x, 1)
            assert ((lse[b, hs].double() - want).abs() <= BOUND + 4 * 2.0 ** -23 * want.abs()).all()
