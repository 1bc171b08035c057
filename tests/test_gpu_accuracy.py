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


# Shared prefixes.  A weight enters as a bf16 pair: its error is uniform within half a step of the residual, 2.45e-6 of the weight in the
# mean square over a binade, independent from weight to weight.  Values of random sign keep that share of the result's norm; values
# of one sign average it away (by the root of the number of tokens).  The tensor core takes 4e-8 of an accumulator away per product of 16
# tokens (a mean; less than 1.2e-7): over n products between two emptyings 4e-8 n / 2 of a sum that grows evenly, 4e-8 n 2/3 of one that
# walks at random.  n is 256 with one row tile, 128 with two, and 8 per tile of a prefix too short to be emptied.
@pytest.mark.parametrize("positive", [True, False])
@pytest.mark.parametrize("what,rows,Hkv,T,bound", [
    ("short", 8, 32, 272, 2.0 ** -18),                   # 2.45e-6 + 24 products: 0.7e-6
    ("hundreds of tiles, one row tile", 20, 48, 100_003, 2.0 ** -16),      # 2.45e-6 + 6.9e-6
    ("hundreds of tiles, two row tiles", 150, 48, 100_003, 2.0 ** -17)])   # 2.45e-6 + 3.4e-6
def test_shared_prefix(what, rows, Hkv, T, bound, positive):
    length, cache, dense = long_cache(rows, 1, Hkv, T, [0], positive)
    shape = P.Shape(1, Hkv, Hkv, 4, T, length)
    q = (torch.randn(rows, Hkv, 128, generator=torch.Generator().manual_seed(rows)) * 0.1).to(torch.bfloat16).cuda()
    out, lse = torch.empty(rows, Hkv, 128, device="cuda"), torch.empty(rows, Hkv, device="cuda")
    P.prefix_attn(shape, cache, q, torch.tensor([0, rows], dtype=torch.int32, device="cuda"), SCALE, out,
                  Bd.new_workspace(shape, Bd.OP_PREFIX_ATTN, rows), lse=lse)
    for h in range(0, Hkv, 7):
        x = q[:, h].double() @ cache.k[0, h].double().T * SCALE
        assert error(out[:, h], torch.softmax(x, 1) @ dense(0, h)) <= bound
        want = torch.logsumexp(x, 1)
        assert ((lse[:, h].double() - want).abs() <= BOUND + 4 * 2.0 ** -23 * want.abs()).all()


@pytest.mark.parametrize("heads", [(4, 1), (28, 4), (8, 8)])
def test_scored_attention_over_short_lists(heads):
    """Three bf16 parts of a weight leave 2^-24 of it; 30 pages: scores and products as above, 2^-20 together."""
    Hq, Hkv = heads
    length, cache, dense = long_cache(Hq, 3, Hkv, 480, [0, 1, 2], False)
    shape = P.Shape(3, Hq, Hkv, 4, 480, length)
    q = (torch.randn(3, Hq, 128, generator=torch.Generator().manual_seed(Hq)) * 0.1).to(torch.bfloat16).cuda()
    out = torch.empty(3, Hq, 128, device="cuda")
    P.decode_attn(shape, cache, q, None, None, SCALE, out, Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, shape.n_pages), score=P.Score(softcap=50.0))
    gq = Hq // Hkv
    for b in range(3):
        for h in range(Hkv):
            hs = slice(h * gq, (h + 1) * gq)
            x = 50.0 * torch.tanh(q[b, hs].double() @ cache.k[b, h].double().T * SCALE / 50.0)
            assert error(out[b, hs], torch.softmax(x, 1) @ dense(b, h)) <= 2.0 ** -20
