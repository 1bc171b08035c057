"""The error of stc_tree_attn as a norm, tight enough to notice accumulators that are emptied half as often."""
import math

import pytest
import torch

import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)


@pytest.mark.parametrize("heads,nodes", [((1, 1), 1), ((8, 1), 16), ((4, 4), 1), ((2, 1), 30)])
def test_error_over_long_caches(heads, nodes):
    """131072 tokens with values around 1 and weights of unit variance in the exponent, as good as 131072 / e = 48000 equal ones.  Norm of
    the error over norm of the result.  What has a sign averages out: a weight's pair, 2^-17 / sqrt(48000) = 4e-8; what is cut off adds
    up: an accumulator takes 64 products between two times it is emptied and grows evenly over them, each cuts off up to 4e-8 of it:
    64 * 4e-8 / 2 = 1.3e-6 (twice as many: 2.6e-6).  Exponentials 2^-22, sums in fp32 1e-7.  Together 1.7e-6."""
    Hq, Hkv = heads
    T, gq = 131072, Hq // Hkv
    g = torch.Generator(device="cuda").manual_seed(11)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    k, packed = rand(1, Hkv, T, 128).to(torch.bfloat16), (0.25 * rand(1, Hkv, 4 * T, 32) + 1).to(torch.bfloat16)
    mask = torch.full((1, Hkv, T), 15, dtype=torch.int16, device="cuda")
    offs = (4 * torch.arange(T + 1, device="cuda")).to(torch.int32).expand(1, Hkv, T + 1).contiguous()
    q, kn, vn = rand(1, nodes, Hq, 128).to(torch.bfloat16), rand(1, Hkv, nodes, 128).to(torch.bfloat16), rand(1, Hkv, nodes, 128).to(torch.bfloat16)
    shape, out, status = P.Shape(1, Hq, Hkv, 4, T), torch.zeros(1, nodes, Hq, 128, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    P.tree_attn(shape, P.Cache(k=k, v_packed=packed, v_mask=mask, v_offs=offs, cap_groups=4 * T), P.Tree(kn, vn), q, None, None, SCALE, out,
                status, Bd.new_workspace(shape, Bd.OP_TREE_ATTN, nodes))
    chain = torch.ones(nodes, nodes, dtype=torch.bool, device="cuda").tril()[:, None]
    for h in range(Hkv):
        keys, values = torch.cat([k[0, h], kn[0, h]]).double(), torch.cat([packed[0, h].view(T, 128), vn[0, h]]).double()
        x = torch.einsum("igd,td->igt", q[0, :, h * gq:(h + 1) * gq].double(), keys) * SCALE
        x[:, :, T:] = torch.where(chain, x[:, :, T:], -math.inf)
        want = torch.softmax(x, -1) @ values
        got = out[0, :, h * gq:(h + 1) * gq].double()
        assert ((got - want).norm() / want.norm()).item() <= 1.8e-6
