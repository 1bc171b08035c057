"""64-bit plain forms of the calls on drafted trees and on whole caches.

Tolerances of the attention: as in operators_ref (every product of two bf16 is exact in fp32; a score is off by its 128
additions, an error d of the scores moves weights within e^{2d}, a weight enters its product as a bf16 pair, each sequential addition
may lose 2^-23)."""
import math
import random

import torch

import operators_ref as R


def random_tree(rng, n, cap):
    """parent list of `cap` entries: the first n a random forest (parents before children), nonsense behind it."""
    parent = []
    for i in range(n):
        parent.append(-1 if i == 0 or rng.random() < 0.1 else rng.randrange(max(0, i - 6), i))
    return parent + [rng.choice([-7, 0, cap, 1 << 20]) for _ in range(cap - n)]


def line(parent, i):
    out = []
    while i >= 0:
        out.append(i)
        i = parent[i]
    return out[::-1]


def tree_rows(q, k, v, at, k_new, v_new, parent, n, pos, sm_scale, softcap=0.0, slope=None, window=0, doc=None, q_doc=0):
    """One KV head of one sequence.  q [n, gq, 128]; k, v [N, 128] of the attended cached tokens `at` [N] (a token may occur twice);
    k_new, v_new [>= n, 128]; pos [n] positions of the nodes; slope [gq].  Returns out [n, gq, 128], lse [n, gq] and tolerances."""
    gq = q.shape[1]
    q, k, v = q[:n].double(), torch.cat([k, k_new[:n]]).double(), torch.cat([v.double(), v_new[:n].double()])
    place = torch.cat([at, pos[:n]])
    kin = torch.zeros(n, n, dtype=torch.bool)
    for i in range(n):
        kin[i, line(parent, i)] = True
    seen = torch.cat([torch.ones(n, at.numel(), dtype=torch.bool), kin], 1)
    if doc is not None:
        seen[:, :at.numel()] &= ((doc[at] < 0) | (doc[at] == q_doc))[None]
    gap = place[None, :] - pos[:n, None]
    seen &= gap <= 0
    if window:
        seen &= -gap < window
    any_seen = seen.any(0)
    k, v = (torch.where(any_seen[:, None], x, torch.zeros_like(x)) for x in (k, v))
    x = torch.einsum("igd,td->igt", q, k) * sm_scale
    d = (R.D * R.EPS32) * torch.einsum("igd,td->igt", q.abs(), k.abs()) * abs(sm_scale) + 4 * R.EPS32 * x.abs()
    if softcap:
        x = softcap * torch.tanh(x / softcap)
        d = d + 6 * R.EPS32 * x.abs()
    if slope is not None:
        bias = slope.double()[None, :, None] * torch.where(seen, gap, torch.zeros_like(gap)).double()[:, None, :]
        x = x + bias
        d = d + 4 * R.EPS32 * (bias.abs() + x.abs())
    hidden = ~seen[:, None, :].expand_as(x)
    x = x.masked_fill(hidden, -math.inf)
    top = x.amax(-1)
    top0 = torch.where(top == -math.inf, torch.zeros_like(top), top)[..., None]
    p = torch.exp(x - top0)
    total = p.sum(-1)
    l1 = torch.where(total > 0, total, torch.ones_like(total))[..., None]
    out = (p @ v) / l1
    lse = torch.where(total > 0, top0[..., 0] + torch.log(l1[..., 0]), torch.full_like(total, -math.inf))
    steps = (x.shape[-1] // 8 + 64) * R.EPS32
    w = torch.exp(2 * d) - 1 + 2.0 ** -16 + 4 * R.EPS32 * (1 + (x - top0).abs().clamp(max=200.0)) + 2 * steps
    w = w.masked_fill(hidden, 0.0)
    share = (p * w).sum(-1) / l1[..., 0]
    tol = ((p * w) @ v.abs()) / l1 + share[..., None] * ((p @ v.abs()) / l1) + 1e-30
    alive = total > 0
    tol_lse = share + 4 * R.EPS32 * (1 + torch.where(alive, lse.abs() + top0[..., 0].abs(), torch.zeros_like(lse)))
    return out, lse, tol, tol_lse


def accept(logits, tokens, parent, n):
    """(path, next) of one sequence; logits [cap, V] in any type."""
    if n == 0:
        return [], -1
    path = [0]
    while True:
        row = logits[path[-1]].double()
        nan = torch.isnan(row)
        top = nan if nan.any() else row == row.max()
        x = int(top.nonzero()[0])
        child = [i for i in range(path[-1] + 1, n) if parent[i] == path[-1] and tokens[i] == x]
        if not child:
            return path, x
        path.append(child[0])


def rng(seed):
    return random.Random(seed)


def dense_of(c, b, h, S):
    """Packed groups of a cache dict by token: list of bf16 [groups kept, 128 / S], and the masks as ints."""
    o = c["v_offs"][b, h].tolist()
    return [c["v_packed"][b, h, o[t]:o[t + 1]] for t in range(len(o) - 1)], [int(x) & 0xFFFF for x in c["v_mask"][b, h]]


def meta(k, n):
    """Page metadata of the first n rows of k [T, 128]: lists of min and max rows."""
    pages = [k[p * 16:min(n, p * 16 + 16)].float() for p in range((n + 15) // 16)]
    return [x.amin(0).bfloat16() for x in pages], [x.amax(0).bfloat16() for x in pages]
