"""64-bit plain forms of the rotary write and of scored attention, and random routed caches to run them on.

Tolerances.  A bf16 output is off by at most half a step (2^-8 relative) plus the fp32 arithmetic before it.
The attention outputs are fp32: with q, k, v in bf16 every product is exact in fp32, so a score is off by
at most `n_adds` additions of 2^-23 (a tensor core may truncate) of sum |q_c k_c|, plus a few
roundings of its own size; an error d of the scores moves the weights by a factor within e^{2d}; a weight
enters the product as a bf16 pair (2^-16); sums over n tokens add 2^-23 each per sequential step."""
import math

import torch

EPS32 = 2.0 ** -23
D = 128


def rope_ref(x, pos, inv_freq, interleaved, scale):
    """x [..., H, 128] with pos [...] broadcast over heads, in 64 bits; returns (value, bound of |a| + |b|)."""
    rot = 2 * inv_freq.numel()
    y = x.double().clone()
    ang = pos.double()[..., None] * inv_freq.double()
    c, s = ang.cos()[..., None, :] * scale, ang.sin()[..., None, :] * scale
    if interleaved:
        a, b = y[..., 0:rot:2].clone(), y[..., 1:rot:2].clone()
        y[..., 0:rot:2], y[..., 1:rot:2] = a * c - b * s, b * c + a * s
    else:
        a, b = y[..., :rot // 2].clone(), y[..., rot // 2:rot].clone()
        y[..., :rot // 2], y[..., rot // 2:rot] = a * c - b * s, b * c + a * s
    size = torch.zeros_like(y)
    m = (a.abs() + b.abs()) * abs(scale)
    if interleaved:
        size[..., 0:rot:2] = size[..., 1:rot:2] = m
    else:
        size[..., :rot // 2] = size[..., rot // 2:rot] = m
    # half a bf16 step, and (cos, sin, product, sum) each within a few fp32 units of |a| + |b|
    return y, 2.0 ** -8 * y.abs() + 8 * EPS32 * size


def make_cache(seed, B, Hkv, T, S, keep, lens, poison=True):
    """Routed cache on the CPU: dict(k, v_packed, v_mask, v_offs, cap, dense f64 [B,Hkv,T,128], lens).
    Keys, packed groups and masks behind a sequence's end hold NaN / ones when `poison`."""
    g = torch.Generator().manual_seed(seed)
    k = torch.randn(B, Hkv, T, D, generator=g).to(torch.bfloat16)
    k[..., ::37] *= 8
    kept = torch.rand(B, Hkv, T, S, generator=g) < keep / S
    for b, n in enumerate(lens):
        kept[b, :, n:] = False
    counts = kept.sum(-1)
    offs = torch.zeros(B, Hkv, T + 1, dtype=torch.int64)
    offs[..., 1:] = counts.cumsum(-1)
    cap = int(offs[..., -1].max()) + 3
    packed = torch.full((B, Hkv, cap, D // S), float("nan"), dtype=torch.bfloat16)
    dense = torch.zeros(B, Hkv, T, S, D // S, dtype=torch.float64)
    for b in range(B):
        for h in range(Hkv):
            n = int(offs[b, h, -1])
            vals = torch.randn(n, D // S, generator=g).to(torch.bfloat16)
            packed[b, h, :n] = vals
            dense[b, h][kept[b, h]] = vals.double()
    mask = (kept.long() << torch.arange(S)).sum(-1)
    if poison:
        for b, n in enumerate(lens):
            k[b, :, n:] = float("nan")
            mask[b, :, n:] = (1 << S) - 1
    mask = torch.where(mask >= 1 << 15, mask - (1 << 16), mask).to(torch.int16)
    return dict(k=k, v_packed=packed, v_mask=mask, v_offs=offs.to(torch.int32), cap=cap,
                dense=dense.reshape(B, Hkv, T, D), lens=list(lens))


def scored_rows(q, k, v, at, pos, sm_scale, softcap=0.0, slope=None, window=0, doc=None, q_doc=None, n_seq=None):
    """Rows q [R,128] over tokens `at` [N] (k, v [N,128], NaN allowed where unseen), row positions pos [R],
    slope [R] or None, doc [N] / q_doc [R].  Returns out, lse, tol_out, tol_lse in 64 bits."""
    q, k, v = q.double(), k.double(), v.double()
    seen = at[None, :] <= pos[:, None]
    if window:
        seen = seen & (pos[:, None] - at[None, :] < window)
    if doc is not None:
        seen = seen & ((doc[None, :] < 0) | (doc[None, :] == q_doc[:, None]))
    any_seen = seen.any(0)
    k = torch.where(any_seen[:, None], k, torch.zeros_like(k))
    v = torch.where(any_seen[:, None], v, torch.zeros_like(v))
    x = q @ k.T * sm_scale
    size = q.abs() @ k.abs().T * abs(sm_scale)          # of the products that a score sums
    d = (D * EPS32) * size + 4 * EPS32 * x.abs()
    if softcap:
        x = softcap * torch.tanh(x / softcap)
        d = d + 6 * EPS32 * x.abs()
    if slope is not None:
        far = torch.where(seen, at[None, :] - pos[:, None], torch.zeros_like(at[None, :])).double()
        bias = slope.double()[:, None] * far
        x = x + bias
        d = d + 4 * EPS32 * (bias.abs() + x.abs())
    x = torch.where(seen, x, torch.full_like(x, -math.inf))
    d = torch.where(seen, d, torch.zeros_like(d))
    top = x.max(1).values if x.shape[1] else torch.full((q.shape[0],), -math.inf, dtype=torch.float64)
    top0 = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.exp(x - top0[:, None])
    l = p.sum(1)
    alive = l > 0
    l1 = torch.where(alive, l, torch.ones_like(l))
    out = torch.where(alive[:, None], (p @ v) / l1[:, None], torch.zeros(1, dtype=torch.float64))
    lse = torch.where(alive, top0 + torch.log(l1), torch.full_like(l, -math.inf))
    steps = (n_seq if n_seq is not None else x.shape[1] // 8 + 64) * EPS32
    w = torch.exp(2 * d) - 1 + 2.0 ** -16 + 4 * EPS32 * (1 + (x - top0[:, None]).abs().clamp(max=200.0)) + 2 * steps
    w = torch.where(seen, w, torch.zeros_like(w))
    share = (p * w).sum(1) / l1                          # relative error of the normaliser
    tol = ((p * w) @ v.abs()) / l1[:, None] + share[:, None] * ((p @ v.abs()) / l1[:, None]) + 1e-30
    tol_lse = share + 4 * EPS32 * (1 + torch.where(alive, lse.abs() + top0.abs(), torch.zeros_like(lse)))
    return out, lse, tol, tol_lse


def assert_rows(got_out, got_lse, out, lse, tol, tol_lse):
    got_out, got_lse = got_out.double().cpu(), got_lse.double().cpu()
    assert torch.isfinite(got_out).all()
    worst = ((got_out - out).abs() / tol).max().item() if out.numel() else 0.0
    assert worst <= 1.0, f"output {worst:.3g} times its tolerance"
    dead = lse == -math.inf
    assert (got_lse[dead] == -math.inf).all() and (got_out[dead] == 0).all()
    if (~dead).any():
        worst = ((got_lse - lse).abs()[~dead] / tol_lse[~dead]).max().item()
        assert worst <= 1.0, f"lse {worst:.3g} times its tolerance"
