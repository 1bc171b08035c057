"""The operators around the cache that are timed and compared: rotary write, scored decode attention, shared prefix.

Every case is one call of a serving program.  With ``own`` false the operators are computed in their plain form
(elementary torch operations in 32 bits); with ``own`` true by the library's calls.

  rope     the projection's q, k, v of the new tokens of a batch are rotated and written where the cache wants them
  scored   one decode step over the listed pages of a routed cache, with capped / biased / windowed / per-document scores
  prefix   one decode step of sequences that share prefixes, joined with the results over their own tokens
"""
import math

import torch

own = False

DEV = "cuda"
D = 128
PAGE = 16


# ---- cases --------------------------------------------------------------------------------------------------------
def _rope(name, batch, hq, hkv, max_new, t_cap, rot, interleaved, scaling, ragged, far):
    return dict(name=name, op="rope", batch=batch, hq=hq, hkv=hkv, max_new=max_new, t_cap=t_cap, rot=rot,
                interleaved=interleaved, scaling=scaling, ragged=ragged, far=far)


def _scored(name, batch, hq, hkv, t, groups, keep, pages, cap, alibi, window, docs, ragged):
    return dict(name=name, op="scored", batch=batch, hq=hq, hkv=hkv, t=t, groups=groups, keep=keep, pages=pages,
                cap=cap, alibi=alibi, window=window, docs=docs, ragged=ragged)


def _prefix(name, prefixes, rows, hq, hkv, t, groups, keep, cap, alibi, window, ragged):
    return dict(name=name, op="prefix", prefixes=prefixes, rows=rows, hq=hq, hkv=hkv, t=t, groups=groups, keep=keep,
                cap=cap, alibi=alibi, window=window, ragged=ragged)


def listed():
    return [
        # one new token for each of 16 long-context sequences: the call of every layer of every decode step
        _rope("rope step 16x1", 16, 32, 8, 1, 512, 128, False, "yarn", False, True),
        # chunked prefill of eight ragged requests on 28 / 4 heads, half of the head rotated, interleaved pairs
        _rope("rope ragged 8x511", 8, 28, 4, 511, 1024, 64, True, "linear", True, False),
        # two whole prompts of 16384 tokens
        _rope("rope prompt 2x16384", 2, 32, 8, 16384, 16384, 128, False, "bands", False, False),
        # the smallest decode step: one sequence, eight single-query heads, capped scores
        _scored("scored cap 1x8", 1, 8, 8, 4096, 8, 4, 64, 30.0, False, 0, 0, False),
        # 32 single-query heads with distance slopes over 32768 cached tokens, 128 selected pages
        _scored("scored alibi 1x32", 1, 32, 32, 32768, 8, 4, 128, 0.0, True, 0, 0, False),
        # eight sequences with 7 query heads per KV head, 16 value groups, capped scores
        _scored("scored cap 8x28/4", 8, 28, 4, 32768, 16, 4, 256, 50.0, False, 0, 0, False),
        # long ragged contexts: window over the recent half, cached documents that only their own queries see
        _scored("scored window docs 16x32/8", 16, 32, 8, 131072, 8, 4, 256, 0.0, False, 65536, 3, True),
        # an image + text prompt of 272 tokens shared by eight answers, single-query heads
        _prefix("prefix 272 8x32", 1, 8, 32, 32, 272, 8, 3, 0.0, False, 0, False),
        # a 32768-token document, eight questions, 7 query heads per KV head
        _prefix("prefix 32768 8x28/4", 1, 8, 28, 4, 32768, 16, 4, 0.0, False, 0, False),
        # three system prompts of odd lengths, 37 sequences split unevenly between them, distance slopes
        _prefix("prefix 3x20011 37x32/8", 3, 37, 32, 8, 20011, 8, 4, 0.0, True, 0, True),
        # a 131072-token context shared by 16 sequences, capped scores
        _prefix("prefix 131072 16x32/8", 1, 16, 32, 8, 131072, 8, 4, 50.0, False, 0, False),
        # a large batch behind one 32768-token prompt: 512 query rows per KV head, bound by the products
        _prefix("prefix 32768 128x32/8", 1, 128, 32, 8, 32768, 8, 4, 0.0, False, 0, False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "scored", "prefix"])
    hq, hkv = rng.choice([(8, 8), (28, 4), (32, 8), (32, 32), (16, 8), (12, 2)])
    groups = rng.choice([4, 8, 16])
    keep = rng.randint(1, groups)
    if op == "rope":
        tokens = _log(rng, 1, 32768)
        batch = min(_log(rng, 1, 64), tokens)
        max_new = max(1, tokens // batch)
        if hq + 2 * hkv > 48:                                   # no more bytes than the largest listed call
            max_new = max(1, max_new // 2)
        return dict(op=op, batch=batch, hq=hq, hkv=hkv, max_new=max_new, t_cap=max_new + rng.randint(0, 700),
                    rot=rng.choice([16, 32, 64, 96, 128]), interleaved=rng.random() < 0.5,
                    scaling=rng.choice(["none", "linear", "yarn", "bands"]), ragged=rng.random() < 0.6,
                    far=rng.random() < 0.5)
    if op == "scored":
        t = _log(rng, 17, 131072)
        batch = min(_log(rng, 1, 32), max(1, 16 * 131072 * 8 // (t * hkv)))
        pages = min((t + PAGE - 1) // PAGE, _log(rng, 1, 256))
        return dict(op=op, batch=batch, hq=hq, hkv=hkv, t=t, groups=groups, keep=keep, pages=pages,
                    cap=rng.choice([0.0, 30.0, 50.0]), alibi=rng.random() < 0.4,
                    window=rng.choice([0, _log(rng, 16, t)]), docs=rng.choice([0, 0, 3]), ragged=rng.random() < 0.5)
    rows = _log(rng, 2, 128)
    prefixes = min(rows, rng.choice([1, 1, 2, 3, 5]))
    most = 32768 * 512 * 8 // (rows * hq)                        # no more products than the largest listed call
    most = min(most, 131072 * 8 // (hkv * prefixes))             # and no more bytes
    t = _log(rng, 17, max(18, min(131072, most)))
    return dict(op=op, prefixes=prefixes, rows=rows, hq=hq, hkv=hkv, t=t, groups=groups, keep=keep,
                cap=rng.choice([0.0, 0.0, 30.0, 50.0]), alibi=rng.random() < 0.3,
                window=rng.choice([0, 0, t + _log(rng, 1, 64)]), ragged=rng.random() < 0.5)


# ---- inputs -------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.bfloat16)


def _lengths(n, most, ragged, least=1):
    """Lengths of n sequences as a list: `most` for all, or spread evenly over least..most in a mixed order, the first `most`."""
    if not ragged:
        return [most] * n
    return [most - int((i * 0.6180339887498949) % 1.0 * (most - least + 1)) for i in range(n)]


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _inv_freq(rot, scaling):
    """Radians per position of each pair, in 64 bits, and the factor on the rotated channels."""
    i = torch.arange(rot // 2, dtype=torch.float64)
    if scaling == "bands":                    # base 500000; wavelengths beyond the trained context / 1 slowed 8 times
        f = 500000.0 ** (-2.0 * i / rot)
        wave, old = 2 * math.pi / f, 8192.0
        smooth = ((old / wave - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
        return (1 - smooth) * f / 8.0 + smooth * f, 1.0
    f = 10000.0 ** (-2.0 * i / rot)
    if scaling == "linear":
        return f / 4.0, 1.0
    if scaling == "yarn":                      # slow pairs interpolated, fast ones kept, a linear ramp between
        old, factor, base = 32768.0, 4.0, 10000.0
        pair = lambda turns: rot * math.log(old / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(pair(32.0)), 0), min(math.ceil(pair(1.0)), rot - 1)
        ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
        return f / factor * ramp + f * (1 - ramp), 0.1 * math.log(factor) + 1.0
    return f, 1.0


def _cache(g, problems0, hkv, t, groups, keep, lens):
    """Keys with four loud channels per head, and a packed value store: every group kept with probability keep / groups."""
    k = _normal(g, problems0, hkv, t, D)
    loud = torch.rand(hkv, D, generator=g, device=DEV).argsort(dim=1)[:, :4]
    scale = torch.ones(hkv, D, dtype=torch.bfloat16, device=DEV).scatter_(1, loud, 8.0)
    k *= scale[None, :, None, :]
    kept = torch.rand(problems0, hkv, t, groups, generator=g, device=DEV) < keep / groups
    length = _i32(lens)
    kept &= (torch.arange(t, device=DEV)[None, :] < length[:, None])[:, None, :, None]
    bits = (kept.to(torch.int32) << torch.arange(groups, device=DEV, dtype=torch.int32)).sum(-1, dtype=torch.int32)
    offs = torch.zeros(problems0, hkv, t + 1, dtype=torch.int32, device=DEV)
    offs[..., 1:] = kept.sum(-1, dtype=torch.int32).cumsum(-1, dtype=torch.int32)
    cap = max(1, int(offs[..., -1].max()))
    v = _normal(g, problems0, hkv, cap, D // groups)
    return dict(k=k, v_packed=v, v_mask=bits.to(torch.int16), v_offs=offs, cap=cap, len=length)


def _slopes(hq):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], dtype=torch.float32, device=DEV)


def _cuts(c):
    """First row of each prefix and the end: equal shares of the sequences, or shares that grow from prefix to prefix."""
    w = [1.0 + i if c["ragged"] else 1.0 for i in range(c["prefixes"])]
    return [0] + [round(c["rows"] * sum(w[:i + 1]) / sum(w)) for i in range(c["prefixes"])]


def prepare(case, seed):
    g = _generator(seed)
    c = case
    s = dict(case=c)
    if c["op"] == "rope":
        B, n, t_cap = c["batch"], c["max_new"], c["t_cap"]
        new = _lengths(B, n, c["ragged"])
        u = torch.rand(B, generator=g, device=DEV, dtype=torch.float64).tolist()
        old = [int(x * (t_cap - m + 1)) for x, m in zip(u, new)]
        # the fused projection's output: a token's q, k and v rows next to each other
        qkv = _normal(g, B, n, c["hq"] + 2 * c["hkv"], D)
        f, scale = _inv_freq(c["rot"], c["scaling"])
        s |= dict(q_in=qkv[:, :, :c["hq"]], k_in=qkv[:, :, c["hq"]:c["hq"] + c["hkv"]], v_in=qkv[:, :, c["hq"] + c["hkv"]:],
                  inv_freq=f.to(DEV), scale=scale, old_len=_i32(old), new_len=_i32([a + b for a, b in zip(old, new)]),
                  count=_i32(new), total=sum(new), pos=None,
                  q_out=torch.zeros(B, n, c["hq"], D, dtype=torch.bfloat16, device=DEV),
                  k=torch.zeros(B, c["hkv"], t_cap, D, dtype=torch.bfloat16, device=DEV),
                  v=torch.zeros(B, c["hkv"], t_cap, D, dtype=torch.bfloat16, device=DEV),
                  status=torch.zeros(B, dtype=torch.int32, device=DEV))
        if c["far"]:                           # tokens of a reduced sequence keep the positions they had in the long one
            first = torch.randint(0, 131072 - n, (B, 1), generator=g, device=DEV, dtype=torch.int32)
            s["pos"] = (first + torch.arange(n, device=DEV, dtype=torch.int32)[None, :]).contiguous()
        return s
    hq, hkv = c["hq"], c["hkv"]
    if c["op"] == "scored":
        B, t = c["batch"], c["t"]
        lens = _lengths(B, t, c["ragged"])
        s |= _cache(g, B, hkv, t, c["groups"], c["keep"], lens)
        pages = (t + PAGE - 1) // PAGE
        # the selection as stc_quest_select leaves it: distinct ids, ascending, the page of the newest token among them
        r = torch.rand(B, hkv, pages, generator=g, device=DEV)
        live = (s["len"] + PAGE - 1) // PAGE
        at = torch.arange(pages, device=DEV)
        r = torch.where(at[None, None] < live[:, None, None], r, 2.0)
        r = torch.where(at[None, None] == (live - 1)[:, None, None], -1.0, r)
        ids = r.argsort(-1)[..., :c["pages"]]
        n_pages = live.clamp(max=c["pages"])
        ids = torch.where(torch.arange(c["pages"], device=DEV)[None, None] < n_pages[:, None, None], ids, pages)
        ids = ids.sort(-1).values
        s |= dict(page_ids=ids.to(torch.int32).contiguous(), n_pages=n_pages[:, None].expand(B, hkv).to(torch.int32).contiguous(),
                  q=_normal(g, B, hq, D), slopes=_slopes(hq) if c["alibi"] else None, q_pos=s["len"] - 1,
                  tok_doc=None, q_doc=None,
                  out=torch.empty(B, hq, D, dtype=torch.float32, device=DEV),
                  lse=torch.empty(B, hq, dtype=torch.float32, device=DEV))
        if c["docs"]:                          # documents in a row; the last belongs to the query, the first (-1) to all
            cut = torch.arange(t, device=DEV, dtype=torch.int64)[None, :] * (c["docs"] + 1) // s["len"].long()[:, None].clamp(min=1)
            s["tok_doc"] = (cut.to(torch.int32).clamp(max=c["docs"]) - 1).contiguous()
            s["q_doc"] = _i32([c["docs"] - 1] * B)
        return s
    G, rows, t = c["prefixes"], c["rows"], c["t"]
    lens = _lengths(G, t, c["ragged"], least=max(1, t // 2))
    s |= _cache(g, G, hkv, t, c["groups"], c["keep"], lens)
    cuts = _cuts(c)
    own_tokens = torch.randint(1, 64, (rows,), generator=g, device=DEV, dtype=torch.int32)
    start = _i32(cuts)
    group = torch.repeat_interleave(torch.arange(G, device=DEV), (start[1:] - start[:-1]).long(), output_size=rows)
    s |= dict(row_start=start, group=group, widest=max(b - a for a, b in zip(cuts, cuts[1:])),
              q=_normal(g, rows, hq, D), slopes=_slopes(hq) if c["alibi"] else None,
              q_pos=(s["len"][group] + own_tokens).contiguous(),
              own_out=torch.randn(rows, hq, D, generator=g, device=DEV),
              own_lse=torch.randn(rows, hq, generator=g, device=DEV) + 6.0,
              out=torch.empty(rows, hq, D, dtype=torch.float32, device=DEV),
              lse=torch.empty(rows, hq, dtype=torch.float32, device=DEV))
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------
def _plain_rope(s):
    c = s["case"]
    rot, half = c["rot"], c["rot"] // 2
    b = torch.repeat_interleave(torch.arange(c["batch"], device=DEV), s["count"].long(), output_size=s["total"])
    first = (s["count"].cumsum(0) - s["count"]).long()
    i = torch.arange(s["total"], device=DEV) - first[b]
    t = s["old_len"].long()[b] + i
    pos = t if s["pos"] is None else s["pos"][b, i].long()
    angle = torch.remainder(pos.double()[:, None] * s["inv_freq"][None, :], 2 * math.pi).float()
    cos, sin = (angle.cos() * s["scale"])[:, None, :], (angle.sin() * s["scale"])[:, None, :]

    def rotated(x):
        x = x.float()
        if c["interleaved"]:
            lo, hi = x[..., 0:rot:2], x[..., 1:rot:2]
            y = torch.stack([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1).flatten(-2)
        else:
            lo, hi = x[..., :half], x[..., half:rot]
            y = torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1)
        return torch.cat([y, x[..., rot:]], dim=-1).to(torch.bfloat16)

    s["q_out"][b, i] = rotated(s["q_in"][b, i])
    s["k"][b, :, t] = rotated(s["k_in"][b, i])
    s["v"][b, :, t] = s["v_in"][b, i]
    return s["q_out"], s["k"], s["v"]


def _plain_values(s, tokens, groups):
    """f32 [B, Hkv, N, 128]: the values of `tokens` [B, Hkv, N], dropped groups zero."""
    bits = torch.gather(s["v_mask"], 2, tokens).int()
    bit = (bits[..., None] >> torch.arange(groups, device=DEV, dtype=torch.int32)) & 1
    at = torch.gather(s["v_offs"], 2, tokens)[..., None] + bit.cumsum(-1) - bit
    B, H = tokens.shape[:2]
    base = (torch.arange(B * H, device=DEV) * s["cap"]).view(B, H, 1, 1)
    rows = s["v_packed"].view(B * H * s["cap"], -1)[base + at.clamp(max=s["cap"] - 1)].float()
    return (rows * 0.0).where(bit[..., None] == 0, rows).flatten(-2)


def _plain_softmax(x, v):
    """out, lse of softmax(x) v over the last axis of x; rows without a finite score give 0 and -inf."""
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    out = torch.where(total > 0, (p @ v) / total, 0.0)
    return out, torch.where(total > 0, top + torch.log(total), -math.inf)[..., 0]


def _plain_scored(s):
    c = s["case"]
    B, hkv, gq = c["batch"], c["hkv"], c["hq"] // c["hkv"]
    tokens = (s["page_ids"].long()[..., None] * PAGE + torch.arange(PAGE, device=DEV)).flatten(2)
    slot_ok = torch.arange(c["pages"], device=DEV) < s["n_pages"][..., None]
    seen = slot_ok.repeat_interleave(PAGE, dim=-1) & (tokens < s["len"][:, None, None])
    pos = s["q_pos"][:, None, None]
    seen &= tokens <= pos
    if c["window"]:
        seen &= pos - tokens < c["window"]
    tokens = torch.where(seen, tokens, 0)
    if c["docs"]:
        doc = torch.gather(s["tok_doc"][:, None, :].expand(B, hkv, -1), 2, tokens)
        seen &= (doc < 0) | (doc == s["q_doc"][:, None, None])
    k = torch.gather(s["k"], 2, tokens[..., None].expand(-1, -1, -1, D)).float()
    x = (s["q"].float().view(B, hkv, gq, D) @ k.transpose(-1, -2)) / math.sqrt(D)
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    if c["alibi"]:
        x = x + s["slopes"].view(1, hkv, gq, 1) * (tokens - pos)[:, :, None, :].float()
    x = x.masked_fill(~seen[:, :, None, :], -math.inf)
    out, lse = _plain_softmax(x, _plain_values(s, tokens, c["groups"]))
    return out.reshape(B, c["hq"], D), lse.reshape(B, c["hq"])


def _plain_prefix(s):
    c = s["case"]
    G, hkv, gq, t, rows, wide = c["prefixes"], c["hkv"], c["hq"] // c["hkv"], c["t"], c["rows"], s["widest"]
    # the sequences of each prefix side by side, the last one repeated where a prefix has fewer
    row = (s["row_start"][:-1, None].long() + torch.arange(wide, device=DEV)).clamp(max=rows - 1)
    q = s["q"].float()[row].view(G, wide, hkv, gq, D).transpose(1, 2).reshape(G, hkv, wide * gq, D)
    x = (q @ s["k"].float().transpose(-1, -2)).view(G, hkv, wide, gq, t) / math.sqrt(D)
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    at = torch.arange(t, device=DEV)
    away = at - s["q_pos"].long()[row][..., None]                 # [G, wide, t], never positive for a visible token
    if c["alibi"]:
        x = x + s["slopes"].view(1, hkv, 1, gq, 1) * away[:, None, :, None, :].float()
    seen = (at < s["len"][:, None, None]) & (away <= 0)
    if c["window"]:
        seen &= -away < c["window"]
    x = x.masked_fill(~seen[:, None, :, None, :], -math.inf)
    every = at.expand(G, hkv, t)
    out, lse = _plain_softmax(x.flatten(2, 3), _plain_values(s, every, c["groups"]))
    # back to the order of the rows
    group, slot = s["group"], torch.arange(rows, device=DEV) - s["row_start"].long()[s["group"]]
    out = out.view(G, hkv, wide, gq, D).transpose(1, 2).reshape(G, wide, c["hq"], D)[group, slot]
    lse = lse.view(G, hkv, wide, gq).transpose(1, 2).reshape(G, wide, c["hq"])[group, slot]
    # joined with the sequences' own tokens
    top = torch.maximum(lse, s["own_lse"])
    top = torch.where(top == -math.inf, 0.0, top)
    a, b = torch.exp(lse - top), torch.exp(s["own_lse"] - top)
    joined = torch.where((a + b)[..., None] > 0, (a[..., None] * out + b[..., None] * s["own_out"]) / (a + b)[..., None], 0.0)
    return joined, top + torch.log(a + b)


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(state):
    s = state
    op = s["case"]["op"]
    if own:
        return {"rope": _own_rope, "scored": _own_scored, "prefix": _own_prefix}[op](s)
    return {"rope": _plain_rope, "scored": _plain_scored, "prefix": _plain_prefix}[op](s)


def _own_rope(s):
    import paper_2604_21335_b200 as P
    c = s["case"]
    shape = P.Shape(c["batch"], c["hq"], c["hkv"], 8, c["t_cap"], s["new_len"])
    rope = P.Rope(s["inv_freq"], interleaved=c["interleaved"], scale=s["scale"])
    P.rope_write(shape, rope, s["old_len"], s["status"], q_in=s["q_in"], k_in=s["k_in"], v_in=s["v_in"],
                 q_out=s["q_out"], k=s["k"], v=s["v"], positions=s["pos"])
    return s["q_out"], s["k"], s["v"]


def _own_cache(P, s, batch):
    c = s["case"]
    shape = P.Shape(batch, c["hq"], c["hkv"], c["groups"], c["t"], s["len"])
    cache = P.Cache(k=s["k"], v_packed=s["v_packed"], v_mask=s["v_mask"], v_offs=s["v_offs"], cap_groups=s["cap"])
    return shape, cache


def _own_scored(s):
    import paper_2604_21335_b200 as P
    c = s["case"]
    shape, cache = _own_cache(P, s, c["batch"])
    if "ws" not in s:                          # the workspace that a serving program allocates once
        s["ws"] = P.binding.new_workspace(shape, P.binding.OP_DECODE_ATTN, c["pages"])
    score = P.Score(softcap=c["cap"], slopes=s["slopes"], q_pos=s["q_pos"], window=c["window"],
                    tok_doc=s["tok_doc"], q_doc=s["q_doc"])
    P.decode_attn(shape, cache, s["q"], s["page_ids"], s["n_pages"], 1 / math.sqrt(D), s["out"], s["ws"],
                  lse=s["lse"], score=score)
    return s["out"], s["lse"]


def _own_prefix(s):
    import paper_2604_21335_b200 as P
    c = s["case"]
    shape, cache = _own_cache(P, s, c["prefixes"])
    if "ws" not in s:
        s["ws"] = P.binding.new_workspace(shape, P.binding.OP_PREFIX_ATTN, c["rows"])
    score = P.Score(softcap=c["cap"], slopes=s["slopes"], q_pos=s["q_pos"], window=c["window"])
    P.prefix_attn(shape, cache, s["q"], s["row_start"], 1 / math.sqrt(D), s["out"], s["ws"], lse=s["lse"],
                  score=score, own_out=s["own_out"], own_lse=s["own_lse"])
    return s["out"], s["lse"]


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "rope":
        tokens = sum(_lengths(c["batch"], c["max_new"], c["ragged"]))
        heads = c["hq"] + 2 * c["hkv"]
        return dict(bytes=tokens * heads * 512.0, flops=tokens * (c["hq"] + c["hkv"]) * c["rot"] * 3.0)
    per_token = 256.0 + 256.0 * c["keep"] / c["groups"] + 2.0
    gq = c["hq"] // c["hkv"]
    if c["op"] == "scored":
        n = 0.0
        for length in _lengths(c["batch"], c["t"], c["ragged"]):
            tokens = min(c["pages"] * PAGE, length)
            if c["window"]:
                tokens *= min(1.0, c["window"] / length)
            if c["docs"]:
                tokens *= 2.0 / (c["docs"] + 1)
            n += tokens * c["hkv"]
        return dict(bytes=n * per_token + c["batch"] * c["hq"] * 772.0, flops=4.0 * n * gq * D)
    lens = _lengths(c["prefixes"], c["t"], c["ragged"], least=max(1, c["t"] // 2))
    cuts = _cuts(c)
    return dict(bytes=sum(lens) * c["hkv"] * per_token + c["rows"] * c["hq"] * (256.0 + 4 * 260.0),
                flops=4.0 * c["hq"] * D * sum(n * (b - a) for n, a, b in zip(lens, cuts, cuts[1:])))


# ---- the definition in 64 bits ------------------------------------------------------------------------------------
def _exact_rope(s):
    c = s["case"]
    rot = c["rot"]
    q, k, v = (torch.zeros(x.shape, dtype=torch.float64, device=DEV) for x in (s["q_out"], s["k"], s["v"]))
    for b, (lo, n) in enumerate(zip(s["old_len"].tolist(), s["count"].tolist())):
        pos = torch.arange(lo, lo + n, device=DEV) if s["pos"] is None else s["pos"][b, :n].long()
        turn = torch.outer(pos.double(), s["inv_freq"])
        unit = torch.polar(torch.full_like(turn, s["scale"]), turn)[:, None, :]

        def spun(x):
            y = x.double().clone()
            pairs = y[..., :rot].unflatten(-1, (-1, 2)) if c["interleaved"] else y[..., :rot].unflatten(-1, (2, -1)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * unit)
            y[..., :rot] = (z if c["interleaved"] else z.transpose(-1, -2)).flatten(-2)
            return y

        q[b, :n] = spun(s["q_in"][b, :n])
        k[b, :, lo:lo + n] = spun(s["k_in"][b, :n]).transpose(0, 1)
        v[b, :, lo:lo + n] = s["v_in"][b, :n].double().transpose(0, 1)
    return q, k, v


def _exact_dense(s, p0, h, length, groups):
    """f64 [length, 128] values of one problem: the packed groups dealt out in the order of the mask's bits."""
    word = s["v_mask"][p0, h, :length].long() & 0xFFFF
    kept = (word[:, None] >> torch.arange(groups, device=DEV)) & 1
    dense = torch.zeros(length, groups, D // groups, dtype=torch.float64, device=DEV)
    dense[kept.bool()] = s["v_packed"][p0, h, :int(kept.sum())].double()
    return dense.view(length, D)


def _exact_head(c, q, k, v, at, pos, slope, seen):
    """out [rows, 128], lse [rows] of rows q over tokens `at`: pos, slope [rows], seen [rows, tokens]."""
    x = q.double() @ k.double().T / math.sqrt(D)
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    if slope is not None:
        x = x + slope.double()[:, None] * (at[None, :] - pos[:, None]).double()
    x[~seen] = -math.inf
    lse = torch.logsumexp(x, dim=1)
    p = torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[:, None])
    return p @ v, lse


def exact(case, seed):
    s = prepare(case, seed)
    c = case
    if c["op"] == "rope":
        return _exact_rope(s)
    gq = c["hq"] // c["hkv"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device=DEV)
    lens = s["len"].tolist()
    if c["op"] == "scored":
        for b, length in enumerate(lens):
            pos = s["q_pos"][b].long()
            for h in range(c["hkv"]):
                ids = s["page_ids"][b, h, :int(s["n_pages"][b, h])].long()
                at = (ids[:, None] * PAGE + torch.arange(PAGE, device=DEV)).flatten()
                at = at[at < length]
                seen = at <= pos
                if c["window"]:
                    seen &= at > pos - c["window"]
                if c["docs"]:
                    doc = s["tok_doc"][b, at]
                    seen &= (doc < 0) | (doc == s["q_doc"][b])
                hs = slice(h * gq, (h + 1) * gq)
                out[b, hs], lse[b, hs] = _exact_head(
                    c, s["q"][b, hs], s["k"][b, h, at], _exact_dense(s, b, h, length, c["groups"])[at], at,
                    pos.expand(gq), s["slopes"][hs] if c["alibi"] else None, seen.expand(gq, -1))
        return out, lse
    cuts = s["row_start"].tolist()
    for p, length in enumerate(lens):
        a, b = cuts[p], cuts[p + 1]
        at = torch.arange(length, device=DEV)
        pos = s["q_pos"][a:b].long().repeat_interleave(gq)
        seen = at[None, :] <= pos[:, None]
        if c["window"]:
            seen &= at[None, :] > pos[:, None] - c["window"]
        for h in range(c["hkv"]):
            hs = slice(h * gq, (h + 1) * gq)
            slope = s["slopes"][hs].repeat(b - a) if c["alibi"] else None
            o, l = _exact_head(c, s["q"][a:b, hs].reshape(-1, D), s["k"][p, h, :length],
                               _exact_dense(s, p, h, length, c["groups"]), at, pos, slope, seen)
            out[a:b, hs], lse[a:b, hs] = o.view(b - a, gq, D), l.view(b - a, gq)
    whole = torch.logaddexp(lse, s["own_lse"].double())
    mix = torch.exp(lse - whole)[..., None] * out + torch.exp(s["own_lse"].double() - whole)[..., None] * s["own_out"].double()
    return mix, whole
