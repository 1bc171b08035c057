"""Speculative decoding on the routed cache, and the cache's own upkeep: what is timed and compared.

Every case is one call of a serving program.  With ``own`` false the operators are computed in their plain form
(elementary torch operations in 32 bits); with ``own`` true by the library's calls.

  tree     all drafted tokens of a tree attend the cache (listed pages or all) and their own ancestors
  accept   the model's choices are followed through the tree: accepted nodes and the next token
  commit   keys and values of the accepted nodes go from the draft buffers into the cache
  fork     whole cached sequences are copied to other rows of a cache
  compact  the listed pages of every KV head are kept, in a smaller cache
"""
import math
import random

import torch

own = False

DEV = "cuda"
D = 128
PAGE = 16


# ---- cases --------------------------------------------------------------------------------------------------------
def _tree(name, batch, hq, hkv, t, groups, keep, pages, nodes, depth, cap, alibi, window, docs, ragged):
    return dict(name=name, op="tree", batch=batch, hq=hq, hkv=hkv, t=t, groups=groups, keep=keep, pages=pages, nodes=nodes,
                depth=depth, cap=cap, alibi=alibi, window=window, docs=docs, ragged=ragged)


def _accept(name, batch, nodes, depth, vocab, bf16):
    return dict(name=name, op="accept", batch=batch, nodes=nodes, depth=depth, vocab=vocab, bf16=bf16)


def _commit(name, batch, hkv, t, groups, keep, nodes, depth, ragged):
    return dict(name=name, op="commit", batch=batch, hkv=hkv, t=t, groups=groups, keep=keep, nodes=nodes, depth=depth,
                ragged=ragged)


def _fork(name, sources, copies, hkv, t, groups, keep, ragged):
    return dict(name=name, op="fork", sources=sources, copies=copies, hkv=hkv, t=t, groups=groups, keep=keep, ragged=ragged)


def _compact(name, batch, hkv, t, groups, keep, pages, ragged):
    return dict(name=name, op="compact", batch=batch, hkv=hkv, t=t, groups=groups, keep=keep, pages=pages, ragged=ragged)


def listed():
    return [
        # the smallest verification step: one sequence, eight single-query heads, eight drafted tokens, distance slopes
        _tree("tree 1x8 n8", 1, 8, 8, 4096, 8, 4, 64, 8, 3, 0.0, True, 0, 0, False),
        # five tokens copied from the prompt as a chain, 7 query heads per KV head, whole ragged caches, capped and windowed
        _tree("tree chain 8x28/4 n5", 8, 28, 4, 20011, 16, 4, 0, 5, 4, 50.0, False, 16384, 0, True),
        # a batch of long contexts with trees of 16 over the selected pages, cached documents that others do not see
        _tree("tree 16x32/8 n16", 16, 32, 8, 131072, 8, 4, 256, 16, 5, 0.0, False, 0, 3, False),
        # the same batch with trees of 64: 256 query rows per KV head, bound by the products
        _tree("tree 16x32/8 n64", 16, 32, 8, 131072, 8, 4, 256, 64, 7, 0.0, False, 0, 0, False),
        # one sequence, 32000 words in fp32
        _accept("accept 1 n8 32000", 1, 8, 3, 32000, False),
        # a batch of trees of 64 over a vocabulary of 152064
        _accept("accept 16 n64 152064", 16, 64, 7, 152064, True),
        # one sequence's accepted tokens
        _commit("commit 1x8 n8", 1, 8, 4096, 8, 4, 8, 3, False),
        # a large batch in the middle of a decode loop
        _commit("commit 64x8 n64", 64, 8, 2048, 8, 4, 64, 7, True),
        # four answers from one prompt, on 4 KV heads of 16 groups
        _fork("fork 4096 1->4", 1, 4, 4, 4096, 16, 4, False),
        # two long prompts, eight answers each
        _fork("fork 16384 2->16", 2, 16, 8, 16384, 8, 4, True),
        # one short cache shrunk to a quarter
        _compact("compact 1x8 4096", 1, 8, 4096, 8, 4, 64, False),
        # a batch of ragged contexts shrunk to the pages that were selected
        _compact("compact 16x8 32768", 16, 8, 32768, 8, 4, 256, True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree", "tree", "accept", "commit", "fork", "compact"])
    groups = rng.choice([4, 8, 16])
    keep = rng.randint(1, groups)
    hq, hkv = rng.choice([(8, 8), (28, 4), (32, 8), (32, 32), (16, 8), (12, 2)])
    nodes = _log(rng, 1, 128)
    depth = min(nodes - 1, rng.randint(0, 12))
    ragged = rng.random() < 0.5
    if op == "tree":
        most = 16 * 8 * 4096 * 64 * 4                            # no more products than the largest listed call
        t = _log(rng, 17, 131072)
        pages = rng.choice([0, _log(rng, 1, 256)])
        seen = min(t, pages * PAGE or t) + nodes
        batch = max(1, min(_log(rng, 1, 16), most // (hq * nodes * seen), 16 * 131072 * 8 // (t * hkv)))
        nodes = max(1, min(nodes, most // (hq * batch * seen)))
        return dict(op=op, batch=batch, hq=hq, hkv=hkv, t=t, groups=groups, keep=keep, pages=min(pages, (t + PAGE - 1) // PAGE),
                    nodes=nodes, depth=min(depth, nodes - 1), cap=rng.choice([0.0, 0.0, 30.0, 50.0]), alibi=rng.random() < 0.3,
                    window=rng.choice([0, 0, _log(rng, 16, t)]), docs=rng.choice([0, 0, 3]), ragged=ragged)
    if op == "accept":
        vocab = _log(rng, 1000, 152064)
        batch = max(1, min(_log(rng, 1, 64), 16 * 64 * 152064 // (nodes * vocab)))
        return dict(op=op, batch=batch, nodes=nodes, depth=depth, vocab=vocab, bf16=rng.random() < 0.6)
    if op == "commit":
        return dict(op=op, batch=_log(rng, 1, 64), hkv=hkv, t=nodes + _log(rng, 17, 2000), groups=groups, keep=keep,
                    nodes=nodes, depth=depth, ragged=ragged)
    if op == "fork":
        copies = _log(rng, 1, 16)
        return dict(op=op, sources=rng.randint(1, min(4, copies)), copies=copies, hkv=hkv, t=_log(rng, 17, 16384 * 8 // max(8, hkv)),
                    groups=groups, keep=min(keep, groups // 2), ragged=ragged)
    t = _log(rng, 17, 32768)
    return dict(op=op, batch=max(1, min(_log(rng, 1, 16), 16 * 32768 * 8 // (t * hkv))), hkv=hkv, t=t, groups=groups, keep=keep,
                pages=min((t + PAGE - 1) // PAGE, _log(rng, 1, 256)), ragged=ragged)


# ---- inputs -------------------------------------------------------------------------------------------------------
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.bfloat16)


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def _spread(i):
    """The i-th of a sequence that fills [0, 1) evenly in a mixed order."""
    return (i * 0.6180339887498949) % 1.0


def _lengths(n, most, ragged):
    """Lengths of n sequences: `most` for all, or spread over most/2 .. most, the first `most`."""
    return [most - int(_spread(i) * (most - most // 2)) if ragged else most for i in range(n)]


def _accepted(c):
    """Drafted tokens that each sequence's verification accepts behind the root."""
    return [int(_spread(i + 1) * (c["depth"] + 1)) for i in range(c["batch"])]


def _nodes(c):
    """Nodes of each sequence's tree (ragged: some of the leaves are missing, never the longest path)."""
    n, d = c["nodes"], c["depth"]
    return [n - int(_spread(i) * (n - d)) if c.get("ragged") else n for i in range(c["batch"])]


def _make_tree(rng, n, cap, depth):
    """parent [cap] with parents before children, and one path of depth + 1 nodes from the root; the others hang anywhere."""
    up, level = [-1], [0]
    for i in range(1, n):
        p = i - 1 if i <= depth else rng.choice([j for j in range(i) if level[j] < max(depth, 1)])
        up.append(p)
        level.append(level[p] + 1)
    # the same tree in a random order that keeps parents before children
    kids, ready, order = [[] for _ in range(n)], [0] if n else [], []
    for i in range(1, n):
        kids[up[i]].append(i)
    while ready:
        i = ready.pop(rng.randrange(len(ready)))
        order.append(i)
        ready += kids[i]
    at = {old: new for new, old in enumerate(order)}
    parent = [-1] * cap
    for old, new in at.items():
        parent[new] = at[up[old]] if up[old] >= 0 else -1
    return parent, [at[i] for i in range(min(depth, n - 1) + 1)]


def _trees(c, seed):
    rng = random.Random(seed * 7919 + 5)
    made = [_make_tree(rng, n, c["nodes"], c["depth"]) for n in _nodes(c)]
    return [p for p, _ in made], [w for _, w in made]


def _cache(g, B, hkv, t, groups, keep, lens, extra=0):
    """Keys with four loud channels per head, a packed value store: every group kept with probability keep / groups."""
    k = _normal(g, B, hkv, t, D)
    loud = torch.rand(hkv, D, generator=g, device=DEV).argsort(dim=1)[:, :4]
    scale = torch.ones(hkv, D, dtype=torch.bfloat16, device=DEV).scatter_(1, loud, 8.0)
    k *= scale[None, :, None, :]
    kept = torch.rand(B, hkv, t, groups, generator=g, device=DEV) < keep / groups
    length = _i32(lens)
    kept &= (torch.arange(t, device=DEV)[None, :] < length[:, None])[:, None, :, None]
    bits = (kept.to(torch.int32) << torch.arange(groups, device=DEV, dtype=torch.int32)).sum(-1, dtype=torch.int32)
    offs = torch.zeros(B, hkv, t + 1, dtype=torch.int32, device=DEV)
    offs[..., 1:] = kept.sum(-1, dtype=torch.int32).cumsum(-1, dtype=torch.int32)
    # room for what any seed keeps (ten standard deviations), and for what is added later
    cap = min(t * groups, t * keep + int(5 * math.sqrt(t * groups)) + 1) + extra
    return dict(k=k, v_packed=_normal(g, B, hkv, cap, D // groups), v_mask=bits.to(torch.int16), v_offs=offs, cap=cap, len=length,
                lens=lens)


def _meta(s):
    """Least and largest key of each page's valid tokens."""
    k, t = s["k"], s["k"].shape[2]
    pages = (t + PAGE - 1) // PAGE
    valid = torch.arange(pages * PAGE, device=DEV)[None, :] < s["len"][:, None]
    full = torch.nn.functional.pad(k, (0, 0, 0, pages * PAGE - t)).view(*k.shape[:2], pages, PAGE, D)
    ok = valid.view(-1, 1, pages, PAGE, 1)
    s["kmin"] = torch.where(ok, full, math.inf).amin(3)
    s["kmax"] = torch.where(ok, full, -math.inf).amax(3)
    return s


def _empty(rows, hkv, t, groups, cap):
    """A cache without anything in it."""
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(*shape, dtype=dtype, device=DEV)  # noqa: E731
    pages = (t + PAGE - 1) // PAGE
    return dict(k=z(rows, hkv, t, D), kmin=z(rows, hkv, pages, D), kmax=z(rows, hkv, pages, D), v_packed=z(rows, hkv, cap, D // groups),
                v_mask=z(rows, hkv, t, dtype=torch.int16), v_offs=z(rows, hkv, t + 1, dtype=torch.int32), cap=cap)


def _selection(g, s, B, hkv, t, pages):
    """Distinct page ids per problem, ascending, the page of the newest token among them, as stc_quest_select_window leaves them."""
    every = (t + PAGE - 1) // PAGE
    live = (s["len"] + PAGE - 1) // PAGE
    at = torch.arange(every, device=DEV)
    r = torch.rand(B, hkv, every, generator=g, device=DEV)
    r = torch.where(at[None, None] < live[:, None, None], r, 2.0)
    r = torch.where(at[None, None] == (live - 1)[:, None, None], -1.0, r)
    n = live.clamp(max=pages)
    ids = r.argsort(-1)[..., :pages]
    ids = torch.where(torch.arange(pages, device=DEV)[None, None] < n[:, None, None], ids, every).sort(-1).values
    return ids.to(torch.int32).contiguous(), n[:, None].expand(B, hkv).to(torch.int32).contiguous()


def prepare(case, seed):
    g = _generator(seed)
    c = case
    s = dict(case=c)
    if c["op"] == "accept":
        B, n, V = c["batch"], c["nodes"], c["vocab"]
        parent, way = _trees(c, seed)
        logits = torch.randn(B, n, V, generator=g, device=DEV, dtype=torch.bfloat16 if c["bf16"] else torch.float32) * 2
        best = _first_max(logits).tolist()
        tokens = torch.randint(0, V, (B, n), generator=g, device=DEV, dtype=torch.int32).tolist()
        for b, a in enumerate(_accepted(c)):
            for i in range(1, n):                               # a drafted token is only right where it is to be
                if tokens[b][i] == best[b][parent[b][i]]:
                    tokens[b][i] = (tokens[b][i] + 1) % V
            for up, down in zip(way[b][:a], way[b][1:a + 1]):
                tokens[b][down] = best[b][up]
        s |= dict(logits=logits, tokens=_i32(tokens), parent=_i32(parent), path=torch.full((B, n), -1, dtype=torch.int32, device=DEV),
                  n_accepted=torch.zeros(B, dtype=torch.int32, device=DEV), next=torch.zeros(B, dtype=torch.int32, device=DEV))
        return s
    hkv, t, groups = c["hkv"], c["t"], c["groups"]
    if c["op"] == "fork":
        S, n = c["sources"], c["copies"]
        s |= _meta(_cache(g, S, hkv, t, groups, c["keep"], _lengths(S, t, c["ragged"])))
        s["to"] = _empty(n, hkv, t, groups, s["cap"])
        s["src"] = [i * S // n for i in range(n)]
        s["dst"] = torch.randperm(n, generator=g, device=DEV).tolist()
        s |= dict(src_row=_i32(s["src"]), dst_row=_i32(s["dst"]), new_len=torch.zeros(n, dtype=torch.int32, device=DEV),
                  total=torch.zeros(n, hkv, dtype=torch.int64, device=DEV), status=torch.zeros(n, hkv, dtype=torch.int32, device=DEV))
        return s
    B = c["batch"]
    if c["op"] == "compact":
        s |= _meta(_cache(g, B, hkv, t, groups, c["keep"], _lengths(B, t, c["ragged"])))
        s["page_ids"], s["n_pages"] = _selection(g, s, B, hkv, t, c["pages"])
        s["to"] = _empty(B, hkv, c["pages"] * PAGE, groups, c["pages"] * PAGE * groups)
        s |= dict(new_len=torch.zeros(B, dtype=torch.int32, device=DEV), total=torch.zeros(B, hkv, dtype=torch.int64, device=DEV),
                  status=torch.zeros(B, hkv, dtype=torch.int32, device=DEV))
        return s
    n = c["nodes"]
    parent, way = _trees(c, seed)
    s |= dict(parent=_i32(parent), n_nodes=_i32(_nodes(c)), k_new=_normal(g, B, hkv, n, D), v_new=_normal(g, B, hkv, n, D))
    if c["op"] == "commit":
        s |= _meta(_cache(g, B, hkv, t, groups, c["keep"], _lengths(B, t - n, c["ragged"]), extra=n * groups))
        for b, a in enumerate(_accepted(c)):
            way[b] = way[b][:a + 1]
        s["way"] = way
        s |= dict(path=_i32([w + [-1] * (n - len(w)) for w in way]), n_accepted=_i32([len(w) for w in way]),
                  new_len=torch.zeros(B, dtype=torch.int32, device=DEV), total=torch.zeros(B, hkv, dtype=torch.int64, device=DEV),
                  status=torch.zeros(B, hkv, dtype=torch.int32, device=DEV))
        return s
    s |= _cache(g, B, hkv, t, groups, c["keep"], _lengths(B, t, c["ragged"]))
    s["page_ids"], s["n_pages"] = _selection(g, s, B, hkv, t, c["pages"]) if c["pages"] else (None, None)
    hq = c["hq"]
    s |= dict(q=_normal(g, B, n, hq, D), slopes=None, tok_doc=None, q_doc=None,
              out=torch.zeros(B, n, hq, D, dtype=torch.float32, device=DEV), lse=torch.zeros(B, n, hq, dtype=torch.float32, device=DEV),
              status=torch.zeros(B, dtype=torch.int32, device=DEV))
    if c["alibi"]:
        s["slopes"] = torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)], dtype=torch.float32, device=DEV)
    if c["docs"]:                              # documents in a row; the last belongs to the sequence, the first (-1) to all
        cut = torch.arange(t, device=DEV, dtype=torch.int64)[None, :] * (c["docs"] + 1) // s["len"].long()[:, None].clamp(min=1)
        s["tok_doc"] = (cut.to(torch.int32).clamp(max=c["docs"]) - 1).contiguous()
        s["q_doc"] = _i32([c["docs"] - 1] * B)
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------
def _first_max(x):
    """Index of the largest value of each row, the lowest of equal ones."""
    top = x.amax(-1, keepdim=True)
    at = torch.arange(x.shape[-1], device=DEV, dtype=torch.int32)
    return torch.where(x == top, at, x.shape[-1]).amin(-1)


def _reach(parent):
    """[B, n, n]: whether node j is node i or one of its ancestors."""
    n = parent.shape[1]
    r = (parent[:, :, None] == torch.arange(n, device=DEV)) | torch.eye(n, dtype=torch.bool, device=DEV)
    for _ in range(7):                         # paths of up to 128 nodes
        r = (r.float() @ r.float()) > 0
    return r


def _plain_values(s, tokens, groups):
    """f32 [B, Hkv, N, 128]: the values of `tokens` [B, Hkv, N], dropped groups zero."""
    bits = torch.gather(s["v_mask"], 2, tokens).int()
    bit = (bits[..., None] >> torch.arange(groups, device=DEV, dtype=torch.int32)) & 1
    at = torch.gather(s["v_offs"], 2, tokens)[..., None] + bit.cumsum(-1) - bit
    B, H = tokens.shape[:2]
    base = (torch.arange(B * H, device=DEV) * s["cap"]).view(B, H, 1, 1)
    rows = s["v_packed"].view(B * H * s["cap"], -1)[base + at.clamp(max=s["cap"] - 1)].float()
    return torch.where(bit[..., None] == 0, 0.0, rows).flatten(-2)


def _plain_tree(s):
    c = s["case"]
    B, hkv, gq, n, t = c["batch"], c["hkv"], c["hq"] // c["hkv"], c["nodes"], c["t"]
    if c["pages"]:
        tokens = (s["page_ids"].long()[..., None] * PAGE + torch.arange(PAGE, device=DEV)).flatten(2)
        seen = (torch.arange(c["pages"], device=DEV) < s["n_pages"][..., None]).repeat_interleave(PAGE, dim=-1)
    else:
        tokens = torch.arange(t, device=DEV).expand(B, hkv, t)
        seen = torch.ones(B, hkv, t, dtype=torch.bool, device=DEV)
    seen = seen & (tokens < s["len"][:, None, None])
    tokens = torch.where(seen, tokens, 0)
    if c["docs"]:
        doc = torch.gather(s["tok_doc"][:, None, :].expand(B, hkv, t), 2, tokens)
        seen &= (doc < 0) | (doc == s["q_doc"][:, None, None])
    reach = _reach(s["parent"])
    pos = s["len"][:, None] + reach.sum(-1) - 1                   # [B, n]
    away = torch.cat([tokens[:, :, None, :] - pos[:, None, :, None],                         # [B, hkv, n, tokens + n]
                      (pos[:, None, None, :] - pos[:, None, :, None]).expand(B, hkv, n, n)], -1)
    seen = torch.cat([seen[:, :, None, :].expand(-1, -1, n, -1), reach[:, None].expand(B, hkv, n, n)], -1)
    if c["window"]:
        seen = seen & (-away < c["window"])
    k = torch.cat([torch.gather(s["k"], 2, tokens[..., None].expand(-1, -1, -1, D)), s["k_new"]], 2).float()
    v = torch.cat([_plain_values(s, tokens, c["groups"]), s["v_new"].float()], 2)
    q = s["q"].float().view(B, n, hkv, gq, D).permute(0, 2, 1, 3, 4)                         # [B, hkv, n, gq, D]
    x = (q.reshape(B, hkv, n * gq, D) @ k.transpose(-1, -2)).view(B, hkv, n, gq, -1) / math.sqrt(D)
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    if c["alibi"]:
        x = x + s["slopes"].view(1, hkv, 1, gq, 1) * away[:, :, :, None, :].float()
    x = x.masked_fill(~seen[:, :, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)                                # a node sees itself: never empty
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    out = (p.flatten(2, 3) @ v).view(B, hkv, n, gq, D) / total
    lse = (top + torch.log(total))[..., 0]
    live = torch.arange(n, device=DEV)[None, :] < s["n_nodes"][:, None]
    s["out"].copy_(torch.where(live[:, :, None, None], out.permute(0, 2, 1, 3, 4).reshape(B, n, -1, D), s["out"]))
    s["lse"].copy_(torch.where(live[:, :, None], lse.permute(0, 2, 1, 3).reshape(B, n, -1), s["lse"]))
    return s["out"], s["lse"]


def _plain_accept(s):
    c = s["case"]
    B, n = c["batch"], c["nodes"]
    best = _first_max(s["logits"])
    at = torch.arange(n, device=DEV, dtype=torch.int32)
    rows = torch.arange(B, device=DEV)
    node = torch.zeros(B, dtype=torch.int32, device=DEV)
    going = torch.ones(B, dtype=torch.bool, device=DEV)
    s["n_accepted"].zero_()
    for i in range(n):
        s["path"][:, i] = torch.where(going, node, s["path"][:, i])
        s["n_accepted"] += going.int()
        choice = best[rows, node.long()]
        s["next"].copy_(torch.where(going, choice, s["next"]))
        child = torch.where((s["parent"] == node[:, None]) & (s["tokens"] == choice[:, None]), at, n).amin(-1)
        going = going & (child < n)
        node = torch.where(going, child, node).to(torch.int32)
    return s["path"], s["n_accepted"], s["next"]


def _parts(x):
    return x["k"], x["kmin"], x["kmax"], x["v_packed"], x["v_mask"], x["v_offs"]


def _plain_commit(s):
    c = s["case"]
    S, H = c["groups"], c["hkv"]
    heads = torch.arange(H, device=DEV)
    b, i = (torch.arange(c["nodes"], device=DEV)[None, :] < s["n_accepted"][:, None]).nonzero(as_tuple=True)
    node, t = s["path"][b, i].long(), s["len"].long()[b] + i
    s["k"][b, :, t] = s["k_new"][b, :, node]
    first = s["v_offs"][b[:, None], heads, s["len"].long()[b][:, None]].long() + i[:, None] * S          # [rows, H]
    values = s["v_new"][b, :, node].view(-1, H, S, D // S)
    s["v_packed"][b[:, None, None], heads[:, None], first[..., None] + torch.arange(S, device=DEV)] = values
    every = (1 << S) - 1
    s["v_mask"][b, :, t] = every - (1 << 16) if every >= 1 << 15 else every
    s["v_offs"][b[:, None], heads, t[:, None] + 1] = (first + S).int()
    s["new_len"].copy_(s["len"] + s["n_accepted"])
    s["total"].copy_(torch.gather(s["v_offs"], 2, s["new_len"].long()[:, None, None].expand(-1, H, 1))[..., 0])
    page = s["len"].long()[:, None] // PAGE + torch.arange(c["nodes"] // PAGE + 2, device=DEV)
    b, j = (page * PAGE < s["new_len"][:, None]).nonzero(as_tuple=True)
    page = page[b, j]
    tok = page[:, None] * PAGE + torch.arange(PAGE, device=DEV)
    ok = (tok < s["new_len"][b][:, None])[:, None, :, None]
    rows = s["k"][b[:, None, None], heads[:, None], tok.clamp(max=c["t"] - 1)[:, None, :]]
    s["kmin"][b, :, page] = torch.where(ok, rows, math.inf).amin(2)
    s["kmax"][b, :, page] = torch.where(ok, rows, -math.inf).amax(2)
    return _parts(s), s["new_len"], s["total"]


def _plain_fork(s):
    to = s["to"]
    for a, d in zip(s["src"], s["dst"]):
        n = s["lens"][a]
        pages = (n + PAGE - 1) // PAGE
        to["k"][d, :, :n] = s["k"][a, :, :n]
        to["kmin"][d, :, :pages] = s["kmin"][a, :, :pages]
        to["kmax"][d, :, :pages] = s["kmax"][a, :, :pages]
        to["v_mask"][d, :, :n] = s["v_mask"][a, :, :n]
        to["v_offs"][d, :, :n + 1] = s["v_offs"][a, :, :n + 1]
        held = torch.arange(s["cap"], device=DEV)[None, :, None] < s["v_offs"][a, :, n][:, None, None]
        to["v_packed"][d] = torch.where(held, s["v_packed"][a], to["v_packed"][d])
        s["new_len"][d] = n
        s["total"][d] = s["v_offs"][a, :, n]
    return _parts(to), s["new_len"], s["total"]


def _plain_compact(s):
    c, to = s["case"], s["to"]
    H = c["hkv"]
    for b, length in enumerate(s["lens"]):
        n = min(c["pages"], (length + PAGE - 1) // PAGE)
        for h in range(H):
            page = s["page_ids"][b, h, :n].long()
            tok = (page[:, None] * PAGE + torch.arange(PAGE, device=DEV)).flatten()
            kept = n * PAGE - (-length) % PAGE                    # the last page is always listed
            tok = tok[:kept]
            to["k"][b, h, :kept] = s["k"][b, h, tok]
            to["kmin"][b, h, :n] = s["kmin"][b, h, page]
            to["kmax"][b, h, :n] = s["kmax"][b, h, page]
            to["v_mask"][b, h, :kept] = s["v_mask"][b, h, tok]
            size = s["v_offs"][b, h, tok + 1] - s["v_offs"][b, h, tok]
            to["v_offs"][b, h, 0] = 0
            to["v_offs"][b, h, 1:kept + 1] = size.cumsum(0)
            listed_page = torch.zeros((c["t"] + PAGE - 1) // PAGE, dtype=torch.bool, device=DEV)
            listed_page[page] = True
            owner = torch.searchsorted(s["v_offs"][b, h, 1:length + 1], torch.arange(s["cap"], device=DEV, dtype=torch.int32), right=True)
            use = listed_page[owner.clamp(max=length - 1) // PAGE] & (owner < length)
            rows = s["v_packed"][b, h][use]
            to["v_packed"][b, h, :rows.shape[0]] = rows
            s["total"][b, h] = rows.shape[0]
        s["new_len"][b] = kept
    return _parts(to), s["new_len"], s["total"]


# ---- one pass -----------------------------------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if own:
        return {"tree": _own_tree, "accept": _own_accept, "commit": _own_commit, "fork": _own_fork, "compact": _own_compact}[op](state)
    return {"tree": _plain_tree, "accept": _plain_accept, "commit": _plain_commit, "fork": _plain_fork,
            "compact": _plain_compact}[op](state)


def _own_cache(P, x):
    return P.Cache(k=x["k"], kmin=x.get("kmin"), kmax=x.get("kmax"), v_packed=x["v_packed"], v_mask=x["v_mask"], v_offs=x["v_offs"],
                   cap_groups=x["cap"])


def _own_shape(P, x, c, length=None):
    B, H, t, _ = x["k"].shape
    return P.Shape(B, c.get("hq", H), H, c["groups"], t, length)


def _own_tree(s):
    import paper_2604_21335_b200 as P
    c = s["case"]
    shape = _own_shape(P, s, c, s["len"])
    tree = P.Tree(s["k_new"], s["v_new"], parent=s["parent"], n_nodes=s["n_nodes"])
    if "ws" not in s:                          # the workspace that a serving program allocates once
        s["ws"] = P.binding.new_workspace(shape, P.binding.OP_TREE_ATTN, c["nodes"])
    score = P.Score(softcap=c["cap"], slopes=s["slopes"], window=c["window"], tok_doc=s["tok_doc"], q_doc=s["q_doc"])
    P.tree_attn(shape, _own_cache(P, s), tree, s["q"], s["page_ids"], s["n_pages"], 1 / math.sqrt(D), s["out"], s["status"],
                s["ws"], lse=s["lse"], score=score)
    return s["out"], s["lse"]


def _own_accept(s):
    import paper_2604_21335_b200 as P
    P.tree_accept(s["logits"], s["tokens"], s["path"], s["n_accepted"], s["next"], parent=s["parent"])
    return s["path"], s["n_accepted"], s["next"]


def _own_commit(s):
    import paper_2604_21335_b200 as P
    shape = _own_shape(P, s, s["case"], s["len"])
    tree = P.Tree(s["k_new"], s["v_new"], parent=s["parent"], n_nodes=s["n_nodes"])
    P.tree_commit(shape, _own_cache(P, s), tree, s["path"], s["n_accepted"], s["new_len"], s["total"], s["status"])
    return _parts(s), s["new_len"], s["total"]


def _own_fork(s):
    import paper_2604_21335_b200 as P
    c = s["case"]
    P.cache_fork(_own_shape(P, s, c, s["len"]), _own_cache(P, s), _own_shape(P, s["to"], c), _own_cache(P, s["to"]), s["src_row"],
                 s["dst_row"], s["new_len"], s["total"], s["status"])
    return _parts(s["to"]), s["new_len"], s["total"]


def _own_compact(s):
    import paper_2604_21335_b200 as P
    c = s["case"]
    P.cache_compact(_own_shape(P, s, c, s["len"]), _own_cache(P, s), s["page_ids"], s["n_pages"], s["new_len"], s["total"],
                    s["status"], dst_shape=_own_shape(P, s["to"], c), dst=_own_cache(P, s["to"]))
    return _parts(s["to"]), s["new_len"], s["total"]


# ---- what a pass cannot do without --------------------------------------------------------------------------------
def work(case):
    c = case
    if c["op"] == "accept":                    # the rows of the accepted nodes
        rows = sum(a + 1 for a in _accepted(c))
        return dict(bytes=rows * c["vocab"] * (2.0 if c["bf16"] else 4.0) + c["batch"] * c["nodes"] * 12.0, flops=0.0)
    value = 256.0 * c["keep"] / c["groups"]
    per_token = 256.0 + value + 2.0            # a cached token of a KV head: key, value groups, mask
    if c["op"] == "commit":
        rows = sum(a + 1 for a in _accepted(c)) * c["hkv"]
        return dict(bytes=rows * (2 * 512.0 + 6.0) + c["batch"] * c["hkv"] * 2 * 512.0, flops=0.0)
    if c["op"] == "fork":
        lens = _lengths(c["sources"], c["t"], c["ragged"])
        copied = sum(lens[i * c["sources"] // c["copies"]] for i in range(c["copies"]))
        return dict(bytes=(sum(lens) + copied) * c["hkv"] * (per_token + 4.0 + 32.0), flops=0.0)
    lens = _lengths(c["batch"], c["t"], c["ragged"])
    if c["op"] == "compact":
        kept = sum(min(c["pages"] * PAGE, n) for n in lens)
        return dict(bytes=2 * kept * c["hkv"] * (per_token + 4.0 + 32.0), flops=0.0)
    n, flops, gq = 0.0, 0.0, c["hq"] // c["hkv"]
    for length, nodes in zip(lens, _nodes(c)):
        tokens = min(c["pages"] * PAGE or length, length)
        if c["window"]:
            tokens *= min(1.0, c["window"] / length)
        if c["docs"]:
            tokens *= 2.0 / (c["docs"] + 1)
        n += tokens * c["hkv"]
        flops += 4.0 * D * gq * c["hkv"] * nodes * (tokens + c["depth"])
    rows = sum(_nodes(c))
    return dict(bytes=n * per_token + rows * (c["hkv"] * 512.0 + c["hq"] * (256.0 + 516.0)), flops=flops)


# ---- the definition in 64 bits ------------------------------------------------------------------------------------
def exact(case, seed):
    c = case
    if c["op"] != "tree":                      # the others choose and move values, they compute none
        return None
    s = prepare(case, seed)
    gq, n = c["hq"] // c["hkv"], c["nodes"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    for b, (length, nodes) in enumerate(zip(s["lens"], s["n_nodes"].tolist())):
        line = []                              # each node's ancestors and itself
        for i, p in enumerate(s["parent"][b, :nodes].tolist()):
            line.append((line[p] if p >= 0 else []) + [i])
        kin = torch.zeros(nodes, nodes, dtype=torch.bool, device=DEV)
        for i, who in enumerate(line):
            kin[i, who] = True
        pos = torch.tensor([length + len(who) - 1 for who in line], device=DEV)
        for h in range(c["hkv"]):
            if c["pages"]:
                ids = s["page_ids"][b, h, :int(s["n_pages"][b, h])].long()
                tok = (ids[:, None] * PAGE + torch.arange(PAGE, device=DEV)).flatten()
                tok = tok[tok < length]
            else:
                tok = torch.arange(length, device=DEV)
            if c["docs"]:
                d = s["tok_doc"][b, tok]
                tok = tok[(d < 0) | (d == s["q_doc"][b])]
            word = s["v_mask"][b, h, tok].long() & 0xFFFF
            bit = ((word[:, None] >> torch.arange(c["groups"], device=DEV)) & 1).bool()
            place = s["v_offs"][b, h, tok].long()[:, None] + torch.cumsum(bit.long(), 1) - 1
            dense = torch.zeros(tok.numel(), c["groups"], D // c["groups"], dtype=torch.float64, device=DEV)
            dense[bit] = s["v_packed"][b, h][place[bit]].double()
            keys = torch.cat([s["k"][b, h, tok], s["k_new"][b, h, :nodes]]).double()
            values = torch.cat([dense.view(-1, D), s["v_new"][b, h, :nodes].double()])
            at = torch.cat([tok, pos])
            see = torch.cat([torch.ones(nodes, tok.numel(), dtype=torch.bool, device=DEV), kin], 1)
            gap = at[None, :] - pos[:, None]
            if c["window"]:
                see &= -gap < c["window"]
            for j in range(gq):
                head = h * gq + j
                x = s["q"][b, :nodes, head].double() @ keys.T / math.sqrt(D)
                if c["cap"]:
                    x = c["cap"] * torch.tanh(x / c["cap"])
                if c["alibi"]:
                    x = x + s["slopes"][head].double() * gap.double()
                x[~see] = -math.inf
                level = torch.logsumexp(x, dim=1)
                out[b, :nodes, head] = torch.exp(x - level[:, None]) @ values
                lse[b, :nodes, head] = level
    return out, lse
