"""stc_tree_attn with given positions and a window: cached tokens between the windows of far apart nodes are seen by no node of the
sequence, and whatever they hold (NaN and infinities here, in keys and values) reaches no row."""
import math

import pytest
import torch

import paper_2604_21335_b200 as P
import test_gpu_tree_attn as TA
import tree_ref as TR

pytestmark = pytest.mark.gpu


def hide(c, q_pos, window, doc=None, q_doc=None):
    """NaN or an infinity in the keys and values of cached tokens that no node of their sequence sees; how many of them lie between two
    windows."""
    between = 0
    for b, (length, n) in enumerate(zip(c["lens"], c["nodes"])):
        t, p = torch.arange(c["T"]), q_pos[b, :n].long()
        gap = p[:, None] - t[None, :]
        seen = ((gap >= 0) & (gap < window)).any(0)
        if n:
            between += int((~seen & (t >= p.min()) & (t < p.max()) & (t < length)).sum())
        if doc is not None:
            seen &= (doc[b] < 0) | (doc[b] == q_doc[b])
        gone = ~seen & (t < length)
        what = float("nan") if b % 2 == 0 else math.inf
        c["k"][b][:, gone] = what
        for h in range(c["heads"][1]):
            o = c["v_offs"][b, h].tolist()
            for i in gone.nonzero().flatten().tolist():
                c["v_packed"][b, h, o[i]:o[i + 1]] = what
        c["dense"][b][:, gone] = float("nan")
    return between


def positions(r, lens, cap):
    """A few far apart places per sequence, before, in and behind the cache, with the nodes in clusters around them."""
    q_pos = torch.zeros(len(lens), cap, dtype=torch.int32)
    for b, n in enumerate(lens):
        places = [r.randint(-30, n + 30) for _ in range(4)] + [n // 5, n * 4 // 5]
        for i in range(cap):
            q_pos[b, i] = r.choice(places) + r.randint(0, 3)
    return q_pos


@pytest.mark.parametrize("heads,S,nodes", [((4, 2), 8, 9), ((28, 4), 16, 5), ((8, 1), 4, 40), ((2, 2), 8, 128), ((3, 3), 16, 1)])
@pytest.mark.parametrize("window", [1, 25, 64])
def test_tokens_between_the_windows(heads, S, nodes, window):
    lens = [900, 333, 16, 0]
    c = TA.make(nodes + window, heads, S, 900, lens, nodes, [nodes, max(1, nodes - 2), nodes, 1])
    q_pos = positions(TR.rng(nodes + window), lens, nodes)
    assert hide(c, q_pos, window) > 0 or nodes == 1
    TA.check(c, *TA.call(c, score=P.Score(q_pos=q_pos.cuda(), window=window)), q_pos=q_pos, window=window)


@pytest.mark.parametrize("distance,window", [(24, 25), (25, 25), (26, 25), (27, 25), (2, 1), (1, 1)])
def test_windows_that_just_meet_or_just_do_not(distance, window):
    c = TA.make(distance, (8, 4), 8, 300, [300, 290], 2, [2, 2])
    q_pos = torch.tensor([[100, 100 + distance], [255 + distance, 255]], dtype=torch.int32)
    assert hide(c, q_pos, window) == 2 * max(0, distance - window)
    TA.check(c, *TA.call(c, score=P.Score(q_pos=q_pos.cuda(), window=window)), q_pos=q_pos, window=window)


@pytest.mark.parametrize("heads,S,nodes", [((8, 8), 8, 20), ((28, 4), 8, 5), ((32, 8), 4, 33)])
@pytest.mark.parametrize("softcap,docs,listed", [(0.0, False, False), (30.0, False, True), (0.0, True, True)])
def test_many_sequences_with_lists_documents_and_caps(heads, S, nodes, softcap, docs, listed):
    """Rows copied over idle lanes too; listed pages in any order."""
    r, B, T, window = TR.rng(nodes), 192 // heads[1], 700, 50
    lens = [r.choice([1, 130, 500, 700]) for _ in range(B)]
    c = TA.make(nodes + 3, heads, S, T, lens, nodes, [r.randint(0, nodes) for _ in range(B)])
    q_pos = positions(r, lens, nodes)
    doc = (torch.arange(T)[None, :] // 37 % 4 - 1).expand(B, T).contiguous().int() if docs else None
    q_doc = torch.tensor([r.choice([1, 2, 9]) for _ in range(B)], dtype=torch.int32) if docs else None
    assert hide(c, q_pos, window, doc, q_doc) > 0
    ids = n_ids = None
    if listed:
        most = 44
        ids = torch.stack([torch.stack([torch.randperm(most, generator=torch.Generator().manual_seed(b * 8 + h)) for h in range(heads[1])])
                           for b in range(B)]).int()
        n_ids = torch.tensor([[r.randint(30, most) for _ in range(heads[1])] for _ in range(B)], dtype=torch.int32)
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    score = P.Score(softcap=softcap, q_pos=q_pos.cuda(), window=window, tok_doc=dev(doc), q_doc=dev(q_doc))
    TA.check(c, *TA.call(c, ids, n_ids, score=score), ids=ids, n_ids=n_ids, softcap=softcap, window=window, doc=doc, q_doc=q_doc, q_pos=q_pos)
