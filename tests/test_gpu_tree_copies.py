"""stc_tree_attn where the rows of a tree are copied over idle tensor-memory lanes and a unit's tiles are split over several CTAs: the copies'
partial results of every CTA are added up by the second kernel."""
import pytest
import torch

import paper_2604_21335_b200 as P
import test_gpu_tree_attn as TA
import tree_ref as TR

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,S,nodes,B", [((8, 8), 8, 32, 3), ((32, 8), 4, 8, 3), ((32, 8), 8, 16, 2), ((28, 4), 16, 5, 3)])
@pytest.mark.parametrize("softcap,alibi,window,docs", [(0.0, False, 0, False), (0.0, False, 9000, True), (20.0, True, 0, False)])
def test_copies_of_rows_in_split_units(heads, S, nodes, B, softcap, alibi, window, docs):
    """Fourteen tiles of 128 tokens per CTA of 148, where up to 25 parts of a row want 4 + 25 / 3 at most."""
    Hkv, r = heads[1], TR.rng(nodes)
    T = 128 * (14 * 148 // (B * Hkv)) + 5
    c = TA.make(nodes + B, heads, S, T, [T - r.randint(0, 300) for _ in range(B)], nodes, [nodes] + [max(1, nodes - 1)] * (B - 1))
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / heads[0]) for h in range(heads[0])]) if alibi else None
    doc = (torch.arange(T)[None, :] // 997 % 4 - 1).expand(B, T).contiguous().int() if docs else None
    q_doc = torch.tensor([r.choice([1, 2]) for _ in range(B)], dtype=torch.int32) if docs else None
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    score = P.Score(softcap=softcap, slopes=dev(slopes), window=window, tok_doc=dev(doc), q_doc=dev(q_doc))
    TA.check(c, *TA.call(c, score=score), softcap=softcap, slopes=slopes, window=window, doc=doc, q_doc=q_doc)
