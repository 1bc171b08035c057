"""Scored decode attention against the 64-bit plain form: cap, slopes, window, documents, empty rows, poisoned memory."""
import math

import pytest
import torch

import operators_ref as R
import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)


def slopes_for(hq):
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)])


def run_case(seed, B, Hq, Hkv, T, S, keep, lens, pages=None, softcap=0.0, alibi=False, window=0, docs=None, q_pos=None,
             poison_unseen=False, score_none=False):
    g = torch.Generator().manual_seed(seed + 1)
    c = R.make_cache(seed, B, Hkv, T, S, keep, lens)
    q = torch.randn(B, Hq, 128, generator=g).to(torch.bfloat16)
    gq, np_all = Hq // Hkv, (T + 15) // 16
    slopes = slopes_for(Hq) if alibi else None
    pos = torch.tensor([n - 1 for n in lens] if q_pos is None else q_pos)
    tok_doc = q_doc = None
    if docs is not None:
        tok_doc = torch.randint(-1, docs, (B, T), generator=g, dtype=torch.int32)
        q_doc = torch.randint(0, docs + 1, (B,), generator=g, dtype=torch.int32)
    ids = n_pages = None
    if pages is not None:
        ids = torch.stack([torch.stack([torch.randperm(np_all, generator=g)[:pages].sort().values for _ in range(Hkv)])
                           for _ in range(B)]).to(torch.int32)
        n_pages = torch.randint(max(0, pages - 3), pages + 1, (B, Hkv), generator=g, dtype=torch.int32)
    if poison_unseen:                            # whatever stands in tokens that no query may see must not matter
        at = torch.arange(T)
        for b in range(B):
            unseen = at > int(pos[b])
            if window:
                unseen |= int(pos[b]) - at >= window
            if docs is not None:
                unseen |= ~((tok_doc[b] < 0) | (tok_doc[b] == q_doc[b]))
            c["k"][b, :, unseen] = float("nan")
            for h in range(Hkv):
                for t in torch.nonzero(unseen[:lens[b]])[:, 0].tolist():
                    lo, hi = int(c["v_offs"][b, h, t]), int(c["v_offs"][b, h, t + 1])
                    c["v_packed"][b, h, lo:hi] = float("inf")
    dev = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor) and k != "dense"}
    shape = P.Shape(B, Hq, Hkv, S, T, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    cache = P.Cache(k=dev["k"], v_packed=dev["v_packed"], v_mask=dev["v_mask"], v_offs=dev["v_offs"], cap_groups=c["cap"])
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    score = None if score_none else P.Score(softcap, cu(slopes), None if q_pos is None else pos.to(torch.int32).cuda(), window,
                                            cu(tok_doc), cu(q_doc))
    out = torch.full((B, Hq, 128), float("nan"), device="cuda")
    lse = torch.full((B, Hq), float("nan"), device="cuda")
    ws = Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, pages if pages is not None else shape.n_pages)
    ws.fill_(0xEF)
    P.decode_attn(shape, cache, q.cuda(), cu(ids), cu(n_pages), SCALE, out, ws, lse=lse, score=score)
    torch.cuda.synchronize()
    assert int(ws[:4].view(torch.int32)[0]) == 0
    for b in range(B):
        for h in range(Hkv):
            at = torch.arange(lens[b])
            if ids is not None:
                at = (ids[b, h, :int(n_pages[b, h])].long()[:, None] * 16 + torch.arange(16)).flatten()
                at = at[at < lens[b]]
            hs = slice(h * gq, (h + 1) * gq)
            ref = R.scored_rows(q[b, hs], c["k"][b, h][at], c["dense"][b, h][at], at, pos[b].expand(gq), SCALE, softcap,
                                None if slopes is None else slopes[hs], window,
                                None if tok_doc is None else tok_doc[b][at],
                                None if q_doc is None else q_doc[b].expand(gq))
            R.assert_rows(out[b, hs], lse[b, hs], *ref)
    return out, lse


@pytest.mark.parametrize("heads", [(8, 8), (28, 4), (6, 2), (8, 1), (2, 1)])
@pytest.mark.parametrize("options", [dict(softcap=30.0), dict(softcap=0.3), dict(alibi=True), dict(window=40), dict(docs=3),
                                     dict(softcap=50.0, alibi=True, window=133, docs=2)], ids=lambda o: "+".join(o))
def test_options_on_every_head_layout(heads, options):
    run_case(11, 3, *heads, 333, 8, 4, [333, 1, 150], **options)


@pytest.mark.parametrize("S", [4, 8, 16])
@pytest.mark.parametrize("T,pages", [(1, None), (17, 2), (1000, 30), (2500, None)])
def test_lengths_and_page_lists(S, T, pages):
    run_case(T, 2, 14, 2, T, S, S // 2, [T, (T + 1) // 2], pages=pages, softcap=20.0, alibi=True, window=max(1, T // 2))


def test_many_problems_and_a_full_wave():
    run_case(5, 16, 32, 8, 700, 8, 3, [700 - 31 * i for i in range(16)], softcap=50.0, window=300)
    run_case(6, 24, 20, 20, 260, 16, 5, [260] * 24, alibi=True, docs=2)


@pytest.mark.parametrize("heads", [(1, 1), (8, 1), (6, 2)])
def test_few_problems_with_long_lists_take_several_clusters(heads):
    run_case(7, 1, *heads, 16 * 1300 + 5, 8, 4, [16 * 1300 + 5], alibi=True, softcap=40.0)
    run_case(8, 2, *heads, 16 * 600, 16, 4, [16 * 600, 40], window=3000, docs=2)


@pytest.mark.parametrize("heads", [(4, 4), (12, 2)])
def test_positions_empty_rows_and_poison(heads):
    """Queries that see nothing, one token, the middle of the cache; NaN and infinities in everything unseen."""
    run_case(21, 6, *heads, 200, 8, 4, [200, 200, 200, 200, 0, 77], q_pos=[-1, 0, 100, 5000, 3, 76], window=60, alibi=True,
             poison_unseen=True)
    run_case(22, 4, *heads, 180, 8, 8, [180, 16, 17, 100], docs=2, softcap=10.0, poison_unseen=True)


def test_bias_of_a_query_far_behind_its_cache():
    """Positions a million tokens on: the common offset must cancel in the weights and appear in lse."""
    run_case(31, 2, 8, 2, 96, 8, 4, [96, 50], q_pos=[1 << 20, 1 << 23], alibi=True)


def test_no_options_are_the_plain_call_bit_for_bit():
    a = run_case(41, 2, 14, 2, 400, 8, 4, [400, 390], pages=20)
    b = run_case(41, 2, 14, 2, 400, 8, 4, [400, 390], pages=20, score_none=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_refusals():
    z = torch.zeros(1, dtype=torch.int32, device="cuda")
    shape = P.Shape(1, 8, 8, 8, 64, z + 64)
    q = torch.zeros(1, 8, 128, dtype=torch.bfloat16, device="cuda")
    c = {k: v.cuda() for k, v in R.make_cache(0, 1, 8, 64, 8, 4, [64]).items() if isinstance(v, torch.Tensor)}
    cache = P.Cache(k=c["k"], v_packed=c["v_packed"], v_mask=c["v_mask"], v_offs=c["v_offs"], cap_groups=c["v_packed"].shape[2])
    out = torch.zeros(1, 8, 128, device="cuda")
    ws = Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, 4)

    def call(score):
        P.decode_attn(shape, cache, q, None, None, SCALE, out, ws, score=score)

    for bad in (P.Score(softcap=-1.0), P.Score(softcap=float("nan")), P.Score(softcap=float("inf")), P.Score(window=-1),
                P.Score(tok_doc=torch.zeros(1, 64, dtype=torch.int32, device="cuda")), P.Score(q_doc=z)):
        with pytest.raises(P.StcError) as e:
            call(bad)
        assert e.value.code == 1
    for bad in (P.Score(slopes=torch.zeros(4, device="cuda")), P.Score(slopes=torch.zeros(8)),
                P.Score(q_pos=torch.zeros(1, dtype=torch.int64, device="cuda")), P.Score(q_pos=torch.zeros(2, dtype=torch.int32, device="cuda")),
                P.Score(tok_doc=torch.zeros(1, 63, dtype=torch.int32, device="cuda"), q_doc=z)):
        with pytest.raises(ValueError):
            call(bad)
