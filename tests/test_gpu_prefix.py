"""Shared-prefix attention against the 64-bit plain form: tile edges, head layouts, groups, joining, options, refusals."""
import math

import pytest
import torch

import operators_ref as R
import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)


def run_case(seed, lens, T, starts, n_rows, Hq, Hkv, S=8, keep=4, softcap=0.0, alibi=False, window=0, docs=None, q_pos=None,
             own=True, poison_keys=False, scale=SCALE, stream=None):
    G = len(lens)
    g = torch.Generator().manual_seed(seed + 1)
    c = R.make_cache(seed, G, Hkv, T, S, keep, lens)
    q = torch.randn(n_rows, Hq, 128, generator=g).to(torch.bfloat16)
    gq = Hq // Hkv
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)]) if alibi else None
    row_len = torch.zeros(n_rows, dtype=torch.int64)
    for i in range(G):
        row_len[starts[i]:starts[i + 1]] = lens[i]
    pos = row_len + torch.randint(0, 9, (n_rows,), generator=g) if q_pos is None else torch.tensor(q_pos)
    tok_doc = q_doc = None
    if docs is not None:
        tok_doc = torch.randint(-1, docs, (G, T), generator=g, dtype=torch.int32)
        q_doc = torch.randint(0, docs + 1, (n_rows,), generator=g, dtype=torch.int32)
    if poison_keys:                              # keys that no row of the prefix sees may hold anything
        at = torch.arange(T)
        for i in range(G):
            p = pos[starts[i]:starts[i + 1], None]
            seen = (at <= p) & ((p - at < window) if window else True)
            if docs is not None:
                seen &= (tok_doc[i] < 0) | (tok_doc[i] == q_doc[starts[i]:starts[i + 1], None])
            c["k"][i, :, ~seen.any(0)] = float("nan")
    own_out = torch.randn(n_rows, Hq, 128, generator=g) if own else None
    own_lse = torch.randn(n_rows, Hq, generator=g) + 4 if own else None
    if own:
        own_lse[n_rows // 2, 0] = -math.inf      # a sequence without own tokens: its out is not to be used
        own_out[n_rows // 2, 0] = float("nan")
    cu = lambda t: None if t is None else t.cuda()  # noqa: E731
    dev = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor) and k != "dense"}
    shape = P.Shape(G, Hq, Hkv, S, T, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    cache = P.Cache(k=dev["k"], v_packed=dev["v_packed"], v_mask=dev["v_mask"], v_offs=dev["v_offs"], cap_groups=c["cap"])
    d_own, d_lse = cu(own_out), cu(own_lse)
    out = torch.full((n_rows, Hq, 128), 7.0, device="cuda")
    lse = torch.full((n_rows, Hq), 7.0, device="cuda")
    ws = Bd.new_workspace(shape, Bd.OP_PREFIX_ATTN, n_rows)
    ws.fill_(0xEF)
    optioned = softcap or alibi or window or docs is not None or q_pos is not None
    score = P.Score(softcap, cu(slopes), pos.to(torch.int32).cuda(), window, cu(tok_doc), cu(q_doc)) if optioned else None
    args = (shape, cache, q.cuda(), torch.tensor(starts, dtype=torch.int32, device="cuda"), scale, out, ws)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        P.prefix_attn(*args, lse=lse, score=score, own_out=d_own, own_lse=d_lse)
    torch.cuda.synchronize()
    assert int(ws[:4].view(torch.int32)[0]) == 0
    got_o, got_l = out.double().cpu(), lse.double().cpu()
    inside = torch.zeros(n_rows, dtype=torch.bool)
    inside[starts[0]:starts[-1]] = True
    assert (got_o[~inside] == 7).all() and (got_l[~inside] == 7).all()
    for i, n in enumerate(lens):
        a, b = starts[i], starts[i + 1]
        if a == b:
            continue
        at = torch.arange(n)
        for h in range(Hkv):
            hs = slice(h * gq, (h + 1) * gq)
            rows = (b - a) * gq
            rep = lambda t: t[a:b].repeat_interleave(gq)  # noqa: E731
            p = rep(pos) if optioned else torch.full((rows,), n)
            o, l, to, tl = R.scored_rows(q[a:b, hs].reshape(rows, 128), c["k"][i, h, :n], c["dense"][i, h, :n], at, p, scale,
                                         softcap, None if slopes is None else slopes[hs].repeat(b - a), window,
                                         None if docs is None else tok_doc[i, :n], None if docs is None else rep(q_doc),
                                         n_seq=n + 64)
            if own:
                oo, ol = own_out[a:b, hs].reshape(rows, 128).double(), own_lse[a:b, hs].reshape(rows).double()
                whole = torch.logaddexp(l, ol)
                dead = whole == -math.inf
                safe = torch.where(dead, torch.zeros_like(whole), whole)
                wa, wb = torch.exp(l - safe), torch.exp(ol - safe)
                oo = torch.where((wb == 0)[:, None], torch.zeros_like(oo), oo)
                fin = lambda t: torch.where(t.isinf(), torch.zeros_like(t), t.abs())  # noqa: E731
                dw = tl * wa * wb + 8 * R.EPS32 * (1 + fin(l) + fin(ol))     # of either weight
                to = wa[:, None] * to + dw[:, None] * (o.abs() + oo.abs()) + 4 * R.EPS32 * (wa[:, None] * o.abs() + wb[:, None] * oo.abs()) + 1e-30
                tl = torch.where(l == -math.inf, torch.zeros_like(tl), tl * wa) + 8 * R.EPS32 * (1 + fin(l) + fin(ol))
                o, l = wa[:, None] * o + wb[:, None] * oo, whole
            R.assert_rows(out[a:b, hs].reshape(rows, 128), lse[a:b, hs].reshape(rows), o, l, to, tl)
    return out, lse


@pytest.mark.parametrize("T", [1, 15, 128, 129, 257, 640])
@pytest.mark.parametrize("own", [False, True])
def test_token_tile_edges(T, own):
    run_case(T, [T], T, [0, 3], 3, 8, 2, own=own)


@pytest.mark.parametrize("heads", [(2, 2), (4, 2), (6, 2), (4, 1), (10, 2), (6, 1), (14, 2), (8, 1)])
@pytest.mark.parametrize("seqs", [1, 19, 70])
def test_row_tiles_of_every_head_layout(heads, seqs):
    """One row, a partial tile, more than one tile; with seven heads a tile holds 126 rows."""
    run_case(seqs, [300], 300, [0, seqs], seqs, *heads, own=seqs == 19)


@pytest.mark.parametrize("rows", [16, 17, 32, 33, 64, 65, 128])
@pytest.mark.parametrize("options", [dict(), dict(softcap=30.0), dict(alibi=True), dict(softcap=30.0, alibi=True, window=700, docs=3)],
                         ids=lambda o: "+".join(o) or "plain")
def test_copies_of_few_rows(rows, options):
    """The row counts at which a tile holds its rows four times, twice, once, and the next tile begins; several CTAs and one."""
    run_case(rows, [2000], 2000, [0, rows], rows, 2, 1, **options)
    run_case(rows, [130, 60], 130, [0, rows, 2 * rows - 1], 2 * rows - 1, 48, 48, keep=2, **options)


def test_accumulators_that_are_emptied():
    """More tiles per CTA than an accumulator takes, and a maximum that moves afterwards."""
    run_case(23, [64 * 36] * 15, 64 * 36, [9 * i for i in range(16)], 135, 48, 48, S=4, keep=1)
    run_case(24, [64 * 40] * 12, 64 * 40, [9 * i for i in range(13)], 108, 48, 48, alibi=True, q_pos=[100 + 290 * (i % 9) for i in range(108)])


def test_more_rows_than_a_unit_and_one_more():
    run_case(3, [200], 200, [0, 257], 257, 1, 1)
    run_case(4, [200], 200, [0, 129], 129, 2, 1, S=4, keep=2)


@pytest.mark.parametrize("S,keep", [(4, 1), (4, 4), (8, 0), (8, 8), (16, 5), (16, 16)])
def test_value_groups(S, keep):
    run_case(S + keep, [500], 517, [0, 9], 9, 8, 4, S=S, keep=keep)


def test_prefixes_of_all_kinds_side_by_side():
    """Empty prefixes, prefixes nobody continues, rows outside, tiny next to long, more units than CTAs."""
    run_case(7, [300, 0, 17, 1, 700, 128], 700, [2, 5, 9, 9, 40, 41, 60], 66, 8, 4)
    n = 40
    run_case(8, [(37 * i) % 150 for i in range(n)], 150, [i * 2 for i in range(n + 1)], 2 * n, 21, 7)


def test_long_prefix_on_all_ctas_one_unit():
    run_case(9, [30000], 30000, [0, 2], 2, 4, 1, S=16, keep=4)


@pytest.mark.parametrize("options", [dict(softcap=30.0), dict(softcap=0.2), dict(alibi=True), dict(window=150), dict(docs=3),
                                     dict(softcap=50.0, alibi=True, window=200, docs=2)], ids=lambda o: "+".join(o))
@pytest.mark.parametrize("seqs", [5, 50])
def test_options(options, seqs):
    run_case(12, [390, 140], 390, [0, seqs, 2 * seqs - 3], 2 * seqs - 3, 12, 4, **options)


def test_positions_inside_the_prefix_rows_that_see_nothing_and_poisoned_keys():
    pos = [-1, 0, 100, 127, 128, 5000, 400, 401, 260]
    run_case(13, [400, 300], 400, [0, 6, 9], 9, 6, 2, window=90, q_pos=pos, poison_keys=True)
    run_case(14, [256], 256, [0, 9], 9, 6, 2, docs=2, q_pos=[300] * 9, poison_keys=True, own=False)
    run_case(15, [256], 256, [0, 2], 2, 2, 2, alibi=True, q_pos=[1 << 20, 1 << 23], own=False)


@pytest.mark.parametrize("scale", [0.0, -0.1, 1.0])
def test_scales(scale):
    run_case(16, [200], 200, [0, 4], 4, 4, 2, scale=scale)


def test_another_stream():
    a = run_case(17, [333], 333, [0, 20], 20, 8, 2)
    b = run_case(17, [333], 333, [0, 20], 20, 8, 2, stream=torch.cuda.Stream())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_repeatable_and_captured():
    lens, T, n = [900, 77], 900, 30
    c = {k: v.cuda() for k, v in R.make_cache(1, 2, 4, T, 8, 4, lens).items() if isinstance(v, torch.Tensor) and k != "dense"}
    length = torch.tensor(lens, dtype=torch.int32, device="cuda")
    shape = P.Shape(2, 16, 4, 8, T, length)
    cache = P.Cache(k=c["k"], v_packed=c["v_packed"], v_mask=c["v_mask"], v_offs=c["v_offs"], cap_groups=c["v_packed"].shape[2])
    q = torch.randn(n, 16, 128, device="cuda").to(torch.bfloat16)
    start = torch.tensor([0, 20, 30], dtype=torch.int32, device="cuda")
    ws = Bd.new_workspace(shape, Bd.OP_PREFIX_ATTN, n)
    out, lse = torch.zeros(n, 16, 128, device="cuda"), torch.zeros(n, 16, device="cuda")
    P.prefix_attn(shape, cache, q, start, SCALE, out, ws, lse=lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.prefix_attn(shape, cache, q, start, SCALE, out, ws, lse=lse)
    for a, b in ((20, lens), (11, [800, 40]), (30, [900, 0]), (0, [3, 77])):     # other splits and lengths, same graph
        start.copy_(torch.tensor([0, a, 30], dtype=torch.int32))
        length.copy_(torch.tensor(b, dtype=torch.int32))
        ref_o, ref_l = torch.full_like(out, 3.0), torch.full_like(lse, 3.0)
        P.prefix_attn(shape, cache, q, start, SCALE, ref_o, ws, lse=ref_l)
        out.fill_(5.0)
        graph.replay()
        assert torch.equal(out, ref_o) and torch.equal(lse, ref_l)


@pytest.mark.parametrize("starts", [[0, 5, 3], [-1, 2, 4], [0, 2, 11]])
def test_row_starts_that_do_not_fit_write_nothing(starts):
    c = {k: v.cuda() for k, v in R.make_cache(1, 2, 2, 64, 8, 4, [64, 64]).items() if isinstance(v, torch.Tensor) and k != "dense"}
    shape = P.Shape(2, 4, 2, 8, 64, None)
    cache = P.Cache(k=c["k"], v_packed=c["v_packed"], v_mask=c["v_mask"], v_offs=c["v_offs"], cap_groups=c["v_packed"].shape[2])
    q = torch.zeros(10, 4, 128, device="cuda", dtype=torch.bfloat16)
    out = torch.full((10, 4, 128), 7.0, device="cuda")
    ws = Bd.new_workspace(shape, Bd.OP_PREFIX_ATTN, 10)
    P.prefix_attn(shape, cache, q, torch.tensor(starts, dtype=torch.int32, device="cuda"), SCALE, out, ws)
    torch.cuda.synchronize()
    assert int(ws[:4].view(torch.int32)[0]) == 1 and (out == 7).all()


def test_cache_without_tokens_hands_on_the_own_results():
    shape = P.Shape(1, 4, 2, 8, 0, None)
    own, own_l = torch.randn(3, 4, 128, device="cuda"), torch.randn(3, 4, device="cuda")
    out, lse = torch.zeros_like(own), torch.zeros_like(own_l)
    ws = Bd.new_workspace(shape, Bd.OP_PREFIX_ATTN, 3)
    q = torch.zeros(3, 4, 128, device="cuda", dtype=torch.bfloat16)
    start = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    P.prefix_attn(shape, P.Cache(), q, start, SCALE, out, ws, lse=lse, own_out=own, own_lse=own_l)
    assert ((out - own).abs() <= 2.0 ** -23 * own.abs()).all() and ((lse - own_l).abs() <= 2.0 ** -21 * (1 + own_l.abs())).all()
    P.prefix_attn(shape, P.Cache(), q, start, SCALE, out, ws, lse=lse)
    assert (out == 0).all() and (lse == -math.inf).all()
