"""stc_tree_attn against the 64-bit plain form: head layouts, trees, lengths, lists, options, and what may stand where nobody looks."""
import math

import pytest
import torch

import operators_ref as R
import paper_2604_21335_b200 as P
import tree_ref as TR
from paper_2604_21335_b200 import binding as Bd

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)
NAN = float("nan")


def make(seed, heads, S, T, lens, cap_nodes, nodes, chain=False, keep=None):
    Hq, Hkv = heads
    B, r = len(lens), TR.rng(seed)
    c = R.make_cache(seed, B, Hkv, T, S, keep or max(1, S // 2), lens)
    g = torch.Generator().manual_seed(seed + 1)
    c["q"] = torch.randn(B, cap_nodes, Hq, 128, generator=g).to(torch.bfloat16)
    c["k_new"], c["v_new"] = (torch.randn(B, Hkv, cap_nodes, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    for b, n in enumerate(nodes):                                       # nobody looks behind the last node
        for x in (c["k_new"][b, :, n:], c["v_new"][b, :, n:], c["q"][b, n:]):
            x.fill_(NAN)
    c["parent"] = [[i - 1 for i in range(cap_nodes)] if chain else TR.random_tree(r, n, cap_nodes) for n in nodes]
    c.update(heads=heads, S=S, T=T, nodes=list(nodes), chain=chain)
    return c


def call(c, ids=None, n_ids=None, score=None, scale=SCALE, buffers=None):
    (Hq, Hkv), B, n = c["heads"], len(c["lens"]), c["q"].shape[1]
    d = {x: c[x].cuda() for x in ("k", "v_packed", "v_mask", "v_offs", "q", "k_new", "v_new")}
    shape = P.Shape(B, Hq, Hkv, c["S"], c["T"], torch.tensor(c["lens"], dtype=torch.int32, device="cuda"))
    cache = P.Cache(k=d["k"], v_packed=d["v_packed"], v_mask=d["v_mask"], v_offs=d["v_offs"], cap_groups=c["cap"])
    tree = P.Tree(d["k_new"], d["v_new"], None if c["chain"] else torch.tensor(c["parent"], dtype=torch.int32, device="cuda"),
                  torch.tensor(c["nodes"], dtype=torch.int32, device="cuda"))
    out, lse = buffers or (torch.full((B, n, Hq, 128), -3.0, device="cuda"), torch.full((B, n, Hq), -3.0, device="cuda"))
    status = torch.full((B,), 77, dtype=torch.int32, device="cuda")
    ws = Bd.new_workspace(shape, Bd.OP_TREE_ATTN, n).fill_(0xAB)
    P.tree_attn(shape, cache, tree, d["q"], None if ids is None else ids.cuda(), None if n_ids is None else n_ids.cuda(), scale, out,
                status, ws, lse=lse, score=score)
    torch.cuda.synchronize()
    assert int(ws[:4].view(torch.int32)[0]) == 0
    return out.cpu(), lse.cpu(), status.cpu()


def check(c, out, lse, status, ids=None, n_ids=None, scale=SCALE, softcap=0.0, slopes=None, window=0, doc=None, q_doc=None, q_pos=None,
          skip=()):
    Hq, Hkv = c["heads"]
    gq = Hq // Hkv
    for b, (length, n) in enumerate(zip(c["lens"], c["nodes"])):
        assert (out[b, n:] == -3).all() and (lse[b, n:] == -3).all()
        if b in skip:
            continue
        assert status[b] == 0
        if n == 0:
            continue
        parent = c["parent"][b]
        pos = torch.tensor([length + len(TR.line(parent, i)) - 1 for i in range(n)]) if q_pos is None else q_pos[b, :n].long()
        pages = (length + 15) // 16
        for h in range(Hkv):
            if ids is None:
                at = torch.arange(length)
            else:
                use = [p for p in ids[b, h, :int(n_ids[b, h])].tolist() if 0 <= p < pages]
                at = torch.tensor([t for p in use for t in range(16 * p, min(length, 16 * p + 16))], dtype=torch.long)
            hs = slice(h * gq, (h + 1) * gq)
            o, l, to, tl = TR.tree_rows(c["q"][b][:, hs], c["k"][b, h][at], c["dense"][b, h][at], at, c["k_new"][b, h], c["v_new"][b, h], parent,
                                        n, pos, scale, softcap, None if slopes is None else slopes[hs], window,
                                        None if doc is None else doc[b], 0 if q_doc is None else int(q_doc[b]))
            R.assert_rows(out[b, :n, hs], lse[b, :n, hs], o, l, to, tl)


@pytest.mark.parametrize("heads,S", [((8, 8), 8), ((28, 4), 16), ((32, 8), 8), ((12, 2), 4), ((5, 1), 8), ((8, 1), 16), ((3, 3), 4)])
@pytest.mark.parametrize("cap_nodes", [1, 7, 32])
def test_heads_and_trees_over_whole_caches(heads, S, cap_nodes):
    nodes = [cap_nodes, max(1, cap_nodes - 3), 0, max(1, cap_nodes // 2)]
    c = make(cap_nodes + S, heads, S, 300, [300, 17, 129, 0], cap_nodes, nodes)
    check(c, *call(c))


@pytest.mark.parametrize("cap_nodes", [33, 64, 65, 100, 128])
@pytest.mark.parametrize("heads", [(2, 2), (4, 1), (14, 2), (8, 1)])
def test_many_nodes(heads, cap_nodes):
    c = make(cap_nodes, heads, 8, 200, [200, 131], cap_nodes, [cap_nodes, cap_nodes - 1])
    check(c, *call(c))


@pytest.mark.parametrize("length", [0, 1, 15, 16, 17, 127, 128, 129, 255, 256, 257, 1000, 2500])
def test_lengths_and_chains(length):
    c = make(length, (6, 2), 8, max(length, 3), [length, max(length - 1, 0)], 6, [6, 5], chain=True)
    check(c, *call(c))


def test_a_cache_without_room():
    c = make(1, (4, 2), 8, 0, [0, 0], 9, [9, 4])
    check(c, *call(c))


@pytest.mark.parametrize("most", [1, 3, 8, 9, 40])
def test_page_lists(most):
    """Unsorted, repeated and outside pages, lists of different lengths; the pages that are not listed hold NaN."""
    heads, T, lens = (12, 4), 1000, [1000, 333, 16, 0]
    r = TR.rng(most)
    c = make(most, heads, 8, T, lens, 10, [10, 3, 7, 2])
    ids, n_ids = torch.full((4, 4, most), 1 << 30, dtype=torch.int32), torch.zeros(4, 4, dtype=torch.int32)
    for b, length in enumerate(lens):
        pages = (length + 15) // 16
        for h in range(4):
            n_ids[b, h] = r.choice([most, most, r.randint(0, most), most + 5, -2])
            for i in range(most):
                ids[b, h, i] = r.choice([r.randrange(pages + 1)] * 6 + [-1, pages, 1 << 28])
            use = ids[b, h, :max(0, min(most, int(n_ids[b, h])))].tolist()
            for p in range(pages):
                if p not in use:
                    c["k"][b, h, 16 * p:16 * p + 16] = NAN
                    o = c["v_offs"][b, h]
                    c["v_packed"][b, h, o[16 * p]:o[min(T, 16 * p + 16)]] = NAN
                    c["dense"][b, h, 16 * p:16 * p + 16] = NAN
    got = call(c, ids, n_ids)
    check(c, *got, ids=ids, n_ids=n_ids.clamp(0, most))


def test_lists_of_no_pages_leave_the_tree():
    c = make(3, (8, 2), 8, 64, [64, 30], 5, [5, 4])
    for most in (0, 3):
        ids, n_ids = torch.zeros(2, 2, most, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32)
        check(c, *call(c, ids, n_ids), ids=ids, n_ids=n_ids)


@pytest.mark.parametrize("heads,S", [((8, 8), 8), ((14, 2), 16), ((8, 1), 4)])
@pytest.mark.parametrize("softcap,alibi,window,docs", [(30.0, False, 0, False), (1.0, False, 0, False), (0.0, True, 0, False), (0.0, False, 1, False),
                                                       (0.0, False, 3, False), (0.0, False, 40, False), (0.0, False, 0, True),
                                                       (5.0, True, 150, True)])
def test_options(heads, S, softcap, alibi, window, docs):
    lens, T = [390, 100, 5], 400
    c = make(S, heads, S, T, lens, 17, [17, 12, 1])
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / heads[0]) for h in range(heads[0])]) if alibi else None
    doc = (torch.arange(T)[None, :] // 37 % 4 - 1).expand(3, T).contiguous().int() if docs else None
    q_doc = torch.tensor([1, 2, 9], dtype=torch.int32) if docs else None
    # tokens that no node of the sequence sees: NaN in keys and values
    for b, length in enumerate(lens):
        gone = torch.zeros(T, dtype=torch.bool)
        if window:
            gone[:max(0, length - window + 1)] = True                   # the least position of a node is the length
        if docs:
            gone |= (doc[b] >= 0) & (doc[b] != q_doc[b])
        gone[length:] = False
        c["k"][b][:, gone] = NAN
        for h in range(heads[1]):
            o = c["v_offs"][b, h].tolist()
            for t in gone.nonzero().flatten().tolist():
                c["v_packed"][b, h, o[t]:o[t + 1]] = NAN
        c["dense"][b][:, gone] = NAN
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    score = P.Score(softcap=softcap, slopes=dev(slopes), window=window, tok_doc=dev(doc), q_doc=dev(q_doc))
    check(c, *call(c, score=score), softcap=softcap, slopes=slopes, window=window, doc=doc, q_doc=q_doc)


@pytest.mark.parametrize("window", [0, 25])
def test_positions_that_are_given(window):
    """Positions inside the cache hide what lies behind them; rows may be left with nothing."""
    lens, n = [130, 40], 9
    c = make(5, (4, 2), 8, 130, lens, n, [9, 9], chain=True)
    q_pos = torch.tensor([[200, 201, 202, 210, 129, 130, 131, 64, 3], [-5, 0, 1, 39, 40, 41, 41, 90, 90]], dtype=torch.int32)
    slopes = torch.tensor([0.5, 0.25, 0.1, 0.01])
    score = P.Score(q_pos=q_pos.cuda(), window=window, slopes=slopes.cuda())
    check(c, *call(c, score=score), q_pos=q_pos, window=window, slopes=slopes)


@pytest.mark.parametrize("scale", [0.0, -0.05, 3.0])
def test_scales(scale):
    c = make(8, (8, 4), 8, 500, [500, 77], 5, [5, 3])
    check(c, *call(c, scale=scale), scale=scale)


def test_a_nan_key_reaches_only_the_rows_that_see_it():
    c = make(6, (6, 2), 8, 300, [300, 300], 12, [12, 12])
    clean = call(c)
    hit = 3
    c["k_new"][0, 1, hit] = NAN
    out, lse, _ = call(c)
    for i in range(12):
        if hit in TR.line(c["parent"][0], i):
            assert torch.isnan(out[0, i, 3:]).all() and torch.isnan(lse[0, i, 3:]).all()
            out[0, i, 3:], lse[0, i, 3:] = clean[0][0, i, 3:], clean[1][0, i, 3:]
    assert torch.equal(out, clean[0]) and torch.equal(lse, clean[1])
    c["k"][1, 0, 250] = NAN
    out, lse, _ = call(c)
    assert torch.isnan(out[1, :, :3]).all() and torch.isnan(lse[1, :, :3]).all() and torch.equal(out[1, :, 3:], clean[0][1, :, 3:])


def test_infinite_keys_are_tokens_without_weight_or_the_only_ones():
    c = make(7, (2, 1), 8, 100, [100], 2, [2], chain=True)
    c["q"][...] = c["q"].abs() + 0.5
    c["k"][0, 0, :50] = -math.inf
    out, lse, _ = call(c)
    c["k"][0, 0, :50] = -1e30
    want, want_lse, _ = call(c)
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and torch.isfinite(out).all()
    c["k"][0, 0] = -math.inf                      # nothing but the nodes themselves has weight
    ids = torch.zeros(1, 1, 0, dtype=torch.int32)
    alone = call(c, ids, torch.zeros(1, 1, dtype=torch.int32))
    out, lse, _ = call(c)
    assert ((out - alone[0]).abs() <= 1e-6 * (1 + alone[0].abs())).all()


@pytest.mark.parametrize("bad", [3, 40, -2])
def test_a_tree_that_is_none_is_reported(bad):
    """A parent that is not below its node counts as none."""
    c = make(4, (8, 4), 8, 64, [64, 64, 20], 5, [5, 4, 5])
    c["parent"][1][3] = bad
    out, lse, status = call(c)
    assert status.tolist() == [0, 1, 0]
    c["parent"][1][3] = -1
    check(c, out, lse, torch.zeros_like(status))


def test_repeatable_and_alone_or_together():
    """The same bits twice, on two streams at once, and replayed from a graph."""
    c = make(9, (16, 4), 8, 3000, [3000, 1234, 2000], 20, [20, 20, 11])
    first = call(c)
    again = call(c)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    d = {x: c[x].cuda() for x in ("k", "v_packed", "v_mask", "v_offs", "q", "k_new", "v_new")}
    shape = P.Shape(3, 16, 4, 8, 3000, torch.tensor(c["lens"], dtype=torch.int32, device="cuda"))
    cache = P.Cache(k=d["k"], v_packed=d["v_packed"], v_mask=d["v_mask"], v_offs=d["v_offs"], cap_groups=c["cap"])
    tree = P.Tree(d["k_new"], d["v_new"], torch.tensor(c["parent"], dtype=torch.int32, device="cuda"),
                  torch.tensor(c["nodes"], dtype=torch.int32, device="cuda"))

    def buffers():
        return dict(out=torch.full((3, 20, 16, 128), -3.0, device="cuda"), lse=torch.full((3, 20, 16), -3.0, device="cuda"),
                    status=torch.zeros(3, dtype=torch.int32, device="cuda"), ws=Bd.new_workspace(shape, Bd.OP_TREE_ATTN, 20))

    def run(s):
        P.tree_attn(shape, cache, tree, d["q"], None, None, SCALE, s["out"], s["status"], s["ws"], lse=s["lse"])

    sets, streams = [buffers(), buffers()], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(8):
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                run(s)
    torch.cuda.synchronize()
    graphed = buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(graphed)
        run(graphed)
    graphed["out"].fill_(-3.0)
    graphed["lse"].fill_(-3.0)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for s in (*sets, graphed):
        assert torch.equal(s["out"].cpu(), first[0]) and torch.equal(s["lse"].cpu(), first[1])


@pytest.mark.parametrize("heads,nodes", [((1, 1), 1), ((8, 1), 16), ((4, 4), 1)])
def test_error_over_long_caches(heads, nodes):
    """131072 tokens.  The error's norm: 2.4e-6 from weights as bf16 pairs (up to 2^-16 each), at most 128 products of 4e-8 between
    two times an accumulator is emptied (half of it on average: 2.6e-6), fp32 sums and scores 1e-6."""
    Hq, Hkv = heads
    T = 131072
    g = torch.Generator(device="cuda").manual_seed(3)
    k = torch.randn(1, Hkv, T, 128, generator=g, device="cuda").to(torch.bfloat16)
    packed = torch.randn(1, Hkv, 4 * T, 32, generator=g, device="cuda").to(torch.bfloat16) + 0.25
    mask = torch.full((1, Hkv, T), 15, dtype=torch.int16, device="cuda")
    offs = (4 * torch.arange(T + 1, device="cuda")).to(torch.int32).expand(1, Hkv, T + 1).contiguous()
    q = torch.randn(1, nodes, Hq, 128, generator=g, device="cuda").to(torch.bfloat16)
    kn, vn = (torch.randn(1, Hkv, nodes, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    shape = P.Shape(1, Hq, Hkv, 4, T)
    out, lse = torch.zeros(1, nodes, Hq, 128, device="cuda"), torch.zeros(1, nodes, Hq, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.tree_attn(shape, P.Cache(k=k, v_packed=packed, v_mask=mask, v_offs=offs, cap_groups=4 * T), P.Tree(kn, vn), q, None, None, SCALE, out,
                status, Bd.new_workspace(shape, Bd.OP_TREE_ATTN, nodes), lse=lse)
    gq = Hq // Hkv
    for h in range(Hkv):
        keys = torch.cat([k[0, h], kn[0, h]]).double()
        values = torch.cat([packed[0, h].view(T, 128), vn[0, h]]).double()
        x = torch.einsum("igd,td->igt", q[0, :, h * gq:(h + 1) * gq].double(), keys) * SCALE
        x[:, :, T:] = torch.where(torch.ones(nodes, nodes, dtype=torch.bool, device="cuda").tril()[:, None], x[:, :, T:], -math.inf)
        want = torch.softmax(x, -1) @ values
        got = out[0, :, h * gq:(h + 1) * gq].double()
        assert ((got - want).norm() / want.norm()).item() <= 6e-6
        assert (lse[0, :, h * gq:(h + 1) * gq].double() - torch.logsumexp(x, -1)).abs().max().item() <= 2e-5


def test_offsets_beyond_32_bits():
    """Keys of 4.4 GB: the last sequence's begin behind 2^31 elements."""
    B, Hkv, Hq, T, S, n, pages = 17, 8, 16, 131072 - 16, 4, 5, 20
    k = torch.empty(B, Hkv, T, 128, dtype=torch.bfloat16, device="cuda")
    assert k.numel() > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(7)
    k[-1].normal_(generator=g)
    packed = torch.empty(B, Hkv, T, 32, dtype=torch.bfloat16, device="cuda")
    packed[-1].normal_(generator=g)
    mask = (1 << (torch.arange(T, device="cuda") % 4)).to(torch.int16).expand(B, Hkv, T).contiguous()
    offs = torch.arange(T + 1, dtype=torch.int32, device="cuda").expand(B, Hkv, T + 1).contiguous()
    ids = torch.randperm(T // 16, generator=g, device="cuda")[:pages].sort().values.to(torch.int32).expand(B, Hkv, pages).contiguous()
    ids[..., -1] = T // 16 - 1
    n_ids = torch.zeros(B, Hkv, dtype=torch.int32, device="cuda")
    n_ids[-1] = pages
    q = torch.randn(B, n, Hq, 128, generator=g, device="cuda").to(torch.bfloat16)
    kn, vn = (torch.randn(B, Hkv, n, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    nodes = torch.zeros(B, dtype=torch.int32, device="cuda")
    nodes[-1] = n
    shape = P.Shape(B, Hq, Hkv, S, T)
    out, lse = torch.zeros(B, n, Hq, 128, device="cuda"), torch.zeros(B, n, Hq, device="cuda")
    status = torch.zeros(B, dtype=torch.int32, device="cuda")
    P.tree_attn(shape, P.Cache(k=k, v_packed=packed, v_mask=mask, v_offs=offs, cap_groups=T), P.Tree(kn, vn, None, nodes), q, ids, n_ids, SCALE,
                out, status, Bd.new_workspace(shape, Bd.OP_TREE_ATTN, n), lse=lse)
    torch.cuda.synchronize()
    assert (out[:-1] == 0).all()
    at = (ids[-1, 0].cpu().long()[:, None] * 16 + torch.arange(16)).flatten()
    for h in range(Hkv):
        dense = torch.zeros(at.numel(), 4, 32, dtype=torch.float64)
        dense[torch.arange(at.numel()), at % 4] = packed[-1, h][at.cuda()].cpu().double()
        o, l, to, tl = TR.tree_rows(q[-1, :, 2 * h:2 * h + 2].cpu(), k[-1, h][at.cuda()].cpu(), dense.reshape(-1, 128), at, kn[-1, h].cpu(),
                                    vn[-1, h].cpu(), [-1, 0, 1, 2, 3], n, T + torch.arange(n), SCALE)
        R.assert_rows(out[-1, :, 2 * h:2 * h + 2], lse[-1, :, 2 * h:2 * h + 2], o, l, to, tl)


# rows of a block (32, 64, 128), copied over the tensor-memory lanes once the call may have more than four tiles per SM
FEW_ROWS = [((8, 8), 8, 32), ((8, 8), 4, 3), ((32, 8), 16, 16), ((28, 4), 8, 5), ((8, 2), 8, 1), ((16, 8), 8, 33)]


@pytest.mark.parametrize("heads,S,nodes", FEW_ROWS)
def test_few_rows_long_caches(heads, S, nodes):
    T = 128 * (600 // (3 * heads[1]) + 1) + 3
    c = make(nodes, heads, S, T, [min(T, 3400), 1500, 129], nodes, [nodes, max(1, nodes - 1), nodes])
    check(c, *call(c))


@pytest.mark.parametrize("heads,S,nodes", FEW_ROWS)
def test_few_rows_many_short_caches(heads, S, nodes):
    """Units that a CTA finishes by itself, several per CTA."""
    r, B, T = TR.rng(nodes), 192 // heads[1], 700
    lens = [r.choice([0, 1, 16, 127, 128, 500, 699, 700]) for _ in range(B)]
    c = make(nodes + 1, heads, S, T, lens, nodes, [r.randint(0, nodes) for _ in range(B)])
    check(c, *call(c))


@pytest.mark.parametrize("heads,nodes", [((8, 8), 20), ((28, 4), 5)])
@pytest.mark.parametrize("softcap,alibi,window,docs", [(30.0, False, 0, False), (0.0, True, 0, False), (0.0, False, 150, True), (5.0, True, 400, True)])
def test_few_rows_with_options(heads, nodes, softcap, alibi, window, docs):
    r, B, T = TR.rng(nodes), 192 // heads[1], 700
    lens = [r.choice([1, 130, 500, 700]) for _ in range(B)]
    c = make(nodes + 2, heads, 8, T, lens, nodes, [r.randint(1, nodes) for _ in range(B)])
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / heads[0]) for h in range(heads[0])]) if alibi else None
    doc = (torch.arange(T)[None, :] // 37 % 4 - 1).expand(B, T).contiguous().int() if docs else None
    q_doc = torch.tensor([r.choice([1, 2, 9]) for _ in range(B)], dtype=torch.int32) if docs else None
    dev = lambda x: None if x is None else x.cuda()  # noqa: E731
    score = P.Score(softcap=softcap, slopes=dev(slopes), window=window, tok_doc=dev(doc), q_doc=dev(q_doc))
    check(c, *call(c, score=score), softcap=softcap, slopes=slopes, window=window, doc=doc, q_doc=q_doc)
