"""stc_tree_commit, stc_cache_fork and stc_cache_compact against copies made on the host, byte for byte."""
import pytest
import torch

import operators_ref as R
import paper_2604_21335_b200 as P
import tree_ref as TR

pytestmark = pytest.mark.gpu
NAMES = ("k", "kmin", "kmax", "v_packed", "v_mask", "v_offs")


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def full(seed, B, Hkv, T, S, lens, room=0, keep=None):
    """A cache dict on the CPU with page metadata and `room` more group rows; nothing in it is NaN, so that copies can be compared."""
    c = R.make_cache(seed, B, Hkv, T, S, keep or max(1, S // 2), lens, poison=False)
    g = torch.Generator().manual_seed(seed + 9)
    cap = c["cap"] + room
    packed = torch.randn(B, Hkv, cap, 128 // S, generator=g).to(torch.bfloat16)
    for b, n in enumerate(lens):
        for h in range(Hkv):
            held = int(c["v_offs"][b, h, n])
            packed[b, h, :held] = c["v_packed"][b, h, :held]
            c["v_offs"][b, h, n + 1:] = 123456789                   # nobody looks behind the length
    c["v_packed"], c["cap"] = packed, cap
    pages = (T + 15) // 16
    c["kmin"], c["kmax"] = (torch.randn(B, Hkv, pages, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    for b, n in enumerate(lens):
        for h in range(Hkv):
            lo, hi = TR.meta(c["k"][b, h], n)
            for p, (x, y) in enumerate(zip(lo, hi)):
                c["kmin"][b, h, p], c["kmax"][b, h, p] = x, y
    return {x: c[x] for x in (*NAMES, "cap", "lens")}


def blank(seed, B, Hkv, T, S, cap):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16)  # noqa: E731
    pages = (T + 15) // 16
    return dict(k=r(B, Hkv, T, 128), kmin=r(B, Hkv, pages, 128), kmax=r(B, Hkv, pages, 128), v_packed=r(B, Hkv, cap, 128 // S),
                v_mask=torch.full((B, Hkv, T), 21, dtype=torch.int16), v_offs=torch.full((B, Hkv, T + 1), 77, dtype=torch.int32), cap=cap)


def clone(c):
    return {n: x.clone() if isinstance(x, torch.Tensor) else x for n, x in c.items()}


def device(c):
    return P.Cache(**{n: c[n].cuda() for n in NAMES}, cap_groups=c["cap"])


def same(cache, want):
    for n in NAMES:
        got = getattr(cache, n).cpu()
        assert torch.equal(got, want[n]), n


def outputs(B, H, rows):
    return (torch.full((B,), -5, dtype=torch.int32, device="cuda"), torch.full((B, H), -5, dtype=torch.int64, device="cuda"),
            torch.full((rows, H), -5, dtype=torch.int32, device="cuda"))


# ---- commit -------------------------------------------------------------------------------------------------------

def commit_on_host(c, S, k_new, v_new, path, n_acc):
    """The cache after the call, new lengths, totals, status."""
    w, T, H = clone(c), c["k"].shape[2], c["k"].shape[1]
    lens, totals, status = list(c["lens"]), [], []
    for b, m in enumerate(n_acc):
        n = c["lens"][b]
        for h in range(H):
            base = int(c["v_offs"][b, h, n])
            for i in range(m):
                w["k"][b, h, n + i] = k_new[b, h, path[b][i]]
                w["v_mask"][b, h, n + i] = (1 << S) - 1 if S < 16 else -1
                w["v_offs"][b, h, n + i + 1] = base + (i + 1) * S
                for j in range(S):
                    if base + i * S + j < c["cap"]:
                        w["v_packed"][b, h, base + i * S + j] = v_new[b, h, path[b][i]].view(S, -1)[j]
            if m:
                lo, hi = TR.meta(w["k"][b, h], n + m)
                for p in range(n // 16, (n + m + 15) // 16):
                    w["kmin"][b, h, p], w["kmax"][b, h, p] = lo[p], hi[p]
            totals.append(base + m * S)
            status.append(4 if base + m * S > c["cap"] else 0)
        lens[b] = n + m
    return w, lens, totals, status


@pytest.mark.parametrize("S", [4, 8, 16])
@pytest.mark.parametrize("Hkv,n_cap,lens,n_acc", [(2, 1, [0, 15, 16], [1, 1, 1]), (3, 8, [0, 31, 40, 100], [8, 0, 3, 5]),
                                                  (1, 128, [0, 1, 130], [128, 128, 100]), (8, 20, [7], [17])])
def test_commit(S, Hkv, n_cap, lens, n_acc):
    B, T = len(lens), max(a + b for a, b in zip(lens, n_acc)) + 3
    c = full(S, B, Hkv, T, S, lens, room=max(n_acc) * S)
    g = torch.Generator().manual_seed(1)
    k_new, v_new = (torch.randn(B, Hkv, n_cap, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    r = TR.rng(S)
    path = [[r.randrange(n_cap) for _ in range(n_cap)] for _ in range(B)]
    for b in range(B):
        path[b][n_acc[b]:] = [99999] * (n_cap - n_acc[b])
    cache = device(c)
    new_len, total, status = outputs(B, Hkv, B)
    shape = P.Shape(B, Hkv, Hkv, S, T, i32(lens))
    P.tree_commit(shape, cache, P.Tree(k_new.cuda(), v_new.cuda()), i32(path), i32(n_acc), new_len, total, status)
    w, ln, tot, st = commit_on_host(c, S, k_new, v_new, path, n_acc)
    same(cache, w)
    assert new_len.tolist() == ln and total.flatten().tolist() == tot and status.flatten().tolist() == st


def test_commit_refuses_sequence_by_sequence_and_fills_a_full_store_no_further():
    S, H, T, lens = 8, 2, 60, [50, 50, 50, 50, 20, 50]
    c = full(3, 6, H, T, S, lens, room=0)
    n_acc = [11, 3, -1, 9, 6, 3]                                        # too long; path outside; negative; more than n_cap; no room; a node that is not there
    path = [[0] * 8, [0, 8, 1] + [0] * 5, [0] * 8, [0] * 8, [1, 3, 5, 7, 0, 2, 0, 0], [0, 1, 6] + [0] * 5]
    c["cap"] = int(c["v_offs"][4, :, 20].max()) + 20
    c["v_packed"] = c["v_packed"][:, :, :c["cap"]].contiguous() if c["cap"] <= c["v_packed"].shape[2] else c["v_packed"]
    c["cap"] = c["v_packed"].shape[2]
    k_new, v_new = (torch.randn(6, H, 8, 128).to(torch.bfloat16) for _ in range(2))
    cache = device(c)
    new_len, total, status = outputs(6, H, 6)
    P.tree_commit(P.Shape(6, H, H, S, T, i32(lens)), cache, P.Tree(k_new.cuda(), v_new.cuda(), None, i32([8, 8, 8, 8, 8, 6])), i32(path), i32(n_acc), new_len,
                  total, status)
    w, ln, tot, st = commit_on_host(c, S, k_new, v_new, path, [0, 0, 0, 0, 6, 0])
    same(cache, w)
    bad = [0, 1, 2, 3, 5]
    assert new_len.tolist() == ln and status[bad].eq(1).all() and total[bad].eq(-5).all()
    assert status[4].tolist() == st[8:10] and total[4].tolist() == tot[8:10]


def test_commit_without_metadata_equals_append_tokens():
    """Accepted nodes 0, 1, 2 .. in order are what stc_append_tokens adds."""
    S, H, T, lens, m = 8, 4, 100, [33, 64], 5
    c = full(5, 2, H, T, S, lens, room=m * S)
    k_new, v_new = (torch.randn(2, H, m, 128).to(torch.bfloat16) for _ in range(2))
    a, b, bare = device(c), device(c), device(c)
    bare.kmin = bare.kmax = None
    outs = [outputs(2, H, 2) for _ in range(3)]
    path = i32([list(range(m))] * 2)
    for cache, o in ((a, outs[0]), (bare, outs[1])):
        P.tree_commit(P.Shape(2, H, H, S, T, i32(lens)), cache, P.Tree(k_new.cuda(), v_new.cuda()), path, i32([m, m]), *o)
    v = torch.zeros(2, H, T, 128, dtype=torch.bfloat16)
    for i, n in enumerate(lens):
        b.k[i, :, n:n + m] = k_new[i].cuda()
        v[i, :, n:n + m] = v_new[i]
    P.append_tokens(P.Shape(2, H, H, S, T, outs[0][0]), b, v.cuda(), i32(lens), m, outs[2][1], outs[2][2])
    for n in NAMES:
        assert torch.equal(getattr(a, n), getattr(b, n)), n
        if getattr(bare, n) is not None:
            assert torch.equal(getattr(bare, n), getattr(a, n)), n
    assert torch.equal(outs[0][1], outs[2][1]) and torch.equal(outs[0][2], outs[2][2])


# ---- fork ---------------------------------------------------------------------------------------------------------

def fork_on_host(c, d, S, pairs):
    w = clone(d)
    for s, t in pairs:
        n = c["lens"][s]
        pages = (n + 15) // 16
        for x, m in (("k", n), ("kmin", pages), ("kmax", pages), ("v_mask", n), ("v_offs", n + 1)):
            w[x][t, :, :m] = c[x][s, :, :m]
        for h in range(c["k"].shape[1]):
            m = min(int(c["v_offs"][s, h, n]), d["cap"])
            w["v_packed"][t, h, :m] = c["v_packed"][s, h, :m]
    return w


@pytest.mark.parametrize("S,Hkv,T,lens", [(8, 4, 70, [70, 33, 0]), (4, 1, 64, [64, 1, 16]), (16, 3, 300, [257, 300, 65])])
def test_fork_into_another_cache(S, Hkv, T, lens):
    c = full(S, 3, Hkv, T, S, lens)
    d = blank(2, 6, Hkv, T + 9, S, c["cap"] + 5)
    src, dst = [0, 0, 2, 1, 0], [5, 0, 3, 1, 4]
    cache = device(d)
    new_len, total, status = outputs(6, Hkv, 5)
    P.cache_fork(P.Shape(3, Hkv, Hkv, S, T, i32(lens)), device(c), P.Shape(6, Hkv, Hkv, S, T + 9), cache, i32(src), i32(dst), new_len, total, status)
    same(cache, fork_on_host(c, d, S, list(zip(src, dst))))
    assert (status == 0).all() and new_len.tolist() == [lens[0], lens[1], -5, lens[2], lens[0], lens[0]]
    for s, t in zip(src, dst):
        assert total[t].tolist() == c["v_offs"][s, :, lens[s]].tolist()
    assert (total[2] == -5).all()


def test_fork_within_one_cache_and_pairs_that_are_left_out():
    S, H, T, lens = 8, 2, 90, [90, 50, 17, 3, 8, 64]
    c = full(4, 6, H, T, S, lens)
    cache = device(c)
    # 0 -> 3 copied; 1 -> 1 stays; 2 -> 4 copied; 2 -> 4 again; 5 -> 0 would overwrite a source; rows outside; 1 -> 5 overwrites a source
    src, dst = [0, 1, 2, 2, 5, 6, 1, -1, 1], [3, 1, 4, 4, 0, 2, 6, 5, 5]
    new_len, total, status = outputs(6, H, 9)
    P.cache_fork(P.Shape(6, H, H, S, T, i32(lens)), cache, P.Shape(6, H, H, S, T), cache, i32(src), i32(dst), new_len, total, status)
    same(cache, fork_on_host(c, c, S, [(0, 3), (2, 4)]))
    assert status[:, 0].tolist() == [0, 0, 0, 1, 1, 1, 1, 1, 1] and torch.equal(status[:, 0], status[:, 1])
    assert new_len.tolist() == [-5, 50, -5, 90, 17, -5]


def test_fork_into_smaller_caches():
    S, H, T, lens = 4, 2, 200, [200, 60, 150]
    c = full(6, 3, H, T, S, lens, keep=3)
    small = 25
    d = blank(3, 3, H, 150, S, small)
    cache = device(d)
    new_len, total, status = outputs(3, H, 3)
    P.cache_fork(P.Shape(3, H, H, S, T, i32(lens)), device(c), P.Shape(3, H, H, S, 150), cache, i32([0, 1, 2]), i32([0, 1, 2]), new_len, total, status)
    same(cache, fork_on_host(c, d, S, [(1, 1), (2, 2)]))
    assert status.tolist() == [[1, 1], [4, 4], [4, 4]] and new_len.tolist() == [-5, 60, 150]
    bare = device(c)
    bare.kmin = bare.kmax = None
    with pytest.raises(P.StcError):                                      # metadata wanted that the source does not have
        P.cache_fork(P.Shape(3, H, H, S, T, i32(lens)), bare, P.Shape(3, H, H, S, 150), cache, i32([0]), i32([0]), new_len, total, status[:1])


def test_fork_of_many_pairs():
    S, H, T, n = 8, 1, 40, 2500
    c = full(8, 4, H, T, S, [40, 17, 1, 0])
    cache = device(blank(3, n, H, T, S, c["cap"]))
    new_len, total, status = outputs(n, H, n)
    src = [i * 4 // n for i in range(n)]
    dst = list(range(n))[::-1]
    P.cache_fork(P.Shape(4, H, H, S, T, i32(c["lens"])), device(c), P.Shape(n, H, H, S, T), cache, i32(src), i32(dst), new_len, total, status)
    same(cache, fork_on_host(c, blank(3, n, H, T, S, c["cap"]), S, list(zip(src, dst))))
    assert (status == 0).all()
    dst[2000] = dst[100]                                                 # the later one is left out
    P.cache_fork(P.Shape(4, H, H, S, T, i32(c["lens"])), device(c), P.Shape(n, H, H, S, T), cache, i32(src), i32(dst), new_len, total, status)
    assert status.sum() == 1 and status[2000] == 1


# ---- compaction ---------------------------------------------------------------------------------------------------

def compact_on_host(c, d, S, lists):
    """lists[b][h]: page ids."""
    w, lens, totals = clone(d), [], []
    for b, per_head in enumerate(lists):
        n = c["lens"][b]
        for h, ids in enumerate(per_head):
            stored, masks = TR.dense_of(c, b, h, S)
            tok = [t for p in ids for t in range(16 * p, min(n, 16 * p + 16))]
            at = 0
            w["v_offs"][b, h, 0] = 0
            for i, t in enumerate(tok):
                w["k"][b, h, i], w["v_mask"][b, h, i] = c["k"][b, h, t], c["v_mask"][b, h, t]
                m = max(0, min(len(stored[t]), d["cap"] - at))
                w["v_packed"][b, h, at:at + m] = stored[t][:m]
                at += len(stored[t])
                w["v_offs"][b, h, i + 1] = at
            for i, p in enumerate(ids):
                w["kmin"][b, h, i], w["kmax"][b, h, i] = c["kmin"][b, h, p], c["kmax"][b, h, p]
            totals.append(at)
        lens.append(len(tok))
    return w, lens, totals


def lists_for(r, lens, Hkv, most, with_last=True):
    out = []
    for n in lens:
        pages = (n + 15) // 16
        m = min(pages, r.randint(0, most)) if pages else 0
        per_head = []
        for _ in range(Hkv):
            if n % 16 and m:
                per_head.append(sorted(r.sample(range(pages - 1), m - 1)) + [pages - 1] if with_last else sorted(r.sample(range(pages - 1), min(m, pages - 1))))
            else:
                per_head.append(sorted(r.sample(range(pages), m)))
        out.append(per_head)
    return out


def pack_lists(lists, most):
    ids = torch.full((len(lists), len(lists[0]), most), -4, dtype=torch.int32)
    n = torch.zeros(len(lists), len(lists[0]), dtype=torch.int32)
    for b, per_head in enumerate(lists):
        for h, x in enumerate(per_head):
            ids[b, h, :len(x)] = torch.tensor(x, dtype=torch.int32)
            n[b, h] = len(x)
    return ids.cuda(), n.cuda()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("S", [4, 8, 16])
@pytest.mark.parametrize("Hkv,T,lens,most", [(2, 100, [100, 33, 0, 16], 7), (1, 1500, [1500, 1499], 94), (3, 700, [640, 555, 700], 20),
                                             (2, 640, [640, 640], 40)])
def test_compact(S, Hkv, T, lens, most, in_place):
    r = TR.rng(S + T)
    c = full(S, len(lens), Hkv, T, S, lens)
    lists = lists_for(r, lens, Hkv, most)
    lists[0] = [x if (most < 40 or in_place) else list(range((lens[0] + 15) // 16)) for x in lists[0]]    # one keeps everything
    ids, n = pack_lists(lists, most)
    d = c if in_place else blank(1, len(lens), Hkv, most * 16, S, c["cap"])
    src = device(c)
    dst = src if in_place else device(d)
    new_len, total, status = outputs(len(lens), Hkv, len(lens))
    shape = P.Shape(len(lens), Hkv, Hkv, S, T, i32(lens))
    P.cache_compact(shape, src, ids, n, new_len, total, status,
                    **({} if in_place else dict(dst_shape=P.Shape(len(lens), Hkv, Hkv, S, most * 16), dst=dst)))
    w, ln, tot = compact_on_host(c, d, S, lists)
    same(dst, w)
    if not in_place:
        same(src, c)
    assert (status == 0).all() and new_len.tolist() == ln and total.flatten().tolist() == tot


def test_compact_long_lists_in_place_again_and_again():
    """Thousands of pages per head move through each other's places; then half of the rest, and so on."""
    S, H, T = 8, 2, 20000
    c = full(11, 1, H, T, S, [T])
    cache, host, r = device(c), clone(c), TR.rng(1)
    length, most = i32([T]), (T + 15) // 16
    for _ in range(3):
        n = int(length[0])
        pages = (n + 15) // 16
        host["lens"] = [n]
        lists = [[sorted(r.sample(range(pages), pages * 3 // 5)) for _ in range(H)]]
        for x in lists[0]:
            if n % 16 and x[-1] != pages - 1:
                x[-1] = pages - 1
        ids, cnt = pack_lists(lists, most)
        new_len, total, status = outputs(1, H, 1)
        P.cache_compact(P.Shape(1, H, H, S, T, length), cache, ids, cnt, new_len, total, status)
        host, ln, tot = compact_on_host(host, host, S, lists)
        same(cache, host)
        assert (status == 0).all() and new_len.tolist() == ln and total.flatten().tolist() == tot
        length = new_len


def test_compact_long_lists_into_another_cache():
    """More pages per CTA than it has threads, and a store that ends in the middle of them."""
    S, H, T, lens = 4, 2, 34000, [34000, 301]
    c, r = full(12, 2, H, T, S, lens, keep=1), TR.rng(2)
    lists = []
    for n in lens:
        pages = (n + 15) // 16
        m = pages - 9
        lists.append([sorted(r.sample(range(pages - 1), m - 1)) + [pages - 1] for _ in range(H)])
    ids, n = pack_lists(lists, 2125)
    for cap in (c["cap"], c["cap"] // 2):
        d = blank(3, 2, H, 2125 * 16, S, cap)
        src, dst = device(c), device(d)
        new_len, total, status = outputs(2, H, 2)
        P.cache_compact(P.Shape(2, H, H, S, T, i32(lens)), src, ids, n, new_len, total, status, dst_shape=P.Shape(2, H, H, S, 2125 * 16), dst=dst)
        w, ln, tot = compact_on_host(c, d, S, lists)
        same(dst, w)
        same(src, c)
        assert new_len.tolist() == ln and total.flatten().tolist() == tot
        assert status.flatten().tolist() == [0 if x <= cap else 4 for x in tot]


def test_compact_dropping_the_last_page_that_is_not_full():
    S, H, T, lens = 8, 2, 200, [185, 200]
    c = full(2, 2, H, T, S, lens)
    lists = [[[0, 3, 5], [1, 2, 10]], [[11], [0]]]
    ids, n = pack_lists(lists, 4)
    cache = device(c)
    new_len, total, status = outputs(2, H, 2)
    P.cache_compact(P.Shape(2, H, H, S, T, i32(lens)), cache, ids, n, new_len, total, status)
    w, ln, _ = compact_on_host(c, c, S, lists)
    same(cache, w)
    assert (status == 0).all() and new_len.tolist() == ln == [48, 16]


def test_compact_leaves_sequences_with_bad_lists_alone():
    S, H, T, L = 8, 2, 96, 90
    cases = [[[2, 1], [0, 5]], [[1, 1], [0, 5]], [[0, 6], [0, 5]], [[-1, 5], [0, 5]], [[0, 5], [5]], [[0, 1], [0, 5]], [[0, 5], [2, 5]]]
    lens = [L] * len(cases)
    c = full(3, len(cases), H, T, S, lens)
    ids, n = pack_lists(cases, 3)
    n[3] = 9                                                             # more than max_pages
    cache = device(c)
    new_len, total, status = outputs(len(cases), H, len(cases))
    P.cache_compact(P.Shape(len(cases), H, H, S, T, i32(lens)), cache, ids, n, new_len, total, status)
    good = len(cases) - 1
    w, ln, tot = compact_on_host(c, c, S, [[list(range(6))] * H] * good + [cases[-1]])
    same(cache, w)
    assert status[:good].eq(1).all() and status[good].eq(0).all() and total[:good].eq(-5).all()
    assert new_len.tolist() == [L] * good + [ln[good]]


def test_compact_into_a_cache_that_is_too_small():
    S, H, T, lens = 4, 2, 160, [160, 160]
    c = full(5, 2, H, T, S, lens, keep=3)
    lists = [[[0, 1, 2, 3], [4, 5, 6, 9]], [[1, 7, 8], [0, 2, 9]]]
    ids, n = pack_lists(lists, 4)
    d = blank(4, 2, H, 48, S, 60)
    cache = device(d)
    new_len, total, status = outputs(2, H, 2)
    P.cache_compact(P.Shape(2, H, H, S, T, i32(lens)), device(c), ids, n, new_len, total, status, dst_shape=P.Shape(2, H, H, S, 48), dst=cache)
    w, ln, tot = compact_on_host(c, d, S, [[[], []], lists[1]])
    w["v_offs"][0, :, 0] = 77
    same(cache, w)
    assert status.tolist() == [[1, 1], [4, 4]] and new_len.tolist() == [160, 48] and total[1].tolist() == tot[2:]


def test_sizes_that_do_not_fit_are_refused():
    S, H, T = 8, 2, 64
    c = device(full(1, 2, H, T, S, [64, 30]))
    shape = P.Shape(2, H, H, S, T, i32([64, 30]))
    ids, n = torch.zeros(2, H, 1, dtype=torch.int32, device="cuda"), torch.zeros(2, H, dtype=torch.int32, device="cuda")
    new_len, total, status = outputs(2, H, 2)
    for bad in (dict(n_pages=n[:1]), dict(page_ids=ids[:, :1]), dict(new_len=new_len[:1]), dict(total_groups=total.int()), dict(dst=c),
                dict(cache=P.Cache(k=c.k[:, :, :32].contiguous(), v_packed=c.v_packed, v_mask=c.v_mask, v_offs=c.v_offs, cap_groups=c.cap_groups)),
                dict(cache=P.Cache(k=c.k, v_packed=c.v_packed, v_mask=c.v_mask, v_offs=c.v_offs, cap_groups=c.cap_groups + 1))):
        with pytest.raises(ValueError):
            P.cache_compact(**{**dict(shape=shape, cache=c, page_ids=ids, n_pages=n, new_len=new_len, total_groups=total, status=status), **bad})
    with pytest.raises(P.StcError):                                      # the lengths that the call reads are not the ones it writes
        P.cache_compact(shape, c, ids, n, shape.seq_len, total, status)
    with pytest.raises(ValueError):
        P.cache_fork(shape, c, P.Shape(3, H, H, S, T), c, i32([0]), i32([1]), new_len, total, status[:1])
    with pytest.raises(P.StcError):
        P.cache_fork(shape, c, P.Shape(2, 2 * H, H, S, T), c, i32([0]), i32([1]), new_len, total, status[:1])
