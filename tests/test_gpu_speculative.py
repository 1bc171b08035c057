"""Speculative decoding as it is used: a loop of rope_write into draft buffers, quest_select, tree_attn, tree_accept and tree_commit, eager and
as one replayed graph, then the cache forked and compacted.  Every step is held against the 64-bit plain forms."""
import math

import pytest
import torch

import operators_ref as R
import paper_2604_21335_b200 as P
import tree_ref as TR
from paper_2604_21335_b200 import binding as Bd

pytestmark = pytest.mark.gpu
SCALE, VOCAB, STEPS = 1 / math.sqrt(128), 96, 6
PARENT = [-1, 0, 0, 1, 1, 3, -1]
NODES = [6, 7]                                              # the second sequence also drafts a second root, which is never reached
DEPTH = [0, 1, 1, 2, 2, 3, 0]
NAMES = ("k", "kmin", "kmax", "v_packed", "v_mask", "v_offs")


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Loop:
    """A one-layer model whose next word mostly follows from the last one, and drafts that know that part."""

    def __init__(self, heads, S, T, lens, budget):
        g = torch.Generator().manual_seed(5)
        self.heads, self.S, self.T, self.n = heads, S, T, len(PARENT)
        Hq, Hkv = heads
        B = len(lens)
        c = R.make_cache(17, B, Hkv, T, S, S // 2, lens, poison=False)
        self.lens, self.k, self.v = list(lens), c["k"].clone(), c["dense"].clone()
        for b, n in enumerate(lens):
            self.k[b, :, n:], self.v[b, :, n:] = 0, 0
        cap = c["cap"] + (STEPS + 1) * self.n * S
        pages = (T + 15) // 16
        packed = torch.zeros(B, Hkv, cap, 128 // S, dtype=torch.bfloat16)
        packed[:, :, :c["cap"]] = c["v_packed"]
        self.cache = P.Cache(k=self.k.cuda(), kmin=torch.zeros(B, Hkv, pages, 128, dtype=torch.bfloat16, device="cuda"),
                             kmax=torch.zeros(B, Hkv, pages, 128, dtype=torch.bfloat16, device="cuda"), v_packed=packed.cuda(),
                             v_mask=c["v_mask"].cuda(), v_offs=c["v_offs"].cuda(), cap_groups=cap)
        self.len = i32(lens)
        self.shape = P.Shape(B, Hq, Hkv, S, T, self.len)
        P.build_page_meta(self.shape, self.cache)
        r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
        # (64 bits outside the calls: whichever product a library picks, eager or captured, rounds to the same bf16)
        self.emb, self.wqkv = r(VOCAB, 64).double().cuda(), (r(64, (Hq + 2 * Hkv) * 128) / 8).double().cuda()
        self.wo, self.follow = (r(Hq * 128, VOCAB) / (8 * math.sqrt(Hq * 128))).double().cuda(), r(VOCAB, VOCAB).double().cuda()
        self.best = self.follow.topk(2, dim=1).indices.to(torch.int32)
        # what the calls read and write; the loop lives on the device
        self.n_nodes, self.parent, self.depth = i32(NODES), i32([PARENT] * B), i32(DEPTH)
        self.tokens = torch.zeros(B, self.n, dtype=torch.int32, device="cuda")
        self.zero, self.rope_status = i32([0] * B), i32([0] * B)
        freq, scale = P.rope_frequencies(128)
        self.rope = P.Rope(freq.cuda(), scale=scale)
        new = lambda *s, t=torch.bfloat16: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731
        self.q, self.k_new, self.v_new = new(B, self.n, Hq, 128), new(B, Hkv, self.n, 128), new(B, Hkv, self.n, 128)
        self.draft = P.Shape(B, Hq, Hkv, S, self.n, self.n_nodes)
        self.tree = P.Tree(self.k_new, self.v_new, self.parent, self.n_nodes)
        most = budget // 16
        self.budget, self.ids, self.n_ids = budget, i32([[[0] * most] * Hkv] * B), i32([[0] * Hkv] * B)
        self.out = new(B, self.n, Hq, 128, t=torch.float32)
        self.path, self.n_accepted, self.next = i32([[0] * self.n] * B), i32([0] * B), i32([1, 2][:B])
        self.new_len, self.total = i32([0] * B), torch.zeros(B, Hkv, dtype=torch.int64, device="cuda")
        self.tree_status, self.commit_status = i32([7] * B), i32([[7] * Hkv] * B)
        self.logits = new(B, self.n, VOCAB, t=torch.float32)
        self.ws_select = Bd.new_workspace(self.shape, Bd.OP_QUEST_SELECT, most)
        self.ws = Bd.new_workspace(self.shape, Bd.OP_TREE_ATTN, self.n)

    def step(self):
        (Hq, Hkv), B, n = self.heads, len(NODES), self.n
        t = self.tokens
        t[:, 0] = self.next
        t[:, 6] = self.next
        for node, up, which in ((1, 0, 0), (2, 0, 1), (3, 1, 0), (4, 1, 1), (5, 3, 0)):
            t[:, node] = self.best[t[:, up].long(), which]
        x = (self.emb[t.long()] @ self.wqkv).to(torch.bfloat16).view(B, n, Hq + 2 * Hkv, 128)
        P.rope_write(self.draft, self.rope, self.zero, self.rope_status, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], self.q,
                     self.k_new, self.v_new, (self.len[:, None] + self.depth[None]).contiguous())
        P.quest_select(self.shape, self.cache, self.q[:, 0].contiguous(), self.budget, self.ids, self.n_ids, self.ws_select, n_recent_pages=1)
        P.tree_attn(self.shape, self.cache, self.tree, self.q, self.ids, self.n_ids, SCALE, self.out, self.tree_status, self.ws)
        self.logits.copy_(self.out.view(B, n, Hq * 128).double() @ self.wo + self.follow[t.long()])
        P.tree_accept(self.logits, t, self.path, self.n_accepted, self.next, self.parent, self.n_nodes)
        P.tree_commit(self.shape, self.cache, self.tree, self.path, self.n_accepted, self.new_len, self.total, self.commit_status)

    def advance(self):
        self.len.copy_(self.new_len)

    def rows(self, b, h, ids, k_new, v_new, q, n):
        """64-bit output of the tree's rows for KV head h over the pages `ids` of the mirrored cache."""
        gq, length = self.heads[0] // self.heads[1], self.lens[b]
        at = torch.tensor([t for p in ids for t in range(16 * p, min(length, 16 * p + 16))], dtype=torch.long)
        pos = torch.tensor([length + d for d in DEPTH[:n]])
        return TR.tree_rows(q[b][:, h * gq:(h + 1) * gq], self.k[b, h][at], self.v[b, h][at], at, k_new[b, h], v_new[b, h], PARENT, n, pos, SCALE)

    def check(self):
        """The step that has just run, and the mirror of the cache brought up to date."""
        Hq, Hkv = self.heads
        gq, words = Hq // Hkv, []
        q, k_new, v_new, out, logits = (x.cpu() for x in (self.q, self.k_new, self.v_new, self.out, self.logits))
        ids, n_ids, tokens = self.ids.cpu(), self.n_ids.cpu(), self.tokens.cpu()
        assert not self.rope_status.any() and not self.tree_status.any() and not self.commit_status.any()
        for b, n in enumerate(NODES):
            for h in range(Hkv):
                o, _, tol, _ = self.rows(b, h, ids[b, h, :int(n_ids[b, h])].tolist(), k_new, v_new, q, n)
                assert ((out[b, :n, h * gq:(h + 1) * gq].double() - o).abs() <= tol).all()
            path, word = TR.accept(logits[b], tokens[b].tolist(), PARENT, n)
            assert self.path[b, :len(path)].tolist() == path and self.n_accepted[b].item() == len(path) and self.next[b].item() == word
            words.append([int(tokens[b, i]) for i in path])
            old = self.lens[b]
            for i, node in enumerate(path):
                self.k[b, :, old + i], self.v[b, :, old + i] = k_new[b, :, node], v_new[b, :, node]
            self.lens[b] = old + len(path)
        assert self.new_len.tolist() == self.lens
        got = self.cache.k.cpu()
        for b, length in enumerate(self.lens):
            assert torch.equal(got[b, :, :length], self.k[b, :, :length])
        return words


def make():
    return Loop((8, 2), 8, 400, [150, 37], 128)


def test_a_loop_of_steps_follows_the_plain_one():
    loop, accepted = make(), 0
    for _ in range(STEPS):
        loop.step()
        accepted += sum(len(w) for w in loop.check())
        loop.advance()
    assert accepted > 2 * STEPS                             # (drafts are taken, else this tests one token per step)


def test_a_captured_step_replayed_gives_the_same_words_and_the_same_cache():
    eager, played = make(), make()
    words = [[], []]
    for loop in (eager, played):
        state = [x.clone() for x in (loop.len, loop.next)] + [getattr(loop.cache, n).clone() for n in NAMES]
        if loop is played:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                loop.step()
            torch.cuda.current_stream().wait_stream(side)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                loop.step()
                loop.advance()
            for x, old in zip([loop.len, loop.next] + [getattr(loop.cache, n) for n in NAMES], state):
                x.copy_(old)
        for _ in range(STEPS):
            if loop is played:
                graph.replay()
            else:
                loop.step()
                loop.advance()
            words[loop is played].append((loop.path.tolist(), loop.n_accepted.tolist(), loop.next.tolist(), loop.out.clone()))
    for (p0, a0, n0, o0), (p1, a1, n1, o1) in zip(*words):
        assert a0 == a1 and n0 == n1 and all(x[:m] == y[:m] for x, y, m in zip(p0, p1, a0))
        assert all(torch.equal(o0[b, :n], o1[b, :n]) for b, n in enumerate(NODES))
    for n in NAMES:
        assert torch.equal(*(getattr(loop.cache, n).view(torch.uint8) for loop in (eager, played))), n      # (bytes: NaN behind the ends)


def test_forked_and_compacted_caches_answer_as_the_first_one():
    loop = make()
    (Hq, Hkv), S, gq = loop.heads, loop.S, loop.heads[0] // loop.heads[1]
    for _ in range(3):
        loop.step()
        loop.check()
        loop.advance()
    loop.step()                                             # a step whose commit is not kept: lens stays as it was
    q, k_new, v_new = (x.cpu() for x in (loop.q, loop.k_new, loop.v_new))
    # both sequences into a cache with three rows: row 0 and 2 from the first one
    B, pages = 3, (loop.T + 15) // 16
    big = P.Cache(k=torch.zeros(B, Hkv, loop.T, 128, dtype=torch.bfloat16, device="cuda"),
                  kmin=torch.zeros(B, Hkv, pages, 128, dtype=torch.bfloat16, device="cuda"),
                  kmax=torch.zeros(B, Hkv, pages, 128, dtype=torch.bfloat16, device="cuda"),
                  v_packed=torch.zeros(B, Hkv, loop.cache.cap_groups, 128 // S, dtype=torch.bfloat16, device="cuda"),
                  v_mask=torch.zeros(B, Hkv, loop.T, dtype=torch.int16, device="cuda"),
                  v_offs=torch.zeros(B, Hkv, loop.T + 1, dtype=torch.int32, device="cuda"), cap_groups=loop.cache.cap_groups)
    rows = [0, 1, 0]
    lens, total, status = i32([0] * B), torch.zeros(B, Hkv, dtype=torch.int64, device="cuda"), i32([[7] * Hkv] * B)
    P.cache_fork(loop.shape, loop.cache, P.Shape(B, Hq, Hkv, S, loop.T), big, i32([0, 0, 1]), i32([0, 2, 1]), lens, total, status)
    assert not status.any() and lens.tolist() == [loop.lens[r] for r in rows]
    tree = P.Tree(loop.k_new[rows].contiguous(), loop.v_new[rows].contiguous(), loop.parent[rows].contiguous(), loop.n_nodes[rows].contiguous())
    shape, qs, ids, n_ids = P.Shape(B, Hq, Hkv, S, loop.T, lens), loop.q[rows].contiguous(), loop.ids[rows].contiguous(), loop.n_ids[rows].contiguous()
    out = torch.zeros(B, loop.n, Hq, 128, device="cuda")
    tree_status, ws = i32([7] * B), Bd.new_workspace(shape, Bd.OP_TREE_ATTN, loop.n)

    def check(cache, shape, ids, n_ids):
        out.fill_(-3)
        P.tree_attn(shape, cache, tree, qs, ids, n_ids, SCALE, out, tree_status, ws)
        assert not tree_status.any()
        for b, r in enumerate(rows):
            for h in range(Hkv):
                o, _, tol, _ = loop.rows(r, h, loop.ids[r, h, :int(loop.n_ids[r, h])].tolist(), k_new, v_new, q, NODES[r])
                assert ((out[b, :NODES[r], h * gq:(h + 1) * gq].cpu().double() - o).abs() <= tol).all()

    check(big, shape, ids, n_ids)
    # only the selected pages stay, in place; whole caches then
    kept = i32([0] * B)
    P.cache_compact(shape, big, ids, n_ids, kept, total, status)
    assert not status.any()
    check(big, P.Shape(B, Hq, Hkv, S, loop.T, kept), None, None)
