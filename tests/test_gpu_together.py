"""The new calls as a decode step uses them: sequences that share a prompt, each with its own tokens behind it.

    rope_write -> append_tokens -> decode_attn (own tokens, scored) -> prefix_attn (the prompt, joined)

eagerly and replayed from one graph, against 64-bit attention over the prompt and the own tokens as one sequence."""
import math

import pytest
import torch

import operators_ref as R
import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)


@pytest.mark.parametrize("heads,S,cap,alibi,window", [((8, 2), 8, 30.0, False, 0), ((4, 4), 16, 0.0, True, 0), ((12, 2), 4, 50.0, True, 150)])
def test_decode_loop_behind_a_shared_prompt(heads, S, cap, alibi, window):
    Hq, Hkv = heads
    B, Tp, T, steps = 5, 197, 48, 20
    gq = Hq // Hkv
    g = torch.Generator().manual_seed(S)
    c = R.make_cache(S, 1, Hkv, Tp, S, S // 2, [Tp], poison=False)
    dev = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor) and k != "dense"}
    p_shape = P.Shape(1, Hq, Hkv, S, Tp, torch.tensor([Tp], dtype=torch.int32, device="cuda"))
    prompt = P.Cache(k=dev["k"], v_packed=dev["v_packed"], v_mask=dev["v_mask"], v_offs=dev["v_offs"], cap_groups=c["cap"])
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / Hq) for h in range(Hq)])
    f, scale = P.rope_frequencies(64, 10000.0, P.ROPE_YARN, factor=4.0, original_len=4096.0)
    rope = P.Rope(f.cuda(), interleaved=False, scale=scale)
    tokens = torch.randn(steps, B, 1, Hq + 2 * Hkv, 128, generator=g).to(torch.bfloat16).cuda()

    def state():
        i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
        length = i32(B)
        shape = P.Shape(B, Hq, Hkv, S, T, length)
        k = torch.zeros(B, Hkv, T, 128, dtype=torch.bfloat16, device="cuda")
        s = dict(shape=shape, cache=P.Cache.allocate(shape, k, T * S), v=torch.zeros_like(k), old=i32(B) - 1, length=length,
                 pos=i32(B, 1), q_pos=i32(B), abs_pos=i32(B), qkv=torch.zeros_like(tokens[0]),
                 q=torch.zeros(B, 1, Hq, 128, dtype=torch.bfloat16, device="cuda"), rope_status=i32(B), status=i32(B, Hkv),
                 total=torch.zeros(B, Hkv, dtype=torch.int64, device="cuda"), start=torch.tensor([0, B], dtype=torch.int32, device="cuda"))
        s["old"].zero_()
        s["slopes"] = slopes.cuda() if alibi else None
        for n in ("own", "out"):
            s[n], s[n + "_lse"] = torch.zeros(B, Hq, 128, device="cuda"), torch.zeros(B, Hq, device="cuda")
        s["ws"] = Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, shape.n_pages)
        s["p_ws"] = Bd.new_workspace(p_shape, Bd.OP_PREFIX_ATTN, B)
        return s

    def step(s):
        s["length"].copy_(s["old"] + 1)
        s["q_pos"].copy_(s["old"])
        s["abs_pos"].copy_(s["old"] + Tp)
        s["pos"].copy_((s["old"] + Tp)[:, None])
        qkv, cache = s["qkv"], s["cache"]
        P.rope_write(s["shape"], rope, s["old"], s["rope_status"], q_in=qkv[:, :, :Hq], k_in=qkv[:, :, Hq:Hq + Hkv], v_in=qkv[:, :, Hq + Hkv:],
                     q_out=s["q"], k=cache.k, v=s["v"], positions=s["pos"])
        P.append_tokens(s["shape"], cache, s["v"], s["old"], 1, s["total"], s["status"])
        q = s["q"][:, 0]
        P.decode_attn(s["shape"], cache, q, None, None, SCALE, s["own"], s["ws"], lse=s["own_lse"],
                      score=P.Score(cap, s["slopes"], s["q_pos"], window))
        P.prefix_attn(p_shape, prompt, q, s["start"], SCALE, s["out"], s["p_ws"], lse=s["out_lse"],
                      score=P.Score(cap, s["slopes"], s["abs_pos"], window), own_out=s["own"], own_lse=s["own_lse"])
        s["old"].add_(1)

    eager, replayed = state(), state()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(replayed)
    for n in range(steps):
        eager["qkv"].copy_(tokens[n])
        replayed["qkv"].copy_(tokens[n])
        step(eager)
        graph.replay()
        torch.cuda.synchronize()
        assert eager["rope_status"].eq(0).all() and eager["status"].eq(0).all()
        for name in ("q", "own", "own_lse", "out", "out_lse"):
            assert torch.equal(eager[name], replayed[name]), name
        if n not in (0, 1, 16, steps - 1):
            continue
        own_k, own_v, q = eager["cache"].k.cpu(), eager["v"].cpu(), eager["q"][:, 0].cpu()
        at = torch.arange(Tp + n + 1)
        for b in range(B):
            for h in range(Hkv):
                hs = slice(h * gq, (h + 1) * gq)
                k = torch.cat([c["k"][0, h], own_k[b, h, :n + 1]])
                v = torch.cat([c["dense"][0, h], own_v[b, h, :n + 1].double()])
                o, l, to, tl = R.scored_rows(q[b, hs], k, v, at, torch.full((gq,), Tp + n), SCALE, cap, slopes[hs] if alibi else None, window,
                                             n_seq=Tp + 256)
                # the join adds roundings of the two log-sum-exps and of the weights they give
                extra = 16 * R.EPS32 * (1 + l.abs())
                R.assert_rows(eager["out"][b, hs], eager["out_lse"][b, hs], o, l, to + extra[:, None] * (o.abs() + v.abs().max()), tl + extra)
