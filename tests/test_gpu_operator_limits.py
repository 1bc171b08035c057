"""The rotary write, the scored attention and the shared-prefix attention at the edges of what they accept: infinities and NaN in
keys that are seen, caches whose offsets pass 32 bits, calls that run at the same time."""
import math

import pytest
import torch

import operators_ref as R
import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd

pytestmark = pytest.mark.gpu
SCALE = 1 / math.sqrt(128)


def setup(seed, lens, T, Hq, Hkv, rows):
    """A routed cache on the device, its CPU copy, and positive queries (an infinite key channel then gives an infinite score)."""
    c = R.make_cache(seed, len(lens), Hkv, T, 8, 4, lens)
    q = (torch.rand(rows, Hq, 128, generator=torch.Generator().manual_seed(seed)) + 0.25).to(torch.bfloat16)
    return c, q


def on_device(c, lens, T, Hq, Hkv):
    dev = {k: v.cuda() for k, v in c.items() if isinstance(v, torch.Tensor) and k != "dense"}
    shape = P.Shape(len(lens), Hq, Hkv, 8, T, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    return shape, P.Cache(k=dev["k"], v_packed=dev["v_packed"], v_mask=dev["v_mask"], v_offs=dev["v_offs"], cap_groups=c["cap"])


def scored(c, q, lens, T, Hq, Hkv, score):
    shape, cache = on_device(c, lens, T, Hq, Hkv)
    out, lse = torch.empty(len(lens), Hq, 128, device="cuda"), torch.empty(len(lens), Hq, device="cuda")
    ws = Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, shape.n_pages)
    P.decode_attn(shape, cache, q.cuda(), None, None, SCALE, out, ws, lse=lse, score=score)
    return out.cpu(), lse.cpu()


def prefix(c, q, lens, T, Hq, Hkv, starts, score=None):
    shape, cache = on_device(c, lens, T, Hq, Hkv)
    out, lse = torch.empty(q.shape[0], Hq, 128, device="cuda"), torch.empty(q.shape[0], Hq, device="cuda")
    ws = Bd.new_workspace(shape, Bd.OP_PREFIX_ATTN, q.shape[0])
    P.prefix_attn(shape, cache, q.cuda(), torch.tensor(starts, dtype=torch.int32, device="cuda"), SCALE, out, ws, lse=lse, score=score)
    return out.cpu(), lse.cpu()


def hide(c, which, tokens):
    """Scores of -inf: those keys hold one -inf and zeros."""
    c["k"][which, :, tokens] = 0.0
    c["k"][which, :, tokens, 3] = -math.inf


@pytest.mark.parametrize("heads", [(4, 4), (12, 2), (1, 1)])
def test_scored_keys_that_give_minus_infinity_are_tokens_without_weight(heads):
    """Whole pages, a whole sequence, the last tokens; one head of a pair alone among several."""
    Hq, Hkv = heads
    lens, T = [200, 90, 16 * 40], 16 * 40
    c, q = setup(1, lens, T, Hq, Hkv, 3)
    hide(c, 0, slice(0, 100))
    hide(c, 1, slice(0, 90))
    hide(c, 2, slice(17, 16 * 40))
    gq = Hq // Hkv
    if gq > 1:                                   # head 1 of every KV head turns its -inf into +0: negative there, no other token infinite
        q[2, 1::gq, 3] = 0.0
        c["k"][2, :, 17:, 3] = torch.where(torch.arange(T - 17) % 2 == 0, -3e38, 0.5).to(torch.bfloat16)
    out, lse = scored(c, q, lens, T, Hq, Hkv, P.Score(window=10 ** 6))
    for b, n in enumerate(lens):
        for h in range(Hkv):
            hs = slice(h * gq, (h + 1) * gq)
            at, k = torch.arange(n), c["k"][b, h, :n].double()
            x = torch.where(torch.isinf(k).any(1), -math.inf, q[b, hs].double() @ torch.where(torch.isinf(k), 0.0, k).T * SCALE)
            x = torch.where(x < -1e30, -math.inf, x)                     # (no weight left in any format)
            w = torch.exp(x - x.max(1, keepdim=True).values.clamp(min=-1e30))
            l = w.sum(1)
            want = torch.where(l[:, None] > 0, w @ c["dense"][b, h, :n] / l.clamp(min=1e-300)[:, None], 0.0)
            # |q.k| stays below 128 * 8 * 1.25 * 5 / 11.3: scores are good to 1e-3, weights and outputs (|v| < 6) to 2e-3 of themselves
            assert ((out[b, hs].double() - want).abs() <= 0.02).all()
            assert (torch.isinf(lse[b, hs]) == (l == 0)).all()


@pytest.mark.parametrize("heads,T", [((4, 4), 640), ((12, 2), 640), ((1, 1), 16 * 1300), ((8, 1), 16 * 1300)])
def test_scored_nan_in_a_seen_key_reaches_its_sequence_only(heads, T):
    Hq, Hkv = heads
    lens = [T, T - 5]
    c, q = setup(2, lens, T, Hq, Hkv, 2)
    clean = scored(c, q, lens, T, Hq, Hkv, P.Score(softcap=30.0, window=T // 2))
    c["k"][0, 0, T - 20, 7] = math.nan
    c["k"][1, 0, 3, 7] = math.nan                # outside the window
    got = scored(c, q, lens, T, Hq, Hkv, P.Score(softcap=30.0, window=T // 2))
    gq = Hq // Hkv
    assert got[0][0, :gq].isnan().all() and got[1][0, :gq].isnan().all()
    assert torch.equal(got[0][0, gq:], clean[0][0, gq:]) and torch.equal(got[0][1], clean[0][1]) and torch.equal(got[1][1], clean[1][1])


@pytest.mark.parametrize("rows", [2, 20, 150])
@pytest.mark.parametrize("T", [60, 900, 9000])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_prefix_nan_in_a_seen_key_and_in_a_query(rows, T, cap):
    """In the first case all rows of the KV head are NaN, in the second that row's heads; nothing else moves."""
    Hq, Hkv, lens, starts = 8, 4, [T, T], [0, rows, rows + 3]
    c, q = setup(3, lens, T, Hq, Hkv, rows + 3)
    score = P.Score(softcap=cap) if cap else None
    clean = prefix(c, q, lens, T, Hq, Hkv, starts, score)
    assert torch.isfinite(clean[0]).all()
    q[1, 0] = math.nan
    got = prefix(c, q, lens, T, Hq, Hkv, starts, score)
    keep = torch.ones(rows + 3, Hq, dtype=torch.bool)
    keep[1, 0] = False
    for a, b in zip(got, clean):
        assert a[~keep].isnan().all() and not a[keep].isnan().any()
        assert (a[keep] - b[keep]).abs().max() <= 1e-4           # (a NaN row moves no maximum of its own, so others may be regrouped)
    q = setup(3, lens, T, Hq, Hkv, rows + 3)[1]
    c["k"][0, 2, T // 3, 100] = math.nan
    got = prefix(c, q, lens, T, Hq, Hkv, starts, score)
    keep = torch.ones(rows + 3, Hq, dtype=torch.bool)
    keep[:rows, 4:6] = False
    for a, b in zip(got, clean):
        assert a[~keep].isnan().all() and torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("heads", [(28, 4), (12, 2), (8, 1)])
@pytest.mark.parametrize("options", [dict(), dict(softcap=30.0), dict(softcap=30.0, slopes=True)], ids=lambda o: "+".join(o) or "plain")
def test_prefix_bits_do_not_depend_on_what_ran_before(heads, options):
    """Tiles that rows do not fill keep what an earlier call left in shared memory; none of it may reach a result."""
    Hq, Hkv = heads
    lens, T, starts, n = [900, 333], 900, [0, 6, 25], 25
    c, q = setup(9, lens, T, Hq, Hkv, n)
    q = torch.randn(n, Hq, 128, generator=torch.Generator().manual_seed(9)).to(torch.bfloat16)
    score = P.Score(options.get("softcap", 0.0), q_pos=torch.full((n,), T, dtype=torch.int32, device="cuda"),
                    slopes=torch.full((Hq,), 0.01, device="cuda") if "slopes" in options else None)
    first = prefix(c, q, lens, T, Hq, Hkv, starts, score)
    other, other_q = setup(10, [900], 900, 32, 4, 64)
    for scale in (0.0, 1e4, math.nan):
        prefix(other, other_q * scale, [900], 900, 32, 4, [0, 64], P.Score(softcap=20.0))
        again = prefix(c, q, lens, T, Hq, Hkv, starts, score)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_prefix_keys_that_give_minus_infinity_are_tokens_without_weight():
    lens, T, starts = [700, 64, 300], 700, [0, 5, 7, 40]
    c, q = setup(4, lens, T, 8, 4, 40)
    clean = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    hide(c, 0, slice(100, 700))
    hide(c, 1, slice(0, 64))
    hide(c, 2, slice(0, 290))
    out, lse = prefix(c, q, lens, T, 8, 4, starts)
    doc = torch.full((3, T), -1, dtype=torch.int32)                      # the same tokens hidden by the mask
    doc[0, 100:], doc[1], doc[2, :290] = 5, 5, 5
    score = P.Score(tok_doc=doc.cuda(), q_doc=torch.zeros(40, dtype=torch.int32, device="cuda"))
    want, want_lse = prefix(clean, q, lens, T, 8, 4, starts, score)
    assert torch.equal(out, want) and torch.equal(lse, want_lse) and (lse[5:7] == -math.inf).all() and (out[5:7] == 0).all()


def test_offsets_beyond_32_bits():
    """Keys of 4.6 GB: the last KV head starts behind 2^31 elements; written, then read by both attentions."""
    Hq, Hkv, S, T = 16, 8, 4, 2_250_000 + 5
    g = torch.Generator(device="cuda").manual_seed(5)
    k = torch.empty(1, Hkv, T, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    assert k.numel() > 2 ** 31
    for h in range(Hkv):
        k[0, h] = torch.randn(T, 128, generator=g, device="cuda").to(torch.bfloat16)
    # every token keeps one group of 32 channels, group t % 4
    packed = torch.empty(1, Hkv, T, 32, dtype=torch.bfloat16, device="cuda")
    packed.normal_(generator=g)
    mask = (1 << (torch.arange(T, device="cuda") % 4)).to(torch.int16).expand(1, Hkv, T).contiguous()
    offs = torch.arange(T + 1, dtype=torch.int32, device="cuda").expand(1, Hkv, T + 1).contiguous()
    length = torch.tensor([T], dtype=torch.int32, device="cuda")
    shape = P.Shape(1, Hq, Hkv, S, T, length)
    cache = P.Cache(k=k, v_packed=packed, v_mask=mask, v_offs=offs, cap_groups=T)
    # the last token's key comes from a projection, unrotated channels included
    new = torch.randn(1, 1, Hkv, 128, generator=g, device="cuda").to(torch.bfloat16)
    f, _ = P.rope_frequencies(64)
    old, status = length - 1, torch.ones(1, dtype=torch.int32, device="cuda")
    P.rope_write(shape, P.Rope(f.cuda()), old, status, k_in=new, k=k, v_in=new, v=v)
    want, tol = R.rope_ref(new[0, 0].cpu(), torch.tensor(T - 1), f, False, 1.0)
    assert ((k[0, :, T - 1].cpu().double() - want).abs() <= tol + 2.0 ** -30).all() and torch.equal(v[0, :, T - 1], new[0, 0])

    q = torch.randn(1, Hq, 128, generator=g, device="cuda").to(torch.bfloat16)
    window = 4000
    score = P.Score(window=window, q_pos=old, softcap=20.0)
    out, lse = torch.empty(2, 1, Hq, 128, device="cuda"), torch.empty(2, 1, Hq, device="cuda")
    P.decode_attn(shape, cache, q, None, None, SCALE, out[0], Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, shape.n_pages), lse=lse[0], score=score)
    ws = Bd.new_workspace(shape, Bd.OP_PREFIX_ATTN, 1)
    P.prefix_attn(shape, cache, q, torch.tensor([0, 1], dtype=torch.int32, device="cuda"), SCALE, out[1], ws, lse=lse[1], score=score)
    torch.cuda.synchronize()
    at = torch.arange(T - window, T)
    for h in range(Hkv):
        dense = torch.zeros(window, 4, 32, dtype=torch.float64)
        dense[torch.arange(window), at % 4] = packed[0, h, T - window:].cpu().double()
        ref = R.scored_rows(q[0, 2 * h:2 * h + 2].cpu(), k[0, h, T - window:].cpu(), dense.reshape(window, 128), at, torch.tensor([T - 1] * 2),
                            SCALE, softcap=20.0, window=window)
        for i in range(2):
            R.assert_rows(out[i, 0, 2 * h:2 * h + 2], lse[i, 0, 2 * h:2 * h + 2], *ref)


def test_calls_on_two_streams_at_once():
    """Own workspaces and outputs, one cache: the bits of calls made one after the other."""
    lens, T, Hq, Hkv, rows = [3000, 2500], 3000, 16, 4, 40
    c, q = setup(6, lens, T, Hq, Hkv, rows)
    shape, cache = on_device(c, lens, T, Hq, Hkv)
    q, start = q.cuda(), torch.tensor([0, 15, 40], dtype=torch.int32, device="cuda")
    score = P.Score(softcap=25.0, window=2000, q_pos=torch.tensor([2999, 2400], dtype=torch.int32, device="cuda"))

    def buffers():
        return dict(own=torch.zeros(2, Hq, 128, device="cuda"), lse=torch.zeros(2, Hq, device="cuda"), out=torch.zeros(rows, Hq, 128, device="cuda"),
                    ws_a=Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, shape.n_pages), ws_p=Bd.new_workspace(shape, Bd.OP_PREFIX_ATTN, rows))

    def calls(s):
        P.decode_attn(shape, cache, q[:2], None, None, SCALE, s["own"], s["ws_a"], lse=s["lse"], score=score)
        P.prefix_attn(shape, cache, q, start, SCALE, s["out"], s["ws_p"])

    alone = buffers()
    calls(alone)
    torch.cuda.synchronize()
    both, streams = [buffers(), buffers()], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(10):
        for s, st in zip(both, streams):
            with torch.cuda.stream(st):
                calls(s)
    torch.cuda.synchronize()
    for s in both:
        assert all(torch.equal(s[name], alone[name]) for name in ("own", "lse", "out"))


@pytest.mark.parametrize("heads", [(8, 8), (8, 2)])
def test_scored_lists_without_pages_attend_nothing(heads):
    c, q = setup(8, [64, 30], 64, *heads, 2)
    shape, cache = on_device(c, [64, 30], 64, *heads)
    out, lse = torch.ones(2, heads[0], 128, device="cuda"), torch.ones(2, heads[0], device="cuda")
    for pages in (0, 3):
        ids = torch.zeros(2, heads[1], pages, dtype=torch.int32, device="cuda")
        n = torch.zeros(2, heads[1], dtype=torch.int32, device="cuda")
        P.decode_attn(shape, cache, q.cuda(), ids, n, SCALE, out.fill_(1), Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, pages),
                      lse=lse.fill_(1), score=P.Score(softcap=5.0))
        assert (out == 0).all() and (lse == -math.inf).all()


def test_scored_sizes_that_do_not_fit_are_refused():
    c, q = setup(7, [64], 64, 8, 8, 1)
    shape, cache = on_device(c, [64], 64, 8, 8)
    q, score = q.cuda(), P.Score(softcap=5.0)
    ws = Bd.new_workspace(shape, Bd.OP_DECODE_ATTN, 4)
    out, lse = torch.zeros(1, 8, 128, device="cuda"), torch.zeros(1, 8, device="cuda")
    ids, n = torch.zeros(1, 8, 4, dtype=torch.int32, device="cuda"), torch.ones(1, 8, dtype=torch.int32, device="cuda")
    P.decode_attn(shape, cache, q, ids, n, SCALE, out, ws, lse=lse, score=score)
    for bad in (dict(q=q[:, :4].contiguous()), dict(out=out[:, :4].contiguous()), dict(lse=lse[:, :4].contiguous()),
                dict(ids=ids[:, :4].contiguous()), dict(n=n[:, :4].contiguous())):
        a = {**dict(q=q, out=out, lse=lse, ids=ids, n=n), **bad}
        with pytest.raises(ValueError):
            P.decode_attn(shape, cache, a["q"], a["ids"], a["n"], SCALE, a["out"], ws, lse=a["lse"], score=score)
