"""Bad arguments of the calls on drafted trees and whole caches are refused before any launch."""
import ctypes as C

import pytest
import torch

import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd
from paper_2604_21335_b200 import build as B

FAKE, ODD, ELSE = C.c_void_p(0x1000), C.c_void_p(0x1008), C.c_void_p(0x2000)
FULL = Bd._Cache(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 100)


@pytest.fixture(scope="module")
def lib():
    B.build()
    return P.load_library()


def tree(k=0x1000, v=0x1000, parent=0, nodes=0, cap=8, reserved=0):
    return Bd._PACK_TREE(k, v, parent, nodes, cap, reserved)


def shape(batch=2, hq=8, hkv=4, S=8, T=4096, **kw):
    return P.Shape(batch, hq, hkv, S, T, **kw).c()


def test_tree_attention(lib):
    def call(shp=shape(), cache=FULL, tr=tree(), q=FAKE, ids=FAKE, n=FAKE, most=4, scale=0.1, score=None, out=FAKE, status=FAKE, ws=FAKE, ws_bytes=16):
        return lib.stc_tree_attn(C.byref(shp), C.byref(cache), tr, q, ids, n, most, scale, score and C.byref(score), out, None, status, ws,
                                 ws_bytes, None)

    assert call() == 3                           # valid but for the workspace
    assert call(ws=C.c_void_p(0x1010), ws_bytes=1 << 40) == 3
    for kw, code in [(dict(tr=None), 1), (dict(tr=tree(cap=0)), 1), (dict(tr=tree(cap=129)), 1), (dict(tr=tree(reserved=1)), 1),
                     (dict(tr=tree(k=0)), 1), (dict(tr=tree(v=0)), 1), (dict(tr=tree(k=0x1008)), 1), (dict(q=None), 1), (dict(q=ODD), 1),
                     (dict(out=None), 1), (dict(out=ODD), 1), (dict(status=None), 1), (dict(n=None), 1), (dict(most=-1), 1),
                     (dict(scale=float("nan")), 1), (dict(cache=Bd._Cache()), 1), (dict(score=Bd._Score(-1.0, 0)), 1),
                     (dict(score=Bd._Score(0.0, -1)), 1), (dict(score=Bd._Score(0.0, 0, None, None, FAKE, None)), 1),
                     (dict(shp=shape(hq=72, hkv=4)), 2), (dict(shp=P.Shape(2, 8, 4, 8, 64, head_dim=64).c()), 2),
                     (dict(shp=shape(batch=200, hq=8, hkv=8, T=(1 << 27) - 16)), 2), (dict(shp=shape(batch=1 << 22, hq=64, hkv=8, T=8), tr=tree(cap=128)), 2),
                     (dict(shp=shape(batch=0)), 0)]:
        assert call(**kw) == code, kw
    assert call(ids=None, n=None) == 3 and call(score=Bd._Score(30.0, 5, FAKE, FAKE, FAKE, FAKE)) == 3
    s = P.Shape(2, 8, 4, 8, 4096)
    n = P.workspace_bytes(s, Bd.OP_TREE_ATTN, 8)
    assert n > 0 and n % 256 == 0 and P.workspace_bytes(s, Bd.OP_TREE_ATTN, 0) == 0
    assert P.workspace_bytes(P.Shape(2, 8, 4, 8, 0), Bd.OP_TREE_ATTN, 4) > 0
    for bad in (-1, 129):
        with pytest.raises(P.StcError):
            P.workspace_bytes(s, Bd.OP_TREE_ATTN, bad)


def test_tree_accept(lib):
    def call(batch=2, cap=8, vocab=100, logits=FAKE, kind=0, step=100, tokens=FAKE, path=FAKE, count=FAKE, nxt=FAKE):
        return lib.stc_tree_accept(batch, cap, vocab, logits, kind, step, tokens, None, None, path, count, nxt, None)

    for kw, code in [(dict(batch=-1), 1), (dict(cap=0), 1), (dict(cap=129), 1), (dict(vocab=0), 1), (dict(step=99), 1), (dict(step=1 << 41), 1),
                     (dict(kind=2), 1), (dict(logits=None), 1), (dict(logits=C.c_void_p(0x1001)), 1), (dict(logits=C.c_void_p(0x1002), kind=1), 1),
                     (dict(tokens=None), 1), (dict(path=None), 1), (dict(count=None), 1), (dict(nxt=None), 1), (dict(batch=1 << 24), 2),
                     (dict(batch=0), 0)]:
        assert call(**kw) == code, kw


def test_tree_commit(lib):
    s = shape()
    s.seq_len = 0x3000

    def call(shp=s, cache=FULL, tr=tree(), path=FAKE, n=FAKE, new_len=ELSE, total=FAKE, status=FAKE):
        return lib.stc_tree_commit(C.byref(shp), C.byref(cache), tr, path, n, new_len, total, status, None)

    half = Bd._Cache(FAKE, FAKE, None, FAKE, FAKE, FAKE, 100)
    for kw, code in [(dict(tr=tree(cap=0)), 1), (dict(tr=tree(v=0)), 1), (dict(tr=tree(v=0x1004)), 1), (dict(cache=Bd._Cache()), 1),
                     (dict(cache=half), 1), (dict(cache=Bd._Cache(FAKE, None, None, ODD, FAKE, FAKE, 100)), 1),
                     (dict(cache=Bd._Cache(FAKE, None, None, FAKE, FAKE, FAKE, -1)), 1), (dict(path=None), 1), (dict(n=None), 1),
                     (dict(new_len=None), 1), (dict(new_len=C.c_void_p(0x3000)), 1), (dict(total=None), 1), (dict(status=None), 1),
                     (dict(shp=shape(S=5)), 2), (dict(shp=shape(batch=0)), 0), (dict(shp=shape(T=0)), 0)]:
        assert call(**kw) == code, kw


def test_cache_fork(lib):
    def call(a=shape(), src=FULL, b=shape(batch=5, T=9000), dst=Bd._Cache(ELSE, FAKE, FAKE, FAKE, FAKE, FAKE, 100), n=3, s=FAKE, d=FAKE, new_len=FAKE,
             total=FAKE, status=FAKE):
        return lib.stc_cache_fork(C.byref(a), C.byref(src), C.byref(b), C.byref(dst), n, s, d, new_len, total, status, None)

    bare = Bd._Cache(FAKE, None, None, FAKE, FAKE, FAKE, 100)
    for kw, code in [(dict(n=-1), 1), (dict(n=4097), 2), (dict(s=None), 1), (dict(d=None), 1), (dict(new_len=None), 1), (dict(total=None), 1),
                     (dict(status=None), 1), (dict(src=Bd._Cache()), 1), (dict(dst=Bd._Cache()), 1), (dict(src=bare), 1),
                     (dict(b=shape(hkv=8)), 1), (dict(b=shape(S=16)), 1), (dict(b=shape(hq=4)), 1), (dict(dst=FULL), 1),
                     (dict(dst=FULL, b=shape(), n=0), 0), (dict(n=0), 0), (dict(a=shape(batch=0)), 0), (dict(b=shape(T=0)), 0),
                     (dict(dst=Bd._Cache(FAKE, FAKE, FAKE, ELSE, FAKE, FAKE, 100), b=shape()), 1),
                     (dict(dst=Bd._Cache(FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 99), b=shape()), 1),
                     (dict(dst=Bd._Cache(C.c_void_p(0x2008), FAKE, FAKE, FAKE, FAKE, FAKE, 100)), 1)]:
        assert call(**kw) == code, kw


def test_cache_compact(lib):
    def call(a=shape(), src=FULL, ids=FAKE, n=FAKE, most=4, b=shape(T=64), dst=Bd._Cache(ELSE, FAKE, FAKE, FAKE, FAKE, FAKE, 100), new_len=FAKE,
             total=FAKE, status=FAKE):
        return lib.stc_cache_compact(C.byref(a), C.byref(src), ids, n, most, C.byref(b), C.byref(dst), new_len, total, status, None)

    bare = Bd._Cache(FAKE, None, None, FAKE, FAKE, FAKE, 100)
    for kw, code in [(dict(most=-1), 1), (dict(ids=None), 1), (dict(n=None), 1), (dict(new_len=None), 1), (dict(total=None), 1), (dict(status=None), 1),
                     (dict(src=bare), 1), (dict(src=Bd._Cache()), 1), (dict(b=shape(batch=3)), 1), (dict(b=shape(S=4)), 1), (dict(dst=FULL), 1),
                     (dict(dst=Bd._Cache(FAKE, ELSE, FAKE, FAKE, FAKE, FAKE, 100), b=shape()), 1),
                     (dict(dst=Bd._Cache(FAKE, FAKE, FAKE, FAKE, ELSE, FAKE, 100), b=shape()), 1), (dict(a=shape(batch=0), b=shape(batch=0)), 0),
                     (dict(b=shape(T=0)), 0)]:
        assert call(**kw) == code, kw


def test_tensors_are_checked_in_the_same_words_with_and_without_the_native_module(lib, monkeypatch):
    assert Bd._native_addresses is not None, "the build makes the native argument check"
    monkeypatch.setattr(Bd, "_current_device", lambda: 0)
    i, bf = lambda *s: torch.zeros(*s, dtype=torch.int32), lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    sh = P.Shape(2, 8, 4, 8, 32, i(2))
    cache = P.Cache(k=bf(2, 4, 32, 128), kmin=bf(2, 4, 2, 128), kmax=bf(2, 4, 2, 128), v_packed=bf(2, 4, 50, 16), v_mask=i(2, 4, 32).short(),
                    v_offs=i(2, 4, 33), cap_groups=50)
    tr, f = P.Tree(bf(2, 4, 3, 128), bf(2, 4, 3, 128)), torch.zeros(2, 3, 8, 128)
    total = torch.zeros(2, 4, dtype=torch.int64)
    cases = [lambda: P.tree_attn(sh, cache, tr, f.bfloat16(), None, None, 1.0, f, i(2), i(9)),
             lambda: P.tree_attn(sh, cache, tr, f[:, :2].bfloat16(), None, None, 1.0, f, i(2), i(9)),
             lambda: P.tree_attn(sh, cache, P.Tree(tr.k, tr.v[:, :, :2]), f.bfloat16(), None, None, 1.0, f, i(2), i(9)),
             lambda: P.tree_attn(sh, cache, tr, f.bfloat16(), None, None, 1.0, f, i(2), i(9), score=P.Score(q_doc=i(3))),
             lambda: P.tree_accept(torch.zeros(2, 3, 5), i(2, 3), i(2, 3), i(2), i(2)),
             lambda: P.tree_commit(sh, cache, tr, i(2, 3), i(2), i(2), total, i(2, 4)),
             lambda: P.tree_commit(sh, cache, tr, i(2, 3), i(2), i(2), total, i(2)),
             lambda: P.tree_commit(sh, P.Cache(**{**vars(cache), "v_mask": i(2, 4, 32)}), tr, i(2, 3), i(2), i(2), total, i(2, 4)),
             lambda: P.cache_fork(sh, cache, sh, cache, i(2), i(3), i(2), total, i(2, 4)),
             lambda: P.cache_compact(sh, cache, i(2, 4, 2), i(2, 4), i(2), total, i(2, 4)),
             lambda: P.cache_compact(sh, cache, i(2, 4, 2), i(2, 4), i(2), total, i(2, 4), dst=cache)]

    def said(f):
        with pytest.raises(ValueError) as e:
            f()
        return str(e.value)

    native = [said(f) for f in cases]
    for name in ("_native_addresses", "_sizes_are", "_native_token_rows"):
        monkeypatch.setattr(Bd, name, None)
    assert [said(f) for f in cases] == native
