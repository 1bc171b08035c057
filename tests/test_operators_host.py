"""Host side of the rotary and scored calls: frequency tables, and bad arguments refused before any launch."""
import ctypes as C
import math

import pytest
import torch

import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd
from paper_2604_21335_b200 import build as B


@pytest.fixture(scope="module")
def lib():
    B.build()
    return P.load_library()


@pytest.mark.parametrize("rot", [16, 64, 128])
def test_unscaled_and_linear_tables(lib, rot):
    f, s = P.rope_frequencies(rot, 10000.0)
    want = [10000.0 ** (-2.0 * i / rot) for i in range(rot // 2)]
    assert s == 1.0 and all(abs(a - b) <= 1e-15 * b for a, b in zip(f.tolist(), want))
    g, s = P.rope_frequencies(rot, 10000.0, P.ROPE_LINEAR, factor=4.0)
    assert s == 1.0 and all(abs(a - b / 4) <= 1e-15 * b for a, b in zip(g.tolist(), want))


def test_banded_table_keeps_fast_pairs_and_slows_slow_ones(lib):
    f, _ = P.rope_frequencies(128, 500000.0)
    g, s = P.rope_frequencies(128, 500000.0, P.ROPE_BANDS, factor=8.0, original_len=8192.0, low=1.0, high=4.0)
    assert s == 1.0
    for a, b in zip(f.tolist(), g.tolist()):
        turns = 8192.0 * a / (2 * math.pi)
        keep = min(max((turns - 1.0) / 3.0, 0.0), 1.0)
        assert abs(b - (keep * a + (1 - keep) * a / 8.0)) <= 1e-14 * a
    assert g[0] == f[0] and abs(g[-1] * 8 - f[-1]) <= 1e-15


def test_ramped_table_and_its_scale(lib):
    f, _ = P.rope_frequencies(128, 10000.0)
    g, s = P.rope_frequencies(128, 10000.0, P.ROPE_YARN, factor=4.0, original_len=32768.0)
    assert abs(s - (0.1 * math.log(4.0) + 1.0)) <= 2.0 ** -23 * 2
    share = (g / f - 0.25) / 0.75                # 1 = kept, 0 = interpolated
    assert abs(share[0] - 1) < 1e-12 and abs(share[-1]) < 1e-12
    assert (share[1:] <= share[:-1] + 1e-12).all()
    pair = lambda turns: 128 * math.log(32768.0 / (turns * 2 * math.pi)) / (2 * math.log(10000.0))  # noqa: E731
    lo, hi = math.floor(pair(32.0)), min(math.ceil(pair(1.0)), 127)
    assert abs(share[lo] - 1) < 1e-12 and share[lo + 1] < 1 and all(share[hi:].abs() < 1e-12)


def test_frequency_refusals(lib):
    for bad, code in [(dict(rot_dim=20), 2), (dict(rot_dim=144), 1), (dict(rot_dim=-16), 1), (dict(rot_dim=64, base=1.0), 1),
                      (dict(rot_dim=64, base=float("inf")), 1), (dict(rot_dim=64, scaling=4), 1),
                      (dict(rot_dim=64, scaling=P.ROPE_LINEAR, factor=0.5), 1),
                      (dict(rot_dim=64, scaling=P.ROPE_YARN, factor=4.0), 1),
                      (dict(rot_dim=64, scaling=P.ROPE_BANDS, factor=4.0, original_len=8192.0, low=4.0, high=1.0), 1)]:
        with pytest.raises(P.StcError) as e:
            P.rope_frequencies(**bad)
        assert e.value.code == code, bad
    assert P.rope_frequencies(0)[0].numel() == 0


def test_rope_write_refusals(lib):
    shape = P.Shape(2, 8, 4, 8, 64).c()
    fake, odd = C.c_void_p(0x1000), C.c_void_p(0x1008)

    def call(rot=64, inter=0, reserved=0, freq=fake, old=fake, max_new=1, q=fake, qs=1024, k=fake, ks=512, v=fake, vs=512,
             q_out=fake, k_out=fake, v_out=fake, status=fake, shp=shape):
        r = Bd._Rope(freq, rot, inter, 1.0, reserved)
        return lib.stc_rope_write(C.byref(shp), C.byref(r), old, max_new, None, q, qs, k, ks, v, vs, q_out, k_out, v_out,
                                  status, None)

    for kw, code in [(dict(rot=24), 2), (dict(rot=144), 1), (dict(rot=-16), 1), (dict(inter=2), 1), (dict(reserved=1), 1),
                     (dict(freq=None), 1), (dict(freq=C.c_void_p(0x1004)), 1), (dict(old=None), 1), (dict(status=None), 1),
                     (dict(max_new=-1), 1), (dict(q=None), 1), (dict(k_out=None), 1), (dict(qs=1016), 1), (dict(qs=1025), 1),
                     (dict(ks=-512), 1), (dict(q=odd), 1), (dict(v_out=odd), 1),
                     (dict(q=None, q_out=None, k=None, k_out=None, v=None, v_out=None), 1)]:
        assert call(**kw) == code, kw
    assert lib.stc_rope_write(C.byref(shape), None, fake, 1, None, fake, 1024, None, 0, None, 0, fake, None, None, fake, None) == 1
    assert call(max_new=0) == 0                  # nothing to do, nothing enqueued
    assert call(shp=P.Shape(0, 8, 4, 8, 64).c()) == 0


def test_scored_attention_refusals(lib):
    cs = P.Shape(1, 8, 8, 8, 4096).c()
    fake = C.c_void_p(0x1000)
    cc = Bd._Cache(fake, fake, fake, fake, fake, fake, 100)

    def call(score):
        return lib.stc_decode_attn_scored(C.byref(cs), C.byref(cc), fake, fake, fake, 64, 0.1, C.byref(score), fake, None, fake,
                                          16, None)

    assert call(Bd._Score(-1.0, 0)) == 1
    assert call(Bd._Score(float("nan"), 0)) == 1
    assert call(Bd._Score(0.0, -3)) == 1
    assert call(Bd._Score(1e-40, 0)) == 1                              # sm_scale / softcap overflows
    assert call(Bd._Score(1e-30, 0)) == 3
    assert call(Bd._Score(0.0, 0, None, None, fake, None)) == 1
    assert call(Bd._Score(0.0, 0, None, None, None, fake)) == 1
    assert call(Bd._Score(30.0, 64, fake, fake, fake, fake)) == 3      # reaches the workspace check


def test_prefix_attention_refusals(lib):
    cs = P.Shape(2, 8, 4, 8, 4096).c()
    fake, odd = C.c_void_p(0x1000), C.c_void_p(0x1008)
    full = Bd._Cache(fake, fake, fake, fake, fake, fake, 100)

    def call(shp=cs, cache=full, n=4, q=fake, start=fake, scale=0.1, score=None, own=None, own_lse=None, out=fake, ws=fake,
             ws_bytes=16):
        return lib.stc_prefix_attn(C.byref(shp), C.byref(cache), n, q, start, scale, score and C.byref(score), own, own_lse, out,
                                   None, ws, ws_bytes, None)

    assert call() == 3                           # valid but for the workspace
    assert call(ws=C.c_void_p(0x1010), ws_bytes=1 << 40) == 3
    for kw, code in [(dict(n=-1), 1), (dict(q=None), 1), (dict(start=None), 1), (dict(out=None), 1), (dict(q=odd), 1),
                     (dict(out=odd), 1), (dict(scale=float("nan")), 1), (dict(own=fake), 1), (dict(own_lse=fake), 1),
                     (dict(cache=Bd._Cache()), 1), (dict(score=Bd._Score(0.0, 5)), 1),
                     (dict(score=Bd._Score(0.0, 0, fake)), 1), (dict(score=Bd._Score(-1.0, 0)), 1), (dict(own=fake, own_lse=C.c_void_p(0x2000)), 1),
                     (dict(shp=P.Shape(200, 8, 8, 8, (1 << 27) - 16).c()), 2), (dict(n=1 << 29), 2),
                     (dict(n=0), 0), (dict(shp=P.Shape(0, 8, 4, 8, 4096).c()), 0)]:
        assert call(**kw) == code, kw
    s = P.Shape(2, 8, 4, 8, 4096)
    n = P.workspace_bytes(s, Bd.OP_PREFIX_ATTN, 4)
    assert n > 0 and n % 256 == 0 and P.workspace_bytes(s, Bd.OP_PREFIX_ATTN, 0) == 0
    assert P.workspace_bytes(P.Shape(2, 8, 4, 8, 0), Bd.OP_PREFIX_ATTN, 4) > 0
    with pytest.raises(P.StcError):
        P.workspace_bytes(s, Bd.OP_PREFIX_ATTN, -1)


def test_argument_checks_agree_with_and_without_the_native_module(lib, monkeypatch):
    """CPU tensors, wrong types, sizes and layouts are refused in the same words by both."""
    assert Bd._native_addresses is not None, "the build makes the native argument check"
    i32 = torch.zeros(2, dtype=torch.int32)
    shape = P.Shape(2, 8, 4, 8, 16, i32)
    x = torch.zeros(2, 1, 8, 128, dtype=torch.bfloat16)
    cases = [lambda: P.rope_write(shape, P.Rope(torch.zeros(8, dtype=torch.float64)), i32, i32, q_in=x, q_out=x),
             lambda: P.rope_write(shape, P.Rope(torch.zeros(8, dtype=torch.float64)), i32, i32),
             lambda: P.decode_attn(shape, P.Cache(), x[:, 0], None, None, 1.0, x[:, 0].float(), i32, score=P.Score(softcap=1.0)),
             lambda: P.decode_attn(shape, P.Cache(), x[:, 0], None, None, 1.0, x[:, 0].float(), i32, score=P.Score(slopes=torch.zeros(3))),
             lambda: P.prefix_attn(shape, P.Cache(), x[:, 0], i32, 1.0, x[:, 0].float(), i32),
             lambda: P.prefix_attn(shape, P.Cache(), x[:, 0], torch.zeros(3, dtype=torch.int32), 1.0, x[:1, 0].float(), i32)]
    monkeypatch.setattr(Bd, "_current_device", lambda: 0)

    def said(f):
        with pytest.raises(ValueError) as e:
            f()
        return str(e.value)

    native = [said(f) for f in cases]
    for name in ("_native_addresses", "_sizes_are", "_native_token_rows"):
        monkeypatch.setattr(Bd, name, None)
    assert [said(f) for f in cases] == native
