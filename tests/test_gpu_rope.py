"""Rotary write against the 64-bit plain form: layouts, partial rotation, far positions, ragged batches, refusals."""
import pytest
import torch

import operators_ref as R
import paper_2604_21335_b200 as P

pytestmark = pytest.mark.gpu


def run_case(B, Hq, Hkv, n, T, rot, interleaved, new, old, scale=1.0, positions=None, fused=True, base=10000.0, seed=0):
    g = torch.Generator().manual_seed(seed)
    wide = torch.randn(B, n, Hq + 2 * Hkv, 128, generator=g).to(torch.bfloat16)
    qkv = wide.cuda()
    parts = [qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]]
    if not fused:
        parts = [p.contiguous() for p in parts]
    f, _ = P.rope_frequencies(rot, base)
    length = torch.tensor([o + m for o, m in zip(old, new)], dtype=torch.int32, device="cuda")
    shape = P.Shape(B, Hq, Hkv, 8, T, length)
    keep = 7.0                                   # what the call must leave alone
    q_out = torch.full((B, n, Hq, 128), keep, dtype=torch.bfloat16, device="cuda")
    k = torch.full((B, Hkv, T, 128), keep, dtype=torch.bfloat16, device="cuda")
    v = torch.full_like(k, keep)
    status = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    pos = None if positions is None else torch.tensor(positions, dtype=torch.int32).reshape(B, n)
    P.rope_write(shape, P.Rope(f.cuda(), interleaved, scale), torch.tensor(old, dtype=torch.int32, device="cuda"), status,
                 *parts, q_out=q_out, k=k, v=v, positions=None if pos is None else pos.cuda())
    torch.cuda.synchronize()
    eq, ek, ev = (torch.full(x.shape, keep, dtype=torch.float64) for x in (q_out, k, v))
    tq, tk = torch.zeros(q_out.shape, dtype=torch.float64), torch.zeros(k.shape, dtype=torch.float64)
    want_status = []
    for b in range(B):
        bad = old[b] < 0 or new[b] < 0 or new[b] > n
        want_status.append(1 if bad else 0)
        if bad:
            continue
        m, o = new[b], old[b]
        p = torch.arange(o, o + m) if pos is None else pos[b, :m]
        y, t = R.rope_ref(wide[b, :m, :Hq], p, f, interleaved, scale)
        eq[b, :m], tq[b, :m] = y, t
        y, t = R.rope_ref(wide[b, :m, Hq:Hq + Hkv], p, f, interleaved, scale)
        ek[b, :, o:o + m], tk[b, :, o:o + m] = y.transpose(0, 1), t.transpose(0, 1)
        ev[b, :, o:o + m] = wide[b, :m, Hq + Hkv:].double().transpose(0, 1)
    assert status.tolist() == want_status
    assert ((q_out.double().cpu() - eq).abs() <= tq).all()
    assert ((k.double().cpu() - ek).abs() <= tk).all()
    assert (v.double().cpu() == ev).all()


@pytest.mark.parametrize("rot", [0, 16, 48, 64, 96, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_layouts_and_partial_rotation(rot, interleaved):
    run_case(2, 14, 2, 5, 40, rot, interleaved, [5, 3], [0, 31], scale=1.1386294, seed=rot)


@pytest.mark.parametrize("n,B", [(1, 1), (1, 16), (33, 7), (700, 4), (2400, 9)])
def test_every_cta_shape_and_ragged_lengths(n, B):
    new = [(n * (i + 1)) // B for i in range(B)]
    old = [(13 * i) % 50 for i in range(B)]
    run_case(B, 4, 1, n, n + 50, 64, False, new, old, fused=n != 33, seed=n)


def test_nothing_new_and_lengths_that_do_not_fit():
    run_case(5, 8, 4, 4, 64, 128, True, [0, 4, 5, 2, 1], [10, 60, 3, -1, 63])


@pytest.mark.parametrize("first", [131072 - 8, (1 << 20) - 8, (1 << 24) + 1, 2**31 - 8, -5])
def test_far_positions(first):
    pos = [first + i for i in range(8)]
    # the fp64 table times the position is itself exact to 2^-53 * 2^31 turns only in 64 bits: keep the reference's
    # own error (2^-22 rad at 2^31) out of the comparison by a base whose table is powers of two
    run_case(1, 8, 2, 8, 16, 128, False, [8], [4], positions=pos, base=2.0 ** 64, seed=9)


def test_angle_is_exact_at_a_position_whose_fp32_product_is_not():
    """One pair with frequency 1: cos / sin of 131071 radians, to bf16."""
    f = torch.zeros(8, dtype=torch.float64)
    f[0] = 1.0
    x = torch.zeros(1, 1, 1, 128, dtype=torch.bfloat16, device="cuda")
    x[..., 0] = 1.0
    out, st = torch.zeros_like(x), torch.zeros(1, dtype=torch.int32, device="cuda")
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    P.rope_write(P.Shape(1, 1, 1, 8, 4, one), P.Rope(f.cuda()), one * 0, st, q_in=x, q_out=out,
                 positions=torch.tensor([[131071]], dtype=torch.int32, device="cuda"))
    a = torch.tensor(131071.0, dtype=torch.float64)
    want = torch.stack([a.cos(), a.sin()])
    got = out[0, 0, 0, [0, 8]].double().cpu()
    assert ((got - want).abs() <= 2.0 ** -8 * want.abs()).all()


def test_in_place_query_and_parts_left_out():
    g = torch.Generator().manual_seed(3)
    x = torch.randn(3, 2, 8, 128, generator=g).to(torch.bfloat16)
    f, _ = P.rope_frequencies(128)
    q = x.cuda()
    st = torch.zeros(3, dtype=torch.int32, device="cuda")
    old = torch.tensor([0, 5, 9], dtype=torch.int32, device="cuda")
    shape = P.Shape(3, 8, 8, 8, 16, old + 2)
    P.rope_write(shape, P.Rope(f.cuda()), old, st, q_in=q, q_out=q)
    for b in range(3):
        y, t = R.rope_ref(x[b], torch.arange(2) + int(old[b]), f, False, 1.0)
        assert ((q[b].double().cpu() - y).abs() <= t).all()
    k = torch.zeros(3, 8, 16, 128, dtype=torch.bfloat16, device="cuda")
    P.rope_write(shape, P.Rope(f.cuda()), old, st, k_in=x.cuda(), k=k)
    for b in range(3):
        lo = int(old[b])
        y, t = R.rope_ref(x[b], torch.arange(2) + lo, f, False, 1.0)
        assert ((k[b, :, lo:lo + 2].double().cpu() - y.transpose(0, 1)).abs() <= t.transpose(0, 1)).all()


def test_captured_call_follows_the_lengths_on_the_device():
    f, _ = P.rope_frequencies(128)
    B, T = 2, 12
    old = torch.zeros(B, dtype=torch.int32, device="cuda")
    length = old + 1
    x = torch.randn(B, 1, 4, 128, device="cuda").to(torch.bfloat16)
    k = torch.zeros(B, 4, T, 128, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(B, dtype=torch.int32, device="cuda")
    shape, rope = P.Shape(B, 4, 4, 8, T, length), P.Rope(f.cuda())
    P.rope_write(shape, rope, old, st, k_in=x, k=k)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.rope_write(shape, rope, old, st, k_in=x, k=k)
    for step in range(1, 5):
        old.add_(1); length.add_(1)
        x.copy_(torch.randn(B, 1, 4, 128, device="cuda"))
        graph.replay()
        y, t = R.rope_ref(x[:, 0].cpu(), torch.full((B,), step), f, False, 1.0)
        assert ((k[:, :, step].double().cpu() - y).abs() <= t).all()


def test_binding_refuses_what_it_cannot_pass_on():
    f, _ = P.rope_frequencies(32)
    rope = P.Rope(f.cuda())
    old, st = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    shape = P.Shape(2, 4, 4, 8, 16, old + 1)
    x = torch.zeros(2, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        P.rope_write(shape, rope, old, st)
    with pytest.raises(ValueError):
        P.rope_write(shape, rope, old, st, q_in=x.float(), q_out=x)
    with pytest.raises(ValueError):
        P.rope_write(shape, rope, old, st, q_in=x, q_out=x[:1])
    with pytest.raises(ValueError):
        P.rope_write(shape, rope, old, st, q_in=x.transpose(2, 3).contiguous().transpose(2, 3), q_out=x)
    with pytest.raises(ValueError):
        P.rope_write(shape, rope, old[:1], st, q_in=x, q_out=x)
    with pytest.raises(P.StcError):
        P.rope_write(shape, rope, old, st, q_in=x)
