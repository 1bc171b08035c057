"""stc_tree_commit, stc_cache_fork and stc_cache_compact at the ends of their ranges: long runs of copies of one prompt, and caches whose
rows begin behind 2^31 pieces of 16 bytes."""
import pytest
import torch

import paper_2604_21335_b200 as P
import test_gpu_cache_ops as CO

pytestmark = pytest.mark.gpu
i32, outputs = CO.i32, CO.outputs


def test_fork_of_long_runs():
    """Hundreds of copies of one source, runs that begin and end anywhere, pairs among them that are left out."""
    S, H, T, lens = 8, 2, 2100, [2100, 1500, 2033, 0]
    c = CO.full(8, 4, H, T, S, lens)
    src = [0] * 5 + [1] * 3 + [0] * 100 + [2] + [0] + [2] * 41 + [3] * 20 + [1] * 70
    n = len(src)
    dst = [(i * 7 + 3) % n for i in range(n)]
    assert sorted(dst) == list(range(n))
    left_out = [0, 1, 8, 9, 10, 15, 16, 17, 31, 47, 48, 107, 110, n - 1]
    for i in left_out:
        dst[i] = -1 if i % 2 else n
    d = CO.blank(3, n, H, T + 20, S, c["cap"] + 1)
    cache = CO.device(d)
    new_len, total, status = outputs(n, H, n)
    P.cache_fork(P.Shape(4, H, H, S, T, i32(lens)), CO.device(c), P.Shape(n, H, H, S, T + 20), cache, i32(src), i32(dst), new_len, total, status)
    CO.same(cache, CO.fork_on_host(c, d, S, [(s, t) for i, (s, t) in enumerate(zip(src, dst)) if i not in left_out]))
    assert status[:, 0].tolist() == [int(i in left_out) for i in range(n)] and torch.equal(status[:, 0], status[:, 1])


def test_copies_of_one_prompt_take_the_time_of_as_many_prompts():
    """The same bytes are written.  (A run of copies shares the reading of its source; when it also shared the few CTAs of one pair, a
    thousand copies took ten times as long as a thousand prompts.)"""
    S, T, n = 8, 2048, 1024
    k = torch.empty(n, 1, T, 128, dtype=torch.bfloat16, device="cuda").normal_()
    offs = (4 * torch.arange(T + 1, device="cuda")).to(torch.int32).expand(n, 1, T + 1).contiguous()

    def cache(k):
        return P.Cache(k=k, kmin=torch.zeros(n, 1, T // 16, 128, dtype=torch.bfloat16, device="cuda"),
                       kmax=torch.zeros(n, 1, T // 16, 128, dtype=torch.bfloat16, device="cuda"),
                       v_packed=torch.zeros(n, 1, 4 * T, 16, dtype=torch.bfloat16, device="cuda"),
                       v_mask=torch.full((n, 1, T), 15, dtype=torch.int16, device="cuda"), v_offs=offs.clone(), cap_groups=4 * T)

    a, b, shape = cache(k), cache(torch.zeros_like(k)), P.Shape(n, 1, 1, S, T)
    new_len, total, status = outputs(n, 1, n)
    dst = torch.arange(n, dtype=torch.int32, device="cuda")
    best = {}
    for _ in range(5):
        for name, src in (("prompts", dst), ("copies", torch.zeros_like(dst))):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            torch.cuda.synchronize()
            start.record()
            P.cache_fork(shape, a, shape, b, src, dst, new_len, total, status)
            end.record()
            torch.cuda.synchronize()
            best[name] = min(best.get(name, 1e9), start.elapsed_time(end))
    assert (status == 0).all() and all(torch.equal(b.k[i], k[0]) for i in (0, 1, 15, 16, n // 2, n - 1))
    assert best["copies"] <= 3 * best["prompts"], best


def test_offsets_beyond_32_bits():
    """35 GB of keys and as much of values: the last rows begin behind 2^31 pieces of 16 bytes.  One row is forked, continued and shrunk,
    in place and into another cache."""
    B, T, S, cap = 130, 1 << 20, 4, 4 << 20
    length = T - 40
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        torch.cuda.empty_cache()
    new = lambda *s, t=torch.bfloat16: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    cache = P.Cache(k=new(B, 1, T, 128), kmin=new(B, 1, T // 16, 128), kmax=new(B, 1, T // 16, 128), v_packed=new(B, 1, cap, 32),
                    v_mask=new(B, 1, T, t=torch.int16), v_offs=new(B, 1, T + 1, t=torch.int32), cap_groups=cap)
    assert (B - 2) * T * 16 >= 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(5)
    a, z = B - 2, B - 1
    cache.v_offs.zero_()
    cache.k[a].normal_(generator=g)
    cache.v_packed[a].normal_(generator=g)
    mask = torch.randint(1, 16, (T,), generator=g, device="cuda")
    count = sum((mask >> j) & 1 for j in range(S))
    mask[length:] = 0
    count[length:] = 0
    cache.v_mask[a, 0] = mask.to(torch.int16)
    cache.v_offs[a, 0, 1:] = count.cumsum(0).to(torch.int32)
    pages = (length + 15) // 16
    cache.kmin[a].normal_(generator=g)
    cache.kmax[a].normal_(generator=g)
    cache.k[z].zero_()
    cache.v_packed[z].zero_()
    seq = torch.zeros(B, dtype=torch.int32, device="cuda")
    seq[a] = length
    shape = P.Shape(B, 1, 1, S, T, seq)
    new_len, total, status = outputs(B, 1, 1)
    P.cache_fork(shape, cache, shape, cache, i32([a]), i32([z]), new_len, total, status)
    groups = int(cache.v_offs[a, 0, length])
    assert status.item() == 0 and new_len[z] == length and total[z, 0] == groups
    assert torch.equal(cache.k[z, 0, :length], cache.k[a, 0, :length]) and torch.equal(cache.v_packed[z, 0, :groups], cache.v_packed[a, 0, :groups])
    assert torch.equal(cache.kmin[z, 0, :pages], cache.kmin[a, 0, :pages]) and torch.equal(cache.kmax[z, 0, :pages], cache.kmax[a, 0, :pages])
    assert torch.equal(cache.v_mask[z, 0, :length], cache.v_mask[a, 0, :length])
    assert torch.equal(cache.v_offs[z, 0, :length + 1], cache.v_offs[a, 0, :length + 1])
    assert (cache.k[z, 0, length:] == 0).all() and (cache.v_packed[z, 0, groups:] == 0).all()

    n_cap, n = 32, 30
    kn, vn = (torch.randn(B, 1, n_cap, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    path = torch.arange(n_cap - 1, -1, -1, dtype=torch.int32, device="cuda").expand(B, n_cap).contiguous()
    took = torch.zeros(B, dtype=torch.int32, device="cuda")
    took[z] = n
    seq[z] = length
    after, total, status = outputs(B, 1, B)
    P.tree_commit(shape, cache, P.Tree(kn, vn), path, took, after, total, status)
    rows = path[z, :n].long()
    assert (status == 0).all() and after[z] == length + n and total[z, 0] == groups + S * n
    assert torch.equal(cache.k[z, 0, length:length + n], kn[z, 0, rows]) and (cache.k[z, 0, length + n:] == 0).all()
    assert torch.equal(cache.v_packed[z, 0, groups:groups + S * n].reshape(n, 128), vn[z, 0, rows]) and (cache.v_packed[z, 0, groups + S * n:] == 0).all()
    assert (cache.v_mask[z, 0, length:length + n] == 15).all()
    assert torch.equal(cache.v_offs[z, 0, length:length + n + 1], groups + S * torch.arange(n + 1, dtype=torch.int32, device="cuda"))
    whole, first, end = length + n, length // 16, (length + n + 15) // 16
    for p in range(first, end):
        part = cache.k[z, 0, 16 * p:min(whole, 16 * p + 16)].float()
        assert torch.equal(cache.kmin[z, 0, p].float(), part.amin(0)) and torch.equal(cache.kmax[z, 0, p].float(), part.amax(0))

    # every third page and the last one, which is not full
    seq[z] = whole
    seq[a] = 0
    ids = torch.arange(0, end, 3, dtype=torch.int32, device="cuda")
    ids = torch.cat([ids[:-1], i32([end - 1])])
    most = ids.numel()
    lists, n_ids = torch.zeros(B, 1, most, dtype=torch.int32, device="cuda"), torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    lists[z, 0] = ids
    n_ids[z] = most
    tok = (ids.long()[:, None] * 16 + torch.arange(16, device="cuda")).flatten()
    tok = tok[tok < whole]
    kept = tok.numel()
    sizes = (cache.v_offs[z, 0, tok + 1] - cache.v_offs[z, 0, tok]).long()
    want_offs = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), sizes.cumsum(0)])
    held = int(want_offs[-1])
    of = torch.repeat_interleave(torch.arange(kept, device="cuda"), sizes)
    from_groups = cache.v_offs[z, 0, tok].long()[of] + torch.arange(held, device="cuda") - want_offs[:-1][of]
    want = dict(k=cache.k[z, 0, tok], v_mask=cache.v_mask[z, 0, tok], v_packed=cache.v_packed[z, 0, from_groups], kmin=cache.kmin[z, 0, ids.long()],
                kmax=cache.kmax[z, 0, ids.long()], v_offs=want_offs.to(torch.int32))
    small_T = most * 16
    to = P.Cache(k=new(B, 1, small_T, 128), kmin=new(B, 1, most, 128), kmax=new(B, 1, most, 128), v_packed=new(B, 1, held, 32),
                 v_mask=new(B, 1, small_T, t=torch.int16), v_offs=new(B, 1, small_T + 1, t=torch.int32), cap_groups=held)
    new_len, total, status = outputs(B, 1, B)
    P.cache_compact(shape, cache, lists, n_ids, new_len, total, status, dst_shape=P.Shape(B, 1, 1, S, small_T), dst=to)
    new_len_in, total_in, status_in = outputs(B, 1, B)
    P.cache_compact(shape, cache, lists, n_ids, new_len_in, total_in, status_in)
    for length, groups, st in ((new_len, total, status), (new_len_in, total_in, status_in)):
        assert (st == 0).all() and length[z] == kept and groups[z, 0] == held and (length[:z] == 0).all() and (groups[:z] == 0).all()
    for got in (to, cache):
        for x, w in want.items():
            assert torch.equal(getattr(got, x)[z, 0, :w.shape[0]], w), x
    del cache, to, want
    torch.cuda.empty_cache()
