"""Caches without room for a token: calls that write lengths and status refuse them instead of leaving both as they were."""
import pytest
import torch

import paper_2604_21335_b200 as P
from paper_2604_21335_b200 import binding as Bd


def parts(B, T, dev):
    """A shape with its cache."""
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device=dev)  # noqa: E731
    bf = lambda *s: torch.zeros(*s, dtype=torch.bfloat16, device=dev)  # noqa: E731
    shape = P.Shape(B, 8, 4, 8, T, i(B))
    n = shape.n_pages
    return shape, P.Cache(k=bf(B, 4, T, 128), kmin=bf(B, 4, n, 128), kmax=bf(B, 4, n, 128), v_packed=bf(B, 4, 1, 16), v_mask=i(B, 4, T).short(),
                          v_offs=i(B, 4, T + 1), cap_groups=1)


@pytest.mark.parametrize("dev", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
@pytest.mark.parametrize("call", ["commit", "fork into", "fork from", "compact into", "compact from", "compact in place"])
def test_a_cache_of_no_tokens_is_refused(call, dev, monkeypatch):
    if dev == "cpu":
        monkeypatch.setattr(Bd, "_current_device", lambda: 0)
    i = lambda *s: torch.full(s, 7, dtype=torch.int32, device=dev)  # noqa: E731
    (s0, c0), (s1, c1), new_len, total, status = parts(2, 0, dev), parts(2, 32, dev), i(2), i(2, 4).long(), i(2, 4)
    node = torch.zeros(2, 4, 3, 128, dtype=torch.bfloat16, device=dev)
    ids, n = i(2, 4, 2), i(2, 4)
    with pytest.raises(ValueError, match="t_cap 0"):
        if call == "commit":
            P.tree_commit(s0, c0, P.Tree(node, node), i(2, 3), i(2), new_len, total, status)
        elif call == "fork into":
            P.cache_fork(s1, c1, s0, c0, i(2), i(2), new_len, total, status)
        elif call == "fork from":
            P.cache_fork(s0, c0, s1, c1, i(2), i(2), new_len, total, status)
        elif call == "compact into":
            P.cache_compact(s1, c1, ids, n, new_len, total, status, dst_shape=s0, dst=c0)
        elif call == "compact from":
            P.cache_compact(s0, c0, ids, n, new_len, total, status, dst_shape=s1, dst=c1)
        else:
            P.cache_compact(s0, c0, ids, n, new_len, total, status)
