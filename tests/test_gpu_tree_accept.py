"""stc_tree_accept against a walk on the host: ties, NaN, infinities, rows that are not aligned, wide rows, odd vocabularies."""
import math

import pytest
import torch

import paper_2604_21335_b200 as P
import tree_ref as TR

pytestmark = pytest.mark.gpu


def run(logits, tokens, parent, nodes):
    B, n = len(tokens), len(tokens[0])
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    path = torch.full((B, n), -9, dtype=torch.int32, device="cuda")
    count, nxt = torch.full((B,), -9, dtype=torch.int32, device="cuda"), torch.full((B,), -9, dtype=torch.int32, device="cuda")
    P.tree_accept(logits, i32(tokens), path, count, nxt, parent=None if parent is None else i32(parent),
                  n_nodes=None if nodes is None else i32(nodes))
    return path.tolist(), count.tolist(), nxt.tolist()


def check(logits, tokens, parent, nodes):
    path, count, nxt = run(logits, tokens, parent, nodes)
    lg = logits.cpu()
    for b in range(len(tokens)):
        n = len(tokens[0]) if nodes is None else max(0, min(nodes[b], len(tokens[0])))
        up = [i - 1 for i in range(len(tokens[0]))] if parent is None else parent[b]
        want, x = TR.accept(lg[b], tokens[b], up, n)
        assert path[b] == want + [-9] * (len(tokens[0]) - len(want)) and count[b] == len(want) and nxt[b] == x


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 33, 1000, 32000, 50257, 151937])
@pytest.mark.parametrize("n", [1, 6])
def test_random_trees(dtype, vocab, n):
    r, B = TR.rng(vocab + n), 5
    g = torch.Generator(device="cuda").manual_seed(vocab)
    logits = torch.randn(B, n, vocab, generator=g, device="cuda").to(dtype)
    best = logits.float().argmax(-1).tolist()
    parent = [TR.random_tree(r, n, n) for _ in range(B)]
    tokens = [[best[b][parent[b][i]] if i and parent[b][i] >= 0 and r.random() < 0.8 else r.randrange(vocab) for i in range(n)] for b in range(B)]
    check(logits, tokens, parent, None)
    check(logits, tokens, parent, [n, 0, 1, n + 4, -3])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("slack", [1, 3, 8, 1000])
def test_rows_of_a_wider_buffer_in_any_alignment(dtype, slack):
    B, n, V = 3, 5, 777
    wide = torch.randn(B, n, V + slack, device="cuda").to(dtype)
    wide[..., V:] = 100.0                                     # not of the row
    logits = wide[..., :V]
    best = logits.float().argmax(-1).tolist()
    tokens = [[0] + [best[b][i - 1] for i in range(1, n)] for b in range(B)]
    tokens[1][3] = (tokens[1][3] + 1) % V
    check(logits, tokens, None, None)
    flat = torch.randn(2 * 3 * 101 + 9, device="cuda").to(dtype)
    for start in range(1, 9):
        view = flat[start:start + 2 * 3 * 101].view(2, 3, 101)
        best = view.float().argmax(-1).tolist()
        check(view, [[5, best[b][0], best[b][1]] for b in range(2)], None, None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ties_zeros_infinities_and_nan(dtype):
    V, n = 5003, 12
    logits = torch.zeros(1, n, V, device="cuda", dtype=dtype)
    logits[0, 0] = -math.inf                                 # all alike: 0
    logits[0, 1, 5:] = -0.0                                  # +0 and -0 are equal
    logits[0, 1, :5] = -1.0
    logits[0, 2, 4999] = math.inf
    logits[0, 3, 3000] = math.nan
    logits[0, 3, 17] = math.inf
    logits[0, 4, 4990] = math.nan
    logits[0, 4, 4000] = math.nan
    logits[0, 5] = -1.0
    logits[0, 5, [77, 1200, 4097, 4098, 5002]] = 2.0
    logits[0, 6] = math.nan
    logits[0, 7] = -3.0
    logits[0, 7, 5002] = -2.0
    logits[0, 8, :] = torch.finfo(dtype).min
    logits[0, 9, 2048:] = 1.0
    logits[0, 10] = -5.0
    logits[0, 10, 3] = -0.0
    logits[0, 10, 4] = 0.0
    want = [0, 5, 4999, 3000, 4000, 77, 0, 5002, 0, 2048, 3, 0]
    check(logits, [[0] + want[:-1]], None, None)
    path, count, nxt = run(logits, [[0] + want[:-1]], None, None)
    assert count == [n] and nxt == [0]


def test_the_lowest_matching_child_and_nodes_that_are_no_children():
    V = 50
    logits = torch.zeros(1, 8, V, device="cuda")
    logits[..., 7] = 1.0
    tokens = [[7, 7, 3, 7, 7, 7, 7, 7]]
    check(logits, tokens, [[-1, -1, 0, 0, 0, 3, 5, 6]], None)         # 0 3 5 6 7
    path, count, _ = run(logits, tokens, [[-1, -1, 0, 0, 0, 3, 5, 6]], None)
    assert path[0][:5] == [0, 3, 5, 6, 7] and count == [5]
    # parents that are not below their node are never followed
    path, count, nxt = run(logits, tokens, [[-1, 1, 2, 5, 9, -4, 100, 7]], None)
    assert path[0][:1] == [0] and count == [1] and nxt == [7]


def test_a_hundred_and_twenty_eight_nodes_of_many_sequences():
    B, n, V = 40, 128, 515
    g = torch.Generator(device="cuda").manual_seed(1)
    logits = torch.randn(B, n, V, generator=g, device="cuda").to(torch.bfloat16)
    best = logits.float()
    best = torch.where(best == best.amax(-1, keepdim=True), torch.arange(V, device="cuda"), V).amin(-1).tolist()
    r = TR.rng(2)
    tokens = [[0] + [best[b][i - 1] if r.random() < 0.97 else 1 for i in range(1, n)] for b in range(B)]
    check(logits, tokens, None, None)


def test_sizes_and_types_that_do_not_fit_are_refused():
    lg = torch.zeros(2, 4, 10, device="cuda")
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    good = dict(logits=lg, tokens=i(2, 4), path=i(2, 4), n_accepted=i(2), next_token=i(2))
    P.tree_accept(**good)
    for bad in (dict(logits=lg.half()), dict(logits=lg[0]), dict(logits=lg[:, :, ::2]), dict(logits=lg.transpose(0, 1)), dict(tokens=i(2, 3)),
                dict(path=i(3, 4)), dict(n_accepted=i(1)), dict(next_token=i(2).long()), dict(logits=lg.cpu()), dict(parent=i(4, 2)),
                dict(n_nodes=i(3))):
        with pytest.raises(ValueError):
            P.tree_accept(**{**good, **bad})
    with pytest.raises(P.StcError):
        P.tree_accept(torch.zeros(1, 129, 4, device="cuda"), i(1, 129), i(1, 129), i(1), i(1))
