"""Masks and positions of drafted trees, and the walk of the chosen tokens, against plain loops."""
import numpy as np
import pytest
import torch

import paper_2603_18815_amd as ra
from tests.draft_util import DEV, ancestors, cu, i32, pack, random_tree

pytestmark = pytest.mark.gpu


def walk(parents, draft, chosen):
    path, cur = [], 0 if len(parents) else -1
    while cur >= 0:
        path.append(cur)
        nxt = [j for j in range(cur + 1, len(parents))
               if parents[j] == cur and chosen[cur] >= 0 and draft[j] == chosen[cur]]
        cur = nxt[0] if nxt else -1
    return path


SIZES = [[1], [0, 1, 2, 63, 64, 65, 0], [16] * 40, [1024, 3, 1000], [200, 0, 129]]


@pytest.mark.parametrize("T", SIZES, ids=lambda t: f"{len(t)}rows_max{max(t)}")
@pytest.mark.parametrize("shape", ["tree", "chain", "star"])
def test_masks_and_walks(device, T, shape):
    rng = np.random.default_rng(len(T) + max(T))
    make = {"tree": lambda t: random_tree(rng, t), "chain": lambda t: np.arange(t) - 1,
            "star": lambda t: np.where(np.arange(t) > 0, 0, -1)}[shape]
    parents = [make(t) for t in T]
    total, pad = sum(T), 3
    few = 1 if shape == "chain" else 2                       # chains are walked to their end
    draft, chosen = rng.integers(0, few, total), rng.integers(0, few, total)
    ctx = rng.integers(0, 50000, len(T))
    flat = np.concatenate(parents + [np.full(pad, -1)])
    words = -(-max(T) // 64) + 1
    mask = torch.full((total + pad, words), 77, dtype=torch.int64, device=DEV)
    pos = torch.full((total + pad,), 77, dtype=torch.int32, device=DEV)
    ra.draft_tree_mask(i32(flat), i32(cu(T)), i32(ctx), max(T), mask, pos)
    seen = [ancestors(p) for p in parents]
    assert np.array_equal(mask[:total].cpu().numpy(), pack(seen, words))
    depth = np.concatenate([s.sum(1) - 1 + c for s, c in zip(seen, ctx)])
    assert np.array_equal(pos[:total].cpu().numpy(), depth)
    assert bool((mask[total:] == 77).all()) and bool((pos[total:] == 77).all())

    full = lambda n: torch.full((n,), 77, dtype=torch.int32, device=DEV)
    path, tokens = full(total + pad), full(total + pad)
    z = lambda x: i32(np.concatenate([x, np.zeros(pad)]))
    _, _, acc, lens, nxt = ra.draft_tree_accept(i32(flat), z(draft), z(chosen), i32(cu(T)), i32(ctx),
                                                max(T), path, tokens)
    assert bool((path[total:] == 77).all()) and bool((tokens[total:] == 77).all())
    path, tokens = path.cpu().numpy(), tokens.cpu().numpy()
    for b, t in enumerate(T):
        at = cu(T)[b]
        want = walk(parents[b], draft[at:at + t], chosen[at:at + t])
        n = len(want)
        assert list(path[at:at + n]) == want and (path[at + n:at + t] == -1).all()
        assert list(tokens[at:at + n]) == [chosen[at + i] for i in want]
        assert (tokens[at + n:at + t] == -1).all()
        assert int(acc[b]) == n and int(lens[b]) == ctx[b] + n
        assert int(nxt[b]) == (chosen[at + want[-1]] if n else -1)


def test_parents_that_name_no_earlier_node(device):
    """Such nodes are roots of their own; only node 0's tree is walked."""
    parents = [5, 0, 2, -7, 3, 1 << 30, 1]
    mask, pos = ra.draft_tree_mask(i32(parents), i32([0, 7]))
    assert mask[:, 0].tolist() == [1, 3, 4, 8, 24, 32, 67] and pos.tolist() == [0, 1, 0, 0, 1, 0, 2]
    draft, chosen = [9, 4, 4, 4, 4, 4, 5], [4, 5, 4, 4, 4, 4, -1]
    path, tokens, acc, lens, nxt = ra.draft_tree_accept(i32(parents), i32(draft), i32(chosen),
                                                        i32([0, 7]), i32([100]))
    assert path.tolist() == [0, 1, 6, -1, -1, -1, -1] and tokens.tolist()[:3] == [4, 5, -1]
    assert acc.tolist() == [3] and lens.tolist() == [103] and nxt.tolist() == [-1]


def test_the_first_of_equal_children_and_negative_tokens(device):
    path, tokens, acc, _, nxt = ra.draft_tree_accept(
        i32([-1, 0, 0, 1, 2]), i32([0, 6, 6, 1, 8]), i32([6, 8, 8, 0, 0]), i32([0, 5]), i32([0]))
    assert path.tolist() == [0, 1, -1, -1, -1] and nxt.tolist() == [8] and acc.tolist() == [2]
    path, tokens, acc, _, nxt = ra.draft_tree_accept(     # a row of nothing but -inf logits
        i32([-1, 0]), i32([0, -1]), i32([-1, 0]), i32([0, 2]), i32([0]))
    assert path.tolist() == [0, -1] and tokens.tolist() == [-1, -1] and nxt.tolist() == [-1]
    assert acc.tolist() == [1]


def test_empty_calls(device):
    none = i32([])
    mask, pos = ra.draft_tree_mask(none, i32([0]))
    assert mask.shape == (0, 1) and pos.shape == (0,)
    got = ra.draft_tree_accept(none, none, none, i32([0]), none)
    assert all(x.numel() == 0 for x in got)


def test_rows_without_any_node_have_results(device):
    none = i32([])
    path, tokens, acc, lens, nxt = ra.draft_tree_accept(none, none, none, i32([0] * 4), i32([0, 7, 90]))
    assert path.numel() == 0 and tokens.numel() == 0
    assert acc.tolist() == [0, 0, 0] and lens.tolist() == [0, 7, 90] and nxt.tolist() == [-1] * 3
