"""Block tables from lengths on the GPU against a plain host loop: exact, element by element."""
import numpy as np
import pytest
import torch

import paper_2603_18815_amd as ra

pytestmark = pytest.mark.gpu


def dev(x, dt=np.int32):
    return torch.as_tensor(np.ascontiguousarray(np.asarray(x, dt)), device="cuda:0")


def host_extend(start, new, free, count, table, total):
    """The definition, row by row; None where the call is to be refused."""
    need = [-(-(s + n) // 16) - -(-s // 16) for s, n in zip(start, new)]
    if (sum(need) > count or sum(new) > total or min([0, *start, *new]) < 0 or
            max([0, *(s + n for s, n in zip(start, new))]) > table.shape[1] * 16):
        return None
    table, slots, top = table.copy(), [], count
    for b, (s, n) in enumerate(zip(start, new)):
        for j in range(-(-s // 16), -(-(s + n) // 16)):
            top -= 1
            table[b, j] = free[top]
        slots += [int(table[b, p // 16]) * 16 + p % 16 for p in range(s, s + n)]
    return table, slots + [-1] * (total - len(slots)), top


def make(rng, start, new, stride, spare=3):
    B = len(start)
    held = [-(-s // 16) for s in start]
    need = sum(-(-(s + n) // 16) for s, n in zip(start, new)) - sum(held)
    pages = rng.permutation(sum(held) + need + spare).astype(np.int32)
    table = np.full((B, stride), -7, np.int32)
    at = 0
    for b, h in enumerate(held):
        table[b, :h] = pages[at:at + h]
        at += h
    free = np.concatenate([pages[at:], np.full(at, -9, np.int32)])   # capacity: every page
    return table, free, pages.size - at


CASES = {
    "one token": ([0], [1], 1, 0),
    "page ends": ([15, 16, 17, 0], [1, 1, 1, 16], 4, 0),
    "no new token": ([0, 5, 16], [0, 0, 0], 4, 2),
    "empty rows between": ([0, 100, 0, 31, 0], [0, 33, 0, 1, 0], 16, 5),
    "behind the last": ([3, 40], [2, 60], 8, 100),
}


@pytest.mark.parametrize("name", list(CASES))
def test_extend_small(name, device):
    start, new, stride, extra = CASES[name]
    check(np.random.default_rng(3), start, new, stride, sum(new) + extra)


@pytest.mark.parametrize("B,hi,nhi", [(64, 4096, 1), (300, 64, 40), (1024, 200, 3), (1025, 100, 9),
                                      (2500, 40, 20), (7, 3000, 5000)])
def test_extend_random(B, hi, nhi, device):
    """Batches of one and several scan steps, calls of one and several workgroups."""
    rng = np.random.default_rng(B)
    start, new = rng.integers(0, hi + 1, B).tolist(), rng.integers(0, nhi + 1, B).tolist()
    check(rng, start, new, (hi + nhi) // 16 + 2, sum(new) + 11)


def check(rng, start, new, stride, total):
    table, free, count = make(rng, start, new, stride)
    want_table, want_slots, left = host_extend(start, new, free, count, table, total)
    t, f, c, s, n = dev(table), dev(free), dev([count]), dev(start), dev(new)
    cu, lens, slots, taken = ra.block_table_extend(t, s, n, f, c, total_new=total)
    assert taken.item() == count - left and c.item() == left
    assert cu.tolist() == [0, *np.cumsum(new).tolist()]
    assert lens.tolist() == [a + b for a, b in zip(start, new)]
    assert np.array_equal(t.cpu().numpy(), want_table)
    assert slots.tolist() == want_slots
    assert np.array_equal(f.cpu().numpy(), free)              # the list is only read
    f[left:] = -1                                             # entries past its end are stale
    released = ra.block_table_release(t, lens, s, f, c)
    assert released.item() == count - left and c.item() == count
    assert np.array_equal(f.cpu().numpy()[:count], free[:count])
    assert np.array_equal(t.cpu().numpy(), want_table)
    # every row ends: all pages are free, each once
    assert ra.block_table_release(t, s, torch.zeros_like(s), f, c,
                                  max_pages=1).item() == sum(-(-a // 16) for a in start)
    assert sorted(f[:c.item()].tolist()) == list(range(c.item()))


@pytest.mark.parametrize("B", [3, 700])
@pytest.mark.parametrize("why", ["pages", "table", "tokens", "negative start", "negative new",
                                 "count", "negative count"])
def test_extend_is_refused_whole(why, B, device):
    """One bad length or one page too few: nothing changes, the outputs are of no new token."""
    rng = np.random.default_rng(5)
    start, new = rng.integers(0, 60, B).tolist(), rng.integers(1, 30, B).tolist()
    table, free, count = make(rng, start, new, 8, spare=0)
    total = sum(new)
    if why == "pages":
        count -= 1
    elif why == "table":
        new[B // 2] = 8 * 16 - start[B // 2] + 1
        total = sum(new)
    elif why == "tokens":
        total -= 1
    elif why == "negative start":
        start[B - 1] = -1
    elif why == "negative new":
        new[1] = -1
    elif why == "count":
        count = free.size + 1
    else:
        count = -1
    t, f, c = dev(table), dev(free), dev([count])
    cu, lens, slots, taken = ra.block_table_extend(t, dev(start), dev(new), f, c, total_new=total)
    assert taken.item() == -1 and c.item() == count
    assert cu.tolist() == [0] * (B + 1) and lens.tolist() == start
    assert slots.tolist() == [-1] * total
    assert np.array_equal(t.cpu().numpy(), table) and np.array_equal(f.cpu().numpy(), free)


@pytest.mark.parametrize("why", ["keep past len", "negative keep", "table", "capacity"])
def test_release_is_refused_whole(why, device):
    rng = np.random.default_rng(6)
    start = rng.integers(1, 100, 40).tolist()
    table, free, count = make(rng, start, [0] * 40, 8)
    keep = [0] * 40
    if why == "keep past len":
        keep[7] = start[7] + 1
    elif why == "negative keep":
        keep[39] = -1
    elif why == "table":
        start[0] = 8 * 16 + 1
    else:
        free = free[:-1].copy()
    t, f, c = dev(table), dev(free), dev([count])
    assert ra.block_table_release(t, dev(start), dev(keep), f, c).item() == -1
    assert c.item() == count and np.array_equal(f.cpu().numpy(), free)


def test_no_rows(device):
    none = dev([])
    f, c = dev([4, 5]), dev([2])
    t = torch.zeros((0, 4), dtype=torch.int32, device="cuda:0")
    cu, lens, slots, taken = ra.block_table_extend(t, none, none, f, c, total_new=3)
    assert cu.tolist() == [0] and taken.item() == 0 and slots.tolist() == [-1] * 3
    assert ra.block_table_release(t, none, none, f, c).item() == 0 and c.item() == 2
