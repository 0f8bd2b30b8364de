"""Forked rows, shared pages' release, page copies and compaction against plain loops."""
import numpy as np
import pytest
import torch

import paper_2603_18815_amd as ra
from tests.draft_util import DEV, cu, i32

pytestmark = pytest.mark.gpu


class Host:
    """The tables, the shares and the free list as plain lists, changed one entry at a time."""

    def __init__(self, seed, B, stride, num, held):
        rng = np.random.default_rng(seed)
        order = list(rng.permutation(num))
        self.stride, self.num = stride, num
        self.table = rng.integers(0, num, (B, stride))
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.free = order[at:]
        self.list = np.concatenate([self.free, rng.integers(0, num, num - len(self.free))])
        self.shares = np.zeros(num, np.int64)
        self.dev = dict(table=i32(self.table), list=i32(self.list), count=i32([len(self.free)]),
                        shares=i32(self.shares))

    def fork(self, src, dst, lens):
        B = len(self.table)
        bad = any(not (0 <= s < B and 0 <= d < B and 0 <= n <= 16 * self.stride)
                  for s, d, n in zip(src, dst, lens))
        bad |= len(set(dst)) < len(dst) or bool(set(src) & set(dst))
        need = sum(n % 16 > 0 for n in lens)
        if bad or need > len(self.free):
            return [-1] * len(src), [-1] * len(src), -1
        cs, cd = [], []
        for s, d, n in zip(src, dst, lens):
            for j in range(n // 16):
                self.table[d, j] = self.table[s, j]
                self.shares[self.table[s, j]] += 1
            if n % 16:
                page = self.free.pop()
                cs.append(self.table[s, n // 16])
                cd.append(page)
                self.table[d, n // 16] = page
            else:
                cs.append(-1)
                cd.append(-1)
        return cs, cd, need

    def release(self, lens, keep):
        if any(k < 0 or k > n or n > 16 * self.stride for n, k in zip(lens, keep)):
            return -1
        entries = [self.table[b, j] for b in range(len(lens))
                   for j in range(-(-keep[b] // 16), -(-lens[b] // 16))]
        entries = [e for e in entries if 0 <= e < self.num]
        freed = {p for p in set(entries) if entries.count(p) > self.shares[p]}
        order = [p for i, p in enumerate(entries) if p in freed and p not in entries[i + 1:]]
        for p in set(entries):
            self.shares[p] = 0 if p in freed else self.shares[p] - entries.count(p)
        self.free += order[::-1]
        return len(order)

    def check(self):
        d = self.dev
        assert np.array_equal(d["table"].cpu().numpy(), self.table)
        assert np.array_equal(d["shares"].cpu().numpy(), self.shares)
        n = int(d["count"])
        assert n == len(self.free) and d["list"][:n].tolist() == [int(p) for p in self.free]

    def do_fork(self, src, dst, lens):
        d = self.dev
        got = ra.block_table_fork(d["table"], i32(src), i32(dst), i32(lens), d["shares"], d["list"],
                                  d["count"])
        want = self.fork(src, dst, lens)
        assert got[0].tolist() == [int(x) for x in want[0]]
        assert got[1].tolist() == [int(x) for x in want[1]]
        assert got[2].tolist() == [want[2]]
        self.check()
        return got

    def do_release(self, lens, keep):
        d = self.dev
        got = ra.block_table_release_shared(d["table"], i32(lens), i32(keep), d["shares"], d["list"],
                                            d["count"])
        assert got.tolist() == [self.release(lens, keep)]
        self.check()


@pytest.mark.parametrize("prompts", [[100], [0, 16, 17, 15], [1, 500, 320, 4000]])
def test_groups_of_rollouts(device, prompts):
    """Prompts forked, their rollouts ended in turn, then the prompts' own rows."""
    group = 4
    B = len(prompts) * group
    held = [-(-prompts[b // group] // 16) if b % group == 0 else 0 for b in range(B)]
    h = Host(1, B, 260, sum(held) + 40, held)
    src = [b // group * group for b in range(B) if b % group]
    dst = [b for b in range(B) if b % group]
    lens = [prompts[b // group] for b in dst]
    h.do_fork(src, dst, lens)
    row = [prompts[b // group] for b in range(B)]
    part = [n if b % 3 else 0 for b, n in enumerate(row)]
    h.do_release(part, [0] * B)                                # some rows, prompts' among them
    h.do_release([n if not b % 3 else 0 for b, n in enumerate(row)], [0] * B)
    assert not h.shares.any()
    assert len(h.free) == h.num                                # every page is back


def test_release_restores_what_a_fork_took(device):
    h = Host(2, 8, 20, 60, [10, 0, 0, 0, 5, 0, 0, 0])
    before = list(h.free)
    h.do_fork([0, 0, 4, 0], [1, 2, 5, 7], [150, 33, 79, 160])
    h.do_release([0, 150, 33, 0, 0, 79, 0, 160], [0] * 8)
    assert h.free == before and not h.shares.any()


def test_whole_pages_cut_and_rows_of_rows(device):
    """A fork of a fork, rows cut back to whole pages, the same page given up by all holders at
    once."""
    h = Host(3, 6, 30, 80, [12, 0, 0, 0, 0, 0])
    h.do_fork([0, 0], [1, 2], [192, 100])
    h.do_fork([1], [3], [192])
    h.do_release([192, 192, 112, 192, 0, 0], [64, 64, 64, 192, 0, 0])
    h.do_release([64, 64, 64, 192, 0, 0], [0] * 6)
    assert not h.shares.any() and len(h.free) == h.num


@pytest.mark.parametrize("args", [
    ([0], [0], [5]), ([0], [6], [5]), ([-1], [1], [5]), ([0], [1], [-1]), ([0], [1], [16 * 12 + 1]),
    ([0, 0], [1, 1], [5, 5]), ([0, 1], [1, 2], [5, 5]), ([2, 0], [1, 2], [5, 5]),
    ([0] * 5, [1, 2, 3, 4, 5], [1] * 5)])
def test_forks_refused_as_a_whole(device, args):
    h = Host(4, 6, 12, 14, [10, 0, 0, 0, 0, 0])
    got = h.do_fork(*args)
    assert got[2].tolist() == [-1]


def test_bad_counts_and_lengths(device):
    h = Host(5, 3, 8, 20, [4, 4, 0])
    for lens, keep in (([129, 0, 0], [0, 0, 0]), ([5, 5, 5], [0, 6, 0]), ([5, 5, 5], [0, -1, 0])):
        h.do_release(lens, keep)
    for count in (-1, 21):
        h.dev["count"].fill_(count)
        for got in (ra.block_table_fork(h.dev["table"], i32([0]), i32([2]), i32([3]), h.dev["shares"],
                                        h.dev["list"], h.dev["count"])[2],
                    ra.block_table_release_shared(h.dev["table"], i32([64, 0, 0]), i32([0, 0, 0]),
                                                  h.dev["shares"], h.dev["list"], h.dev["count"])):
            assert got.tolist() == [-1] and h.dev["count"].tolist() == [count]
    h.dev["count"].fill_(len(h.free))
    h.check()


def test_entries_that_name_no_page_are_passed_over(device):
    h = Host(6, 2, 8, 20, [4, 0])
    h.table[0, 1], h.table[0, 3] = -5, 20
    h.dev["table"] = i32(h.table)
    h.do_release([64, 0], [0, 0])


def test_nothing_to_do(device):
    h = Host(7, 2, 8, 20, [4, 0])
    h.do_fork([], [], [])
    h.do_fork([0], [1], [0])
    h.do_release([0, 0], [0, 0])
    none = torch.empty((0, 8), dtype=torch.int32, device=DEV)
    r = ra.block_table_release_shared(none, i32([]), i32([]), h.dev["shares"], h.dev["list"],
                                      h.dev["count"])
    assert r.tolist() == [0]
    h.check()


def test_many_rows_and_long_prompts(device):
    """More forks than a workgroup's threads, more entries than a release's step."""
    B = 700
    h = Host(8, B, 330, 1500, [320] + [0] * (B - 1))
    lens = [5120 - 7 * (i % 50) for i in range(B - 1)]
    h.do_fork([0] * (B - 1), list(range(B - 1, 0, -1)), lens)
    rows = [5120] + [lens[B - 1 - b] for b in range(1, B)]
    d = h.dev
    got = ra.block_table_release_shared(d["table"], i32(rows), i32([0] * B), d["shares"], d["list"],
                                        d["count"])
    assert not bool(d["shares"].any())
    n = int(d["count"])
    assert n == h.num and sorted(d["list"][:n].tolist()) == list(range(h.num))
    assert got.tolist() == [h.num - len(h.free)]


def pools(seed, num, hkv, fp8):
    g = torch.Generator(device=DEV).manual_seed(seed)
    dt = torch.uint8 if fp8 else torch.int16
    k = torch.randint(0, 127 if fp8 else 32767, (num, hkv, 16, 128), generator=g, device=DEV).to(dt)
    v = torch.randint(0, 127 if fp8 else 32767, (num, hkv, 128, 16), generator=g, device=DEV).to(dt)
    view = (lambda x: x) if fp8 else (lambda x: x.view(torch.bfloat16))
    return k, v, lambda table: ra.PagedKV(view(k), view(v), table, *((1.0, 1.0) if fp8 else ()))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hkv", [1, 3, 8])
def test_page_copy(device, hkv, fp8):
    k, v, kv = pools(1, 40, hkv, fp8)
    src = [0, 5, -1, 7, 7, 40, 3, 12]
    dst = [20, 21, 22, 23, 24, 25, -1, 12]
    wk, wv = k.clone(), v.clone()
    for s, d in zip(src, dst):
        if 0 <= s < 40 and 0 <= d < 40:
            wk[d], wv[d] = k[s], v[s]
    ra.kv_page_copy(kv(i32([[0]])), i32(src), i32(dst))
    assert torch.equal(k, wk) and torch.equal(v, wv)
    ra.kv_page_copy(kv(i32([[0]])), i32([]), i32([]))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("hkv", [1, 8])
@pytest.mark.parametrize("T", [[1], [0, 1, 2, 17, 64, 100], [300, 5]], ids=lambda t: str(max(t)))
@pytest.mark.parametrize("dense", [0.15, 0.6, 1.0])
def test_compact(device, T, hkv, fp8, dense):
    rng = np.random.default_rng(sum(T) + hkv)
    B = len(T)
    start = rng.integers(0, 40, B)
    stride = -(-(40 + max(T)) // 16)
    table = rng.permutation(B * stride + 2)[:B * stride].reshape(B, stride)
    k, v, kv = pools(2, B * stride + 2, hkv, fp8)
    keep = [np.flatnonzero(rng.random(t) < dense) for t in T]
    index = np.full(sum(T) + 2, -1)
    for b in range(B):
        index[cu(T)[b]:cu(T)[b] + len(keep[b])] = keep[b]
    wk, wv = k.clone(), v.clone()
    for b in range(B):
        for i, j in enumerate(keep[b]):
            s, d = start[b] + j, start[b] + i
            ps, pd = table[b, s // 16], table[b, d // 16]
            wk[pd, :, d % 16] = k[ps, :, s % 16]
            wv[pd, :, :, d % 16] = v[ps, :, :, s % 16]
    ra.kv_page_compact(kv(i32(table)), i32(start), i32(cu(T)), i32(index),
                       i32([len(x) for x in keep]), max(T))
    assert torch.equal(k, wk) and torch.equal(v, wv)


def test_compact_whole_rows_and_broken_indices(device):
    """Without counts all of a row's entries are kept tokens; entries that would move a token back
    or come from past the table stay where they are."""
    k, v, kv = pools(3, 6, 2, False)
    table = np.array([[1, 4], [3, 0]])
    wk, wv = k.clone(), v.clone()
    for b, start, moves in ((0, 3, [(4, 1), (9, 2)]), (1, 30, [(1, 0)])):
        for s, d in moves:
            s, d = s + start, d + start
            wk[table[b, d // 16], :, d % 16] = k[table[b, s // 16], :, s % 16]
            wv[table[b, d // 16], :, :, d % 16] = v[table[b, s // 16], :, :, s % 16]
    ra.kv_page_compact(kv(i32(table)), i32([3, 30]), i32([0, 4, 7]), i32([0, 4, 9, 2, 1, 2, 900]))
    assert torch.equal(k, wk) and torch.equal(v, wv)
