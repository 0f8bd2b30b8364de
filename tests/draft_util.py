"""Inputs and plain 64-bit references of the operators on drafted trees (test helpers)."""
import math

import numpy as np
import torch

DEV = "cuda:0"
SCALE = 1.0 / math.sqrt(128)


def i32(x, dev=DEV):
    return torch.as_tensor(np.ascontiguousarray(np.asarray(x, np.int32)), device=dev)


def cu(T):
    return np.concatenate([[0], np.cumsum(T)])


def random_tree(rng, T, back=6):
    """Parents of T nodes: -1 for the root, else one of the `back` nodes before."""
    return np.array([-1] + [int(rng.integers(max(0, i - back), i)) for i in range(1, T)][:max(T - 1, 0)],
                    np.int64)[:T]


def ancestors(parents):
    """bool [T][T]: node j is node i or above it."""
    T = len(parents)
    sees = np.zeros((T, T), bool)
    for i in range(T):
        j = i
        while j >= 0:
            sees[i, j] = True
            j = parents[j] if 0 <= parents[j] < j else -1
    return sees


def pack(masks, words):
    """int64 [sum T][words] of bool [T][T] masks."""
    out = np.zeros((sum(len(m) for m in masks), words * 64), bool)
    at = 0
    for m in masks:
        if len(m):
            out[at:at + len(m), :m.shape[1]] = m
        at += len(m)
    return np.packbits(out, axis=1, bitorder="little").view(np.int64)


class Cache:
    """Pools with every row's pages shuffled among decoys; whatever no token owns holds NaN."""

    def __init__(self, seed, lens, hkv, fp8=False, spare=3, stride=None):
        g = torch.Generator(device=DEV).manual_seed(seed)
        rng = np.random.default_rng(seed)
        pages = [-(-n // 16) for n in lens]
        self.num = sum(pages) + spare
        order = rng.permutation(self.num)
        stride = max(1, max(pages, default=1)) + 1 if stride is None else stride
        table = np.full((len(lens), stride), order[-1], np.int64)
        at = 0
        for b, n in enumerate(pages):
            table[b, :n] = order[at:at + n]
            at += n
        self.lens, self.fp8, self.hkv = list(lens), fp8, hkv
        self.scales = (0.02, 0.03) if fp8 else (1.0, 1.0)
        k = torch.randn((self.num, hkv, 16, 128), generator=g, device=DEV)
        v = torch.randn((self.num, hkv, 128, 16), generator=g, device=DEV)
        used = np.zeros((self.num, 16), bool)
        for b, n in enumerate(lens):
            for p in range(pages[b]):
                used[table[b, p], :min(16, n - 16 * p)] = True
        dead = torch.as_tensor(~used, device=DEV)
        if fp8:
            self.k = (k * 30).to(torch.float8_e4m3fn).view(torch.uint8)
            self.v = (v * 30).to(torch.float8_e4m3fn).view(torch.uint8)
            nan = 0x7f
        else:
            self.k, self.v = k.bfloat16(), v.bfloat16()
            nan = float("nan")
        self.k.masked_fill_(dead[:, None, :, None], nan)
        self.v.masked_fill_(dead[:, None, None, :], nan)
        self.table_host = table
        self.table = i32(table)

    def kv(self):
        import paper_2603_18815_amd as ra
        return ra.PagedKV(self.k, self.v, self.table, *(self.scales if self.fp8 else ()))

    def place(self, b, pos):
        return int(self.table_host[b, pos // 16]), pos % 16

    def row(self, b, n):
        """Keys and values of the row's first n tokens, fp64 [n][Hkv][128]."""
        pages = torch.as_tensor(self.table_host[b, :-(-n // 16)], device=DEV)
        val = (lambda x, s: x.view(torch.float8_e4m3fn).double() * np.float64(np.float32(s))) \
            if self.fp8 else (lambda x, s: x.double())
        k = val(self.k[pages], self.scales[0]).permute(0, 2, 1, 3).reshape(-1, self.hkv, 128)
        v = val(self.v[pages], self.scales[1]).permute(0, 3, 1, 2).reshape(-1, self.hkv, 128)
        return k[:n], v[:n]


def tree_reference(q, T, ctx, masks, cache, scale=SCALE):
    """(out, lse, tolerance of out, tolerance of lse), fp64, from the definition.

    Tolerances: a score is a sum of 128 products, exact in fp32, off by at most 132 half steps
    (2^-24) of the sum of their sizes, with the scaling and the exponential's own; a weight is
    taken in two bf16 parts, off by 2^-16 of itself; sums over L keys are off by L half steps."""
    total, Hq, _ = q.shape
    out = torch.zeros((total, Hq, 128), dtype=torch.float64, device=q.device)
    lse = torch.full((total, Hq), float("-inf"), dtype=torch.float64, device=q.device)
    otol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    at = 0
    for b, n in enumerate(T):
        if n == 0:
            continue
        L = ctx[b] + n
        k, v = cache.row(b, L)
        sees = torch.ones((n, L), dtype=torch.bool, device=q.device)
        sees[:, ctx[b]:] = torch.as_tensor(masks[b], device=q.device)
        G = Hq // k.shape[1]
        for h in range(Hq):
            kh, vh, x = k[:, h // G], v[:, h // G], q[at:at + n, h].double()
            s = (x @ torch.nan_to_num(kh, 0, 0, 0).t()) * scale
            size = (x.abs() @ torch.nan_to_num(kh, 0, 0, 0).abs().t()) * abs(scale)
            s = s.masked_fill(~sees, float("-inf"))
            z = torch.logsumexp(s, 1)
            some = torch.isfinite(z)
            w = torch.where(some[:, None], torch.exp(s - torch.where(some, z, 0.0)[:, None]), 0.0)
            clean = torch.nan_to_num(vh, 0, 0, 0)
            out[at:at + n, h] = w @ clean
            lse[at:at + n, h] = torch.where(some, z, float("-inf"))
            es = 2.0**-24 * 132 * size.masked_fill(~sees, 0).amax(1) if L else 0
            ltol[at:at + n, h] = es + (L + 8 + 4 * z.abs().nan_to_num(0, 0, 0)) * 2.0**-24
            otol[at:at + n, h] = (2.0**-16 + 2 * es + 2 * L * 2.0**-24)[:, None] * (w @ clean.abs()) + 1e-30
        at += n
    return out, lse, otol, ltol


def assert_within(got, want, tol, what):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    bad = torch.isfinite(want)
    assert torch.equal(got[~bad & ~torch.isnan(want)], want[~bad & ~torch.isnan(want)]), what
    worst = ((got - want).abs() / tol)[bad]
    assert worst.numel() == 0 or float(worst.max()) <= 1.0, (what, float(worst.max()))
