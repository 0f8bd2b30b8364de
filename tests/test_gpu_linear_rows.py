"""Linear attention on the GPU, each row and head by itself, against the recurrence in 64 bits.

With A the state's sum of magnitudes (A_t = l A_{t-1} + |k_t| |v_t|^T) and M = scale A^T |q|:

out, each element. The result's rounding to bf16: 2^-8 |o|. Of M: the state and the scores in
two bf16 parts each, 2^-17 twice; their products' fp32 sums over 128 dims (two of them) and
64 tokens, 2.5 * 2^-17; the decays inside a chunk, powers of 2 up to 2^-126 whose exponents have
24 bits, 2^-17; the state's own error, below 2^-17: 6.5 * 2^-17 < 2^-14 in all. Decode has
fp32 sums over 128 dims alone: 2^-16.
states, each (slot, KV head), relative to its 2-norm: fp32 products and sums, the decayed values in
three parts (2^-24), over at most T / 64 chunk steps whose errors of 2^-24 add up where a
state remembers them all: (4 + T / 64) 2^-24.
"""
import math

import numpy as np
import pytest
import torch

import paper_2603_18815_amd as ra

pytestmark = pytest.mark.gpu
SCALE = 1.0 / math.sqrt(128)
DEV = "cuda:0"


def i32(x):
    return torch.as_tensor(np.ascontiguousarray(np.asarray(x, np.int32)), device=DEV)


def make(T, ctx, Hq, Hkv, seed, decay=None):
    g = torch.Generator(device=DEV).manual_seed(seed)
    B, total = len(T), sum(T)
    r = lambda h: torch.randn((total, h, 128), generator=g, device=DEV).bfloat16()
    if decay is None:
        decay = -torch.exp(torch.linspace(0.5, -9.0, Hkv))
    return dict(q=r(Hq), k=r(Hkv), v=r(Hkv), cu=i32(np.concatenate([[0], np.cumsum(T)])),
                ctx=i32(ctx), decay=torch.as_tensor(decay, dtype=torch.float32, device=DEV),
                slots=torch.randperm(B + 2, generator=g, device=DEV)[:B].to(torch.int32),
                states=3 * torch.randn((B + 2, Hkv, 128, 128), generator=g, device=DEV))


def recurrence(d, T, fresh):
    """All rows token by token: out, M, the same by root sums of squares (R), and states."""
    q, k, v = (d[n].double() for n in ("q", "k", "v"))
    Hkv = k.shape[1]
    lam = torch.exp(torch.nan_to_num(d["decay"].double(), nan=0.0, neginf=-1e300).clamp(max=0))
    lam = lam[None, :, None, None]
    slots, states = d["slots"].long(), d["states"].double()
    fresh = torch.as_tensor(fresh, device=DEV)[:, None, None, None]
    S = torch.where(fresh, 0.0, states[slots])
    A = S.abs()
    out, M, R = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
    first, T = d["cu"][:-1].long(), torch.as_tensor(T, device=DEV)
    for t in range(int(T.max())):
        rows = torch.nonzero(T > t).flatten()
        at = first[rows] + t
        S[rows] = lam * S[rows] + k[at][..., :, None] * v[at][..., None, :]
        A[rows] = lam * A[rows] + k[at].abs()[..., :, None] * v[at].abs()[..., None, :]
        qt = q[at].view(len(rows), Hkv, -1, 128)
        out[at] = SCALE * torch.matmul(qt, S[rows]).view_as(out[at])
        M[at] = SCALE * torch.matmul(qt.abs(), A[rows]).view_as(out[at])
        R[at] = SCALE * torch.matmul(qt.square(), A[rows].square()).sqrt().view_as(out[at])
    new = states.clone()
    some = T > 0
    new[slots[some]] = S[some]
    return out, M, R, new


def by_head(x):
    return x.double().flatten(2).norm(dim=2)


def check(d, T, ctx, out, states):
    want, M, _, wstates = recurrence(d, T, [c <= 0 for c in ctx])
    off = (out.double() - want).abs() - 2.0 ** -8 * want.abs() - 2.0 ** -14 * M
    assert off.max().item() <= 0, f"{(off > 0).sum().item()} of {off.numel()} elements"
    bound = (4 + max(T) / 64) * 2.0 ** -24 * by_head(wstates)
    assert (by_head(states.double() - wstates) <= bound).all()
    kept = torch.ones(len(states), dtype=torch.bool, device=DEV)
    kept[d["slots"].long()[torch.as_tensor(T, device=DEV) > 0]] = False
    assert torch.equal(states[kept], d["states"][kept])


def append(d, **kw):
    states = d["states"].clone()
    return ra.linear_append(d["q"], d["k"], d["v"], d["cu"], d["ctx"], states, d["slots"],
                            d["decay"], **kw), states


@pytest.mark.parametrize("Hq,Hkv", [(3, 3), (8, 4), (5, 1), (32, 1)])
def test_rows_of_all_lengths(Hq, Hkv, device):
    T = [1, 0, 2, 15, 16, 17, 63, 64, 65, 127, 0, 128, 129, 300, 0]
    ctx = [b % 3 for b in range(len(T))]
    d = make(T, ctx, Hq, Hkv, seed=Hq)
    check(d, T, ctx, *append(d))


# rows cut into stretches: alone, among short rows, many stretches of one KV head, of one chunk
@pytest.mark.parametrize("T,Hq,Hkv", [
    ([5000], 2, 2), ([3001, 17, 1024], 2, 1), ([3] * 150 + [2000] + [1] * 30 + [1100, 0, 2], 4, 4),
    ([1, 0, 700, 129, 0, 640], 1, 1), ([412, 493], 32, 8), ([8200], 16, 1), ([4100], 8, 2)])
def test_cut_rows(T, Hq, Hkv, device):
    ctx = [(b + 1) % 3 for b in range(len(T))]
    d = make(T, ctx, Hq, Hkv, seed=len(T))
    assert ra.linear_append_workspace_size(len(T), Hq, Hkv, sum(T), max(T)) > 0
    check(d, T, ctx, *append(d))


# workgroups that share a row's heads: more rows than a wave orders by their length, an odd
# number of heads each, two and four at once
@pytest.mark.parametrize("T,Hq,Hkv", [
    ([400] + [40, 95, 1, 0, 64] * 20, 16, 4), ([400] + [90, 0, 150] * 33 + [2], 24, 4),
    ([500, 130, 490, 0, 7, 500, 480, 500, 500], 16, 8),
    ([512, 130, 450, 0, 500, 1, 512, 64, 401], 32, 8), ([600, 40, 580, 590, 0, 600, 3, 600, 599], 64, 8)])
def test_rows_whose_heads_are_shared(T, Hq, Hkv, device):
    ctx = [(b + 1) % 3 for b in range(len(T))]
    d = make(T, ctx, Hq, Hkv, seed=len(T))
    need = ra.linear_append_workspace_size(len(T), Hq, Hkv, sum(T), max(T))
    assert need == len(T) * Hkv * 65536                   # a state a row
    check(d, T, ctx, *append(d))


@pytest.mark.parametrize("decay", [[0.0, -1e-6], [-1e-4, -50.0], [float("-inf"), -1000.0],
                                   [0.5, float("nan")]])
@pytest.mark.parametrize("T", [[333, 70], [1500]])
def test_decays_head_by_head(T, decay, device):
    ctx = [9, 0][:len(T)]
    d = make(T, ctx, 4, 2, seed=4, decay=decay)
    check(d, T, ctx, *append(d))


@pytest.mark.parametrize("T,Hq,Hkv", [([1000, 40], 2, 1), ([1000, 40], 3, 3), ([3000], 4, 2),
                                      ([500] * 9, 16, 8)])
def test_a_large_common_part_that_the_queries_do_not_see(T, Hq, Hkv, device):
    """Keys and values with a common part, and queries across it: the state is some hundred
    times what a result takes from it. Each (row, head), in 2-norms: the result's rounding and,
    as the roundings of the 128 dims are independent, eight times 2^-17 of R."""
    d = make(T, [0] * len(T), Hq, Hkv, seed=Hq, decay=[-1e-4] * Hkv)
    u = torch.where(torch.arange(128, device=DEV) % 3 > 0, 1.0, -1.0)
    d["k"] = (d["k"].float() + 4 * u).bfloat16()
    d["v"] = (d["v"].float() + 1).bfloat16()
    q = d["q"].float()
    d["q"] = (q - (q @ u)[..., None] * u / 128).bfloat16()
    out, states = append(d)
    want, M, R, wstates = recurrence(d, T, [True] * len(T))
    at = 0
    for n in T:
        rows = slice(at, at + n)
        norm = lambda x: x[rows].double().transpose(0, 1).flatten(1).norm(dim=1)
        assert (norm(R) > 50 * norm(want)).all() or n < 500   # what the test is about
        assert (norm(out.double() - want) <= 2.0 ** -8 * norm(want) + 2.0 ** -14 * norm(R)).all()
        at += n
    bound = (4 + max(T) / 64) * 2.0 ** -24 * by_head(wstates)
    assert (by_head(states.double() - wstates) <= bound).all()


@pytest.mark.parametrize("Hq,Hkv,B", [(1, 1, 1), (32, 8, 3), (8, 8, 70), (32, 1, 2), (6, 2, 9),
                                      (32, 32, 40)])
def test_decode_each_element(Hq, Hkv, B, device):
    d = make([1] * B, [0] * B, Hq, Hkv, B)
    lens = np.random.default_rng(B).integers(1, 5, B)
    lens[0] = 7
    states = d["states"].clone()
    out = ra.linear_decode(d["q"], d["k"], d["v"], states, d["slots"], i32(lens), d["decay"])
    want, M, _, wstates = recurrence(d, [1] * B, [n <= 1 for n in lens])
    assert ((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -16 * M).all()
    assert (by_head(states.double() - wstates) <= 4 * 2.0 ** -24 * by_head(wstates)).all()
