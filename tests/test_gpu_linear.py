"""Linear attention on the GPU against the token-by-token recurrence in 64 bits.

Tolerances, relative to a tensor's 2-norm. out: three roundings to bf16 (the scores, the
state as the query meets it, the result), each at most 2^-8 relative to its value: 3 * 2^-8.
Decode rounds the result alone: 2^-8. states: fp32 products and sums, the decayed values in
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


def i32(x):
    return torch.as_tensor(np.ascontiguousarray(np.asarray(x, np.int32)), device="cuda:0")


def rel(a, b):
    n = b.norm().item()
    d = (a.double() - b).norm().item()
    return d / n if n else d


def make(T, ctx, Hq, Hkv, seed, extra=0, decay=None, num_slots=None):
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    B, total = len(T), sum(T) + extra
    r = lambda h: torch.randn((total, h, 128), generator=g, device="cuda:0").bfloat16()
    num_slots = num_slots or B + 2
    slots = torch.randperm(num_slots, generator=g, device="cuda:0")[:B].to(torch.int32)
    if decay is None:
        decay = -torch.exp(torch.linspace(0.5, -9.0, Hkv))
    decay = torch.as_tensor(decay, dtype=torch.float32, device="cuda:0")
    states = 3 * torch.randn((num_slots, Hkv, 128, 128), generator=g, device="cuda:0")
    return dict(q=r(Hq), k=r(Hkv), v=r(Hkv), cu=i32(np.concatenate([[0], np.cumsum(T)])),
                ctx=i32(ctx), slots=slots, decay=decay, states=states)


def recurrence(d, T, fresh, scale=SCALE):
    """(out, states) in 64 bits; rows without tokens and slots outside the pool left out."""
    q, k, v, states = (d[n].double() for n in ("q", "k", "v", "states"))
    out = torch.zeros_like(q)
    lam = torch.exp(torch.nan_to_num(d["decay"].double(), nan=0.0, neginf=-1e300).clamp(max=0))
    lam = lam[:, None, None]
    at = 0
    for b, n in enumerate(T):
        slot = d["slots"][b].item()
        if n and 0 <= slot < states.shape[0]:
            S = torch.zeros_like(states[slot]) if fresh[b] else states[slot].clone()
            for t in range(at, at + n):
                S = lam * S + k[t][:, :, None] * v[t][:, None, :]
                out[t] = scale * torch.matmul(q[t].view(S.shape[0], -1, 128), S).view(-1, 128)
            states[slot] = S
        at += n
    return out, states


def run_append(d, T, scale=None, **kw):
    states = d["states"].clone()
    out = ra.linear_append(d["q"], d["k"], d["v"], d["cu"], d["ctx"], states, d["slots"],
                           d["decay"], scale=scale, **kw)
    return out, states


def check_append(T, ctx, Hq, Hkv, seed=0, **kw):
    d = make(T, ctx, Hq, Hkv, seed, **kw)
    out, states = run_append(d, T)
    want, wstates = recurrence(d, T, [c <= 0 for c in ctx])
    n = sum(T)
    assert rel(out[:n], want[:n]) <= 3 * 2.0 ** -8
    assert rel(states, wstates) <= (4 + max(T) / 64) * 2.0 ** -24
    rows = [i for i in range(states.shape[0]) if i not in
            [d["slots"][b].item() for b in range(len(T)) if T[b]]]
    assert torch.equal(states[rows], d["states"][rows])       # nobody else's state moved
    return d, out, states


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300, 1000])
def test_append_lengths(T, device):
    check_append([T], [5], 4, 2, seed=T)
    check_append([T], [0], 2, 2, seed=T)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 8), (8, 2), (16, 1), (32, 1), (3, 3), (6, 2), (10, 2),
                                    (12, 1)])
def test_append_heads(Hq, Hkv, device):
    check_append([100, 33], [7, 0], Hq, Hkv, seed=Hq)


def test_append_ragged_rows(device):
    T = [0, 5, 0, 200, 64, 1, 0, 129, 0]
    check_append(T, [3, 0, 0, 9, 1, 0, 5, 77, 2], 4, 2, seed=1)


def test_append_long_row_in_stretches(device):
    check_append([5000], [0], 2, 2, seed=2)
    check_append([3001, 17, 1024], [4, 0, 6], 2, 1, seed=3)


@pytest.mark.parametrize("T,Hkv", [
    ([3] * 150 + [2000] + [1] * 30 + [1100, 0, 2], 4),   # more rows than stretches
    ([1, 0, 700, 129, 0, 640], 1),
    ([2] * 64 + [900], 1), ([900] + [2] * 65, 1)])
def test_append_long_rows_among_short_ones(T, Hkv, device):
    d, out, states = check_append(T, [b % 3 for b in range(len(T))], Hkv, Hkv, seed=len(T))
    need = ra.linear_append_workspace_size(len(T), Hkv, Hkv, sum(T), max(T))
    assert 0 < need <= (2 * 256 + Hkv) * 65536            # two stretches a compute unit
    tight = torch.empty(need, dtype=torch.uint8, device="cuda:0").fill_(0xff)
    again, states2 = run_append(d, T, workspace=tight)
    assert torch.equal(again, out) and torch.equal(states2, states)


@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (16, 8), (64, 8)])
def test_append_rows_shared_by_their_heads(Hq, Hkv, device):
    """Few rows of some length: workgroups that share a row's query heads, one of which
    writes the state. With an empty row, one of a token, one without a slot, one that is new."""
    T = [512, 130, 450, 0, 500, 1, 512, 64, 401]
    ctx = [3, 0, 1, 5, 9, 7, 0, 2, 4]
    d = make(T, ctx, Hq, Hkv, seed=Hq)
    d["slots"][4] = -1
    states = d["states"].clone()
    need = ra.linear_append_workspace_size(len(T), Hq, Hkv, sum(T), max(T))
    assert need == len(T) * Hkv * 65536                   # a state a row
    ws = torch.empty(need, dtype=torch.uint8, device="cuda:0").fill_(0xff)
    out = ra.linear_append(d["q"], d["k"], d["v"], d["cu"], d["ctx"], states, d["slots"],
                           d["decay"], workspace=ws)
    want, wstates = recurrence(d, T, [c <= 0 for c in ctx])
    assert rel(out, want) <= 3 * 2.0 ** -8
    assert (out[sum(T[:4]):sum(T[:5])] == 0).all()
    assert rel(states, wstates) <= (4 + max(T) / 64) * 2.0 ** -24
    kept = [i for i in range(states.shape[0]) if i not in
            [d["slots"][b].item() for b in range(len(T)) if T[b]]]
    assert torch.equal(states[kept], d["states"][kept])


@pytest.mark.parametrize("T,at", [([200, 40], 70), ([200, 40], 199), ([200, 40], 0), ([3000], 1500),
                                  ([3000], 2999)])
@pytest.mark.parametrize("what", ["k", "v"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_append_keeps_what_is_not_finite_behind(T, at, what, bad, device):
    """An infinite or NaN key or value changes its own token and later ones alone: for a key
    all of the KV head's dims, for a value its dim."""
    d = make(T, [3] * len(T), 4, 2, seed=at)
    out, states = run_append(d, T)
    d[what][at, 1, 37] = bad
    out2, states2 = run_append(d, T)
    own = torch.zeros_like(out, dtype=torch.bool)
    kept = torch.zeros_like(states, dtype=torch.bool)
    slot = d["slots"][0].item()
    if what == "k":
        own[at:T[0], 2:] = True
        kept[slot, 1, 37] = True
    else:
        own[at:T[0], 2:, 37] = True
        kept[slot, 1, :, 37] = True
    assert torch.equal(out2[~own], out[~own])
    assert torch.equal(states2[~kept], states[~kept])
    assert not torch.isfinite(out2[at, 2:][own[at, 2:]]).any()
    assert not torch.isfinite(states2[kept]).any()


@pytest.mark.parametrize("decay", [[0.0, -1e-6], [-1e-4, -50.0], [float("-inf"), -1000.0],
                                   [0.5, float("nan")]])
def test_append_decays(decay, device):
    """No decay, hardly any, all of it; values above 0 and NaN count as none."""
    check_append([333, 70], [9, 0], 2, 2, seed=4, decay=decay)


def test_fresh_rows_ignore_the_pool(device):
    d = make([90, 40], [0, 0], 4, 2, 5)
    d["states"].fill_(float("nan"))
    out, states = run_append(d, [90, 40])
    want, ws = recurrence(d, [90, 40], [True, True])
    assert rel(out, want) <= 3 * 2.0 ** -8
    used = d["slots"].long()
    assert rel(states[used], ws[used]) <= 8 * 2.0 ** -24
    o1 = ra.linear_decode(d["q"][:2].contiguous(), d["k"][:2].contiguous(),
                          d["v"][:2].contiguous(), d["states"], d["slots"], i32([1, 1]), d["decay"])
    assert torch.isfinite(o1).all()


def test_tokens_behind_the_last_row_and_bad_slots(device):
    T = [70, 20, 33]
    d = make(T, [1, 1, 1], 4, 2, 6, extra=19)
    d["slots"][1] = 99                                # outside the pool
    out = torch.full((sum(T) + 19, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda:0")
    states = d["states"].clone()
    ra.linear_append(d["q"], d["k"], d["v"], d["cu"], d["ctx"], states, d["slots"], d["decay"],
                     out=out)
    want, ws = recurrence(d, T, [False] * 3)
    assert rel(out[:sum(T)], want[:sum(T)]) <= 3 * 2.0 ** -8
    assert (out[70:90] == 0).all() and (out[sum(T):] == 7.0).all()
    assert rel(states, ws) <= 8 * 2.0 ** -24


@pytest.mark.parametrize("Hq,Hkv,B", [(1, 1, 1), (32, 8, 3), (8, 8, 70), (16, 1, 5), (32, 1, 2),
                                      (6, 2, 9), (32, 32, 40)])
def test_decode(Hq, Hkv, B, device):
    d = make([1] * B, [0] * B, Hq, Hkv, B)
    lens = np.random.default_rng(B).integers(1, 5, B)
    lens[0] = 7
    if B > 2:
        lens[1], lens[2] = 1, 0
        d["slots"][B - 1] = -1
    states = d["states"].clone()
    out = ra.linear_decode(d["q"], d["k"], d["v"], states, d["slots"], i32(lens), d["decay"])
    T = [int(n > 0) for n in lens]
    full = [1] * B
    want, ws = recurrence(dict(d, slots=torch.where(i32(lens) > 0, d["slots"], -1)), full,
                          [n <= 1 for n in lens])
    assert rel(out, want) <= 2.0 ** -8
    assert rel(states, ws) <= 4 * 2.0 ** -24
    for b in range(B):
        if not T[b]:
            assert (out[b] == 0).all()


@pytest.mark.parametrize("scale", [0.0, -0.5, 3.0])
def test_scale(scale, device):
    d = make([100], [3], 4, 2, 8)
    out, states = run_append(d, [100], scale)
    want, ws = recurrence(d, [100], [False], scale)
    assert rel(out, want) <= 3 * 2.0 ** -8 and rel(states, ws) <= 8 * 2.0 ** -24


def test_append_equals_decode_steps(device):
    """The same tokens one at a time: the states agree to fp32 sums, the outputs to bf16."""
    T = 90
    d = make([T], [4], 8, 2, 9)
    out, states = run_append(d, [T])
    st = d["states"].clone()
    for t in range(T):
        o = ra.linear_decode(d["q"][t:t + 1], d["k"][t:t + 1], d["v"][t:t + 1], st, d["slots"],
                             i32([5 + t]), d["decay"])
        assert rel(o[0], out[t].double()) <= 4 * 2.0 ** -8
    assert rel(st, states.double()) <= (8 + T) * 2.0 ** -24


def test_chunks_of_one_row_continue(device):
    """A row appended in pieces keeps its history: the state after them is that of one call."""
    d = make([400], [0], 4, 2, 10)
    out, states = run_append(d, [400])
    st, at, outs = d["states"].clone(), 0, []
    for n in (1, 150, 64, 185):
        sl = slice(at, at + n)
        outs.append(ra.linear_append(d["q"][sl], d["k"][sl], d["v"][sl], i32([0, n]), i32([at]),
                                     st, d["slots"], d["decay"]))
        at += n
    want, ws = recurrence(d, [400], [True])
    assert rel(torch.cat(outs), want) <= 3 * 2.0 ** -8
    assert rel(st, ws) <= 16 * 2.0 ** -24


def test_refusals(device):
    d = make([10], [0], 4, 2, 0)
    call = lambda **kw: ra.linear_append(**dict(dict(
        q=d["q"], k_new=d["k"], v_new=d["v"], cu_q=d["cu"], ctx_lens=d["ctx"], states=d["states"],
        slots=d["slots"], log_decay=d["decay"]), **kw))
    with pytest.raises(ValueError, match="k_new"):
        call(k_new=d["k"][:, :1].contiguous())
    with pytest.raises(ValueError, match="contiguous"):
        call(q=d["q"].transpose(1, 2))
    with pytest.raises(ValueError, match="states"):
        call(states=d["states"][..., :64].contiguous())
    with pytest.raises(TypeError, match="states"):
        call(states=d["states"].bfloat16())
    with pytest.raises(ra.RolloutAttnError):
        call(q=d["q"][:, :3].contiguous())
    with pytest.raises(ra.RolloutAttnError):
        call(scale=float("nan"))
    empty = ra.linear_append(d["q"][:0], d["k"][:0], d["v"][:0], i32([0, 0]), d["ctx"],
                             d["states"], d["slots"], d["decay"])
    assert empty.shape == (0, 4, 128)


@pytest.mark.parametrize("T,Hq,Hkv", [([900, 3, 0, 40], 2, 2), ([512, 300, 480, 512, 512, 500, 401], 32, 8)])
def test_append_workspace_at_16_bytes_and_no_larger_than_asked(T, Hq, Hkv, device):
    d = make(T, [1] * len(T), Hq, Hkv, 9)
    out, states = run_append(d, T)
    need = ra.linear_append_workspace_size(len(T), Hq, Hkv, sum(T), max(T))
    assert need > 0
    store = torch.full((need + 512,), 0xab, dtype=torch.uint8, device="cuda:0")
    out2, states2 = run_append(d, T, workspace=store[16:16 + need])
    assert torch.equal(out2, out) and torch.equal(states2, states)
    assert (store[:16] == 0xab).all() and (store[16 + need:] == 0xab).all()
