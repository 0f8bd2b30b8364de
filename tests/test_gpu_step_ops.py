"""The step operators as a rollout uses them: together, captured, and on other streams.

A step of a small model with one paged layer and one linear layer: pages reserved for the
new token, its key and value written, paged decode, linear decode, logits, a token drawn.
"""
import math

import numpy as np
import pytest
import torch

import paper_2603_18815_amd as ra
from tests.test_gpu_sample import host

pytestmark = pytest.mark.gpu
B, HQ, HKV, V, STRIDE = 5, 8, 2, 900, 16
DEV = "cuda:0"


def i32(x):
    return torch.as_tensor(np.ascontiguousarray(np.asarray(x, np.int32)), device=DEV)


class Model:
    """Random weights; a token's q, k, v of both layers are rows of an embedding."""

    def __init__(self, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device=DEV)
        self.q, self.k, self.v = rnd(V, HQ, 128).bfloat16(), rnd(V, HKV, 128).bfloat16(), rnd(V, HKV, 128).bfloat16()
        self.head = rnd(HQ * 128, V) / math.sqrt(HQ * 128) * 4
        self.decay = -torch.exp(torch.tensor([0.0, -4.0], device=DEV))
        self.u = torch.rand((64, B), generator=g, device=DEV)
        self.top_p = torch.full((B,), 0.95, device=DEV)
        self.top_k = i32([0, 50, 5, 0, 300])
        self.temperature = torch.tensor([1.0, 0.8, 0.0, 1.2, 1.0], device=DEV)
        pages = B * STRIDE
        self.table = torch.zeros((B, STRIDE), dtype=torch.int32, device=DEV)
        self.free = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
        self.count = i32([pages])
        self.kv = ra.PagedKV(torch.zeros((pages, HKV, 16, 128), dtype=torch.bfloat16, device=DEV),
                             torch.zeros((pages, HKV, 128, 16), dtype=torch.bfloat16, device=DEV),
                             self.table)
        self.states = torch.full((B + 1, HKV, 128, 128), float("nan"), device=DEV)
        self.slots = i32([4, 0, 5, 1, 2])
        self.lens = i32([0] * B)
        self.one = i32([1] * B)
        self.tokens = i32([7, 100, 3, 899, 42])
        self.turn = torch.zeros((1,), dtype=torch.int64, device=DEV)

    def everything(self):
        return [self.table, self.free, self.count, self.kv.k_pool, self.kv.v_pool, self.states,
                self.lens, self.tokens, self.turn]

    def prompt(self, lens, tokens):
        """The prompts' tokens through both layers; the next token is theirs last one's."""
        total = sum(lens)
        cu, kv_lens, slots, taken = ra.block_table_extend(self.table, self.lens, i32(lens), self.free,
                                                          self.count, total_new=total)
        q, k, v = self.q[tokens], self.k[tokens], self.v[tokens]
        paged, _ = ra.append_write(q, k, v, cu, self.lens, self.kv, max_q_len=max(lens),
                                   max_kv_len=max(lens))
        linear = ra.linear_append(q, k, v, cu, self.lens, self.states, self.slots, self.decay,
                                  max_q_len=max(lens))
        self.lens.copy_(kv_lens)
        return paged, linear, taken

    def step(self):
        cu, kv_lens, slots, taken = ra.block_table_extend(self.table, self.lens, self.one, self.free,
                                                          self.count, total_new=B)
        t = self.tokens.long()
        q, k, v = self.q[t], self.k[t], self.v[t]
        ra.kv_page_write(k, v, cu, self.lens, self.kv, max_new=1, max_pos=STRIDE * 16)
        paged, _ = ra.decode(q, self.kv, kv_lens, max_kv_len=STRIDE * 16)
        linear = ra.linear_decode(q, k, v, self.states, self.slots, kv_lens, self.decay)
        logits = (paged + linear.float()).view(B, -1) @ self.head
        u = self.u.index_select(0, self.turn).view(B)
        tokens, logp = ra.token_sample(logits, u, self.temperature, self.top_k, self.top_p,
                                       want_logprob=True)
        self.lens.copy_(kv_lens)
        self.tokens.copy_(tokens)
        self.turn.add_(1)
        return dict(cu=cu, slots=slots, taken=taken, paged=paged, linear=linear, logits=logits,
                    tokens=tokens, logp=logp)


def test_a_rollout(device):
    """A prompt, 40 steps (across page ends), every piece checked; then the rows end."""
    m = Model(1)
    lens = [3, 0, 17, 1, 64]
    rng = np.random.default_rng(2)
    history = [rng.integers(0, V, n).tolist() for n in lens]
    toks = torch.tensor(sum(history, []), device=DEV)
    paged, linear, taken = m.prompt(lens, toks)
    assert taken.item() == sum(-(-n // 16) for n in lens)
    for step in range(40):
        for b, t in enumerate(m.tokens.tolist()):
            history[b].append(t)
        o = m.step()
        assert o["cu"].tolist() == list(range(B + 1))
        assert m.lens.tolist() == [len(h) for h in history]
        z, u = o["logits"].double().cpu().numpy(), m.u[step].tolist()
        for b in range(B):
            want = host(z[b], u[b], m.temperature[b].item(), m.top_k[b].item(), m.top_p[b].item())
            assert o["tokens"][b].item() == want[0], (step, b)
            assert abs(o["logp"][b].item() - want[1]) <= 2.0 ** -24 * abs(want[1]) + 2.0 ** -28
    # the whole history at once: the paged layer's last outputs and the linear layer's state
    for b in range(B):
        h = torch.tensor(history[b], device=DEV)
        n = len(history[b])
        q, k, v = m.q[h], m.k[h], m.v[h]
        state = torch.zeros((1, HKV, 128, 128), device=DEV)
        lin = ra.linear_append(q, k, v, i32([0, n]), i32([0]), state, i32([0]), m.decay, max_q_len=n)
        got = m.states[m.slots[b].long()]
        assert (got - state[0]).norm() / state.norm() <= (16 + n) * 2.0 ** -24
        # one rounding of decode's result against three of append's
        assert (lin[-1].double() - o["linear"][b].double()).norm() / lin[-1].double().norm() <= 4 * 2.0 ** -8
        kk, vv = k.double().repeat_interleave(HQ // HKV, 1), v.double().repeat_interleave(HQ // HKV, 1)
        p = torch.softmax(torch.einsum("hd,khd->hk", q[-1].double().cpu(), kk.cpu()) / math.sqrt(128), 1)
        ref = torch.einsum("hk,khd->hd", p, vv.cpu())
        assert (o["paged"][b].double().cpu() - ref).norm() / ref.norm() <= 5e-3
    gone = ra.block_table_release(m.table, m.lens, torch.zeros_like(m.lens), m.free, m.count)
    assert gone.item() == sum(-(-len(h) // 16) for h in history)
    assert sorted(m.free.tolist()) == list(range(B * STRIDE))
    assert torch.isnan(m.states[3]).all()                 # the slot that no row has


def test_a_refused_reservation_writes_nothing(device):
    """Too few pages: the outputs of extend make the following page write one of no token."""
    m = Model(3)
    m.count.fill_(B - 1)
    before = [x.clone() for x in m.everything()]
    cu, kv_lens, slots, taken = ra.block_table_extend(m.table, m.lens, m.one, m.free, m.count, total_new=B)
    ra.kv_page_write(m.k[:B].contiguous(), m.v[:B].contiguous(), cu, m.lens, m.kv, max_new=1,
                     max_pos=STRIDE * 16)
    torch.cuda.synchronize()
    assert taken.item() == -1 and kv_lens.tolist() == [0] * B
    for x, y in zip(before, m.everything()):
        assert torch.equal(torch.nan_to_num(x.float()), torch.nan_to_num(y.float()))


def test_step_replays_in_a_graph(device):
    """Eager steps and replays of one captured step from the same start: the same bits."""
    eager, m = Model(5), Model(5)
    toks = torch.arange(30, device=DEV)
    for x in (eager, m):
        x.prompt([6] * B, toks)
    start = [x.clone() for x in m.everything()]
    want = [eager.step() for _ in range(20)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        m.step()                                           # warm-up
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = m.step()
    for x, x0 in zip(m.everything(), start):
        x.copy_(x0)
    for turn, w in enumerate(want):
        graph.replay()
        torch.cuda.synchronize()
        for name in w:
            assert torch.equal(out[name], w[name]), (turn, name)
        torch.randn(1000, device=DEV).sum()                # eager work between the replays
        torch.cuda.synchronize()
    assert torch.equal(m.states[m.slots.long()], eager.states[eager.slots.long()])


def test_prompt_calls_replay_in_a_graph(device):
    """Cut and whole rows of linear_append, many-page tables: replays equal the eager call."""
    g = torch.Generator(device=DEV).manual_seed(9)
    T = [900, 1, 77]
    total = sum(T)
    rnd = lambda h: torch.randn((total, h, 128), generator=g, device=DEV).bfloat16()
    q, k, v = rnd(4), rnd(2), rnd(2)
    cu, ctx, slots = i32([0, 900, 901, 978]), i32([0, 5, 3]), i32([0, 1, 2])
    decay = torch.tensor([-0.5, -0.001], device=DEV)
    first = torch.randn((3, 2, 128, 128), generator=g, device=DEV)
    states, out = first.clone(), torch.empty_like(q)
    ws = torch.empty(max(1, ra.linear_append_workspace_size(3, 4, 2, total, 900)), dtype=torch.uint8,
                     device=DEV)
    start, new = i32([5] * 600), i32([20] * 600)
    table = torch.arange(600 * 8, device=DEV).to(torch.int32).view(600, 8).clone()
    free, count = torch.arange(5000, 9000, device=DEV).to(torch.int32), i32([4000])
    outs = [torch.empty(601, dtype=torch.int32, device=DEV), torch.empty(600, dtype=torch.int32, device=DEV),
            torch.empty(12000, dtype=torch.int64, device=DEV), torch.empty(1, dtype=torch.int32, device=DEV)]
    gone = torch.empty(1, dtype=torch.int32, device=DEV)
    z = torch.randn((3, 20000), generator=g, device=DEV)
    u, p = torch.rand(3, generator=g, device=DEV), torch.full((3,), 0.9, device=DEV)
    tok, lp = torch.empty(3, dtype=torch.int32, device=DEV), torch.empty(3, device=DEV)
    sws = torch.empty(max(1, ra.token_sample_workspace_size(3, 20000)), dtype=torch.uint8, device=DEV)

    def call():
        states.copy_(first)
        ra.linear_append(q, k, v, cu, ctx, states, slots, decay, max_q_len=900, out=out, workspace=ws)
        ra.block_table_extend(table, start, new, free, count, 12000, *outs)
        ra.block_table_release(table, outs[1], start, free, count, released=gone)
        ra.token_sample(z, u, None, None, p, None, tok, lp, workspace=sws)
    call()
    torch.cuda.synchronize()
    results = [out, states, table, free, count, *outs, gone, tok, lp]
    want = [x.clone() for x in results]
    assert gone.item() == outs[3].item() > 0
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        ws.fill_(0xFF)
        sws.fill_(0xFF)
        for x in (out, tok, lp, gone):
            x.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, w in zip(results, want):
            assert torch.equal(x, w)


@pytest.mark.parametrize("handle", ["stream", "int"])
def test_side_streams_with_binding_allocations(handle, device):
    """Two calls of each operator at once, on streams of their own, while the default stream
    allocates and fills memory: the results are those of the default stream."""
    g = torch.Generator(device=DEV).manual_seed(11)
    z = torch.randn((40, 70001), generator=g, device=DEV)
    u, p = torch.rand(40, generator=g, device=DEV), torch.full((40,), 0.8, device=DEV)
    T = 1500
    q = torch.randn((T, 4, 128), generator=g, device=DEV).bfloat16()
    k, v = (torch.randn((T, 2, 128), generator=g, device=DEV).bfloat16() for _ in range(2))
    decay, slots = torch.tensor([-0.1, -0.01], device=DEV), i32([0])
    zero = lambda: torch.zeros((1, 2, 128, 128), device=DEV)
    start, new, lens1 = i32([3] * 100), i32([40] * 100), i32([9])

    def calls(stream, states, table, free, count):
        kw = {} if stream is None else dict(stream=stream if handle == "stream" else stream.cuda_stream)
        a = ra.token_sample(z, u, top_p=p, want_logprob=True, **kw)
        b = ra.linear_append(q, k, v, i32c, i32z, states, slots, decay, max_q_len=T, **kw)
        c = ra.linear_decode(q[:1], k[:1], v[:1], states, slots, lens1, decay, **kw)
        d = ra.block_table_extend(table, start, new, free, count, total_new=4000, **kw)
        return [*a, b, c, *d]
    i32c, i32z = i32([0, T]), i32([0])
    inputs = lambda: (zero(), torch.zeros((100, 4), dtype=torch.int32, device=DEV),
                      torch.arange(400, device=DEV).to(torch.int32), i32([400]))
    ref_in = inputs()
    ref = calls(None, *ref_in)
    ins = [inputs(), inputs()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [calls(s, *x) for s, x in zip(streams, ins)]
    for r in range(4):
        held = [torch.full((n,), 0xFF - r, dtype=torch.uint8, device=DEV) for n in (1 << 22, 1 << 16, 4096)]
        del held
    torch.cuda.synchronize()
    for outs, x in zip(got, ins):
        for a, b in zip(outs, ref):
            assert torch.equal(a, b)
        for a, b in zip(x, ref_in):
            assert torch.equal(a, b)
