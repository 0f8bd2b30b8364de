"""Penalties, biases and masks on logits against plain loops in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2603_18815_amd as ra
from tests.draft_util import DEV, ancestors, cu, i32, pack, random_tree

pytestmark = pytest.mark.gpu
PARAMS = ("repetition", "frequency", "presence")


def f32(x):
    return torch.as_tensor(np.asarray(x, np.float32), device=DEV)


def reference(z, rows, hist, lens, prompt, par, bias, allowed, which, paths):
    """fp64 [N][V] and where an element is not concerned. rows[n]: its history row; paths[n]:
    drafted tokens of its nodes."""
    N, V = z.shape
    out, plain = z.astype(np.float64), np.ones((N, V), bool)
    for n in range(N):
        b = rows[n]
        if b < 0:
            continue
        tokens = [] if hist is None else list(hist[b][:max(lens[b], 0)])
        split = 0 if prompt is None else max(prompt[b], 0)
        ok = lambda ids: [int(t) for t in ids if 0 <= t < V]
        answer = ok(tokens[split:] + paths[n])
        known = set(ok(tokens[:split])) | set(answer)
        get = lambda name, off, good: (float(par[name][b]) if par.get(name) is not None and
                                       np.isfinite(par[name][b]) and good(par[name][b]) else off)
        r = get("repetition", 1.0, lambda x: x > 0)
        f, p = get("frequency", 0.0, lambda x: True), get("presence", 0.0, lambda x: True)
        for v in known:
            out[n, v] = out[n, v] / r if out[n, v] > 0 else out[n, v] * r
            plain[n, v] = False
        for v in set(answer):
            out[n, v] -= f * answer.count(v) + p
        for v, x in (bias[b] if bias else {}).items():
            if 0 <= v < V:
                out[n, v] += x
                plain[n, v] = False
        if allowed is not None:
            m = n if which is None else which[n]
            if 0 <= m < len(allowed):
                out[n, ~allowed[m][:V]] = -np.inf
                plain[n, ~allowed[m][:V]] = False
    return out, plain


def check(got, z, want, plain):
    """Untouched elements keep their bits; the others are off by three roundings in fp32 (each
    half a step of what it rounds, at most |z| repetition + |f c| + |p| + |b|) and one to the
    type."""
    bits = lambda x: x.contiguous().view(torch.int16 if x.dtype == torch.bfloat16 else torch.int32)
    keep = torch.as_tensor(plain, device=DEV)
    assert torch.equal(bits(got)[keep], bits(z)[keep])
    g, w = got.double().cpu().numpy()[~plain], want[~plain]
    assert np.array_equal(np.isinf(g), np.isinf(w)) and np.array_equal(np.isnan(g), np.isnan(w))
    f = np.isfinite(w)
    step = torch.finfo(got.dtype).eps / 2
    size = np.abs(w[f]) + 400.0                         # sizes met on the way in these tests
    assert (np.abs(g[f] - w[f]) <= step * 1.01 * np.abs(w[f]) + 5 * 2.0**-24 * size).all()


def case(seed, B, V, lens, use, dtype=torch.float32, nodes=None, pad=0, odd=False):
    """Arguments of the call and the host's view of them."""
    rng = np.random.default_rng(seed)
    N, rows, paths, kw = B, list(range(B)), [[] for _ in range(B)], {}
    if nodes is not None:
        N, rows = sum(nodes), list(np.repeat(np.arange(B), nodes))
        trees = [ancestors(random_tree(rng, t)) for t in nodes]
        draft = rng.integers(0, V, N)
        paths = [[int(draft[cu(nodes)[b] + j]) for j in np.flatnonzero(trees[b][i])]
                 for b in range(B) for i in range(nodes[b])]
        words = max(1, -(-max(nodes) // 64))
        kw.update(cu_rows=i32(cu(nodes)), draft_tokens=i32(draft),
                  tree_mask=torch.as_tensor(pack(trees, words), device=DEV))
    store = torch.as_tensor(rng.normal(0, 4, (N, V + pad)).astype(np.float32), device=DEV).to(dtype)
    z = store[:, :V]
    hist = prompt = None
    if "history" in use:
        longest = max(max(lens), 1) + 5
        # few tokens, so that they repeat, among them ids of no token
        hist = rng.integers(-2 if odd else 0, (V + 3) if odd else V, (B, longest))
        hist = np.where(rng.random(hist.shape) < 0.5, hist % min(V, 7), hist)
        kw.update(history=i32(hist), history_lens=i32(lens))
        if "prompt" in use:
            prompt = rng.integers(0, longest, B)
            kw["prompt_lens"] = i32(prompt)
    par = {}
    for name, lo, hi in (("repetition", 0.7, 1.6), ("frequency", -0.2, 0.5), ("presence", -0.3, 0.8)):
        if name in use:
            par[name] = rng.uniform(lo, hi, B).astype(np.float32)
            kw[name] = f32(par[name])
    bias = None
    if "bias" in use:
        n = rng.integers(0, 20, B)
        ids = rng.integers(-1 if odd else 0, min(V, 40) + (1 if odd else 0), int(n.sum()) + 2)
        val = rng.normal(0, 3, ids.size).astype(np.float32)
        at = cu(n)
        bias = [{int(ids[e]): float(val[e]) for e in range(at[b], at[b + 1])} for b in range(B)]
        kw.update(bias_tokens=i32(ids), bias_values=f32(val), cu_bias=i32(at))
    allowed = which = None
    if "allowed" in use:
        M = N if use == "allowed" else 3
        allowed = rng.random((M, -(-V // 32) * 32)) < 0.5
        kw["allowed"] = i32(np.packbits(allowed, axis=1, bitorder="little").view(np.int32))
        if M != N:
            which = rng.integers(-1, M + 1, N)
            kw["allowed_rows"] = i32(which)
    host = dict(rows=rows, hist=hist, lens=lens, prompt=prompt, par=par, bias=bias, allowed=allowed,
                which=which, paths=paths)
    return z, kw, host


ALL = "history prompt repetition frequency presence bias allowed "
USES = ["history repetition", "history prompt frequency presence", "bias", "allowed", ALL]


@pytest.mark.parametrize("use", USES)
@pytest.mark.parametrize("V,pad", [(1, 0), (37, 0), (8191, 3), (8193, 0), (30011, 5)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows(device, V, pad, use, dtype):
    lens = [0, 1, 700, 33, 64]
    z, kw, host = case(V, 5, V, lens, use, dtype, pad=pad, odd=True)
    want, plain = reference(z.double().cpu().numpy(), **host)
    out = ra.token_logits_adjust(z, **kw)
    assert out.is_contiguous()
    check(out, z, want, plain)
    store = torch.full((5, V + 9), 5.0, dtype=dtype, device=DEV)     # another alignment
    ra.token_logits_adjust(z, **kw, out=store[:, 2:V + 2])
    assert torch.equal(store[:, 2:V + 2].contiguous(), out)
    assert bool((store[:, :2] == 5.0).all()) and bool((store[:, V + 2:] == 5.0).all())
    before = z.clone()
    assert ra.token_logits_adjust(z, **kw, out=z) is z
    assert torch.equal(z.contiguous(), out) and not torch.equal(before, z) or V == 1


@pytest.mark.parametrize("nodes", [[1, 1], [3, 0, 64, 1], [100, 7]])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_trees(device, nodes, dtype):
    V = 9001
    B = len(nodes)
    z, kw, host = case(3, B, V, [50, 3, 900, 0][:B], ALL, dtype, nodes=nodes)
    want, plain = reference(z.double().cpu().numpy(), **host)
    out = ra.token_logits_adjust(z, **kw)
    check(out, z, want, plain)
    ra.token_logits_adjust(z, **kw, out=z)
    assert torch.equal(z, out)


def test_rows_behind_the_last_tree_stay(device):
    z, kw, host = case(4, 3, 500, [9, 9, 9], ALL, nodes=[2, 0, 3])
    N = z.shape[0]
    more = lambda t: torch.cat([t, t[:2]])
    z2 = more(z)
    kw.update(draft_tokens=more(kw["draft_tokens"]), tree_mask=more(kw["tree_mask"]),
              allowed_rows=more(kw["allowed_rows"]))
    out = torch.full_like(z2, 3.25)
    ra.token_logits_adjust(z2, **kw, out=out)
    assert torch.equal(out[:N], ra.token_logits_adjust(z, **{**kw, "draft_tokens": kw["draft_tokens"][:N],
                                                             "tree_mask": kw["tree_mask"][:N],
                                                             "allowed_rows": kw["allowed_rows"][:N]}))
    assert bool((out[N:] == 3.25).all())


def test_many_rows_of_few_trees(device):
    """More nodes than a workgroup's rows, over several histories."""
    nodes = [200, 1, 0, 333, 64]
    z, kw, host = case(5, 5, 70001, [10, 2000, 5, 300, 0], "history repetition frequency", nodes=nodes)
    want, plain = reference(z.double().cpu().numpy(), **host)
    check(ra.token_logits_adjust(z, **kw), z, want, plain)


def test_a_large_call_equals_its_trees_one_by_one(device):
    """Rows enough for the most that a workgroup takes, of trees that begin anywhere in them."""
    rng = np.random.default_rng(6)
    V, nodes = 100003, rng.integers(0, 65, 60)
    B, at = len(nodes), cu(nodes)
    N = at[-1]
    z = torch.randn((N, V), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV).bfloat16()
    history, tokens = i32(rng.integers(0, 3000, (B, 500))), i32(rng.integers(0, 3000, N))
    mask = torch.as_tensor(pack([ancestors(random_tree(rng, t)) for t in nodes], 1), device=DEV)
    lens = rng.integers(0, 501, B)
    par = {k: f32(rng.uniform(0.8, 1.5, B)) for k in PARAMS}
    out = ra.token_logits_adjust(z, history=history, history_lens=i32(lens), cu_rows=i32(at),
                                 draft_tokens=tokens, tree_mask=mask, **par)
    for b in range(B):
        rows = slice(at[b], at[b + 1])
        if nodes[b] == 0:
            continue
        one = ra.token_logits_adjust(z[rows], history=history[b:b + 1], history_lens=i32(lens[b:b + 1]),
                                     cu_rows=i32([0, nodes[b]]), draft_tokens=tokens[rows],
                                     tree_mask=mask[rows], **{k: v[b:b + 1] for k, v in par.items()})
        assert torch.equal(out[rows], one), b


def test_special_values(device):
    inf, nan = float("inf"), float("nan")
    z = f32([[inf, -inf, nan, 0.0, -0.0, 2.0, -2.0, 1e38]] * 4)
    out = ra.token_logits_adjust(z, history=i32([list(range(8))] * 4), history_lens=i32([8] * 4),
                                 repetition=f32([2.0, inf, -1.0, nan]),
                                 frequency=f32([0.5, nan, inf, 0.0]), presence=f32([0.0, 0.0, nan, 0.0]))
    assert torch.equal(torch.nan_to_num(out[0], 9.0), torch.nan_to_num(
        f32([inf, -inf, nan, -0.5, -0.5, 0.5, -4.5, 5e37]), 9.0))
    for n in (1, 2, 3):                              # parameters that are off
        assert torch.equal(torch.nan_to_num(out[n], 9.0), torch.nan_to_num(z[n], 9.0))
    # a mask that leaves nothing, and what follows it
    none = torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    masked = ra.token_logits_adjust(z[:1], allowed=none)
    assert bool((masked == -inf).all())
    tok, _ = ra.token_sample(masked, f32([0.5]))
    assert tok.tolist() == [-1]


def test_nan_payload_of_untouched_logits_stays(device):
    z = torch.tensor([[0x7fc12345, 0x3f800000]], dtype=torch.int32, device=DEV).view(torch.float32)
    out = ra.token_logits_adjust(z, history=i32([[1]]), history_lens=i32([1]), repetition=f32([2.0]))
    assert out.view(torch.int32).tolist() == [[0x7fc12345, 0x3f000000]]


def test_no_adjustment_is_a_copy(device):
    z = torch.randn((3, 1000), device=DEV)
    assert torch.equal(ra.token_logits_adjust(z), z)
    assert torch.equal(ra.token_logits_adjust(z, repetition=f32([2.0] * 3)), z)   # no history
    before = z.clone()
    ra.token_logits_adjust(z, out=z)
    assert torch.equal(z, before)


def test_strided_history_and_masks(device):
    z, kw, host = case(6, 4, 3001, [40, 50, 60, 0], ALL)
    want = ra.token_logits_adjust(z, **kw)
    wide = torch.full((4, kw["history"].shape[1] + 11), 1, dtype=torch.int32, device=DEV)
    wide[:, 3:3 + kw["history"].shape[1]] = kw["history"]
    bits = torch.zeros((3, kw["allowed"].shape[1] + 3), dtype=torch.int32, device=DEV)
    bits[:, 1:1 + kw["allowed"].shape[1]] = kw["allowed"]
    kw.update(history=wide[:, 3:3 + kw["history"].shape[1]], allowed=bits[:, 1:1 + kw["allowed"].shape[1]])
    assert torch.equal(ra.token_logits_adjust(z, **kw), want)


def test_lengths_past_the_history_and_below_zero(device):
    z = torch.randn((2, 50), device=DEV)
    h = i32([[1, 2, 3], [4, 5, 6]])
    kw = dict(history=h, frequency=f32([1.0, 1.0]))
    a = ra.token_logits_adjust(z, history_lens=i32([1000, -3]), **kw)
    b = ra.token_logits_adjust(z, history_lens=i32([3, 0]), **kw)
    assert torch.equal(a, b) and torch.equal(a[1], z[1])
    # of rows cut out of wider ones too
    wide = i32([[9, 9, 1, 2, 3], [9, 9, 4, 5, 6]])[:, 2:]
    c = ra.token_logits_adjust(z, history_lens=i32([1000, -3]), history=wide, frequency=kw["frequency"])
    assert torch.equal(a, c)


def test_bias_offsets_past_the_lists(device):
    z = torch.randn((2, 50), device=DEV)
    kw = dict(bias_tokens=i32([3, 4, 5]), bias_values=f32([1.0, 2.0, 3.0]))
    a = ra.token_logits_adjust(z, cu_bias=i32([0, 2, 1 << 30]), **kw)
    b = ra.token_logits_adjust(z, cu_bias=i32([0, 2, 3]), **kw)
    assert torch.equal(a, b)


def test_masks_of_few_rows_and_ids_outside(device):
    """Without allowed_rows row n has mask n; rows past the masks have none."""
    z = torch.randn((3, 40), device=DEV)
    one = torch.zeros((1, 2), dtype=torch.int32, device=DEV)
    out = ra.token_logits_adjust(z, allowed=one)
    assert bool((out[0] == float("-inf")).all()) and torch.equal(out[1:], z[1:])
    out = ra.token_logits_adjust(z, allowed=one, allowed_rows=i32([-1, 1, 0]))
    assert torch.equal(out[:2], z[:2]) and bool((out[2] == float("-inf")).all())


# Calls whose workgroups take several rows and count a tree's history once: rows of logits a
# multiple of 16 bytes apart, and N rows in ceil(V / 8184) chunks over 512 workgroups.
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,pad,nodes,lens", [
    (16384, 0, [200, 1, 0, 333, 64], [10, 120, 5, 90, 0]),      # 4 rows a workgroup
    (16384, 16, [7] * 90, list(range(90))),                     # 4, of several trees
    (12000, 8, [3, 1000, 0, 70], [40, 60, 9, 0]),               # 5; paths through nodes past 512
    (1200, 0, [1024, 1024], [30, 0]),                           # 4
])
def test_rows_that_share_a_history(device, V, pad, nodes, lens, dtype):
    for use in (ALL, "history frequency"):
        z, kw, host = case(7, len(nodes), V, lens, use, dtype, nodes=nodes, pad=pad, odd=True)
        want, plain = reference(z.double().cpu().numpy(), **host)
        out = ra.token_logits_adjust(z, **kw)
        check(out, z, want, plain)
        ra.token_logits_adjust(z, **kw, out=z)
        assert torch.equal(z.contiguous(), out)


def test_rows_that_share_a_history_take_off_each_others_paths(device):
    """Leaves of one root in falling and rising order of their tokens: a path that stayed would be
    counted in the rows behind it."""
    V, T = 8192, 1024
    N = 2 * T
    sees = np.eye(T, dtype=bool)
    sees[:, 0] = True
    draft = np.concatenate([np.arange(T), np.arange(T)[::-1]]) * 8 % V
    z = torch.zeros((N, V), device=DEV)
    out = ra.token_logits_adjust(
        z, history=i32([[5, 13], [8000, 5]]), history_lens=i32([2, 2]), frequency=f32([1.0, 1.0]),
        cu_rows=i32([0, T, N]), draft_tokens=i32(draft),
        tree_mask=torch.as_tensor(pack([sees, sees], T // 64), device=DEV))
    want = torch.zeros((N, V), device=DEV)
    for b, seen in enumerate(([5, 13], [8000, 5])):
        rows = slice(b * T, (b + 1) * T)
        for v in seen:
            want[rows, v] -= 1
        want[rows, int(draft[b * T])] -= 1                # the root
        at = torch.arange(b * T + 1, (b + 1) * T, device=DEV)
        want[at, torch.as_tensor(draft[b * T + 1:(b + 1) * T], device=DEV)] -= 1
    assert torch.equal(out, want)


@pytest.mark.parametrize("use", USES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_logit_in_place(device, use, dtype):
    z, kw, _ = case(8, 5, 1, [0, 1, 700, 33, 64], use, dtype, odd=True)
    out = ra.token_logits_adjust(z, **kw)
    assert ra.token_logits_adjust(z, **kw, out=z) is z
    assert torch.equal(z, out)


def test_a_nodes_history_is_the_rows_then_its_path_with_the_root(device):
    """The history ends before the root, whose token is the first of every path: a row of a tree is
    the row whose history goes on with the path's tokens. A history that holds the root already
    counts it twice."""
    V, nodes, lens = 600, [9, 0, 4], [40, 3, 0]
    z, kw, host = case(9, 3, V, lens, ALL, nodes=nodes)
    out = ra.token_logits_adjust(z, **kw)
    longest = max(lens) + max(nodes) + 1
    for root_twice in (False, True):
        if root_twice:                                    # as if the root had been appended
            wide = torch.zeros((3, longest), dtype=torch.int32, device=DEV)
            wide[:, :kw["history"].shape[1]] = kw["history"]
            for b, n in enumerate(nodes):
                if n:
                    wide[b, lens[b]] = kw["draft_tokens"][cu(nodes)[b]]
            out = ra.token_logits_adjust(z, **{**kw, "history": wide, "history_lens": i32(np.add(lens, 1))})
        for n, b in enumerate(host["rows"]):
            path = host["paths"][n]
            tokens = [int(t) for t in host["hist"][b][:lens[b]]] + path[:1] * root_twice + path
            one = dict(history=i32([tokens]), history_lens=i32([len(tokens)]),
                       prompt_lens=i32([min(int(host["prompt"][b]), lens[b] + root_twice)]),
                       bias_tokens=kw["bias_tokens"], bias_values=kw["bias_values"],
                       cu_bias=kw["cu_bias"][b:b + 2].contiguous(), allowed=kw["allowed"],
                       allowed_rows=kw["allowed_rows"][n:n + 1], **{k: kw[k][b:b + 1] for k in PARAMS})
            assert torch.equal(ra.token_logits_adjust(z[n:n + 1], **one), out[n:n + 1]), (n, root_twice)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_of_one_history_and_trees_without_one(device, dtype):
    """cu_rows alone: several rows of logits for a history, no path; and paths alone."""
    V, nodes, lens = 16384, [250, 0, 90, 260], [80, 4, 0, 31]        # 4 rows a workgroup
    z, kw, host = case(10, 4, V, lens, ALL, dtype, nodes=nodes)
    rows = {k: v for k, v in kw.items() if k not in ("draft_tokens", "tree_mask")}
    paths = {k: v for k, v in kw.items() if k not in ("history", "history_lens", "prompt_lens")}
    for args, view in ((rows, dict(host, paths=[[] for _ in host["paths"]])),
                       (paths, dict(host, hist=None, prompt=None))):
        want, plain = reference(z.double().cpu().numpy(), **view)
        out = ra.token_logits_adjust(z, **args)
        check(out, z, want, plain)
        again = z.clone()
        assert torch.equal(ra.token_logits_adjust(again, **args, out=again), out)
