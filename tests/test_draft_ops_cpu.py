"""Refusals of the operators on drafted trees, logits and shared pages that need no GPU: through
the C ABI with addresses that are never dereferenced, and through the binding."""
import ctypes
import math
import random

import pytest
import torch

import paper_2603_18815_amd as ra
from paper_2603_18815_amd import _lib

BIG = 1 << 40


def at(i):
    """Addresses far apart."""
    return ctypes.c_void_p(0x1000 + i * BIG)


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def call(fn, names, defaults, **kw):
    assert set(kw) <= set(defaults), kw
    d = dict(defaults, **kw)
    return fn(*[d[n] for n in names.split()])


def pools(**kw):
    d = dict(k=0x100000, v=0x200000, bt=0x300000, num=10, stride=8, hkv=2, page=16, dim=128, dt=0,
             ks=1.0, vs=1.0)
    d.update(kw)
    return _lib.RaPagedKV(*d.values())


NULL, SHAPE, UNSUPPORTED = _lib.RA_ERR_NULL, _lib.RA_ERR_SHAPE, _lib.RA_ERR_UNSUPPORTED
WORKSPACE, OK = _lib.RA_ERR_WORKSPACE, _lib.RA_OK


def test_draft_tree_mask_validation(lib):
    names = "parents cu ctx B total mq words mask pos stream"
    base = dict(parents=at(1), cu=at(2), ctx=at(3), B=2, total=20, mq=10, words=1, mask=at(4),
                pos=at(5), stream=None)
    go = lambda **kw: call(lib.draft_tree_mask, names, base, **kw)
    for n in ("parents", "cu", "mask"):
        assert go(**{n: None}) == NULL
    for n in ("B", "total", "mq"):
        assert go(**{n: -1}) == SHAPE
        assert go(**{n: 0}) == OK
    assert go(words=0) == SHAPE and go(mq=65) == SHAPE and go(words=-1) == SHAPE
    assert go(mq=1025, words=17) == UNSUPPORTED and go(B=65536) == UNSUPPORTED
    for a, b in (("mask", "parents"), ("pos", "parents"), ("pos", "mask"), ("mask", "cu"), ("pos", "ctx")):
        assert go(**{a: base[b]}) == UNSUPPORTED


def test_draft_tree_accept_validation(lib):
    names = "parents draft chosen cu ctx B total mq path tokens acc lens nxt stream"
    arrays = names.split()[:5] + names.split()[8:13]
    base = dict({n: at(i + 1) for i, n in enumerate(arrays)}, B=2, total=20, mq=10, stream=None)
    go = lambda **kw: call(lib.draft_tree_accept, names, base, **kw)
    for n in arrays:
        assert go(**{n: None}) == NULL
    for n in ("cu", "ctx", "acc", "lens", "nxt"):      # rows without nodes have results too
        assert go(total=0, **{n: None}) == NULL and go(mq=0, **{n: None}) == NULL
    assert go(B=0) == OK
    for n in ("B", "total", "mq"):
        assert go(**{n: -1}) == SHAPE
    assert go(mq=1025) == UNSUPPORTED and go(B=65536) == UNSUPPORTED
    for out in ("path", "tokens", "acc", "lens", "nxt"):
        for other in arrays:
            if other != out:
                assert go(**{out: base[other]}) == UNSUPPORTED, (out, other)


def test_decode_tree_validation(lib):
    names = "q cu ctx mask words kv B Hq total mq mk scale out lse ws bytes stream"
    kv = pools()
    base = dict(q=at(1), cu=at(2), ctx=at(3), mask=at(4), words=1, kv=ctypes.byref(kv), B=2, Hq=8,
                total=20, mq=10, mk=128, scale=0.1, out=at(5), lse=None, ws=at(6), bytes=BIG,
                stream=None)
    go = lambda **kw: call(lib.rollout_attn_decode_tree, names, base, **kw)
    for n in ("q", "cu", "ctx", "mask", "out", "kv"):
        assert go(**{n: None}) == NULL
    for n in ("B", "total", "mq"):
        assert go(**{n: -1}) == SHAPE
        assert go(**{n: 0}) == OK
    assert go(Hq=0) == SHAPE and go(Hq=7) == SHAPE and go(mk=-1) == SHAPE and go(mk=129) == SHAPE
    assert go(words=0) == SHAPE and go(mq=65) == SHAPE
    for s in (float("nan"), float("inf")):
        assert go(scale=s) == SHAPE
    assert go(Hq=514) == UNSUPPORTED and go(B=65536) == UNSUPPORTED
    assert go(mq=1025, words=17) == UNSUPPORTED
    for n in ("q", "out"):
        assert go(**{n: ctypes.c_void_p(0x1008)}) == UNSUPPORTED
    bad = pools(k=0x100008)
    assert go(kv=ctypes.byref(bad)) == UNSUPPORTED
    for kw, want in ((dict(page=32), UNSUPPORTED), (dict(dt=7), UNSUPPORTED), (dict(bt=0), NULL),
                     (dict(dt=1, ks=0.0), SHAPE)):
        bad = pools(**kw)
        assert go(kv=ctypes.byref(bad)) == want
    far = pools(stride=1 << 27)
    assert go(kv=ctypes.byref(far), mk=(1 << 30) + 1) == UNSUPPORTED
    long = pools(stride=4096)
    need = lib.rollout_attn_decode_tree_workspace_size(2, 8, 2, 20, 10, 40000)
    assert need > 0
    big = dict(kv=ctypes.byref(long), mk=40000)
    assert go(**big, bytes=need - 1) == WORKSPACE and go(**big, ws=None) == WORKSPACE
    assert go(**big, ws=ctypes.c_void_p(0x1004)) == UNSUPPORTED
    size = lib.rollout_attn_decode_tree_workspace_size
    for zero in ((0, 8, 2, 20, 10, 128), (2, 7, 2, 20, 10, 128), (2, 8, 2, 0, 10, 128),
                 (2, 8, 2, 20, 1025, 128), (2, 8, 2, 20, 10, 0)):
        assert size(*zero) == 0


def adjust(**kw):
    a = _lib.RaLogitsAdjust()
    for k, v in kw.items():
        setattr(a, k, v.value if isinstance(v, ctypes.c_void_p) else v)
    return a


def test_token_logits_adjust_validation(lib):
    names = "z dt N V stride a B out ostride stream"
    base = dict(z=at(1), dt=0, N=4, V=100, stride=100, B=4, out=at(2), ostride=100, stream=None)

    def go(args=None, **kw):
        a = adjust(**(args or {}))
        return call(lib.token_logits_adjust, names, dict(base, a=ctypes.byref(a)), **kw)
    assert go(z=None) == NULL and go(out=None) == NULL and go(a=None) == NULL
    assert go(N=-1) == SHAPE and go(B=-1) == SHAPE and go(V=0) == SHAPE
    assert go(stride=99) == SHAPE and go(ostride=99) == SHAPE
    assert go(B=3) == SHAPE and go(dt=2) == UNSUPPORTED
    assert go(V=(1 << 24) + 1, stride=1 << 25, ostride=1 << 25) == UNSUPPORTED
    assert go(N=1 << 21, B=1 << 21, V=1 << 24, stride=1 << 24, ostride=1 << 24) == UNSUPPORTED
    assert go(N=0, B=0, z=None, out=None) == OK
    assert go(dict(cu_rows=at(3)), B=0) == OK
    assert go(dict(history=at(3))) == NULL
    assert go(dict(history=at(3), history_lens=at(4), history_width=-1)) == SHAPE
    assert go(dict(history=at(3), history_lens=at(4), history_width=9, history_stride=8)) == SHAPE
    assert go(dict(bias_tokens=at(3), bias_values=at(4), cu_bias=at(5), num_bias=-1)) == SHAPE
    assert go(dict(bias_tokens=at(3), bias_values=at(4))) == NULL
    assert go(dict(bias_tokens=at(3), cu_bias=at(4))) == NULL
    assert go(dict(allowed=at(3), allowed_stride=3, num_allowed=4)) == SHAPE
    assert go(dict(allowed=at(3), allowed_stride=4, num_allowed=-1)) == SHAPE
    tree = dict(cu_rows=at(3), draft_tokens=at(4), tree_mask=at(5), mask_words=1)
    assert go(dict(tree, mask_words=0)) == SHAPE
    for n in ("draft_tokens", "tree_mask", "cu_rows"):
        assert go({k: v for k, v in tree.items() if k != n}) == NULL
    # what is written must not be read elsewhere: in place, or apart
    assert go(out=ctypes.c_void_p(0x1000 + BIG + 4)) == UNSUPPORTED
    assert go(out=at(1), ostride=200) == UNSUPPORTED
    full = dict(tree, history=at(6), history_lens=at(7), history_stride=9, history_width=9, num_bias=5, prompt_lens=at(8),
                repetition=at(9), frequency=at(10), presence=at(11), bias_tokens=at(12),
                bias_values=at(13), cu_bias=at(14), allowed=at(15), allowed_stride=4, num_allowed=2,
                allowed_rows=at(16))
    for n in set(full) - {"mask_words", "history_stride", "history_width", "num_bias",
                          "allowed_stride", "num_allowed"}:
        assert go(dict(full, **{n: at(2)})) == UNSUPPORTED, n


def test_fork_and_release_validation(lib):
    names = "src dst lens n table B stride shares num free count cap cs cd taken stream"
    arrays = "src dst lens table shares free count cs cd taken".split()
    base = dict({n: at(i + 1) for i, n in enumerate(arrays)}, n=3, B=4, stride=8, num=50, cap=50,
                stream=None)
    go = lambda **kw: call(lib.kv_block_table_fork, names, base, **kw)
    for n in arrays:
        assert go(**{n: None}) == NULL
    for n in ("n", "B", "cap", "num"):
        assert go(**{n: -1}) == SHAPE
    assert go(num=0) == SHAPE and go(stride=0) == SHAPE
    assert go(n=65536) == UNSUPPORTED and go(B=65536) == UNSUPPORTED and go(stride=1 << 27) == UNSUPPORTED
    for out in ("table", "shares", "count", "cs", "cd", "taken"):
        for other in arrays:
            if other != out:
                assert go(**{out: base[other]}) == UNSUPPORTED, (out, other)

    names = "lens keep table B stride shares num free count cap released ws bytes stream"
    arrays = "lens keep table shares free count released ws".split()
    base = dict({n: at(i + 1) for i, n in enumerate(arrays)}, B=4, stride=8, num=50, cap=50,
                bytes=1 << 20, stream=None)
    go = lambda **kw: call(lib.kv_block_table_release_shared, names, base, **kw)
    for n in arrays[:-1]:
        assert go(**{n: None}) == NULL
    need = lib.kv_block_table_release_shared_workspace_size(4)
    assert go(ws=None) == WORKSPACE and go(bytes=need - 1) == WORKSPACE
    assert go(ws=ctypes.c_void_p(0x1008)) == WORKSPACE
    assert go(B=-1) == SHAPE and go(num=0) == SHAPE and go(cap=49) == SHAPE and go(stride=0) == SHAPE
    assert go(B=65536) == UNSUPPORTED and go(B=1 << 10, stride=1 << 20) == UNSUPPORTED
    for out in ("shares", "free", "count", "released", "ws"):
        for other in arrays:
            if other != out:
                assert go(**{out: base[other]}) == UNSUPPORTED, (out, other)
    assert lib.kv_block_table_release_shared_workspace_size(-1) == 0


def test_page_copy_and_compact_validation(lib):
    kv, bare = pools(), pools(bt=0)
    copy = lambda k, s, d, n: lib.kv_page_copy(k, s, d, n, None)
    assert copy(None, at(1), at(2), 1) == NULL
    assert copy(ctypes.byref(kv), None, at(2), 1) == NULL
    assert copy(ctypes.byref(kv), at(1), None, 1) == NULL
    assert copy(ctypes.byref(kv), at(1), at(2), -1) == SHAPE
    assert copy(ctypes.byref(kv), None, None, 0) == OK
    assert copy(ctypes.byref(bare), None, None, 0) == OK           # the table is not used
    assert copy(ctypes.byref(kv), at(1), at(2), 1 << 30) == UNSUPPORTED
    for kw, want in ((dict(k=0), NULL), (dict(k=0x100004), UNSUPPORTED), (dict(dim=64), UNSUPPORTED)):
        bad = pools(**kw)
        assert copy(ctypes.byref(bad), at(1), at(2), 1) == want
    names = "kv start cu src counts B total most stream"
    base = dict(kv=ctypes.byref(kv), start=at(1), cu=at(2), src=at(3), counts=None, B=2, total=5,
                most=4, stream=None)
    go = lambda **kw: call(lib.kv_page_compact, names, base, **kw)
    for n in ("kv", "start", "cu", "src"):
        assert go(**{n: None}) == NULL
    for n in ("B", "total", "most"):
        assert go(**{n: -1}) == SHAPE
        assert go(**{n: 0}) == OK
    assert go(B=65536) == UNSUPPORTED
    assert go(kv=ctypes.byref(bare)) == NULL


def test_the_binding_refuses_host_tensors_and_missing_partners():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)
    z = torch.zeros((2, 10))
    for f in (lambda: ra.draft_tree_mask(i(3), i(2)),
              lambda: ra.draft_tree_accept(i(3), i(3), i(3), i(2), i(1)),
              lambda: ra.token_logits_adjust(z),
              lambda: ra.block_table_fork(i(2, 4), i(1), i(1), i(1), i(9), i(9), i(1)),
              lambda: ra.block_table_release_shared(i(2, 4), i(2), i(2), i(9), i(9), i(1))):
        with pytest.raises(ValueError, match="GPU tensor"):
            f()


def test_page_copy_takes_pools_without_a_table(lib):
    """Nothing that describes the block table is looked at."""
    for kw in (dict(bt=0, stride=0), dict(stride=0), dict(bt=0, stride=-1), dict(bt=0)):
        bare = pools(**kw)
        assert lib.kv_page_copy(ctypes.byref(bare), None, None, 0, None) == OK, kw
        assert lib.kv_page_copy(ctypes.byref(bare), None, at(2), 1, None) == NULL, kw
    for kw, want in ((dict(k=0), NULL), (dict(v=0), NULL), (dict(num=0), SHAPE), (dict(hkv=0), SHAPE)):
        bad = pools(bt=0, stride=0, **kw)
        assert lib.kv_page_copy(ctypes.byref(bad), at(1), at(2), 1, None) == want, kw


def test_launches_of_more_threads_than_a_grid_can_have_are_refused(lib):
    """A launch has fewer than 2^32 threads: calls just past that, of sizes whose arrays fit the
    GPU's memory."""
    z = ctypes.byref(adjust())
    trees = ctypes.byref(adjust(cu_rows=at(3)))
    for N, V, a in ((1 << 23, 2, z), (1 << 22, 9000, z), (1 << 28, 2, trees)):
        for dt in (0, 1):
            assert lib.token_logits_adjust(at(1), dt, N, V, V, a, N, at(2), V, None) == UNSUPPORTED
    two, many, wide, cut = pools(), pools(hkv=257), pools(hkv=129, stride=16), pools(hkv=256, stride=512)
    ref = ctypes.byref
    assert lib.kv_page_copy(ref(two), at(1), at(2), 1 << 23, None) == UNSUPPORTED
    assert lib.kv_page_compact(ref(many), at(1), at(2), at(3), None, 65535, 5, 4, None) == UNSUPPORTED
    for kv, heads, total, nodes, keys in ((many, 257, 65535, 1, 16), (wide, 129, 65535, 129, 200),
                                          (cut, 256, 1 << 18, 4, 8192)):
        assert lib.rollout_attn_decode_tree(
            at(1), at(2), at(3), at(4), 3, ref(kv), 65535, heads, total, nodes, keys, 0.1, at(5), None,
            at(6), BIG, None) == UNSUPPORTED, heads


@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (8, 1), (12, 4), (5, 5), (200, 1)])
def test_one_workspace_holds_every_call_of_a_loop(Hq, Hkv):
    """The size of a call can fall as rows, nodes or keys grow; the largest size is that of the
    largest call that a loop can make, and not more than a call of it can need."""
    rng = random.Random(Hq)
    size, most = ra.decode_tree_workspace_size, ra.decode_tree_max_workspace_size
    spread = lambda n: min(n, int(2 ** rng.uniform(0, math.log2(n + 1))))
    falls = False
    for _ in range(60):
        B, T, L = spread(300), spread(1024), spread(40000)
        bound, largest = most(B, Hq, Hkv, T, L), 0
        # trees just within each size of tile, rows just within and past what is not cut
        nodes = {t for r in (1, 16, 32, 128, 256, T * Hq) for t in (r * Hkv // Hq,) if 1 <= t <= T} | {1, T}
        keys = {n for n in (512, 513, 4096, 4097, L, *(spread(L) for _ in range(20))) if n <= L}
        for b in {1, B, *(spread(B) for _ in range(10))}:
            for t in nodes | {spread(T) for _ in range(4)}:
                for n in keys:
                    need = size(b, Hq, Hkv, b * t, t, n)
                    assert need <= bound, (B, T, L, b, t, n)
                    largest = max(largest, need)
        falls |= size(B, Hq, Hkv, B * T, T, L) < largest
        if L > 4096:
            assert bound <= largest + 8 * 300 + 256, (B, T, L, bound, largest)
    assert falls
    for zero in ((0, Hq, Hkv, 8, 5000), (4, Hq, Hkv, 0, 5000), (4, Hq, Hkv, 1025, 5000),
                 (4, Hq, Hkv, 8, 0), (4, Hq, Hkv, 8, 512), (4, Hq + 1, Hkv + 1, 8, 512)):
        assert most(*zero) == 0, zero
