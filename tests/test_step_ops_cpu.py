"""Refusals of the step operators (tables, sampling, linear attention) that need no GPU:
through the C ABI with addresses that are never dereferenced, and through the binding."""
import ctypes

import pytest
import torch

import paper_2603_18815_amd as ra
from paper_2603_18815_amd import _lib

FAKE = ctypes.c_void_p(0x1000)
INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def lib():
    return _lib.load()


def test_token_sample_validation(lib):
    def call(**kw):
        d = dict(z=FAKE, dt=_lib.RA_LOGITS_FP32, N=4, V=100, stride=100, u=FAKE, t=FAKE, ws=FAKE,
                 bytes=1 << 40)
        d.update(kw)
        return lib.token_sample(d["z"], d["dt"], d["N"], d["V"], d["stride"], None, None, None,
                                None, d["u"], d["t"], None, d["ws"], d["bytes"], None)
    for name in ("z", "u", "t"):
        assert call(**{name: None}) == _lib.RA_ERR_NULL
    assert call(N=-1) == _lib.RA_ERR_SHAPE
    assert call(V=0) == _lib.RA_ERR_SHAPE
    assert call(stride=99) == _lib.RA_ERR_SHAPE
    assert call(dt=2) == _lib.RA_ERR_UNSUPPORTED
    assert call(V=(1 << 19) + 1, stride=1 << 20) == _lib.RA_ERR_UNSUPPORTED
    assert call(N=(1 << 20) + 1) == _lib.RA_ERR_UNSUPPORTED
    assert call(N=0, z=None, u=None, t=None, ws=None) == _lib.RA_OK
    size = lib.token_sample_workspace_size
    assert size(0, 100) == 0 and size(4, 0) == 0 and size(4, (1 << 19) + 1) == 0
    need = size(4, 1 << 19)
    assert call(V=1 << 19, stride=1 << 19, bytes=need - 1) == _lib.RA_ERR_WORKSPACE
    assert call(V=1 << 19, stride=1 << 19, ws=None) == _lib.RA_ERR_WORKSPACE
    assert call(ws=ctypes.c_void_p(0x1008)) == _lib.RA_ERR_WORKSPACE          # 16 bytes


LINEAR = dict(q=FAKE, k=FAKE, v=FAKE, cu=FAKE, lens=FAKE, st=FAKE, slots=FAKE, ns=8, g=FAKE, B=4,
              Hq=8, Hkv=2, total=1000, mq=500, scale=0.1, out=FAKE, ws=FAKE, bytes=1 << 40)


def _decode(lib, **kw):
    d = dict(LINEAR, **kw)
    return lib.rollout_linear_attn_decode(
        d["q"], d["k"], d["v"], d["st"], d["slots"], d["ns"], d["lens"], d["g"], d["B"], d["Hq"],
        d["Hkv"], d["scale"], d["out"], None)


def _append(lib, **kw):
    d = dict(LINEAR, **kw)
    return lib.rollout_linear_attn_append(
        d["q"], d["k"], d["v"], d["cu"], d["lens"], d["st"], d["slots"], d["ns"], d["g"], d["B"],
        d["Hq"], d["Hkv"], d["total"], d["mq"], d["scale"], d["out"], d["ws"], d["bytes"], None)


@pytest.mark.parametrize("call", [_decode, _append])
def test_linear_validation(lib, call):
    for name in ("q", "k", "v", "lens", "st", "slots", "g", "out"):
        assert call(lib, **{name: None}) == _lib.RA_ERR_NULL, name
    assert call(lib, B=-1) == _lib.RA_ERR_SHAPE
    assert call(lib, Hq=7) == _lib.RA_ERR_SHAPE
    assert call(lib, Hkv=0) == _lib.RA_ERR_SHAPE
    assert call(lib, ns=0) == _lib.RA_ERR_SHAPE
    for bad in (INF, -INF, NAN):
        assert call(lib, scale=bad) == _lib.RA_ERR_SHAPE
    assert call(lib, Hq=66) == _lib.RA_ERR_UNSUPPORTED
    assert call(lib, B=65536) == _lib.RA_ERR_UNSUPPORTED
    assert call(lib, Hq=65568, Hkv=2049) == _lib.RA_ERR_UNSUPPORTED
    assert call(lib, B=65535, Hq=1024, Hkv=1024) == _lib.RA_ERR_UNSUPPORTED     # pairs
    for name in ("q", "k", "v", "st", "out"):
        assert call(lib, **{name: ctypes.c_void_p(0x1002)}) == _lib.RA_ERR_UNSUPPORTED, name
    assert call(lib, B=0, q=None, st=None) == _lib.RA_OK


def test_linear_append_validation(lib):
    assert _append(lib, cu=None) == _lib.RA_ERR_NULL
    assert _append(lib, total=-1) == _lib.RA_ERR_SHAPE
    assert _append(lib, mq=-1) == _lib.RA_ERR_SHAPE
    assert _append(lib, total=0, q=None) == _lib.RA_OK
    assert _append(lib, mq=0, q=None) == _lib.RA_OK
    size = lib.rollout_linear_attn_append_workspace_size
    assert size(0, 8, 2, 100, 50) == 0 and size(4, 7, 2, 100, 50) == 0
    assert size(4, 8, 2, 0, 50) == 0 and size(4, 8, 2, 100, 0) == 0
    need = size(1, 32, 32, 16384, 16384)
    one = dict(B=1, Hq=32, Hkv=32, total=16384, mq=16384)
    assert _append(lib, bytes=need - 1, **one) == _lib.RA_ERR_WORKSPACE
    assert _append(lib, ws=None, **one) == _lib.RA_ERR_WORKSPACE
    assert _append(lib, ws=ctypes.c_void_p(0x1008), **one) == _lib.RA_ERR_WORKSPACE
    assert size(256, 32, 32, 25600, 100) == 0                         # whole rows need none
    # the stretches of cut rows take the place, however many rows there are beside them
    state = 128 * 128 * 4
    assert size(60000, 8, 8, 200000, 140000) <= (2 * 256 + 8) * state
    assert size(1, 8, 8, 16384, 2**31 - 1) == size(1, 8, 8, 16384, 16384) <= (256 + 8) * state
    assert _append(lib, B=65535, Hq=65, Hkv=65) == _lib.RA_ERR_UNSUPPORTED   # 2^22 pairs


def test_table_validation(lib):
    def extend(**kw):
        d = dict(s=FAKE, n=FAKE, free=FAKE, count=FAKE, cap=10, bt=FAKE, B=4, stride=8, total=100,
                 cu=FAKE, lens=FAKE, slots=FAKE, taken=FAKE)
        d.update(kw)
        return lib.kv_block_table_extend(d["s"], d["n"], d["free"], d["count"], d["cap"], d["bt"],
                                         d["B"], d["stride"], d["total"], d["cu"], d["lens"],
                                         d["slots"], d["taken"], None)

    def release(**kw):
        d = dict(s=FAKE, n=FAKE, bt=FAKE, B=4, stride=8, free=FAKE, count=FAKE, cap=10, most=32,
                 taken=FAKE)
        d.update(kw)
        return lib.kv_block_table_release(d["s"], d["n"], d["bt"], d["B"], d["stride"], d["free"],
                                          d["count"], d["cap"], d["most"], d["taken"], None)
    for call in (extend, release):
        for name in ("s", "n", "bt", "free", "count", "taken"):
            assert call(**{name: None}) == _lib.RA_ERR_NULL, name
        assert call(B=-1) == _lib.RA_ERR_SHAPE
        assert call(stride=0) == _lib.RA_ERR_SHAPE
        assert call(cap=-1) == _lib.RA_ERR_SHAPE
        assert call(B=65536) == _lib.RA_ERR_UNSUPPORTED
        assert call(stride=1 << 27) == _lib.RA_ERR_UNSUPPORTED
    for name in ("cu", "lens"):
        assert extend(**{name: None}) == _lib.RA_ERR_NULL
    assert extend(total=-1) == _lib.RA_ERR_SHAPE
    assert release(most=-1) == _lib.RA_ERR_SHAPE


def test_host_tensors_are_refused():
    z, u = torch.zeros((2, 8)), torch.zeros(2)
    with pytest.raises(ValueError, match="GPU tensor"):
        ra.token_sample(z, u)
    q = torch.zeros((2, 2, 128), dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU tensor"):
        ra.linear_decode(q, q, q, torch.zeros((2, 2, 128, 128)), i, i, torch.zeros(2))
    with pytest.raises(ValueError, match="GPU tensor"):
        ra.linear_append(q, q, q, i, i[:1], torch.zeros((2, 2, 128, 128)), i[:1], torch.zeros(2))
    with pytest.raises(ValueError, match="GPU tensor"):
        ra.block_table_extend(torch.zeros((2, 4), dtype=torch.int32), i, i, i, i[:1])
    with pytest.raises(ValueError, match="GPU tensor"):
        ra.block_table_release(torch.zeros((2, 4), dtype=torch.int32), i, i, i, i[:1])
