"""Block-table calls whose outputs share memory with another array: refused before anything is
launched (a workgroup could still be reading what another has written)."""
import ctypes

import pytest

from paper_2603_18815_amd import _lib

# 4 rows of 8 pages, a free list of 10, 100 slots: arrays 4 KB apart, never dereferenced
BASE = {n: 0x10000 + 0x1000 * i for i, n in enumerate(
    ("start", "new", "free", "count", "table", "cu", "lens", "slots", "taken"))}
ROWS, TABLE, FREE, SLOTS = 16, 128, 40, 800


def extend(lib, **kw):
    d = {n: ctypes.c_void_p(kw.get(n, a)) for n, a in BASE.items()}
    return lib.kv_block_table_extend(d["start"], d["new"], d["free"], d["count"], 10, d["table"], 4,
                                     8, 100, d["cu"], d["lens"], d["slots"], d["taken"], None)


def release(lib, **kw):
    d = {n: ctypes.c_void_p(kw.get(n, a)) for n, a in BASE.items()}
    return lib.kv_block_table_release(d["start"], d["new"], d["table"], 4, 8, d["free"], d["count"],
                                      10, 32, d["taken"], None)


@pytest.mark.parametrize("call,which,at", [
    (extend, "lens", BASE["start"]), (extend, "lens", BASE["new"]), (extend, "cu", BASE["new"]),
    (extend, "lens", BASE["start"] + ROWS - 4), (extend, "lens", BASE["start"] - ROWS + 4),
    (extend, "cu", BASE["lens"] - ROWS), (extend, "taken", BASE["count"]),
    (extend, "taken", BASE["free"] + FREE - 4), (extend, "slots", BASE["start"] - SLOTS + 8),
    (extend, "start", BASE["table"] + TABLE - 4), (extend, "count", BASE["free"] + 36),
    (release, "taken", BASE["start"] + 12), (release, "taken", BASE["count"]),
    (release, "free", BASE["table"] + TABLE - 4), (release, "count", BASE["new"])])
def test_arrays_that_share_memory_are_refused(call, which, at):
    assert call(_lib.load(), **{which: at}) == _lib.RA_ERR_UNSUPPORTED
