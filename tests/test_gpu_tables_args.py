"""Arguments of the block-table calls that stand at the edge of what is documented."""
import numpy as np
import pytest
import torch

import paper_2603_18815_amd as ra

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.as_tensor(np.ascontiguousarray(np.asarray(x, np.int32)), device="cuda:0")


def pool(B, stride=4, pages=32):
    return dev(np.full((B, stride), -7)), dev(np.arange(pages)), dev([pages])


# sums below zero, past every row's table, and past 32 bits
@pytest.mark.parametrize("new", [[-5, 3], [-1], [-2**31, -2**31, 1], [1, 100], [65] * 3,
                                 [2**31 - 1, 2**31 - 1], [2**31 - 1] * 2 + [7]])
def test_total_new_left_out_for_lengths_out_of_range(new, device):
    """The call refuses as a whole; nothing is raised, and the slot map is no longer than the
    tables."""
    B = len(new)
    table, free, count = pool(B)
    start = dev([2] * B)
    cu, lens, slots, taken = ra.block_table_extend(table, start, dev(new), free, count)
    assert taken.item() == -1 and count.item() == 32
    assert cu.tolist() == [0] * (B + 1) and lens.tolist() == [2] * B
    assert slots.numel() <= B * 4 * 16 and (slots == -1).all()
    assert (table == -7).all() and free.tolist() == list(range(32))


def test_total_new_beyond_32_bits_is_refused(device):
    table, free, count = pool(2)
    with pytest.raises(ValueError, match="total_new"):
        ra.block_table_extend(table, dev([0, 0]), dev([1, 1]), free, count, total_new=2**32 + 2)
    assert count.item() == 32 and (table == -7).all()


def test_lengths_in_place_are_refused(device):
    """Other workgroups may not have read the old lengths yet."""
    table, free, count = pool(3)
    start, new = dev([2, 3, 4]), dev([1, 1, 1])
    for kw in (dict(kv_lens=start), dict(kv_lens=new)):
        with pytest.raises(ra.RolloutAttnError):
            ra.block_table_extend(table, start, new, free, count, total_new=3, **kw)
    with pytest.raises(ra.RolloutAttnError):
        ra.block_table_release(table, start, new, free, count, released=count)
    assert start.tolist() == [2, 3, 4] and new.tolist() == [1, 1, 1] and count.item() == 32
    # what is only read may be the same
    assert ra.block_table_release(table, start, start, free, count).item() == 0


@pytest.mark.parametrize("B,nhi", [(1, 1), (64, 1), (40, 300), (1100, 9)])
def test_without_a_slot_map(B, nhi, device):
    """Through the C ABI: the same tables, lengths and list as with one."""
    from paper_2603_18815_amd import _lib
    rng = np.random.default_rng(B)
    start, new = dev(rng.integers(0, 64, B)), dev(rng.integers(0, nhi + 1, B))
    stride, total = (64 + nhi) // 16 + 1, int(new.sum())
    sides = []
    for slots in (True, False):
        table, free, count = pool(B, stride, B * stride)
        cu, lens, taken = dev(np.full(B + 1, 9)), dev(np.full(B, 9)), dev([9])
        out = torch.full((total,), 5, dtype=torch.int64, device="cuda:0") if slots else None
        s = _lib.load().kv_block_table_extend(
            start.data_ptr(), new.data_ptr(), free.data_ptr(), count.data_ptr(), free.numel(),
            table.data_ptr(), B, stride, total, cu.data_ptr(), lens.data_ptr(),
            out.data_ptr() if slots else None, taken.data_ptr(),
            torch.cuda.current_stream().cuda_stream)
        assert s == _lib.RA_OK
        sides.append((table, free, count, cu, lens, taken))
    assert all(torch.equal(a, b) for a, b in zip(*sides))
    assert sides[0][5].item() >= 0
