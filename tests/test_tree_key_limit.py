"""reform_tree_attend counts a sequence's keys, and what its loops add to them, in 32-bit signed integers: more keys than these
hold are refused on the host (no GPU is needed: no call here gets past its checks)."""
import ctypes

import pytest

from paper_2506_01215_amd import binding

FAKE = 0x1000
MOST = (1 << 31) - 512


def desc(max_cache_len, n_nodes, dtype, head_dim):
    row = 64 * head_dim
    return binding.TreeDesc(struct_size=ctypes.sizeof(binding.TreeDesc), dtype=dtype, n_seq=1, n_q_heads=1, n_kv_heads=1, head_dim=head_dim,
                            n_nodes=n_nodes, max_cache_len=max_cache_len, capacity=(1 << 31) - 1, scale=0.5, q_seq_stride=row,
                            q_head_stride=row, q_row_stride=head_dim, o_seq_stride=row, o_head_stride=row, o_row_stride=head_dim,
                            kv_seq_stride=0, kv_head_stride=0)


def call(d):
    return binding.load_library().reform_tree_attend(ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, None, None, FAKE, None, None, 0, None)


@pytest.mark.parametrize("dtype,head_dim", [(0, 4), (0, 256), (1, 64), (1, 128)])
@pytest.mark.parametrize("n_nodes", [1, 5, 64])
def test_key_counts_outside_32_bits_are_refused(dtype, head_dim, n_nodes):
    query = binding.load_library().reform_tree_attend_workspace
    for keys in (MOST + 1, (1 << 31) - 64, (1 << 31) - 16, (1 << 31) - 1):
        d = desc(keys - n_nodes, n_nodes, dtype, head_dim)
        assert query(ctypes.byref(d)) == 0 and call(d) == 2, keys
    # the most that is taken is shared out, so without a workspace the call ends there
    d = desc(MOST - n_nodes, n_nodes, dtype, head_dim)
    assert query(ctypes.byref(d)) > 0 and call(d) == 3


def test_the_limit_covers_the_largest_sum():
    """Tiles of 16, 32 and 64 keys, two groups of waves at most: the number of tiles is formed as (keys + 63) / 64, and the
    key that comes after a group's next but one tile is the largest count that a loop compares."""
    for tile, groups in ((16, 1), (32, 1), (64, 1), (64, 2)):
        tiles = (MOST + tile - 1) // tile
        steps = -(-tiles // groups)
        assert MOST + tile - 1 < 1 << 31
        assert ((steps + 1) * groups + groups) * tile < 1 << 31
