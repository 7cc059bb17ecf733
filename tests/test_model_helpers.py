"""Pool.kv_cache and Pool.adapters, on a pool that was never created (CPU)."""
import numpy as np
import pytest

from paper_2601_21473_amd import binding as B

P = 0x100000


@pytest.fixture
def pool():
    pool = B.Pool.__new__(B.Pool)
    pool._h, pool.n_agents, pool._capacity = None, 4, 8
    pool._units = np.ones(4, np.uint32)
    pool._chunk = np.array([8192, 4096], np.uint64)
    pool._bases = [P, 2 * P]
    pool.block_table = lambda: (P, P)
    return pool


@pytest.mark.parametrize("k_offset,v_offset", [(0, 0), (0, 2048), (4096, 64), (64, 4080)])
def test_keys_and_values_in_the_same_bytes(pool, k_offset, v_offset):
    """A page of 16 x 2 x 64 16-bit values is 4,096 bytes; keys and values may share a
    plane, not bytes of it."""
    with pytest.raises(ValueError, match="overlap"):
        pool.kv_cache(0, 0, page_tokens=16, n_heads=2, head_dim=64, type=B.SS_BF16, k_offset=k_offset,
                      v_offset=v_offset)


@pytest.mark.parametrize("k_offset,v_offset", [(0, 4096), (4096, 0), (0, 2176)])
def test_keys_and_values_in_one_plane(pool, k_offset, v_offset):
    kind = B.SS_E4M3 if v_offset == 2176 else B.SS_BF16        # 2,048 codes and 32 scales
    c = pool.kv_cache(0, 0, page_tokens=16, n_heads=2, head_dim=64, type=kind, k_offset=k_offset,
                      v_offset=v_offset)
    assert (c.k, c.v, c.k_unit_bytes, c.v_unit_bytes) == (P + k_offset, P + v_offset, 8192, 8192)
