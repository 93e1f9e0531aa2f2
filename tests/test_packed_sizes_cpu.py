"""Packed caches: sizes next to what integers hold (no GPU)."""
import pytest

import paper_2412_05693_b200 as bm
from paper_2412_05693_b200.build import build

MOST_RUNS = 148 * 12      # warps that share a call, and leave two shares each


@pytest.fixture(scope="module", autouse=True)
def built():
    build()


def test_workspaces_of_the_largest_configs():
    """Samples, heads, queries and rows multiply to more than 64 bits hold: the workspace stays that of a full GPU's warps."""
    for queries, heads in ((1 << 24, 1 << 20), (1 << 24, 1 << 30), (1, 1 << 30), (1 << 24, 8)):
        for batch, capacity in ((1 << 12, 1 << 24), (1 << 20, 1 << 16)):
            cfg = bm.PackedConfig(batch=batch, n_q_heads=heads, n_kv_heads=8, head_dim=128, capacity=capacity, queries_max=queries)
            assert bm.packed_arena_bytes(cfg) > 0
            shares = MOST_RUNS * 2 * 8 * 132 * 4
            assert shares <= bm.packed_workspace_bytes(cfg) <= shares + 4 * batch * 8 * 64 + 4096


def test_workspaces_of_configs_without_an_arena_are_refused():
    cfg = bm.PackedConfig(batch=2 ** 31 - 1, n_q_heads=1 << 20, n_kv_heads=1 << 20, head_dim=128, capacity=1 << 24, n_layers=2 ** 31 - 1)
    for query in (bm.packed_arena_bytes, bm.packed_workspace_bytes):
        with pytest.raises(bm.BMError) as e:
            query(cfg)
        assert e.value.code == 1
