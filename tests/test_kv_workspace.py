"""The scratch of molora_kv_attend as a size that a caller asks for once: what is enough for a step's most tokens is enough for fewer (no GPU)."""
import pytest

import paper_2603_15965_b200 as M


@pytest.mark.parametrize("dt", ["BF16", "F32"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 8), (6, 2), (8, 2), (5, 1), (8, 1), (24, 1), (1024, 1)])
def test_size_never_falls_as_tokens_grow(dt, dim, heads, kv_heads):
    last = 0
    for most in list(range(1, 140)) + [1000, 10 ** 6, 2 ** 31, 2 ** 40, 2 ** 53, 2 ** 62, 2 ** 63 - 1]:
        size = M.molora_kv_attend_workspace_bytes(getattr(M, dt), heads, kv_heads, dim, most)
        assert size >= last > -1 and size > 0, (most, size, last)
        last = size
