"""Results over inputs that the same call still reads: refused on the host, before anything is enqueued, wherever rows share a byte, and only there (no
GPU; calls that are not refused here are left to end with their next argument)."""
import ctypes
import itertools

import pytest

import paper_2603_15965_b200 as M
from test_kv_refusals import INVALID, WORKSPACE, cache, seqs

BASE = 0x100000


def append(N, dt, q, ldq, q_out, ldqo, k=0x9000000, ldk=256, v=0xA000000, ldv=256):
    return M.load_library().molora_kv_append(ctypes.byref(cache()), ctypes.byref(seqs()), dt, N, k, ldk, v, ldv, q, ldq, q_out, ldqo, 4, None, 0, 0, None, None)


def attend(N, dt, q, ldq, out, ldo):
    """With a workspace that is too small: a call that is not refused for its rows ends there."""
    return M.load_library().molora_kv_attend(ctypes.byref(cache()), ctypes.byref(seqs()), dt, N, q, ldq, out, ldo, None, 4, 0.1, 1, 0, 1, 0x10000, 16, None, None)


@pytest.fixture(autouse=True)
def nothing_enqueued():
    before = M.molora_launch_count()
    yield
    assert M.molora_launch_count() == before


def _share(N, size, a, lda, b, ldb, width):
    rows = [(a + i * lda * size, b + i * ldb * size) for i in range(N)]
    return any(x < y + width * size and y < x + width * size for x, _ in rows for _, y in rows)


@pytest.mark.parametrize("dt,size", [("BF16", 2), ("F32", 4)])
@pytest.mark.parametrize("lda,ldb", [(512, 512), (1024, 1024), (1536, 1536), (1032, 1032), (512, 1024), (1024, 512), (2048, 1024), (1536, 1024)])
@pytest.mark.parametrize("N", [1, 2, 5])
def test_attention_refuses_exactly_what_overlaps(N, lda, ldb, dt, size):
    for d in itertools.chain(range(-6 * 2048, 6 * 2048 + 1, 256), (-520, -512, -504, 504, 520, 1016, 1032, 1544)):
        out = BASE + d * size
        if out % 16:
            continue
        want = INVALID if _share(N, size, BASE, lda, out, ldb, 512) else WORKSPACE
        assert attend(N, getattr(M, dt), BASE, lda, out, ldb) == want, d


@pytest.mark.parametrize("d", [-1016, -504, -8, 8, 256, 504, 520, 1024, -1024, 2048])
def test_append_refuses_q_out_over_other_rows_of_q(d):
    assert append(4, M.BF16, BASE, 1024, BASE + 2 * d, 1024) == INVALID


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("d", [-504, -8, 0, 8, 248, 520, 1024, -1024])
def test_append_refuses_q_out_over_k_or_v(which, d):
    """Packed rows of q, k, v: q_out one buffer that reaches into k's or v's columns, or rows."""
    at = BASE + 2 * 512
    assert append(4, M.BF16, 0x8000000, 512, at + 2 * d, 1024, **{which: at, "ld" + which: 1024}) == INVALID
