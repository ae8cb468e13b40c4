"""molora_kv_attend where units of rows are many, are cut between shares, or meet each other: every number of rows that has a kernel of
its own, prompts of several tiles, key axes that many shares divide, streams and graphs.  Bounds from _kv_reference.attend."""
import pytest
import torch

import _kv_reference as R
import paper_2603_15965_b200 as M
from test_gpu_kv_attend import check, problem, run

pytestmark = pytest.mark.gpu

# heads, kv_heads, most new tokens: 4, 8, 16, 24 and 32 rows, and numbers that do not fill them
ROWS = [(4, 1, 1), (6, 2, 1), (8, 1, 1), (10, 2, 1), (8, 2, 4), (5, 1, 3), (8, 1, 3), (12, 2, 4), (8, 1, 4), (10, 2, 5)]


@pytest.mark.parametrize("heads,kv_heads,most", ROWS)
@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 130)])
def test_rows_of_a_few_tokens(heads, kv_heads, most, page, causal, window):
    """A long sequence that many shares divide, between short ones and one without new tokens."""
    new, lens = (1, most, 0, most, 1), (3, 9000, 77, 257, 128)
    p = problem(40 + heads, new, lens, heads, kv_heads, 128, page, "bf16")
    out, lse = run(p, causal=causal, window=window)
    check(p, out, lse, causal=causal, window=window)


@pytest.mark.parametrize("most", [1, 2, 3, 4])
def test_many_sequences_of_a_few_tokens(most):
    """More units than shares, and with them shares of several units."""
    new = tuple(1 + (i * 7) % most for i in range(400))
    lens = tuple(n + (i * i) % 500 for i, n in enumerate(new))
    p = problem(50 + most, new, lens, 8, 1, 128, 64, "bf16")
    out, lse = run(p)
    check(p, out, lse)


PROMPTS = [
    # new, lens, heads, kv_heads, page
    ((700,), (700,), 4, 1, 64),
    ((300, 1, 0, 513, 64), (1000, 50, 0, 513, 3000), 8, 2, 16),
    ((2100,), (2100,), 2, 2, 128),
    ((40,), (30000,), 4, 1, 64),                                         # one unit, cut wherever shares end
    ((257, 31, 257, 128, 129), (257, 31, 900, 129, 193), 3, 3, 32),
    ((1500, 300), (1500, 1300), 4, 2, 32),
    ((257, 31, 700, 128, 129, 256), (2257, 31, 900, 129, 193, 256), 12, 3, 128),
    ((90,) * 12, tuple(90 + 70 * i for i in range(12)), 16, 4, 16),
    (tuple(20 + i % 50 for i in range(60)), tuple(20 + i % 50 + (i % 7) * 40 for i in range(60)), 4, 2, 64),
]


@pytest.mark.parametrize("dim,dtype", [(128, "bf16"), (64, "f32")])
@pytest.mark.parametrize("new,lens", [((1, 3), (300, 90)), ((60, 9), (50, 200))])
def test_a_window_of_everything(dim, dtype, new, lens):
    """The largest window is no window, also where more tokens are new than there are."""
    p = problem(56, new, lens, 8, 2, dim, 64, dtype)
    out, lse = run(p)
    for window in (2 ** 30, 2 ** 31 - 1):
        again, z = run(p, window=window)
        assert torch.equal(out, again) and torch.equal(lse, z)


@pytest.mark.parametrize("most", [1, 3, 6, 1000])
def test_longest_sequence_need_not_be_known(most):
    """max_tokens chooses the kernel; sequences longer than it are served all the same."""
    new, lens = (5, 70, 1, 200), (900, 70, 30, 450)
    p = problem(55, new, lens, 8, 2, 128, 64, "bf16")
    out, lse = run(p, max_tokens=most)
    check(p, out, lse)


@pytest.mark.parametrize("which", range(len(PROMPTS)))
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 200)])
def test_prompts_of_several_tiles(which, causal, window):
    new, lens, heads, kv_heads, page = PROMPTS[which]
    p = problem(60 + which, new, lens, heads, kv_heads, 128, page, "bf16")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = run(p, causal=causal, window=window, dev_status=status)
    assert int(status) == 0
    check(p, out, lse, causal=causal, window=window)


@pytest.mark.parametrize("new", [1, 20])
def test_one_key_against_many_alike(new):
    """A key that has half of the weight and values of zero, 60000 keys alike: what they are off by adds up.  Up to 32 rows a weight is off by
    2^-11 of itself and by 2^-20 where the row's largest is 2^5 or more, so by 2^-25 of the largest; the bound takes that for all."""
    length = 60001
    p = problem(70 + new, (new,), (length,), 2, 1, 128, 128, "bf16")
    pool, table = p["pool"], p["table"][0].long()
    p["q"][:] = 1.0
    pool.k[:], pool.v[:] = 0, R.encode(torch.full((), 3.0, dtype=torch.float64))
    pool.k[table[0], 0, 0] = R.encode(torch.full((), 124.0 / 128, dtype=torch.float64))      # about ln 60000 with a scale of 1 / 11
    pool.v[table[0], 0, 0] = 0
    pool.k_scale[:], pool.v_scale[:] = 1.0, 1.0
    scale = 1 / 11.0
    out, lse = run(p, scale=scale, causal=False)
    o, z, eo, ez = R.attend(p["q"], pool, p["table"], p["new"], p["lens"], scale, False, 0)
    assert 0.3 < float(o[0, 0, 0]) / 3 < 0.7
    largest = 0.7
    check(p, out, lse, ref=(o, z, eo + length * 2.0 ** -25 * largest * 3.0, ez))


@pytest.mark.parametrize("new,lens", [((1,) * 30, tuple(range(50, 3050, 100))), ((90, 300), (400, 300))])
def test_two_streams_with_workspaces_of_their_own(new, lens):
    p = problem(80, new, lens, 8, 2, 128, 64, "bf16")
    first, z = run(p)
    check(p, first, z)
    args = [p["q"].cuda(), p["pool"].cuda(M), p["table"].cuda(), R.offsets(new).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()]
    size = M.molora_kv_attend_workspace_bytes(M.BF16, 8, 2, 128, max(new))
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [torch.zeros_like(first) for _ in streams]
    spaces = [torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda") for _ in streams]      # (need not be cleared)
    torch.cuda.synchronize()
    for _ in range(10):
        for s, o, ws in zip(streams, outs, spaces):
            with torch.cuda.stream(s):
                M.molora_kv_attend(*args, max_tokens=max(new), out=o, ws=ws)
    torch.cuda.synchronize()
    for o in outs:
        assert torch.equal(o, first)


def test_prompts_in_a_graph_over_changing_lengths():
    """A captured call serves what the lengths on the device say, from a single token to the whole prompt."""
    heads, kv_heads, page, rows = 8, 2, 64, 600
    full = problem(81, (rows,), (1500,), heads, kv_heads, 128, page, "bf16")
    q, cache, table = full["q"].cuda(), full["pool"].cuda(M), full["table"].cuda()
    table2 = torch.cat([table, table])
    cu, lens = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    ws = torch.empty(M.molora_kv_attend_workspace_bytes(M.BF16, heads, kv_heads, 128, rows), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        M.molora_kv_attend(q, cache, table2, cu, lens, max_tokens=rows, out=out, ws=ws)
    for new, have in (((rows, 0), (1500, 0)), ((1, 1), (1000, 30)), ((0, 599), (0, 599)), ((200, 400), (200, 1500))):
        cu.copy_(R.offsets(new))
        lens.copy_(torch.tensor(have, dtype=torch.int32))
        out.fill_(7.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        n = sum(new)
        p = dict(full, new=new, lens=have, q=full["q"][:n], table=torch.cat([full["table"]] * 2))
        check(p, out, None)
        assert bool((out[n:] == 7).all())


@pytest.mark.parametrize("dim,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32")])
@pytest.mark.parametrize("new", [(1, 0, 2), (50, 0, 3)])
def test_a_pool_without_pages(dim, dtype, new):
    gen = torch.Generator().manual_seed(82)
    q = torch.randn(sum(new), 4, dim, generator=gen).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    codes, scales = torch.zeros(0, 2, 64, dim, dtype=torch.uint8, device="cuda"), torch.zeros(0, 2, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = torch.zeros(sum(new), 4, device="cuda")
    out = M.molora_kv_attend(q, M.KVCache(codes, codes.clone(), scales, scales.clone()), torch.zeros(3, 1, dtype=torch.int32, device="cuda"), R.offsets(new).cuda(),
                             torch.zeros(3, dtype=torch.int32, device="cuda"), max_tokens=max(new), lse=lse, dev_status=status)
    assert bool((out == 0).all()) and bool((lse == -float("inf")).all()) and int(status) == 8
