"""molora_kv_attend on the GPU against attention in 64 bits; bounds from _kv_reference.attend."""
import math

import pytest
import torch

import _kv_reference as R
import paper_2603_15965_b200 as M

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def problem(seed, new, lens, heads, kv_heads, dim, page, dtype, tail=0, size=1.0):
    gen = torch.Generator().manual_seed(seed)
    table, pages = R.tables(lens, page, gen)
    pool = R.Pool(pages, kv_heads, page, dim, gen)
    q = (torch.randn(sum(new) + tail, heads, dim, generator=gen) * size).to(TYPES[dtype])
    return dict(new=new, lens=lens, table=table, pool=pool, q=q, gen=gen)


def run(p, scale=None, causal=True, window=0, max_tokens=None, lse=True, out=None, **kw):
    q = p["q"].cuda()
    z = torch.full(q.shape[:2], 7.0, device="cuda") if lse else None
    cache = p["pool"].cuda(M)
    out = M.molora_kv_attend(q, cache, p["table"].cuda(), R.offsets(p["new"]).cuda(), torch.tensor(p["lens"], dtype=torch.int32).cuda(), scale=scale, causal=causal,
                             window=window, max_tokens=max(p["new"]) if max_tokens is None else max_tokens, out=out, lse=z, **kw)
    torch.cuda.synchronize()
    return out, z


def check(p, out, lse, scale=None, causal=True, window=0, rows=None, ref=None):
    scale = p["q"].shape[2] ** -0.5 if scale is None else scale
    o, z, eo, ez = ref or R.attend(p["q"].cpu(), p["pool"], p["table"], p["new"], p["lens"], scale, causal, window, 2 if out.dtype == torch.float32 else 1)
    got = out[:o.shape[0]].cpu().double()
    half = torch.finfo(out.dtype).eps / 2
    bound = eo + half * (o.abs() + eo)
    sel = slice(None) if rows is None else rows
    err = (got - o).abs()
    assert bool((err <= bound)[sel].all()), (float((err - bound)[sel].max()), float((err / bound)[sel].nan_to_num(0).max()))
    if lse is not None:
        g = lse[:o.shape[0]].cpu().double()
        assert torch.equal(g.isinf()[sel], z.isinf()[sel])
        fin = z.isfinite()
        fin = fin if rows is None else fin & torch.zeros_like(fin).index_fill(0, torch.tensor(rows), True)
        assert bool(((g - z).abs() <= ez)[fin].all()), float((g - z).abs()[fin].max())


SHAPES = [
    # new, lens, heads, kv_heads, dim, page
    ((1,), (1,), 2, 1, 128, 64),
    ((1, 1, 1), (17, 64, 1000), 16, 8, 128, 64),
    ((1,) * 5, (3, 129, 16, 15, 700), 12, 4, 64, 16),
    ((1, 1), (2500, 31), 7, 1, 128, 32),
    ((1,), (5000,), 8, 8, 128, 128),
    ((5, 3, 0, 8), (5, 300, 40, 90), 8, 2, 128, 64),                     # drafts: 20, 12, 0, 32 rows
    ((2, 7), (33, 257), 24, 1, 64, 128),                                 # 24 heads share one: 48 and 168 rows
    ((100, 1, 33), (100, 77, 400), 6, 2, 128, 64),                       # chunks beside a single token
    ((130,), (517,), 5, 5, 64, 32),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 50)])
def test_against_64_bits(shape, dtype, causal, window):
    new, lens, heads, kv_heads, dim, page = SHAPES[shape]
    p = problem(shape, new, lens, heads, kv_heads, dim, page, dtype)
    out, lse = run(p, causal=causal, window=window)
    check(p, out, lse, causal=causal, window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size,scale", [(40.0, None), (1e-20, 1e18), (1e15, 1e-14), (3.0, 0.7)])
def test_sizes_of_q_and_scale(dtype, size, scale):
    p = problem(20, (1, 4), (300, 90), 4, 2, 128, 64, dtype, size=size)
    out, lse = run(p, scale=scale)
    check(p, out, lse, scale=scale)


def test_growing_scores_and_uneven_blocks():
    """Scores that keep rising along the keys (the reference of a row has to move), scales of v from 2^-60 to 2^60."""
    p = problem(21, (1, 2), (900, 400), 4, 2, 128, 16, "f32")
    pool = p["pool"]
    q = torch.ones(3, 4, 128)
    p["q"] = q
    for b, l in enumerate(p["lens"]):
        for i in range(-(-l // 16)):
            pool.k[p["table"][b, i].long()] = R.encode(torch.full((), 100.0 + i, dtype=torch.float64))
    pool.k_scale[:] = 2.0 ** -9
    out, lse = run(p, scale=1.0)
    check(p, out, lse, scale=1.0)
    p = problem(22, (1, 2), (900, 400), 4, 2, 128, 16, "bf16")
    p["pool"].v_scale[:] = torch.pow(2.0, torch.randint(-60, 61, p["pool"].v_scale.shape, generator=p["gen"]).float())
    out, lse = run(p)
    o, z, eo, ez = R.attend(p["q"], p["pool"], p["table"], p["new"], p["lens"], 128 ** -0.5, True, 0)
    # weights below 2^-32 of what a row's largest contributes come out in steps; the reference's bound knows that by the largest scale
    check(p, out, lse, ref=(o, z, eo, ez))


def test_scales_that_are_no_powers_of_two():
    p = problem(23, (1, 6), (500, 130), 8, 4, 128, 64, "f32")
    p["pool"].k_scale *= 1 + 0.9 * torch.rand(p["pool"].k_scale.shape, generator=p["gen"])
    p["pool"].v_scale *= 1 + 0.9 * torch.rand(p["pool"].v_scale.shape, generator=p["gen"])
    out, lse = run(p)
    check(p, out, lse)
    p["pool"].k_scale[:], p["pool"].v_scale[:] = 0.0, 0.0                # blocks of nothing, as others may write them
    out, lse = run(p)
    assert bool((out.abs() <= 448 * 2.0 ** -100).all())
    check(p, lse.new_zeros(out.shape), lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,lens", [((1, 1), (50, 20)), ((6, 20), (50, 20)), ((140, 3), (300, 40))])
def test_codes_that_no_row_sees_leave_no_trace(dtype, new, lens):
    """NaN codes behind the sequences' ends, in foreign pages, and at keys that the earlier rows of a tile do not see."""
    p = problem(24, new, lens, 4, 2, 128, 64, dtype)
    clean, clean_lse = run(p)
    check(p, clean, clean_lse)
    pool, page = p["pool"], p["pool"].page
    used = torch.zeros(pool.k.shape[0], page, dtype=torch.bool)
    for b, l in enumerate(lens):
        for j in range(l):
            used[int(p["table"][b, j // page]), j % page] = True
    for codes in (pool.k, pool.v):
        codes.transpose(1, 2)[~used] = 0x7F
    out, lse = run(p)
    assert torch.equal(out, clean) and torch.equal(lse, clean_lse)
    if max(new) == 1:
        return
    for which in ("k", "v"):                                             # the last token of sequence 0: only its last row sees it
        q = problem(24, new, lens, 4, 2, 128, 64, dtype)
        at = lens[0] - 1
        getattr(q["pool"], which)[int(q["table"][0, at // page]), 1, at % page, 77] = 0xFF
        out, lse = run(q)
        rows = [r for r in range(sum(new)) if r != new[0] - 1]
        assert torch.equal(out[rows], clean[rows]) and torch.equal(lse[rows], clean_lse[rows])
        assert bool(out[new[0] - 1, 2:].isnan().any(-1).all()) and torch.equal(out[new[0] - 1, :2], clean[new[0] - 1, :2])


def test_window_hides_nan_in_front():
    p = problem(25, (3,), (200,), 2, 1, 64, 16, "bf16")
    clean, z = run(p, window=40)
    check(p, clean, z, window=40)
    p["pool"].v[int(p["table"][0, 157 // 16]), 0, 157 % 16, 3] = 0x7F      # rows see from 158, 159 and 160 on
    p["pool"].k[int(p["table"][0, 150 // 16]), 0, 150 % 16, 3] = 0x7F
    out, lse = run(p, window=40)
    assert torch.equal(out, clean) and torch.equal(lse, z)
    p["pool"].v[int(p["table"][0, 158 // 16]), 0, 158 % 16, 3] = 0x7F
    out, lse = run(p, window=40)
    assert bool(out[0].isnan().any()) and torch.equal(out[1:], clean[1:])


def test_nan_in_q_stays_in_its_row():
    p = problem(26, (9,), (90,), 4, 2, 128, 64, "bf16")
    clean, z = run(p)
    p["q"][4, 1, 100] = math.nan
    out, lse = run(p)
    keep = torch.ones(9, 4, dtype=torch.bool)
    keep[4, 1] = False
    assert torch.equal(out.cpu()[keep], clean.cpu()[keep]) and bool(out[4, 1].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [(2, 1, 3), (40, 1, 150)])
def test_rows_that_see_nothing(dtype, new):
    """An empty cache, and more new tokens than the cache has: rows of position below 0."""
    p = problem(27, new, (new[0], 0, new[2] - 2), 4, 2, 64, 16, dtype, tail=5)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out0 = torch.full(p["q"].shape, 7.0, dtype=p["q"].dtype, device="cuda")
    out, lse = run(p, out=out0, dev_status=status)
    assert int(status) == 8
    n = sum(new)
    assert bool((out[n:] == 7).all()) and bool((lse[n:] == 7).all())      # rows of no sequence
    empty = [new[0], new[0] + 1, new[0] + 2]
    assert bool((out[empty] == 0).all()) and bool((lse[empty] == -math.inf).all())
    good = dict(p, new=(new[0],), lens=(new[0],))
    check(good, out[:new[0]], lse[:new[0]])


def test_pages_outside_the_pool_are_left_out_and_reported():
    p = problem(28, (1, 1), (100, 100), 2, 1, 64, 16, "bf16")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    clean, _ = run(p, dev_status=status)
    assert int(status) == 0
    p["table"][0, 2] = p["pool"].k.shape[0]
    out, lse = run(p, dev_status=status)
    assert int(status) == 8 and torch.equal(out[1], clean[1])
    # what is left: the keys of the other pages
    keep = torch.cat([torch.arange(32), torch.arange(48, 100)])
    k, v = (p["pool"].sequence(w, p["table"][0].clamp(0, p["pool"].k.shape[0] - 1), 100)[0][keep] for w in "kv")
    w = torch.softmax(p["q"][0].double() @ k.T * 64 ** -0.5, -1)
    assert float((out[0].cpu().double() - w @ v).abs().max()) < 0.02
    status.zero_()
    q = dict(p, lens=(100, 4000))                                        # longer than its page table
    out, lse = run(q, dev_status=status)
    assert int(status) == 8


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_key_axis_and_many_short_sequences(dtype):
    p = problem(29, (1, 1), (20000, 9), 8, 2, 128, 64, dtype)
    out, lse = run(p)
    check(p, out, lse)
    lens = tuple(1 + (37 * i) % 90 for i in range(700))
    p = problem(30, (1,) * 700, lens, 2, 1, 64, 16, dtype)
    out, lse = run(p)
    check(p, out, lse)


def test_offsets_beyond_32_bits():
    """A pool of more than 2^31 codes, the sequence in its last pages."""
    pages = 2 ** 31 // (8 * 128 * 128) + 40
    k = torch.zeros(pages, 8, 128, 128, dtype=torch.uint8, device="cuda")
    v = torch.zeros_like(k)
    ks, vs = torch.ones(pages, 8, device="cuda"), torch.ones(pages, 8, device="cuda")
    p = problem(31, (4,), (300,), 8, 8, 128, 128, "bf16")
    n = p["pool"].k.shape[0]
    for big, small in ((k, p["pool"].k), (v, p["pool"].v), (ks, p["pool"].k_scale), (vs, p["pool"].v_scale)):
        big[pages - n:] = small.cuda()
    table = torch.where(p["table"] >= 0, p["table"] + pages - n, p["table"]).cuda()
    out = M.molora_kv_attend(p["q"].cuda(), M.KVCache(k, v, ks, vs), table, R.offsets((4,)).cuda(), torch.tensor([300], dtype=torch.int32).cuda())
    check(p, out, None)
    new_k = torch.randn(4, 8, 128, device="cuda").bfloat16()
    M.molora_kv_append(new_k, new_k, M.KVCache(k, v, ks, vs), table, R.offsets((4,)).cuda(), torch.tensor([300], dtype=torch.int32).cuda())
    got = R.decode(k[int(table[0, 2]), :, 40:44].cpu()) * ks[int(table[0, 2])].cpu().double()[:, None, None]
    assert bool(((got - new_k.cpu().double().transpose(0, 1)).abs() <= 2.0 ** -4 * new_k.cpu().double().abs().transpose(0, 1) + 2.0 ** -6).all())
    assert int(k[:pages - n].count_nonzero()) == 0


def test_strided_q_shared_workspace_and_graphs():
    """q inside a packed projection; two captured graphs that share one workspace, replayed in turn; a stream of its own."""
    a, b = problem(32, (1, 1), (900, 60), 16, 8, 128, 64, "bf16"), problem(33, (3, 5), (200, 77), 16, 8, 128, 64, "bf16")
    ws = torch.empty(M.molora_kv_attend_workspace_bytes(M.BF16, 16, 8, 128, 5), dtype=torch.uint8, device="cuda")
    state = []
    for p in (a, b):
        n = sum(p["new"])
        wide = torch.randn(n, 32, 128, device="cuda").bfloat16()
        wide[:, 4:20] = p["q"].cuda()
        state.append(dict(q=wide[:, 4:20], cache=p["pool"].cuda(M), table=p["table"].cuda(), cu=R.offsets(p["new"]).cuda(),
                          lens=torch.tensor(p["lens"], dtype=torch.int32).cuda(), out=torch.zeros(n, 20, 128, dtype=torch.bfloat16, device="cuda")))
    graphs = []
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for st in state:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            M.molora_kv_attend(st["q"], st["cache"], st["table"], st["cu"], st["lens"], max_tokens=5, out=st["out"][:, 1:17], ws=ws)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for p, st in zip((a, b), state):
        check(p, st["out"][:, 1:17], None)
        assert bool((st["out"][:, 0] == 0).all()) and bool((st["out"][:, 17:] == 0).all())


def test_results_do_not_depend_on_the_run():
    p = problem(34, (1,) * 20, tuple(range(100, 2100, 100)), 8, 4, 128, 64, "bf16")
    first = run(p)
    for _ in range(3):
        again = run(p)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
