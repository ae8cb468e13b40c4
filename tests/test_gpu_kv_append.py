"""molora_kv_append on the GPU against the rotation and the quantisation in 64 bits."""
import math

import pytest
import torch

import _kv_reference as R
import paper_2603_15965_b200 as M

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def problem(seed, new, before, heads, kv_heads, dim, page, dtype, rotary, packed=True, tail=0):
    gen = torch.Generator().manual_seed(seed)
    lens = [n + c for n, c in zip(new, before)]
    table, pages = R.tables(lens, page, gen)
    pool = R.Pool(pages, kv_heads, page, dim, gen)
    N = sum(new) + tail
    wide = torch.randn(N, (heads + 2 * kv_heads) if packed else heads, dim, generator=gen) * torch.exp2(torch.randint(-3, 4, (N, 1, 1), generator=gen).float())
    wide = wide.to(TYPES[dtype])
    if packed:
        q, k, v = wide[:, :heads], wide[:, heads:heads + kv_heads], wide[:, heads + kv_heads:]
    else:
        q = wide
        k, v = (torch.randn(N, kv_heads, dim, generator=gen).to(TYPES[dtype]) for _ in range(2))
    f = torch.pow(torch.tensor(10000.0, dtype=torch.float64), -torch.arange(0, rotary, 2).double() / max(rotary, 1)).float() if rotary else None
    return dict(new=new, lens=lens, table=table, pool=pool, q=q, k=k, v=v, f=f, N=N, wide=wide if packed else None, heads=heads, kv_heads=kv_heads)


def expected(p, interleaved):
    """(q rotated [rows, heads, dim], its bound, k codes, v codes, scales as dicts of what the call has to leave) in 64 bits."""
    pool, page = p["pool"], p["pool"].page
    rows = sum(p["new"])
    pos = torch.cat([torch.arange(l - n, l) for n, l in zip(p["new"], p["lens"])])
    q = R.rotate(p["q"][:rows].double(), pos, p["f"], interleaved)
    k = R.rotate(p["k"][:rows].double(), pos, p["f"], interleaved)
    v = p["v"][:rows].double()
    blocks = []                                   # (which, page id, head, first row, rows, values [rows, dim], scale, older codes expected)
    at = 0
    for b, (n, l) in enumerate(zip(p["new"], p["lens"])):
        for first in range((l - n) // page * page, l if n else 0, page):
            i = int(p["table"][b, first // page])
            lo, hi = max(first, l - n), min(first + page, l)
            for which, x, codes, scales in (("k", k, pool.k, pool.k_scale), ("v", v, pool.v, pool.v_scale)):
                for h in range(p["kv_heads"]):
                    val = x[at + lo - (l - n):at + hi - (l - n), h]
                    fin = val.abs()[val.isfinite()]
                    scale = R.scale_for(float(fin.max()) if fin.numel() else 0.0)
                    older = None
                    if lo > first:
                        old = float(scales[i, h])
                        scale = max(scale, old)
                        older = R.encode(R.decode(codes[i, h, :lo - first]) * (old / scale)) if scale > old else codes[i, h, :lo - first]
                    blocks.append((which, i, h, lo - first, hi - lo, val, scale, older))
        at += n
    return q, blocks


def run(p, interleaved=False, q_out=None, with_q=True, stream=None, status=None, fp8=True):
    cache = p["pool"].cuda(M, fp8)
    if p["wide"] is not None:
        w = p["wide"].cuda()
        q, k, v = w[:, :p["heads"]], w[:, p["heads"]:p["heads"] + p["kv_heads"]], w[:, p["heads"] + p["kv_heads"]:]
    else:
        q, k, v = p["q"].cuda(), p["k"].cuda(), p["v"].cuda()
    out = M.molora_kv_append(k, v, cache, p["table"].cuda(), R.offsets(p["new"]).cuda(), torch.tensor(p["lens"], dtype=torch.int32).cuda(), q=q if with_q else None,
                             inv_freq=None if p["f"] is None else p["f"].cuda(), interleaved=interleaved, q_out=q if q_out == "in place" else q_out, dev_status=status, stream=stream)
    torch.cuda.synchronize()
    return out, cache


def check(p, out, cache, interleaved):
    q, blocks = expected(p, interleaved)
    rows = q.shape[0]
    if out is not None:
        # cos and sin to 2^-23 each, two products and a sum in fp32, then half a step of the type
        half = torch.finfo(out.dtype).eps / 2
        rot = 2.0 ** -21 * p["q"][:rows].double().abs().amax(-1, keepdim=True) * math.sqrt(2) if p["f"] is not None else 0.0
        err = (out[:rows].cpu().double() - q).abs()
        assert bool((err <= half * q.abs() + rot * (1 + half)).all()), float((err - half * q.abs()).max())
    got = {"k": cache.k.view(torch.uint8).cpu(), "v": cache.v.view(torch.uint8).cpu()}
    scales = {"k": cache.k_scale.cpu(), "v": cache.v_scale.cpu()}
    want_codes = {"k": p["pool"].k.clone(), "v": p["pool"].v.clone()}
    touched = {"k": torch.zeros(p["pool"].k.shape[:3], dtype=torch.bool), "v": torch.zeros(p["pool"].k.shape[:3], dtype=torch.bool)}
    marked = {w: torch.zeros(p["pool"].k_scale.shape, dtype=torch.bool) for w in "kv"}
    for which, i, h, r0, n, val, scale, older in blocks:
        assert float(scales[which][i, h]) == scale, (which, i, h, float(scales[which][i, h]), scale)
        if older is not None:
            assert torch.equal(got[which][i, h, :r0], older), (which, i, h)
        x = R.decode(got[which][i, h, r0:r0 + n]) * scale
        rot = 2.0 ** -21 * val.abs().nan_to_num(0, 0, 0).amax(-1, keepdim=True) * math.sqrt(2) if which == "k" and p["f"] is not None else 0.0
        ok = (x - val).abs() <= torch.maximum(2.0 ** -4 * val.abs(), torch.tensor(2.0 ** -10 * scale)) + rot * (1 + 2.0 ** -4)
        assert bool(ok[val.isfinite()].all()), (which, i, h)
        assert bool(x[val.isnan()].isnan().all()) and not bool(x[~val.isnan()].isnan().any())
        touched[which][i, h, :r0 + n] = True
        marked[which][i, h] = True
    for w, codes, scale in (("k", p["pool"].k, p["pool"].k_scale), ("v", p["pool"].v, p["pool"].v_scale)):
        assert torch.equal(got[w][~touched[w]], codes[~touched[w]]) and torch.equal(scales[w][~marked[w]], scale[~marked[w]])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,before,heads,kv_heads,dim,page,rotary,interleaved", [
    ((1,), (0,), 4, 2, 128, 64, 128, False),                             # the first token of all
    ((1, 1, 1, 1), (63, 64, 65, 200), 16, 8, 128, 64, 128, False),       # one token each: end, beginning and middle of a page
    ((5, 0, 2, 8, 1), (60, 7, 0, 15, 130), 6, 2, 64, 16, 32, True),      # drafts across pages, a sequence without new tokens
    ((100, 17, 1), (0, 33, 500), 7, 1, 128, 32, 64, True),
    ((333, 9), (5, 120), 12, 4, 64, 128, 64, False),                     # pages of 128, a piece just over a warp's tokens
    ((300,), (0,), 3, 3, 128, 128, 16, False),
    ((1025, 64, 700), (0, 64, 1), 10, 10, 128, 64, 128, False),          # more rows than the one-row runs take; more heads than a CTA
    ((2, 3), (10, 11), 1, 1, 64, 16, 0, False),                          # no rotation
])
def test_against_64_bits(dtype, new, before, heads, kv_heads, dim, page, rotary, interleaved):
    p = problem(hash((new, heads)) % 1000, new, before, heads, kv_heads, dim, page, dtype, rotary)
    out, cache = run(p, interleaved)
    check(p, out, cache, interleaved)
    again = M.KVCache(cache.k.clone(), cache.v.clone(), cache.k_scale.clone(), cache.v_scale.clone())      # the same call again changes nothing
    w = p["wide"].cuda()
    M.molora_kv_append(w[:, heads:heads + kv_heads], w[:, heads + kv_heads:], cache, p["table"].cuda(), R.offsets(new).cuda(), torch.tensor(p["lens"], dtype=torch.int32).cuda(),
                       inv_freq=None if p["f"] is None else p["f"].cuda(), interleaved=interleaved)
    assert all(torch.equal(getattr(cache, n).view(torch.uint8) if n in "kv" else getattr(cache, n), getattr(again, n).view(torch.uint8) if n in "kv" else getattr(again, n))
               for n in ("k", "v", "k_scale", "v_scale"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_without_q_and_separate_tensors(dtype):
    p = problem(5, (3, 40), (9, 70), 4, 2, 128, 64, dtype, 128, packed=False)
    out, cache = run(p, q_out="in place")
    check(p, out, cache, False)
    out, cache = run(p, with_q=False, fp8=False)
    assert out is None
    check(p, None, cache, False)


def test_far_positions():
    """Angles of a position of a million: fp32 would be off by 0.03 radians and more."""
    p = problem(6, (2,), (999_950,), 2, 1, 128, 128, "f32", 128)
    out, cache = run(p)
    check(p, out, cache, False)


def test_what_is_not_finite():
    p = problem(7, (40, 1), (0, 20), 2, 2, 64, 32, "f32", 0, packed=False)
    p["k"][3, 0, 5], p["k"][4, 0, 6], p["v"][7, 1, 0] = math.inf, math.nan, -math.inf
    p["k"][33, 1] = math.nan
    p["v"][40] = math.inf                                                # a whole block addition without one finite value
    out, cache = run(p)
    check(p, out, cache, False)
    page = p["pool"].page
    row = cache.k.view(torch.uint8)[int(p["table"][0, 3 // page]), 0, 3 % page].cpu()
    assert int(row[5]) == 0x7E                                           # saturated


@pytest.mark.parametrize("size", [0.0, 1e-30, 1e30, 3e-19, 448.0, 448.5])
def test_extreme_sizes(size):
    p = problem(8, (20,), (0,), 1, 1, 64, 16, "f32", 0, packed=False)
    p["k"] = torch.full_like(p["k"], size)
    p["v"] = torch.randn_like(p["v"]) * size
    out, cache = run(p)
    if size <= 1e20:
        check(p, out, cache, False)
    else:                                                                # beyond 448 * 2^64: saturated
        assert float(cache.k_scale.max()) == 2.0 ** 64 and bool((cache.k.view(torch.uint8)[p["table"][0, 0].long()] == 0x7E).all())


def test_growing_scale_moves_the_older_codes():
    p = problem(9, (1, 1), (30, 31), 2, 2, 128, 32, "bf16", 0, packed=False)
    p["k"] *= 2.0 ** 6
    p["v"] *= 2.0 ** 12
    before = p["pool"].k_scale.clone()
    out, cache = run(p)
    check(p, out, cache, False)
    assert bool((cache.k_scale.cpu() > before).any())


def test_rows_behind_the_last_sequence_stay():
    p = problem(10, (3, 4), (1, 2), 2, 1, 64, 16, "bf16", 64, tail=9)
    q_out = torch.full((p["N"], 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    out, cache = run(p, q_out=q_out)
    check(p, out, cache, False)
    assert bool((q_out[7:] == 7).all())


def test_bad_pages_and_lengths_are_left_out_and_reported():
    p = problem(11, (4, 4, 4), (10, 10, 10), 2, 1, 64, 16, "bf16", 64)
    good_q, good = expected(p, False)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    bad = int(p["table"][1, 0])
    p["table"][1, 0] = p["pool"].k.shape[0]                              # just outside
    out, cache = run(p, status=status)
    assert int(status) == 8
    got = cache.k.view(torch.uint8).cpu()
    assert torch.equal(got[bad], p["pool"].k[bad])                       # nothing written where it would have gone
    p["table"][1, 0] = bad
    for which, i, h, r0, n, val, scale, older in good:                   # the other sequences are as ever
        if i != bad and which == "k":
            assert float(cache.k_scale[i, h]) == scale
    for table, lens, flag in ((-1, None, 8), (None, (14, 2, 14), 8), (None, (14, 400, 14), 8), (None, (14, 14, 14), 0)):
        t = p["table"].clone()
        if table is not None:
            t[2, 0] = table
        status.zero_()
        w = p["wide"].cuda()
        cache = p["pool"].cuda(M)
        M.molora_kv_append(w[:, 2:3], w[:, 3:4], cache, t.cuda(), R.offsets(p["new"]).cuda(), torch.tensor(lens or p["lens"], dtype=torch.int32).cuda(),
                           q=w[:, :2], inv_freq=p["f"].cuda(), dev_status=status)
        torch.cuda.synchronize()
        assert int(status) == flag


def test_other_stream_and_replayed_graph():
    p = problem(12, (2, 30), (5, 40), 4, 2, 128, 64, "bf16", 128)
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        out, cache = run(p)
    check(p, out, cache, False)
    w, table, cu, lens, f = p["wide"].cuda(), p["table"].cuda(), R.offsets(p["new"]).cuda(), torch.tensor(p["lens"], dtype=torch.int32).cuda(), p["f"].cuda()
    cache = p["pool"].cuda(M)
    out = torch.zeros(32, 4, 128, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.molora_kv_append(w[:, 4:6], w[:, 6:], cache, table, cu, lens, q=w[:, :4], inv_freq=f, q_out=out)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    check(p, out, cache, False)
