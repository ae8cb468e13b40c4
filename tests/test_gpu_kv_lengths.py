"""Lengths that do not fit the page table, and rows that do not fit the call: what is left out is left out, and nothing else moves.  Every token keeps
the position that its sequence's length gives it."""
import pytest
import torch

import _kv_reference as R
import paper_2603_15965_b200 as M
import test_gpu_kv_append as A
import test_gpu_kv_attend as T

pytestmark = pytest.mark.gpu

PAGE, WIDTH = 16, 3
ROOM = PAGE * WIDTH


def _append(p, cu, lens, status, q_out):
    w = p["wide"].cuda()
    h, hk = p["heads"], p["kv_heads"]
    cache = p["pool"].cuda(M)
    M.molora_kv_append(w[:, h:h + hk], w[:, h + hk:], cache, p["table"].cuda(), torch.tensor(cu, dtype=torch.int32).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(),
                       q=w[:, :h], inv_freq=p["f"].cuda(), q_out=q_out, dev_status=status)
    torch.cuda.synchronize()
    return cache


def _rows(cu, lens, N):
    """(row, sequence, position) of the tokens that the call has."""
    return [(i, b, lens[b] - cu[b + 1] + i) for b in range(len(lens)) for i in range(max(0, cu[b]), min(N, cu[b + 1]))]


# cu_tokens (of sequences of at most 8 new tokens), kv_lens
CALLS = [
    ((0, 1, 2), (ROOM, ROOM + 1)),                                       # one token just inside, one just behind the table
    ((0, 8, 16), (ROOM + 3, 30)),                                        # five inside, three behind
    ((0, 8, 16), (ROOM + 8, ROOM + 1000)),                               # none inside
    ((0, 8, 16), (30, 2 ** 31 - 1)),
    ((0, 8, 16), (2 ** 30 + 4, 20)),
    ((0, 8, 19), (40, 40)),                                              # three rows that the call does not have
    ((-3, 8, 16), (40, 20)),
    ((0, 8, 16), (ROOM + 20, 5)),                                        # behind the table; the other in front of its beginning
    ((0, 8, 16), (-4, 20)),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cu,lens", CALLS)
def test_append_moves_no_token(cu, lens, dtype):
    N = min(16, cu[-1])
    p = A.problem(100, (N,), (0,), 2, 2, 64, PAGE, dtype, 64)
    gen = torch.Generator().manual_seed(7)
    p["table"], pages = R.tables([ROOM, ROOM], PAGE, gen)
    p["pool"] = R.Pool(pages, 2, PAGE, 64, gen)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q_out = torch.full((N, 2, 64), 7.0, dtype=p["q"].dtype, device="cuda")
    cache = _append(p, cu, lens, status, q_out)
    assert int(status) == 8
    # what the call has to leave, piece by piece, as if every sequence's tokens inside the table were a call of their own
    rows = _rows(cu, lens, N)
    got = {"k": cache.k.view(torch.uint8).cpu(), "v": cache.v.view(torch.uint8).cpu()}
    scales = {"k": cache.k_scale.cpu(), "v": cache.v_scale.cpu()}
    want, kept = {"k": p["pool"].k.clone(), "v": p["pool"].v.clone()}, {"k": p["pool"].k_scale.clone(), "v": p["pool"].v_scale.clone()}
    pos = torch.tensor([r[2] for r in rows])
    x = {"q": p["q"], "k": p["k"], "v": p["v"]}
    turned = {n: (R.rotate(x[n].double()[[r[0] for r in rows]], pos, p["f"], False) if n != "v" else x[n].double()[[r[0] for r in rows]]) for n in x}
    slack = {n: 2.0 ** -21 * turned[n].abs().amax(-1, keepdim=True) * 2 for n in x}       # as in the tests of the rotation
    written = {n: torch.zeros(p["pool"].k.shape[:3], dtype=torch.bool) for n in "kv"}
    for b in range(2):
        inside = [i for i, r in enumerate(rows) if r[1] == b and 0 <= r[2] < ROOM]
        for block in sorted({rows[i][2] // PAGE for i in inside}):
            mine = [i for i in inside if rows[i][2] // PAGE == block]
            page, first = int(p["table"][b, block]), rows[mine[0]][2] % PAGE
            for n in "kv":
                for h in range(2):
                    val = turned[n][mine, h]
                    scale = R.scale_for(float(val.abs().max()))
                    if first > 0:
                        old = float(kept[n][page, h])
                        scale = max(scale, old)
                        older = R.encode(R.decode(want[n][page, h, :first]) * (old / scale)) if scale > old else want[n][page, h, :first]
                        assert torch.equal(got[n][page, h, :first], older)
                    assert float(scales[n][page, h]) == scale
                    err = (R.decode(got[n][page, h, first:first + len(mine)]) * scale - val).abs()
                    room = slack[n][mine, h] if n == "k" else 0.0
                    assert bool((err <= torch.maximum(2.0 ** -4 * val.abs(), torch.tensor(2.0 ** -10 * scale)) + room * (1 + 2.0 ** -4)).all())
                    written[n][page, h, :first + len(mine)] = True
                    kept[n][page, h] = scale
    for n in "kv":                                                       # nothing else has changed
        assert torch.equal(got[n][~written[n]], want[n][~written[n]]) and torch.equal(scales[n], kept[n])
    # q is rotated by the position that the length gives, wherever the token's page is; tokens in front of the beginning are left as they are
    half = torch.finfo(p["q"].dtype).eps / 2
    for i, (row, b, at) in enumerate(rows):
        if at < 0:
            assert bool((q_out[row] == 7).all())
        elif at < 2 ** 24:
            err = (q_out[row].cpu().double() - turned["q"][i]).abs()
            assert bool((err <= half * turned["q"][i].abs() + slack["q"][i] * (1 + half)).all())


@pytest.mark.parametrize("dim,dtype,heads,kv_heads", [(128, "bf16", 4, 2), (128, "bf16", 24, 1), (64, "bf16", 4, 2), (64, "f32", 8, 2), (128, "f32", 4, 2)])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 12), (False, 0)])
@pytest.mark.parametrize("cu,lens", CALLS + [((0, 40, 56), (ROOM + 21, ROOM + 9)), ((0, 40, 70), (60, 40))])
def test_attention_moves_no_token(cu, lens, causal, window, dim, dtype, heads, kv_heads):
    _attention(cu, lens, causal, window, dim, dtype, heads, kv_heads, min(cu[-1], 56 if cu[1] == 40 else 16))


@pytest.mark.parametrize("causal,window", [(True, 0), (True, 12), (False, 0)])
@pytest.mark.parametrize("cu,lens", [((0, 700, 1290), (ROOM + 600, ROOM + 9)), ((0, 700, 1400), (ROOM - 5, ROOM + 300)), ((-30, 700, 1290), (2 ** 31 - 1, ROOM + 1))])
def test_attention_of_prompts_moves_no_token(cu, lens, causal, window):
    """More units of 32 rows than the kernel for few rows is given."""
    _attention(cu, lens, causal, window, 128, "bf16", 16, 8, 1290)


def _attention(cu, lens, causal, window, dim, dtype, heads, kv_heads, N):
    gen = torch.Generator().manual_seed(8)
    table, pages = R.tables([ROOM, ROOM], PAGE, gen)
    pool = R.Pool(pages, kv_heads, PAGE, dim, gen)
    q = torch.randn(N, heads, dim, generator=gen).to(T.TYPES[dtype])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lse = torch.full((N, heads), 7.0, device="cuda")
    out = M.molora_kv_attend(q.cuda(), pool.cuda(M), table.cuda(), torch.tensor(cu, dtype=torch.int32).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), causal=causal,
                             window=window, lse=lse, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 8
    # row by row: a call of one token whose cache ends with what the row sees
    for row, b, at in _rows(cu, lens, N):
        readable = max(0, min(lens[b], ROOM))
        seen = min(max(at + 1, 0), readable) if causal else readable
        left = window - max(0, at + 1 - seen) if window else 0           # of the window, in front of the last readable key
        if seen == 0 or (window and left <= 0):
            assert bool((out[row] == 0).all()) and bool((lse[row] == -float("inf")).all()), (row, b, at)
            continue
        p = dict(q=q[row:row + 1], pool=pool, table=table[b:b + 1], new=(1,), lens=(seen,))
        T.check(p, out[row:row + 1], lse[row:row + 1], causal=True, window=left)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("front", [1, 3, 40])
@pytest.mark.parametrize("new", [(1, 1, 1), (5, 0, 30), (70, 2, 9)])
def test_rows_in_front_of_the_first_sequence(front, new, dtype):
    """A call whose first sequence does not begin with row 0 leaves what the same rows leave as a call of their own."""
    n = sum(new)
    p = A.problem(160, new, (10, 0, 25), 4, 2, 64, PAGE, dtype, 64)
    f, table, lens = p["f"].cuda(), p["table"].cuda(), torch.tensor(p["lens"], dtype=torch.int32).cuda()
    rows = torch.cat([torch.randn(front, 8, 64).to(p["wide"].dtype), p["wide"]]).cuda()
    results = []
    for at, w in ((0, rows[front:].contiguous()), (front, rows)):
        cache, status = p["pool"].cuda(M), torch.zeros(1, dtype=torch.int32, device="cuda")
        cu = (R.offsets(new) + at).cuda()
        q = torch.full((at + n, 4, 64), 7.0, dtype=rows.dtype, device="cuda")
        M.molora_kv_append(w[:, 4:6], w[:, 6:], cache, table, cu, lens, q=w[:, :4], inv_freq=f, q_out=q, dev_status=status)
        out, lse = torch.full_like(q, 7.0), torch.full((at + n, 4), 7.0, device="cuda")
        M.molora_kv_attend(q, cache, table, cu, lens, max_tokens=max(new), out=out, lse=lse, dev_status=status)
        torch.cuda.synchronize()
        assert int(status) == 0 and all(bool((t[:at] == 7).all()) for t in (q, out, lse))
        results.append([q[at:], out[at:], lse[at:], cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scale, cache.v_scale])
    for a, b in zip(*results):
        assert torch.equal(a, b)
