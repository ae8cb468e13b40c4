"""molora_kv_attend's kernel for many rows where not every row sees every key: calls of more units of 32 rows than the kernel for few rows is given.
Bounds from _kv_reference.attend."""
import math

import pytest
import torch

import _kv_reference as R
import paper_2603_15965_b200 as M
from test_gpu_kv_attend import check, problem, run

pytestmark = pytest.mark.gpu

HEADS, KV_HEADS, NEW, LENS = 16, 8, (640, 3), (900, 40)


def prompts(seed, page=64):
    return problem(seed, NEW, LENS, HEADS, KV_HEADS, 128, page, "bf16")


def put(p, which, token, head, element, code):
    """A code of sequence 0."""
    page = p["pool"].page
    getattr(p["pool"], which)[int(p["table"][0, token // page]), head, token % page, element] = code


@pytest.mark.parametrize("page", [16, 64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_codes_that_no_row_sees_leave_no_trace(page, causal):
    """NaN codes behind the sequences' ends and in foreign pages."""
    p = prompts(170, page)
    clean, z = run(p, causal=causal)
    check(p, clean, z, causal=causal)
    used = torch.zeros(p["pool"].k.shape[0], page, dtype=torch.bool)
    for b, l in enumerate(LENS):
        for j in range(l):
            used[int(p["table"][b, j // page]), j % page] = True
    for codes in (p["pool"].k, p["pool"].v):
        codes.transpose(1, 2)[~used] = 0x7F
    out, lse = run(p, causal=causal)
    assert torch.equal(out, clean) and torch.equal(lse, z)


@pytest.mark.parametrize("which", ["k", "v"])
@pytest.mark.parametrize("token", [899, 700, 517, 260, 5])
def test_a_nan_reaches_the_rows_that_see_it(which, token):
    """New tokens stand at 260 to 899; query heads 2 and 3 read key / value head 1."""
    p = prompts(171)
    clean, z = run(p)
    put(p, which, token, 1, 77, 0xFF)
    out, lse = run(p)
    sees = torch.zeros(sum(NEW), HEADS, dtype=torch.bool)
    sees[max(0, token - 260):640, 2:4] = True
    assert torch.equal(out.cpu()[~sees], clean.cpu()[~sees]) and torch.equal(lse.cpu()[~sees], z.cpu()[~sees])
    assert bool(out.cpu()[sees].isnan().any(-1).all())


@pytest.mark.parametrize("window", [1, 40, 300])
def test_window_hides_nan_in_front(window):
    p = prompts(172)
    clean, z = run(p, window=window)
    check(p, clean, z, window=window)
    first = 260 - window + 1                                             # the first key that any row of sequence 0 sees
    for token in range(max(0, first)):
        put(p, "k", token, 3, token % 128, 0x7F)
        put(p, "v", token, 3, 127 - token % 128, 0xFF)
    out, lse = run(p, window=window)
    assert torch.equal(out, clean) and torch.equal(lse, z)
    if first >= 0:
        put(p, "v", first, 3, 9, 0x7F)
        out, lse = run(p, window=window)
        assert bool(out[0, 6:8].isnan().any(-1).all()) and torch.equal(out[1:], clean[1:]) and torch.equal(out[0, :6], clean[0, :6])


@pytest.mark.parametrize("page,missing", [(16, (3, 4, 56)), (64, (0,)), (64, (5, 14)), (128, (2, 7))])
@pytest.mark.parametrize("outside", [-1, 10 ** 6])
def test_pages_outside_the_pool_are_left_out_and_reported(page, missing, outside):
    """Without a causal limit the order of the keys does not matter: what is left is the sequence without those pages."""
    p = prompts(173, page)
    whole = p["table"].clone()
    p["table"][0, list(missing)] = outside
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = run(p, causal=False, dev_status=status)
    assert int(status) == 8
    kept = [i for i in range(-(-LENS[0] // page)) if i not in missing]
    lost = sum(min(page, LENS[0] - i * page) for i in missing)
    table = whole.clone()
    table[0, :len(kept)] = whole[0, kept]
    check(dict(p, table=table, lens=(LENS[0] - lost, LENS[1])), out, lse, causal=False)


def test_more_new_tokens_than_the_cache_has():
    new, lens = (700, 5, 700), (700, 0, 650)
    p = problem(174, new, lens, HEADS, KV_HEADS, 128, 32, "bf16", tail=9)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out0 = torch.full(p["q"].shape, 7.0, dtype=torch.bfloat16, device="cuda")
    out, lse = run(p, out=out0, dev_status=status)
    assert int(status) == 8 and bool((out[1405:] == 7).all()) and bool((lse[1405:] == 7).all())
    assert bool((out[700:755] == 0).all()) and bool((lse[700:755] == -math.inf).all())
    check(dict(p, new=(700,), lens=(700,)), out[:700], lse[:700])
    check(dict(p, q=p["q"][755:1405], table=p["table"][2:], new=(650,), lens=(650,)), out[755:1405], lse[755:1405])


def test_two_graphs_share_a_workspace():
    """Prompts and a single token, captured with one workspace, replayed in turn."""
    a, b = prompts(175), problem(176, (1, 1), (900, 60), HEADS, KV_HEADS, 128, 64, "bf16")
    ws = torch.empty(M.molora_kv_attend_workspace_bytes(M.BF16, HEADS, KV_HEADS, 128, 640), dtype=torch.uint8, device="cuda")
    state = []
    for p in (a, b):
        state.append((p["q"].cuda(), p["pool"].cuda(M), p["table"].cuda(), R.offsets(p["new"]).cuda(), torch.tensor(p["lens"], dtype=torch.int32).cuda()))
        run(p)
    outs, graphs, stream = [torch.zeros_like(s[0]) for s in state], [], torch.cuda.Stream()
    torch.cuda.synchronize()
    for p, s, o in zip((a, b), state, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            M.molora_kv_attend(*s, max_tokens=max(p["new"]), out=o, ws=ws)
        graphs.append(g)
    for _ in range(3):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for p, o in zip((a, b), outs):
        check(p, o, None)
