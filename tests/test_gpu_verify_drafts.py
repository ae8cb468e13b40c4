"""molora_verify_drafts on the GPU against the acceptance rule and the inverse CDF in 64 bits (exact: whole numbers)."""
import numpy as np
import pytest
import torch

import paper_2603_15965_b200 as M

pytestmark = pytest.mark.gpu


def reference(target, draft, drafted, u, n_drafted):
    B, S = drafted.shape
    tokens, accepted = np.full((B, S + 1), -1, dtype=np.int64), np.zeros(B, dtype=np.int64)
    for b in range(B):
        n, a = int(n_drafted[b]), 0
        while a < n:
            x = int(drafted[b, a])
            if not 0 <= x < target.shape[2]:
                break
            q = 1.0 if draft is None else float(draft[b, a, x])
            if not float(u[b, a]) * q < float(target[b, a, x]):
                break
            a += 1
        p = target[b, a].astype(np.float64)
        left = p
        if a < n:
            if draft is None:
                left = p.copy()
                if 0 <= drafted[b, a] < p.size:
                    left[drafted[b, a]] = 0
            else:
                left = np.maximum(p - draft[b, a].astype(np.float64), 0)
        if not left.sum() > 0:
            left = p
        cum = np.cumsum(left)
        tokens[b, :a], accepted[b] = drafted[b, :a], a
        tokens[b, a] = -1 if not cum[-1] > 0 else int(np.argmax(cum > float(u[b, S]) * cum[-1]))
    return tokens, accepted


def problem(seed, B, S, V, bf16=False, sharp=2.0, close=0.7, with_draft=True):
    gen = torch.Generator().manual_seed(seed)
    z = torch.randn(B, S + 1, V, generator=gen) * sharp
    target = torch.softmax(z, -1)
    q = torch.softmax(z[:, :S] + close * torch.randn(B, S, V, generator=gen), -1)
    drafted = torch.multinomial(q.reshape(B * S, V), 1, generator=gen).reshape(B, S).to(torch.int32) if S else torch.zeros(B, 0, dtype=torch.int32)
    if not with_draft:
        drafted = z[:, :S].argmax(-1).to(torch.int32)
    t = torch.bfloat16 if bf16 else torch.float32
    return target.to(t), q.to(t) if with_draft else None, drafted, torch.rand(B, S + 1, generator=gen)


def check(target, draft, drafted, u, n=None, **kw):
    B, S = drafted.shape
    want = reference(target.float().numpy(), None if draft is None else draft.float().numpy(), drafted.numpy(), u.numpy(), [S] * B if n is None else n.clamp(0, S).numpy())
    tokens, accepted = M.molora_verify_drafts(target.cuda(), None if draft is None else draft.cuda(), drafted.cuda(), u.cuda(), n_drafted=None if n is None else n.cuda(), **kw)
    torch.cuda.synchronize()
    assert np.array_equal(accepted.cpu().numpy(), want[1])
    assert np.array_equal(tokens.cpu().numpy(), want[0])
    return want


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("with_draft", [True, False])
@pytest.mark.parametrize("B,S,V", [(1, 1, 1), (1, 4, 7), (3, 5, 1000), (2, 2, 4096), (1, 3, 32000), (5, 4, 50257), (300, 2, 999), (2, 31, 130), (1, 1, 160000), (4, 0, 5000)])
def test_against_64_bits(B, S, V, with_draft, bf16):
    for seed in range(3):
        check(*problem(seed, B, S, V, bf16, with_draft=with_draft))


def test_ragged_drafts():
    t, q, d, u = problem(4, 40, 5, 777)
    want = check(t, q, d, u, torch.randint(0, 6, (40,), dtype=torch.int32))
    assert len(set(want[1].tolist())) > 2
    check(t, q, d, u, torch.full((40,), 99, dtype=torch.int32))          # clamped to the drafts there are
    check(t, q, d, u, torch.full((40,), -3, dtype=torch.int32))


def test_ties_zeros_and_equal_distributions():
    B, S, V = 6, 2, 10
    t = torch.zeros(B, S + 1, V)
    t[:, :, 3] = t[:, :, 7] = 0.5
    q = t[:, :S].clone()
    d = torch.full((B, S), 3, dtype=torch.int32)
    u = torch.zeros(B, S + 1)
    u[1, S], u[2, S], u[3, :S] = 0.5, 0.49999997, 0.99999994            # exactly on the border between the two tokens, just below it
    d[4] = 0                                                             # a token without probability under either: refused, and nothing is left of p - q: p
    q[5] *= 2                                                            # q above p everywhere: half of the random numbers refuse; nothing left, p again
    u[5, 0] = 0.75
    want = check(t, q, d, u)
    assert want[0][1, 2] == 7 and want[0][2, 2] == 3 and want[1][4] == 0 and want[1][5] == 0


def test_odd_pitches_rows_out_of_step_and_given_outputs():
    t, q, d, u = problem(5, 3, 3, 4001)                                  # rows begin anywhere modulo 16 bytes
    T = torch.full((3, 4, 4100), 9.0)
    T[:, :, 5:4006] = t
    Q = torch.full((3, 3, 4007), 9.0)
    Q[:, :, 3:4004] = q
    want = reference(t.numpy(), q.numpy(), d.numpy(), u.numpy(), [3] * 3)
    tokens, accepted = torch.full((3, 4), 5, dtype=torch.int32, device="cuda"), torch.full((3,), 5, dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    a, b, c, e = T.cuda()[:, :, 5:4006], Q.cuda()[:, :, 3:4004], d.cuda(), u.cuda()
    torch.cuda.synchronize()
    M.molora_verify_drafts(a, b, c, e, tokens=tokens, accepted=accepted, stream=s)
    torch.cuda.synchronize()
    assert np.array_equal(tokens.cpu().numpy(), want[0]) and np.array_equal(accepted.cpu().numpy(), want[1])


def test_bad_drafts_and_empty_distributions_are_reported():
    t, q, d, u = problem(6, 3, 2, 100)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    d[1, 0] = 100
    check(t, q, d, u, dev_status=status)
    assert int(status) == 0x10
    status.zero_()
    d[1, 0] = -1
    check(t, None, d, u, dev_status=status)
    assert int(status) == 0x10
    status.zero_()
    d[1, 0] = 1
    check(t, q, d, u, dev_status=status)
    assert int(status) == 0
    t[2] = 0
    check(t, q, d, u, dev_status=status)
    assert int(status) == 0x10


def test_frequencies_follow_the_target():
    """What comes out first is distributed as p whatever q is (the point of the rule): 40000 trials of a small vocabulary, 5 sigma."""
    B, V = 40000, 6
    gen = torch.Generator().manual_seed(0)
    p, q = torch.tensor([0.05, 0.3, 0.0, 0.25, 0.3, 0.1]), torch.tensor([0.4, 0.1, 0.1, 0.1, 0.25, 0.05])
    d = torch.multinomial(q, B, True, generator=gen).reshape(B, 1).to(torch.int32)
    tokens, _ = M.molora_verify_drafts(p.expand(B, 2, V).contiguous().cuda(), q.expand(B, 1, V).contiguous().cuda(), d.cuda(), torch.rand(B, 2, generator=gen).cuda())
    seen = torch.bincount(tokens[:, 0].cpu().long(), minlength=V).double() / B
    assert bool(((seen - p).abs() <= 5 * (p * (1 - p) / B).sqrt()).all())


def test_replayed_graph():
    t, q, d, u = problem(7, 4, 3, 9000)
    want = reference(t.numpy(), q.numpy(), d.numpy(), u.numpy(), [3] * 4)
    a = [x.cuda() for x in (t, q, d, u)]
    tokens, accepted = torch.zeros(4, 4, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        M.molora_verify_drafts(*a, tokens=tokens, accepted=accepted)
    for _ in range(3):
        tokens.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(tokens.cpu().numpy(), want[0]) and np.array_equal(accepted.cpu().numpy(), want[1])
