"""The operators in the order in which a serving step uses them: the adapted q / k / v projections, append with rotation, attention, the
adapted output projection; then verification of the drafts, the cache cut back to what was accepted, and the next step on top of it."""
import pytest
import torch

import _kv_reference as R
import paper_2603_15965_b200 as M

pytestmark = pytest.mark.gpu

H, HK, D, PAGE, C, RANK = 8, 2, 64, 16, 4, 16
HIDDEN = H * D


def _layer(gen):
    def w(*shape, by):
        return (torch.randn(*shape, generator=gen) * by).bfloat16().cuda()
    width = {"qkv": (H + 2 * HK) * D, "o": HIDDEN}
    return {n: (w(HIDDEN, width[n], by=HIDDEN ** -0.5), w(C, HIDDEN, RANK, by=HIDDEN ** -0.5), w(C, RANK, width[n], by=0.1)) for n in width}


def _adapted(layer, name, x, route):
    W, A, B = layer[name]
    y = x @ W
    M.molora_group_apply_batched(route, [M.ProjDesc(x, y, A, B, 1.0)])
    return y


def _step(layer, x, route, cache, table, new, lens, freq):
    qkv = _adapted(layer, "qkv", x, route).view(-1, H + 2 * HK, D)
    cu, kv = R.offsets(new).cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    q = M.molora_kv_append(qkv[:, H:H + HK], qkv[:, H + HK:], cache, table, cu, kv, q=qkv[:, :H], inv_freq=freq)
    a = M.molora_kv_attend(q, cache, table, cu, kv, max_tokens=max(new))
    return _adapted(layer, "o", a.view(-1, HIDDEN), route), q, qkv


def _dense(qkv_all, pos0, freq):
    """Attention of one sequence in 64 bits on unquantised keys and values."""
    n = qkv_all.shape[0]
    x = qkv_all.cpu().double()
    pos = torch.arange(pos0, pos0 + n)
    q, k, v = R.rotate(x[:, :H], pos, freq.cpu(), False), R.rotate(x[:, H:H + HK], pos, freq.cpu(), False), x[:, H + HK:]
    k, v = k.repeat_interleave(H // HK, 1), v.repeat_interleave(H // HK, 1)
    s = torch.einsum("nhd,lhd->hnl", q, k) * D ** -0.5
    s = s.masked_fill(torch.arange(n)[None] > torch.arange(n)[:, None], float("-inf"))
    return torch.einsum("hnl,lhd->nhd", torch.softmax(s, -1), v)


def test_prompt_then_drafts_then_cut_back():
    gen = torch.Generator().manual_seed(1)
    layer = _layer(gen)
    freq = torch.pow(torch.tensor(10000.0), -torch.arange(0, D, 2) / D).cuda()
    B, prompt = 3, (37, 1, 50)
    table, pages = R.tables([p + 40 for p in prompt], PAGE, gen)
    table = table.clamp(min=0).cuda()
    cache = M.KVCache(*(torch.full((pages, HK, PAGE, D), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2)),      # never written: NaN codes
                      *(torch.full((pages, HK), float("nan"), device="cuda") for _ in range(2)))
    lens, history = [0] * B, [[] for _ in range(B)]
    for step, new in enumerate((prompt, (4, 4, 4), (4, 4, 4), (1, 2, 4))):
        x = torch.randn(sum(new), HIDDEN, generator=gen).bfloat16().cuda()
        route = torch.randint(0, C, (sum(new),), generator=gen).to(torch.int32).cuda()
        lens = [l + n for l, n in zip(lens, new)]
        out, q, qkv = _step(layer, x, route, cache, table, new, lens, freq)
        assert out.shape == (sum(new), HIDDEN) and bool(out.isfinite().all())
        attended = M.molora_kv_attend(q, cache, table, R.offsets(new).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), max_tokens=max(new))
        at = 0
        for b, n in enumerate(new):
            history[b].append(qkv[at:at + n])
            every = torch.cat(history[b])
            assert every.shape[0] == lens[b]
            want = _dense(every, 0, freq)[-n:]
            got = attended[at:at + n].cpu().double()
            # keys and values carry half a step of e4m3 each, 2^-4 of themselves: a score is off by up to 2^-4 |q| |k| scale, taken at its
            # root mean square over D elements; values by 2^-4; 0.25 covers both at four times what they come to here
            assert float((got - want).norm() / want.norm()) < 0.25
            at += n
        if step == 0:
            continue
        # verification: five distributions per sequence, drafts partly refused; what was refused leaves the cache by its length
        S, V = max(new), 500
        target = torch.softmax(torch.randn(B, S + 1, V, generator=gen) * 2, -1).cuda()
        drafted = torch.multinomial(target[:, :S].reshape(B * S, V).cpu(), 1, generator=gen).reshape(B, S).to(torch.int32).cuda()
        draft = torch.softmax(target[:, :S].log() + 0.8 * torch.randn(B, S, V, generator=gen).cuda(), -1)
        tokens, accepted = M.molora_verify_drafts(target, draft, drafted, torch.rand(B, S + 1, generator=gen).cuda(), n_drafted=torch.tensor(new, dtype=torch.int32).cuda())
        keep = accepted.tolist()
        for b, n in enumerate(new):
            assert 0 <= keep[b] <= n and tokens[b, :keep[b]].tolist() == drafted[b, :keep[b]].tolist() and 0 <= int(tokens[b, keep[b]]) < V
            drop = n - keep[b]
            lens[b] -= drop
            history[b][-1] = history[b][-1][:n - drop]
