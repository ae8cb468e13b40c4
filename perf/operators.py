"""What stands between the adapted projections of a serving step, as measured work: writing keys and values into the
8-bit paged cache, attention over that cache, and the verification of drafted tokens.

A case is one call of one of them.  `prepare` makes what a serving engine has in hand before the call (the step's
projections, the cache pool, page tables, lengths, the drafter's and the target's probabilities, random numbers), `run`
is the call: in its plain form, or through the package's entry points where `own` is true.

Keys of a case
  op           "append", "attend" or "verify"
  dtype        of q, k, v and the attention's result, or of the probabilities: "bf16" | "f32"
  seqs         sequences of the step
  append / attend:
    new_min, new_max   new tokens of a sequence (1, 1: decode; 2 .. 8: drafted tokens; more: a chunk of a prompt)
    len_min, len_max   tokens of a sequence in the cache before the step
    heads, kv_heads, dim, page
    lengths            seed of the lengths: they belong to the case, inputs to the seed of `prepare`
    rotary (append)    rotated leading dimensions of a head; 0: none
    interleaved (append)   pairs (2i, 2i + 1) instead of (i, i + rotary / 2)
    causal, window (attend)   window 0: all earlier keys
    lse (attend)       also the logarithm of the softmax's sum
  verify:
    drafts       drafted tokens a sequence (the most; ragged: fewer for some)
    vocab
    draft_probs  whether the drafter gives its distributions; without, its tokens count as certain
    ragged
"""
import math
import random

import torch

own = False

ROTARY_BASE = 1e6


def _append(name, seqs, new, length, heads, kv_heads, dim=128, page=64, dtype="bf16", rotary=None, interleaved=False, lengths=1):
    case = dict(op="append", dtype=dtype, seqs=seqs, new_min=new[0], new_max=new[1], len_min=length[0], len_max=length[1], heads=heads, kv_heads=kv_heads,
                dim=dim, page=page, rotary=dim if rotary is None else rotary, interleaved=interleaved, lengths=lengths)
    return dict(case, name=name) if name else case


def _attend(name, seqs, new, length, heads, kv_heads, dim=128, page=64, dtype="bf16", causal=True, window=0, lse=False, lengths=1):
    case = dict(op="attend", dtype=dtype, seqs=seqs, new_min=new[0], new_max=new[1], len_min=length[0], len_max=length[1], heads=heads, kv_heads=kv_heads,
                dim=dim, page=page, causal=causal, window=window, lse=lse, lengths=lengths)
    return dict(case, name=name) if name else case


def _verify(name, seqs, drafts, vocab, dtype="f32", draft_probs=True, ragged=False):
    case = dict(op="verify", dtype=dtype, seqs=seqs, drafts=drafts, vocab=vocab, draft_probs=draft_probs, ragged=ragged)
    return dict(case, name=name) if name else case


def listed():
    return [
        # A nearly idle server: one token of one sequence goes into the cache, between two small launches.
        _append("append-1", 1, (1, 1), (776, 776), 16, 8),
        # A full decode batch of ragged sequences, one token each, blocks half full.
        _append("append-decode-256", 256, (1, 1), (0, 700), 16, 8),
        # A prefill step of eight prompts of the wide model: whole blocks are written.
        _append("append-prefill-8192", 8, (1024, 1024), (0, 0), 32, 8),
        # A small fp32 model, ragged chunks, interleaved pairs, half of the head rotated.
        _append("append-f32-ragged", 9, (1, 333), (0, 500), 12, 4, dim=64, page=16, dtype="f32", rotary=32, interleaved=True),
        # One token of one sequence against a medium context: latency.
        _attend("attend-1", 1, (1, 1), (776, 776), 16, 8),
        # A full decode batch, contexts from a few tokens to four thousand.
        _attend("attend-decode-256", 256, (1, 1), (3, 4095), 16, 8),
        # Two users with very long contexts: the key axis has to be spread over the device.
        _attend("attend-long-2", 2, (1, 1), (100000, 131071), 32, 8, lse=True),
        # Drafted tokens under verification: five new tokens of each sequence of the wide model.
        _attend("attend-drafts-64", 64, (5, 5), (100, 2043), 32, 8),
        # A prefill step of eight prompts.
        _attend("attend-prefill-8192", 8, (1024, 1024), (0, 0), 32, 8),
        # A chunk of a long prompt against what is in the cache already.
        _attend("attend-chunk-2048", 1, (2048, 2048), (14336, 14336), 32, 8),
        # Verification at a vocabulary with image and audio tokens, the drafter's distributions given.
        _verify("verify-64", 64, 5, 160000),
        # One sequence, drafts looked up in the prompt (no distributions): latency.
        _verify("verify-1-certain", 1, 4, 32000, draft_probs=False),
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high + 0.5)))))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "verify"])
    if op == "verify":
        vocab = _log_int(rng, 1000, 160000)
        seqs = max(1, min(_log_int(rng, 1, 256), 64 * 160000 // vocab))
        return _verify(None, seqs, rng.randint(1, 5), vocab, rng.choice(["f32", "f32", "bf16"]), rng.random() < 0.7, rng.random() < 0.5)
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = min(32, kv_heads * rng.choice([1, 2, 3, 4, 7, 8]))
    heads -= heads % kv_heads
    dim, page = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    kind = rng.choice(["one", "drafts", "chunk"])
    lengths = rng.randint(0, 10 ** 6)
    if op == "append":
        seqs = _log_int(rng, 1, 256)
        new = {"one": (1, 1), "drafts": (0, rng.randint(2, 8)), "chunk": (1, _log_int(rng, 9, max(9, 8192 // seqs)))}[kind]
        rotary = rng.choice([dim, dim, dim // 2, 0])
        return _append(None, seqs, new, (0, _log_int(rng, 1, 700)), heads, kv_heads, dim, page, dtype, rotary, rng.random() < 0.3, lengths)
    if kind == "chunk":
        seqs = _log_int(rng, 1, 16)
        new = (1, _log_int(rng, 9, (256 if dtype == "f32" else 4096) // seqs))
        length = (0, _log_int(rng, 1, 4096 // seqs))
    else:
        seqs = _log_int(rng, 1, 256)
        new = (1, 1) if kind == "one" else (0, rng.randint(2, 8))
        length = (0, _log_int(rng, 1, min(65536, 256 * 2048 // seqs)))
    causal = rng.random() < 0.8
    window = _log_int(rng, 1, 4096) if causal and rng.random() < 0.25 else 0
    return _attend(None, seqs, new, length, heads, kv_heads, dim, page, dtype, causal, window, rng.random() < 0.5, lengths)


# ---------------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """(new tokens, tokens in the cache once they are in) of every sequence; they go with the case."""
    rng = random.Random(case["lengths"])
    new = [rng.randint(case["new_min"], case["new_max"]) for _ in range(case["seqs"])]
    if not any(new):
        new[0] = case["new_max"]
    return new, [n + rng.randint(case["len_min"], case["len_max"]) for n in new]


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _tables(case, new, length, gen):
    """Page table (pages of the pool in random order, as a pool in use hands them out), offsets and lengths."""
    page = case["page"]
    need = [-(-n // page) for n in length]
    total = sum(need) + 3
    order = torch.randperm(total, device="cuda", generator=gen).to(torch.int32)
    width = max(max(need), 1)
    at = torch.tensor([0] + need[:-1], device="cuda").cumsum(0)[:, None] + torch.arange(width, device="cuda")[None]
    used = torch.arange(width, device="cuda")[None] < torch.tensor(need, device="cuda")[:, None]
    table = torch.where(used, order[at.clamp(max=total - 1)], 0).to(torch.int32)
    cu = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
    return table, cu, torch.tensor(length, device="cuda", dtype=torch.int32), total


def _pool(case, pages, gen):
    """A pool in use: blocks of normal values of changing size, 8-bit codes and a scale for each block and head."""
    shape = (pages, case["kv_heads"], case["page"], case["dim"])
    x = torch.randn(shape, device="cuda", generator=gen)
    size = torch.exp2(torch.randint(-2, 3, shape[:2], device="cuda", generator=gen).float())
    amax = x.abs().amax((2, 3))
    m, e = torch.frexp(amax / 448)
    scale = torch.exp2((e - (m == 0.5).int()).float())
    codes = (x / scale[..., None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, scale * size


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = dict(case=case)
    if case["op"] == "verify":
        B, S, V = case["seqs"], case["drafts"], case["vocab"]
        z = torch.randn(B, S + 1, V, device="cuda", generator=gen) * 2.5
        st["target"] = torch.softmax(z, -1).to(_type(case))
        st["draft"] = None
        if case["draft_probs"]:
            q = torch.softmax(z[:, :S] + torch.randn(B, S, V, device="cuda", generator=gen) * 0.5, -1)
            st["draft"] = q.to(_type(case))
            drafted = torch.multinomial(q.reshape(B * S, V), 1, generator=gen).reshape(B, S)
        else:
            drafted = z[:, :S].argmax(-1)
        st["drafted"] = drafted.to(torch.int32)
        st["uniform"] = torch.rand(B, S + 1, device="cuda", generator=gen)
        st["n_drafted"] = torch.randint(0, S + 1, (B,), device="cuda", generator=gen).to(torch.int32) if case["ragged"] else None
        return st
    new, length = _lengths(case)
    st["most_new"], st["most_len"] = max(new), max(length)
    st["table"], st["cu"], st["kv_lens"], pages = _tables(case, new, length, gen)
    N, D, dt = sum(new), case["dim"], _type(case)
    st["k"], st["k_scale"] = _pool(case, pages, gen)
    st["v"], st["v_scale"] = _pool(case, pages, gen)
    # q, k and v are slices of one packed projection, as an engine has them
    wide = case["heads"] + (2 * case["kv_heads"] if case["op"] == "append" else 0)
    qkv = torch.randn(N, wide * D, device="cuda", generator=gen).to(dt).view(N, wide, D)
    st["q"] = qkv[:, :case["heads"]]
    if case["op"] == "append":
        st["new_k"] = qkv[:, case["heads"]:case["heads"] + case["kv_heads"]]
        st["new_v"] = qkv[:, case["heads"] + case["kv_heads"]:]
        r = case["rotary"]
        st["inv_freq"] = torch.pow(torch.tensor(ROTARY_BASE, dtype=torch.float64), -torch.arange(0, r, 2, dtype=torch.float64) / max(r, 1)).float().cuda() if r else None
        st["q_out"] = torch.zeros(N, case["heads"], D, device="cuda", dtype=dt)
    else:
        st["out"] = torch.zeros(N, case["heads"], D, device="cuda", dtype=dt)
        st["lse"] = torch.zeros(N, case["heads"], device="cuda") if case["lse"] else None
    return st


# ---------------------------------------------------------------------------------------------------- plain forms
def _token_places(cu, kv_lens, N):
    """(sequence, index among its new tokens, position) of every row."""
    row = torch.arange(N, device=cu.device)
    seq = torch.searchsorted(cu[1:].long().contiguous(), row, right=True)
    j = row - cu.long()[seq]
    return seq, j, kv_lens.long()[seq] - (cu[1:] - cu[:-1]).long()[seq] + j


def _rotate(x, pos, inv_freq, interleaved):
    x = x.float()
    if inv_freq is None:
        return x
    angle = pos.double()[:, None] * inv_freq.double()[None]
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    r = 2 * inv_freq.numel()
    if interleaved:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([y, x[..., r:]], -1)


def _blocks_written(codes, scale, values, st):
    """Write one of K and V: whole blocks that the step's tokens touch are read, extended and written back."""
    page, cu, kv_lens = st["case"]["page"], st["cu"].long(), st["kv_lens"].long()
    new = cu[1:] - cu[:-1]
    start = kv_lens - new
    most = -(-st["most_new"] // page) + 1
    block = start[:, None] // page + torch.arange(most, device=cu.device)[None]                # [B, most]
    touched = (block * page < kv_lens[:, None]) & (new > 0)[:, None]
    seq = torch.arange(len(new), device=cu.device)[:, None].expand_as(block)[touched]
    block = block[touched]
    ids = st["table"].long()[seq, block]
    pos = block[:, None] * page + torch.arange(page, device=cu.device)[None]                   # [T, page]
    fresh = (pos >= start[seq, None]) & (pos < kv_lens[seq, None])
    older = pos < start[seq, None]
    row = (cu[:-1][seq, None] + pos - start[seq, None]).clamp(0, values.shape[0] - 1)
    x = values[row].permute(0, 2, 1, 3)                                                        # [T, H, page, D]
    amax = (x.abs() * fresh[:, None, :, None]).amax((2, 3))
    m, e = torch.frexp(amax)                                                                   # amax = m 2^e; 448 = 0.875 * 2^9
    grown = torch.exp2((e - 9 + (m > 0.875).int()).clamp(-64, 64).float())
    grown = torch.where(amax > 0, grown, 2.0 ** -64)
    before = scale[ids]
    grown = torch.where(older.any(1)[:, None], torch.maximum(grown, before), grown)
    held = codes[ids]
    moved = held.view(torch.float8_e4m3fn).float() * (before / grown)[..., None, None]
    moved = moved.to(torch.float8_e4m3fn).view(torch.uint8)
    written = (x / grown[..., None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    codes[ids] = torch.where(fresh[:, None, :, None], written, torch.where(older[:, None, :, None], moved, held))
    scale[ids] = grown


def _append_plain(st):
    q, k = st["q"], st["new_k"]
    _, _, pos = _token_places(st["cu"], st["kv_lens"], q.shape[0])
    st["q_out"].copy_(_rotate(q, pos, st["inv_freq"], st["case"]["interleaved"]))
    _blocks_written(st["k"], st["k_scale"], _rotate(k, pos, st["inv_freq"], st["case"]["interleaved"]), st)
    _blocks_written(st["v"], st["v_scale"], st["new_v"].float(), st)


def _gathered(codes, scale, table, width):
    """[B, H, width * page, D] of the sequences' blocks."""
    ids = table[:, :width].long()
    x = codes[ids].view(torch.float8_e4m3fn).float() * scale[ids][..., None, None]
    B, W, H, page, D = x.shape
    return x.transpose(1, 2).reshape(B, H, W * page, D)


def _attend_plain(st):
    case, q, cu, kv_lens = st["case"], st["q"], st["cu"].long(), st["kv_lens"].long()
    N, H, D = q.shape
    Hk, G, T, width = case["kv_heads"], H // case["kv_heads"], st["most_new"], -(-st["most_len"] // case["page"])
    K, V = _gathered(st["k"], st["k_scale"], st["table"], width), _gathered(st["v"], st["v_scale"], st["table"], width)
    new = cu[1:] - cu[:-1]
    j = torch.arange(T, device=q.device)
    rows = (cu[:-1, None] + j[None]).clamp(max=N - 1)
    Q = q[rows].float().view(-1, T, Hk, G, D).permute(0, 2, 1, 3, 4).reshape(-1, Hk, T * G, D)
    s = Q @ K.transpose(2, 3)
    s *= D ** -0.5
    key = torch.arange(K.shape[2], device=q.device)
    pos = (kv_lens - new)[:, None] + j[None]                                                    # [B, T]
    seen = (key[None, None] < kv_lens[:, None, None]).expand(-1, T, -1)
    if case["causal"]:
        seen = seen & (key[None, None] <= pos[..., None])
    if case["window"]:
        seen = seen & (key[None, None] > pos[..., None] - case["window"])
    s.view(-1, Hk, T, G, K.shape[2]).masked_fill_(~seen[:, None, :, None], -math.inf)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    s -= m
    p = s.exp_()
    total = p.sum(-1, keepdim=True)
    o = (p @ V) / torch.where(total > 0, total, 1.0)
    seq, jj, _ = _token_places(st["cu"], st["kv_lens"], N)
    o = o.view(-1, Hk, T, G, D)[seq, :, jj]
    st["out"].copy_(o.reshape(N, H, D))
    if st["lse"] is not None:
        st["lse"].copy_((m + total.log()).view(-1, Hk, T, G)[seq, :, jj].reshape(N, H))


def _verify_plain(target, draft, drafted, uniform, n_drafted):
    B, S = drafted.shape
    x = drafted.long()[..., None]
    n = torch.full((B,), S, device=x.device) if n_drafted is None else n_drafted.long()
    p_x = target[:, :S].gather(2, x)[..., 0].double()
    q_x = torch.ones_like(p_x) if draft is None else draft.gather(2, x)[..., 0].double()
    ok = (uniform[:, :S].double() * q_x < p_x) & (torch.arange(S, device=x.device)[None] < n[:, None])
    accepted = ok.long().cumprod(1).sum(1)
    b = torch.arange(B, device=x.device)
    p = target[b, accepted].double()
    at = accepted.clamp(max=max(S - 1, 0))
    if draft is None:
        q = torch.zeros_like(p).scatter_(1, x[b, at], math.inf)
    else:
        q = draft[b, at].double()
    left = torch.where((accepted < n)[:, None], (p - q).clamp(min=0), p)
    left = torch.where(left.sum(1, keepdim=True) > 0, left, p)
    cum = left.cumsum(1)
    token = (cum > uniform[:, S:].double() * cum[:, -1:]).long().argmax(1)
    out = torch.where(torch.arange(S + 1, device=x.device)[None] < accepted[:, None], torch.cat([x[..., 0], x[:, :1, 0]], 1), -1)
    out.scatter_(1, accepted[:, None], token[:, None])
    return out.to(torch.int32), accepted.to(torch.int32)


def run(st):
    case = st["case"]
    if case["op"] == "verify":
        if own:
            import paper_2603_15965_b200 as molora
            tokens, accepted = molora.molora_verify_drafts(st["target"], st["draft"], st["drafted"], st["uniform"], n_drafted=st["n_drafted"])
        else:
            tokens, accepted = _verify_plain(st["target"], st["draft"], st["drafted"], st["uniform"], st["n_drafted"])
        return {"tokens": tokens, "accepted": accepted}
    if case["op"] == "append":
        if own:
            import paper_2603_15965_b200 as molora
            cache = molora.KVCache(st["k"], st["v"], st["k_scale"], st["v_scale"])
            molora.molora_kv_append(st["new_k"], st["new_v"], cache, st["table"], st["cu"], st["kv_lens"], q=st["q"], inv_freq=st["inv_freq"],
                                    interleaved=case["interleaved"], q_out=st["q_out"])
        else:
            _append_plain(st)
        return {"q": st["q_out"], "k": st["k"].view(torch.float8_e4m3fn), "v": st["v"].view(torch.float8_e4m3fn), "k_scale": st["k_scale"], "v_scale": st["v_scale"]}
    if own:
        import paper_2603_15965_b200 as molora
        cache = molora.KVCache(st["k"], st["v"], st["k_scale"], st["v_scale"])
        molora.molora_kv_attend(st["q"], cache, st["table"], st["cu"], st["kv_lens"], causal=case["causal"], window=case["window"], max_tokens=st["most_new"],
                                out=st["out"], lse=st["lse"])
    else:
        _attend_plain(st)
    return {"out": st["out"]} if st["lse"] is None else {"out": st["out"], "lse": st["lse"]}


# ---------------------------------------------------------------------------------------------------- from the definition, in 64 bits
def _exact_attend(case, st):
    new, length = _lengths(case)
    H, Hk, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    if sum(n * l for n, l in zip(new, length)) * H > 4e9:
        return None
    outs, lses, at = [], [], 0
    for b, (n, l) in enumerate(zip(new, length)):
        if n == 0:
            continue
        ids = st["table"][b, :-(-l // page)].long()
        k = (st["k"][ids].view(torch.float8_e4m3fn).double() * st["k_scale"][ids].double()[..., None, None]).transpose(0, 1).reshape(Hk, -1, D)[:, :l]
        v = (st["v"][ids].view(torch.float8_e4m3fn).double() * st["v_scale"][ids].double()[..., None, None]).transpose(0, 1).reshape(Hk, -1, D)[:, :l]
        q = st["q"][at:at + n].double()
        i, t = torch.arange(l - n, l, device=q.device)[:, None], torch.arange(l, device=q.device)[None]
        hidden = torch.zeros(n, l, dtype=torch.bool, device=q.device)
        if case["causal"]:
            hidden |= t > i
        if case["window"]:
            hidden |= t <= i - case["window"]
        o, z = [], []
        for h in range(H):
            w = torch.einsum("nd,ld->nl", q[:, h], k[h * Hk // H]) / math.sqrt(D)
            w[hidden] = -math.inf
            z.append(torch.logsumexp(w, 1))
            o.append(torch.exp(w - z[-1][:, None]) @ v[h * Hk // H])
        outs.append(torch.stack(o, 1))
        lses.append(torch.stack(z, 1))
        at += n
    out = {"out": torch.cat(outs)}
    if case["lse"]:
        out["lse"] = torch.cat(lses)
    return out


def _turned(x, positions, case):
    """The rotation as a product of complex numbers."""
    r, x = case["rotary"], x.double()
    if r == 0:
        return x
    freq = torch.pow(torch.tensor(ROTARY_BASE, dtype=torch.float64), -torch.arange(0, r, 2, dtype=torch.float64) / r).float().double().to(x.device)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=x.device), torch.outer(positions.double(), freq))[:, None]
    y = x.clone()
    if case["interleaved"]:
        z = torch.complex(x[..., 0:r:2], x[..., 1:r:2]) * turn
        y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
    else:
        z = torch.complex(x[..., :r // 2], x[..., r // 2:r]) * turn
        y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
    return y


def _two_to(e):
    """2^e for whole e, exactly."""
    return torch.ldexp(torch.ones_like(e), e.int())


def _nearest_code_value(x):
    """The e4m3 value next to x (64 bits, |x| <= 448), ties to the even mantissa."""
    a = x.abs()
    e = torch.floor(torch.log2(a.clamp(min=2.0 ** -6)))
    e = torch.where(_two_to(e) > a.clamp(min=2.0 ** -6), e - 1, e)
    step = _two_to(e - 3)
    return torch.copysign(torch.round(a / step) * step, x)


def _exact_append(case, st):
    new, length = _lengths(case)
    page = case["page"]
    positions = torch.cat([torch.arange(l - n, l) for n, l in zip(new, length)]).to(st["q"].device)
    out = {"q": _turned(st["q"], positions, case)}
    for name, x in (("k", _turned(st["new_k"], positions, case)), ("v", st["new_v"].double())):
        values = st[name].view(torch.float8_e4m3fn).double()
        scales = st[name + "_scale"].double()
        at = 0
        for b, (n, l) in enumerate(zip(new, length)):
            for first in range((l - n) // page * page, l if n else 0, page):
                i = int(st["table"][b, first // page])
                lo, hi = max(first, l - n), min(first + page, l)
                block = x[at + lo - (l - n):at + hi - (l - n)].transpose(0, 1)                    # [H, tokens, D]
                top = block.abs().amax((1, 2)) / 448
                e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -64)))
                e = torch.where(_two_to(e - 1) >= top, e - 1, e)
                e = torch.where(_two_to(e) < top, e + 1, e).clamp(-64, 64)
                if lo > first:
                    e = torch.maximum(e, torch.round(torch.log2(scales[i])))
                    values[i, :, :lo - first] = _nearest_code_value(values[i, :, :lo - first] * (scales[i] * _two_to(-e))[:, None, None])
                values[i, :, lo - first:hi - first] = _nearest_code_value((block * _two_to(-e)[:, None, None]).clamp(-448, 448))
                scales[i] = _two_to(e)
            at += n
        out[name], out[name + "_scale"] = values, scales
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(case, st)
    if case["op"] == "append":
        return _exact_append(case, st)
    return None          # whole numbers


def work(case):
    if case["op"] == "verify":
        size = 4 if case["dtype"] == "f32" else 2
        B, S, V = case["seqs"], case["drafts"], case["vocab"]
        # one row of the target's probabilities per sequence, whatever is accepted; random numbers, drafts and their probabilities; the answer
        return {"bytes": B * (V * size + (S + 1) * 4 + S * (4 + size * (2 if case["draft_probs"] else 1)) + (S + 2) * 4), "flops": B * V}
    new, length = _lengths(case)
    size = 4 if case["dtype"] == "f32" else 2
    H, Hk, D, page, N = case["heads"], case["kv_heads"], case["dim"], case["page"], sum(new)
    if case["op"] == "append":
        blocks = sum(-(-l // page) - (l - n) // page for n, l in zip(new, length) if n)
        return {"bytes": N * D * (size * (2 * H + 2 * Hk) + 2 * Hk) + blocks * Hk * 8, "flops": N * (H + Hk) * case["rotary"] * 3}
    keys, pairs = 0, 0
    for n, l in zip(new, length):
        if n == 0:
            continue
        w = case["window"] or l + n
        keys += min(l, n - 1 + w)
        if case["causal"]:
            full = max(0, min(n, l - w + 1 if case["window"] else 0))          # rows whose window is full: the last ones
            pairs += full * w + sum(range(l - n + 1, l - full + 1))
        else:
            pairs += n * l
    return {"bytes": 2 * N * H * D * size + 2 * keys * Hk * D + -(-keys // page) * Hk * 8 + (N * H * 4 if case["lse"] else 0), "flops": 4 * pairs * H * D}
