"""What the entry points of the paged cache and of draft verification refuse on the host, before anything is enqueued (no GPU)."""
import ctypes

import pytest
import torch

import paper_2603_15965_b200 as M
from paper_2603_15965_b200.binding import _KvCacheC, _SequencesC

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
P = 0x1000                                # never dereferenced: validation fails first


def cache(**kw):
    a = dict(k=P, v=P, k_scale=P, v_scale=P, n_pages=9, kv_heads=2, page=64, dim=128)
    a.update(kw)
    return _KvCacheC(*(a[n] for n, _ in _KvCacheC._fields_))


def seqs(**kw):
    a = dict(page_table=P, ld_table=5, cu_tokens=P, kv_lens=P, B=3, max_pages=5)
    a.update(kw)
    return _SequencesC(*(a[n] for n, _ in _SequencesC._fields_))


def append(c=None, s=None, **kw):
    a = dict(dt=M.BF16, N=4, k=P, ldk=256, v=P, ldv=256, q=P, ldq=512, q_out=0x2000, ldqo=512, heads=4, inv_freq=P, rotary=128, interleaved=0)
    a.update(kw)
    return M.load_library().molora_kv_append(ctypes.byref(c or cache()), ctypes.byref(s or seqs()), *a.values(), None, None)


def attend(c=None, s=None, **kw):
    a = dict(dt=M.BF16, N=4, q=P, ldq=512, out=0x2000, ldo=512, lse=None, heads=4, scale=0.1, causal=1, window=0, max_tokens=1, ws=0x10000, ws_bytes=1 << 40)
    a.update(kw)
    return M.load_library().molora_kv_attend(ctypes.byref(c or cache()), ctypes.byref(s or seqs()), *a.values(), None, None)


def verify(**kw):
    a = dict(target=P, tls=400, tl=100, draft=P, dls=300, dl=100, dt=M.F32, drafted=P, n=None, uniform=P, B=2, S=3, V=100, tokens=P, accepted=P)
    a.update(kw)
    return M.load_library().molora_verify_drafts(*a.values(), None, None)


@pytest.fixture(autouse=True)
def nothing_enqueued():
    before = M.molora_launch_count()
    yield
    assert M.molora_launch_count() == before


@pytest.mark.parametrize("call", [append, attend])
@pytest.mark.parametrize("kw,status", [
    (dict(c=dict(page=48)), UNSUPPORTED), (dict(c=dict(page=256)), UNSUPPORTED), (dict(c=dict(dim=96)), UNSUPPORTED), (dict(c=dict(kv_heads=0)), INVALID),
    (dict(c=dict(n_pages=-1)), INVALID), (dict(c=dict(k=None)), INVALID), (dict(c=dict(v=0x1004)), INVALID), (dict(c=dict(k_scale=None)), INVALID),
    (dict(s=dict(B=-1)), INVALID), (dict(s=dict(cu_tokens=None)), INVALID), (dict(s=dict(kv_lens=None)), INVALID), (dict(s=dict(page_table=None)), INVALID),
    (dict(s=dict(ld_table=4)), INVALID), (dict(s=dict(max_pages=-1)), INVALID), (dict(N=-1), INVALID), (dict(N=2 ** 31), UNSUPPORTED), (dict(dt=7), UNSUPPORTED),
    (dict(q=None), INVALID), (dict(q=0x1008), INVALID), (dict(ldq=504), INVALID), (dict(ldq=516), UNSUPPORTED), (dict(heads=-1), INVALID),
    (dict(c=dict(kv_heads=1025)), UNSUPPORTED), (dict(c=dict(n_pages=2 ** 24)), UNSUPPORTED), (dict(c=dict(n_pages=2 ** 31 - 1, kv_heads=1024)), UNSUPPORTED),
])
def test_cache_calls(call, kw, status):
    kw = dict(kw)
    if "c" in kw:
        kw["c"] = cache(**kw["c"])
    if "s" in kw:
        kw["s"] = seqs(**kw["s"])
    assert call(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(k=None), INVALID), (dict(v=0x1002), INVALID), (dict(ldk=248), INVALID), (dict(ldv=260), UNSUPPORTED), (dict(q_out=None), INVALID), (dict(rotary=24), UNSUPPORTED),
    (dict(rotary=144), INVALID), (dict(rotary=-16), INVALID), (dict(inv_freq=None), INVALID), (dict(heads=1025), UNSUPPORTED), (dict(q_out=P, ldqo=1024), INVALID),
])
def test_append(kw, status):
    assert append(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(heads=3), INVALID), (dict(heads=0), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(window=-1), INVALID), (dict(window=5, causal=0), UNSUPPORTED), (dict(out=None), INVALID), (dict(ldo=256), INVALID),
    (dict(out=P), INVALID), (dict(max_tokens=-1), INVALID), (dict(ws=None), WORKSPACE), (dict(ws_bytes=1000), WORKSPACE), (dict(ws=0x10010), WORKSPACE),
])
def test_attend(kw, status):
    assert attend(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(B=-1), INVALID), (dict(S=-1), INVALID), (dict(S=32), UNSUPPORTED), (dict(V=0), INVALID), (dict(V=1 << 30), UNSUPPORTED), (dict(dt=3), UNSUPPORTED),
    (dict(target=None), INVALID), (dict(target=0x1002), INVALID), (dict(draft=0x1001), INVALID), (dict(drafted=None), INVALID), (dict(uniform=None), INVALID),
    (dict(tokens=None), INVALID), (dict(accepted=None), INVALID), (dict(tl=99), INVALID), (dict(tls=399), INVALID), (dict(dl=99), INVALID), (dict(dls=299), INVALID),
])
def test_verify(kw, status):
    assert verify(**kw) == status


def test_calls_without_work_are_no_calls():
    assert append(N=0) == 0 and append(s=seqs(B=0)) == 0 and attend(N=0) == 0 and attend(s=seqs(B=0)) == 0 and verify(B=0) == 0
    assert append(N=0, k=None, q=None) == 0 and attend(N=0, ws=None) == 0


def test_workspace_of_what_would_be_refused():
    assert M.molora_kv_attend_workspace_bytes(M.BF16, 4, 3, 128, 1) == 0 and M.molora_kv_attend_workspace_bytes(M.BF16, 4, 0, 128, 1) == 0
    assert M.molora_kv_attend_workspace_bytes(M.BF16, 4, 2, 96, 1) == 0 and M.molora_kv_attend_workspace_bytes(M.BF16, 4, 2, 128, 1) > 0


def test_host_tensors_are_refused():
    f, i = torch.zeros(2, 2, 128), torch.zeros(3, dtype=torch.int32)
    c = M.KVCache(torch.zeros(4, 2, 64, 128, dtype=torch.uint8), torch.zeros(4, 2, 64, 128, dtype=torch.uint8), torch.ones(4, 2), torch.ones(4, 2))
    with pytest.raises(ValueError):
        M.molora_kv_append(f, f, c, i[None], i, i[:2])
    with pytest.raises(ValueError):
        M.molora_kv_attend(f, c, i[None], i, i[:2])
    with pytest.raises(ValueError):
        M.molora_verify_drafts(f, None, i[None], f[0])
    with pytest.raises(TypeError):
        M.molora_kv_append(None, None, c, i, i, i)
