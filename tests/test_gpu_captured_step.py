"""A serving step with drafts captured into ONE graph: adapted q / k / v projections, append with rotation, attention, adapted output projection,
verification.  Lengths, page table, routes and activations lie in buffers at fixed addresses and change between replays; the same step run
call by call has to leave the same bits, and what the replayed attention says is compared with 64 bits."""
import pytest
import torch

import _kv_reference as R
import paper_2603_15965_b200 as M
from test_gpu_kv_attend import check

pytestmark = pytest.mark.gpu

HK, C, RANK, PAGE, SEQS, V = 2, 4, 16, 16, 3, 1000


class Step:
    """One step of a layer and the end of it, for at most `rows` new tokens, `most` of a sequence, in buffers of its own."""

    def __init__(self, heads, dim, rows, most, drafts, seed):
        gen = torch.Generator().manual_seed(seed)
        self.heads, self.dim, self.rows, self.most, self.gen = heads, dim, rows, most, gen
        hidden, wide = heads * dim, (heads + 2 * HK) * dim

        def w(*shape, by):
            return (torch.randn(*shape, generator=gen) * by).bfloat16().cuda()
        self.qkv_weights = w(C, hidden, RANK, by=hidden ** -0.5), w(C, RANK, wide, by=0.3)
        self.o_weights = w(C, hidden, RANK, by=hidden ** -0.5), w(C, RANK, hidden, by=0.3)
        self.x, self.base = w(rows, hidden, by=1.0), w(rows, wide, by=1.0)      # base: what the unadapted projection gives
        self.qkv, self.q = torch.zeros_like(self.base), torch.zeros(rows, heads, dim, dtype=torch.bfloat16, device="cuda")
        self.a, self.y = torch.zeros_like(self.q), torch.zeros_like(self.x)
        self.route = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.freq = torch.pow(torch.tensor(10000.0), -torch.arange(0, dim, 2) / dim).cuda()
        table, pages = R.tables([400] * SEQS, PAGE, gen)
        self.table, self.cu, self.lens = table.cuda(), torch.zeros(SEQS + 1, dtype=torch.int32, device="cuda"), torch.zeros(SEQS, dtype=torch.int32, device="cuda")
        self.cache = M.KVCache(*(torch.full((pages, HK, PAGE, dim), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(2)),       # never written: NaN
                               *(torch.full((pages, HK), float("nan"), device="cuda") for _ in range(2)))
        self.ws = torch.empty(M.molora_kv_attend_workspace_bytes(M.BF16, heads, HK, dim, most), dtype=torch.uint8, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.target = torch.zeros(SEQS, drafts + 1, V, device="cuda")
        self.draft, self.drafted = torch.zeros(SEQS, drafts, V, device="cuda"), torch.zeros(SEQS, drafts, dtype=torch.int32, device="cuda")
        self.n_drafted, self.uniform = torch.zeros(SEQS, dtype=torch.int32, device="cuda"), torch.zeros(SEQS, drafts + 1, device="cuda")
        self.tokens, self.accepted = torch.zeros(SEQS, drafts + 1, dtype=torch.int32, device="cuda"), torch.zeros(SEQS, dtype=torch.int32, device="cuda")

    def calls(self):
        h = self.heads
        self.qkv.copy_(self.base)
        M.molora_group_apply_batched(self.route, [M.ProjDesc(self.x, self.qkv, *self.qkv_weights, 1.0)])
        p = self.qkv.view(self.rows, h + 2 * HK, self.dim)
        M.molora_kv_append(p[:, h:h + HK], p[:, h + HK:], self.cache, self.table, self.cu, self.lens, q=p[:, :h], inv_freq=self.freq, q_out=self.q, dev_status=self.status)
        M.molora_kv_attend(self.q, self.cache, self.table, self.cu, self.lens, max_tokens=self.most, out=self.a, ws=self.ws, dev_status=self.status)
        self.y.copy_(self.x)
        M.molora_group_apply_batched(self.route, [M.ProjDesc(self.a.view(self.rows, -1), self.y, *self.o_weights, 1.0)])
        M.molora_verify_drafts(self.target, self.draft, self.drafted, self.uniform, n_drafted=self.n_drafted, tokens=self.tokens, accepted=self.accepted, dev_status=self.status)

    def fill(self, new, lens, source):
        """The inputs of a step of `new` tokens that ends at `lens`; rows behind them keep values of the step before."""
        n = sum(new)
        self.x[:n], self.base[:n] = source["x"][:n].cuda(), source["base"][:n].cuda()
        self.route[:] = -1
        self.route[:n] = source["route"][:n].cuda()
        self.cu.copy_(R.offsets(new))
        self.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        for name in ("target", "draft", "drafted", "uniform", "n_drafted"):
            getattr(self, name).copy_(source[name])
        torch.cuda.synchronize()

    def results(self):
        return dict(qkv=self.qkv, q=self.q, a=self.a, y=self.y, tokens=self.tokens, accepted=self.accepted, status=self.status, k=self.cache.k, v=self.cache.v,
                    k_scale=self.cache.k_scale.view(torch.int32), v_scale=self.cache.v_scale.view(torch.int32))


def _source(s, drafts, seed):
    gen = torch.Generator().manual_seed(seed)
    target = torch.softmax(torch.randn(SEQS, drafts + 1, V, generator=gen) * 2, -1)
    draft = torch.softmax(target[:, :drafts].log() + 0.8 * torch.randn(SEQS, drafts, V, generator=gen), -1)
    return dict(x=torch.randn(s.rows, s.heads * s.dim, generator=gen).bfloat16(), base=torch.randn(s.rows, (s.heads + 2 * HK) * s.dim, generator=gen).bfloat16(),
                route=torch.randint(-1, C, (s.rows,), generator=gen).to(torch.int32), target=target, draft=draft,
                drafted=torch.multinomial(draft.reshape(-1, V), 1, generator=gen).reshape(SEQS, drafts).to(torch.int32), uniform=torch.rand(SEQS, drafts + 1, generator=gen),
                n_drafted=torch.randint(0, drafts + 1, (SEQS,), generator=gen).to(torch.int32))


@pytest.mark.parametrize("heads,dim", [(8, 64), (8, 128)])
@pytest.mark.parametrize("rows,most,steps", [(15, 5, [(5, 5, 5), (1, 1, 1), (5, 0, 3), (2, 4, 5)]),             # drafts
                                             (96, 90, [(70, 1, 20), (3, 0, 90), (1, 1, 1), (5, 60, 5)])])      # chunks of prompts beside single tokens
def test_a_captured_step_serves_every_step(heads, dim, rows, most, steps):
    drafts = 5
    eager, replayed = Step(heads, dim, rows, most, drafts, 3), Step(heads, dim, rows, most, drafts, 3)
    warm = Step(heads, dim, rows, most, drafts, 3)                       # (first calls set up what is kept per device, which a capture must not)
    warm.calls()
    torch.cuda.synchronize()
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=stream):
        replayed.calls()
    length = [0] * SEQS
    for i, new in enumerate(steps):
        lens = [l + n for l, n in zip(length, new)]
        for s in (eager, replayed):
            s.fill(new, lens, _source(s, drafts, 50 + i))
        eager.calls()
        graph.replay()
        torch.cuda.synchronize()
        a, b = eager.results(), replayed.results()
        for name in a:
            assert torch.equal(a[name].view(torch.uint8), b[name].view(torch.uint8)), (i, name)
        assert int(replayed.status) == 0
        # the attention of the replay, from the codes that are in its cache
        pool = R.Pool(1, 1, PAGE, 64, torch.Generator().manual_seed(0))
        pool.k, pool.v, pool.k_scale, pool.v_scale = (t.cpu() for t in (replayed.cache.k, replayed.cache.v, replayed.cache.k_scale, replayed.cache.v_scale))
        used = pool.v_scale.isfinite()                                   # (the bound knows the pool by its largest scale)
        assert bool(used.any())
        pool.k_scale[~pool.k_scale.isfinite()], pool.v_scale[~used] = 0.0, 0.0
        n = sum(new)
        check(dict(q=replayed.q[:n].cpu(), pool=pool, table=replayed.table.cpu(), new=new, lens=lens), replayed.a[:n], None)
        # the cache is cut back to what stands: all of a prompt, the accepted ones of drafts
        kept = [min(k, n) if n <= drafts else n for k, n in zip(replayed.accepted.tolist(), new)]
        length = [l + k for l, k in zip(length, kept)]
