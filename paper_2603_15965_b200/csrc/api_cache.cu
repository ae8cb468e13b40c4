// C ABI of the paged cache and of draft verification: argument validation on the host, then enqueue.
#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <utility>

#include "kv_cache.cuh"

using namespace molora;

namespace {

constexpr int32_t kMaxHeads = 1024;

// MOLORA_OK, or why cache and sequences are refused
molora_status_t check_cache(const molora_kv_cache_t* c, const molora_sequences_t* s, molora_dtype_t dt, int64_t N)
{
    if (c == nullptr || s == nullptr || N < 0 || s->B < 0 || s->max_pages < 0 || c->n_pages < 0 || c->kv_heads < 1) return MOLORA_ERR_INVALID_ARG;
    if (N >= INT32_MAX || (dt != MOLORA_F32 && dt != MOLORA_BF16) || c->kv_heads > kMaxHeads) return MOLORA_ERR_UNSUPPORTED;
    if (c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) return MOLORA_ERR_UNSUPPORTED;
    if (c->dim != 64 && c->dim != 128) return MOLORA_ERR_UNSUPPORTED;
    if ((int64_t)c->n_pages * c->kv_heads * c->page > INT32_MAX) return MOLORA_ERR_UNSUPPORTED;       // lines of the pool (of 64 bytes or more each)
    if (N == 0 || s->B == 0) return MOLORA_OK;
    if (s->cu_tokens == nullptr || s->kv_lens == nullptr || (s->max_pages > 0 && s->page_table == nullptr)) return MOLORA_ERR_INVALID_ARG;
    if (s->B > 1 && s->ld_table < s->max_pages) return MOLORA_ERR_INVALID_ARG;
    if (c->n_pages > 0 && (c->k == nullptr || c->v == nullptr || c->k_scale == nullptr || c->v_scale == nullptr)) return MOLORA_ERR_INVALID_ARG;
    if (!aligned16(c->k) || !aligned16(c->v)) return MOLORA_ERR_INVALID_ARG;
    return MOLORA_OK;
}

molora_status_t check_rows(const void* p, int64_t ld, int64_t width)
{
    if (p == nullptr || !aligned16(p) || ld < width) return MOLORA_ERR_INVALID_ARG;
    return ld % 8 == 0 ? MOLORA_OK : MOLORA_ERR_UNSUPPORTED;
}

// Whether N rows of width_a bytes from pa on, lda bytes apart, share a byte with N rows of width_b bytes from pb on (pitches of at least the widths).
bool rows_overlap(const void* pa, int64_t lda, int64_t width_a, const void* pb, int64_t ldb, int64_t width_b, int64_t N)
{
    const int64_t a = (int64_t)reinterpret_cast<intptr_t>(pa), b = (int64_t)reinterpret_cast<intptr_t>(pb);
    if (a + (N - 1) * lda + width_a <= b || b + (N - 1) * ldb + width_b <= a) return false;
    if (N == 1) return true;
    if (lda == ldb) {                                 // slices of one buffer: row j of b begins r bytes behind the beginning of row j + k of a
        const int64_t k = (b - a >= 0 ? b - a : b - a - lda + 1) / lda, r = b - a - k * lda;
        return (r < width_a && std::abs(k) < N) || (r + width_b > lda && std::abs(k + 1) < N);
    }
    for (int64_t i = 0; i < N; ++i) {                 // the first row of b that ends behind the beginning of a's row i
        const int64_t at = a + i * lda, j = at < b + width_b ? 0 : (at - b - width_b) / ldb + 1;
        if (j < N && b + j * ldb < at + width_a) return true;
    }
    return false;
}

KvView view_of(const molora_kv_cache_t& c, const molora_sequences_t& s)
{
    KvView v;
    v.k = static_cast<uint8_t*>(c.k);
    v.v = static_cast<uint8_t*>(c.v);
    v.k_scale = c.k_scale;
    v.v_scale = c.v_scale;
    v.n_pages = c.n_pages, v.kv_heads = c.kv_heads, v.dim = c.dim;
    v.page_log2 = c.page == 16 ? 4 : c.page == 32 ? 5 : c.page == 64 ? 6 : 7;
    v.table = s.page_table, v.ld_table = s.ld_table;
    v.cu = s.cu_tokens, v.kv_lens = s.kv_lens;
    v.B = s.B, v.max_pages = s.max_pages;
    return v;
}

// rows of the longest sequence, per key / value head; what is beyond 2^31 tokens is no call's
int64_t rows_of(int64_t max_tokens, int32_t group) { return std::min(max_tokens, (int64_t)INT32_MAX) * group; }

// Whether bf16 rows with heads of 128 go to the kernel for few rows, in units of 32: always up to that, and for more where its units find a worker
// each and read few keys over again -- two units a sequence, or no more than four tiles of 128 keys a worker if every page of the table is in use.
// (16 new tokens of one sequence, 4 heads a key / value head, behind 20,000: 36 us against 47; 40 behind 460: 19 against 28; 16 of each of 16
// sequences, 384 units: 44 both; 32 of each, 640 units: 73 against 46.)  The lengths are on the device, so what stands for them is the width of
// the page table: calls of more than 2 kMaxStreamRows rows with a table much wider than their sequences go to the other kernel.
bool few_rows(int64_t rows, int64_t N, int32_t group, const molora_kv_cache_t& c, const molora_sequences_t& s)
{
    if (rows <= kMaxStreamRows) return true;
    const int64_t units = c.kv_heads * (s.B + N * group / kMaxStreamRows), workers = 2 * sm_count();
    const int64_t tiles = ((int64_t)s.max_pages * c.page + 127) / 128;
    return units <= workers && (rows <= 2 * kMaxStreamRows || units * tiles <= 4 * workers);
}

}  // namespace

extern "C" {

molora_status_t molora_kv_append(const molora_kv_cache_t* cache, const molora_sequences_t* seqs, molora_dtype_t dt, int64_t N, const void* k,
                                 int64_t ldk, const void* v, int64_t ldv, const void* q, int64_t ldq, void* q_out, int64_t ldqo,
                                 int32_t heads, const float* inv_freq, int32_t rotary, int32_t interleaved, uint32_t* dev_status,
                                 void* stream)
{
    if (const molora_status_t st = check_cache(cache, seqs, dt, N)) return st;
    if (heads < 0 || rotary < 0 || rotary > cache->dim) return MOLORA_ERR_INVALID_ARG;
    if (heads > kMaxHeads || rotary % 16 != 0) return MOLORA_ERR_UNSUPPORTED;
    if (N == 0 || seqs->B == 0) return MOLORA_OK;
    if (rotary > 0 && inv_freq == nullptr) return MOLORA_ERR_INVALID_ARG;
    const int64_t wide = (int64_t)cache->kv_heads * cache->dim;
    if (const molora_status_t st = check_rows(k, ldk, wide)) return st;
    if (const molora_status_t st = check_rows(v, ldv, wide)) return st;
    if (heads > 0) {
        if (const molora_status_t st = check_rows(q, ldq, (int64_t)heads * cache->dim)) return st;
        if (const molora_status_t st = check_rows(q_out, ldqo, (int64_t)heads * cache->dim)) return st;
        const int64_t size = dt == MOLORA_F32 ? 4 : 2, q_bytes = (int64_t)heads * cache->dim * size;
        if (q == q_out ? ldq != ldqo && N > 1 : rows_overlap(q, ldq * size, q_bytes, q_out, ldqo * size, q_bytes, N)) return MOLORA_ERR_INVALID_ARG;
        for (const auto& [p, ld] : {std::pair<const void*, int64_t>(k, ldk), std::pair<const void*, int64_t>(v, ldv)})      // (read by other CTAs)
            if (rows_overlap(p, ld * size, wide * size, q_out, ldqo * size, q_bytes, N)) return MOLORA_ERR_INVALID_ARG;
    }
    return launch_kv_append(view_of(*cache, *seqs), dt, N, k, ldk, v, ldv, q, ldq, q_out, ldqo, heads, inv_freq, rotary, interleaved != 0, dev_status,
                            static_cast<cudaStream_t>(stream));
}

size_t molora_kv_attend_workspace_bytes(molora_dtype_t dt, int32_t heads, int32_t kv_heads, int32_t dim, int64_t max_tokens)
{
    if ((dim != 64 && dim != 128) || kv_heads < 1 || heads < 1 || heads % kv_heads != 0 || max_tokens < 1 || (dt != MOLORA_F32 && dt != MOLORA_BF16)) return 0;
    const int64_t rows = rows_of(max_tokens, heads / kv_heads);
    // Enough for fewer rows too: a call is cut down to the tokens that it has, and a workspace made for a step's most serves every step.
    if (dt != MOLORA_BF16 || dim != 128) return attend_rows_workspace_bytes(dt, dim, rows);
    // (more rows may go to either kernel, by what else the call has)
    return rows <= kMaxStreamRows ? attend_stream_workspace_bytes(rows) : std::max(attend_stream_workspace_bytes(rows), attend_tiles_workspace_bytes());
}

molora_status_t molora_kv_attend(const molora_kv_cache_t* cache, const molora_sequences_t* seqs, molora_dtype_t dt, int64_t N, const void* q,
                                 int64_t ldq, void* out, int64_t ldo, float* lse, int32_t heads, float scale, int32_t causal,
                                 int32_t window, int64_t max_tokens, void* ws, size_t ws_bytes, uint32_t* dev_status, void* stream)
{
    if (const molora_status_t st = check_cache(cache, seqs, dt, N)) return st;
    if (heads < 1 || heads % cache->kv_heads != 0 || window < 0 || max_tokens < 0 || !(scale > 0.f) || !std::isfinite(scale)) return MOLORA_ERR_INVALID_ARG;
    if (heads > kMaxHeads || (window > 0 && !causal)) return MOLORA_ERR_UNSUPPORTED;
    if (N == 0 || seqs->B == 0) return MOLORA_OK;
    if (const molora_status_t st = check_rows(q, ldq, (int64_t)heads * cache->dim)) return st;
    if (const molora_status_t st = check_rows(out, ldo, (int64_t)heads * cache->dim)) return st;
    const int64_t size = dt == MOLORA_F32 ? 4 : 2, row_bytes = (int64_t)heads * cache->dim * size;
    if (rows_overlap(q, ldq * size, row_bytes, out, ldo * size, row_bytes, N)) return MOLORA_ERR_INVALID_ARG;      // (units read rows of q after others have been written)
    if (max_tokens == 0 || max_tokens > N) max_tokens = N;
    const size_t need = molora_kv_attend_workspace_bytes(dt, heads, cache->kv_heads, cache->dim, max_tokens);
    if (need > 0 && (ws == nullptr || ws_bytes < need || (reinterpret_cast<uintptr_t>(ws) & 255u) != 0)) return MOLORA_ERR_WORKSPACE;
    AttendArgs a;
    a.c = view_of(*cache, *seqs);
    a.N = N;
    a.q = q, a.ldq = ldq, a.out = out, a.ldo = ldo, a.lse = lse;
    a.heads = heads, a.group = heads / cache->kv_heads, a.causal = causal != 0, a.window = std::min(window, kMaxTokens);
    a.scale_log2 = (float)((double)scale * 1.4426950408889634);
    a.dev_status = dev_status;
    const int64_t rows = rows_of(max_tokens, a.group);
    if (dt != MOLORA_BF16 || cache->dim != 128) return launch_attend_rows(a, dt, rows, ws, static_cast<cudaStream_t>(stream));
    if (few_rows(rows, N, a.group, *cache, *seqs)) return launch_attend_stream(a, rows, ws, static_cast<cudaStream_t>(stream));
    return launch_attend_tiles(a, ws, static_cast<cudaStream_t>(stream));
}

molora_status_t molora_verify_drafts(const void* target, int64_t target_ld_seq, int64_t target_ld, const void* draft, int64_t draft_ld_seq,
                                     int64_t draft_ld, molora_dtype_t dt, const int32_t* drafted, const int32_t* n_drafted,
                                     const float* uniform, int32_t B, int32_t S, int32_t V, int32_t* tokens, int32_t* accepted,
                                     uint32_t* dev_status, void* stream)
{
    if (B < 0 || S < 0 || V < 1) return MOLORA_ERR_INVALID_ARG;
    if ((dt != MOLORA_F32 && dt != MOLORA_BF16) || S > MOLORA_MAX_DRAFTS || V >= (1 << 30) || B > (1 << 27)) return MOLORA_ERR_UNSUPPORTED;
    if (B == 0) return MOLORA_OK;
    const uintptr_t size = dt == MOLORA_F32 ? 4 : 2;
    if (target == nullptr || uniform == nullptr || tokens == nullptr || accepted == nullptr || (S > 0 && drafted == nullptr)) return MOLORA_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(target) % size != 0 || reinterpret_cast<uintptr_t>(draft) % size != 0) return MOLORA_ERR_INVALID_ARG;
    if ((S > 0 && target_ld < V) || (B > 1 && target_ld_seq < S * target_ld + V)) return MOLORA_ERR_INVALID_ARG;
    if (draft != nullptr && S > 0 && ((S > 1 && draft_ld < V) || (B > 1 && draft_ld_seq < (S - 1) * draft_ld + V))) return MOLORA_ERR_INVALID_ARG;
    return launch_verify_drafts(target, target_ld_seq, target_ld, draft, draft_ld_seq, draft_ld, dt, drafted, n_drafted, uniform, B, S, V, tokens,
                                accepted, dev_status, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
