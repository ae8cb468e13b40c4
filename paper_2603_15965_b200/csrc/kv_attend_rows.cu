// Attention over the paged 8-bit cache for tiles of 16 query rows (molora_kv_attend): single tokens, drafted tokens, fp32.
//
// A row of a sequence is (new token, query head of the group that shares a key / value head); 16 consecutive rows, one
// key / value head and the keys that they see are a UNIT.  The units' keys, cut into steps of 16, form one long list; every warp
// of the grid takes an equal, contiguous share of it, whatever the lengths of the sequences.  A unit that lies inside one
// share is written at once; one that is cut leaves its pieces (sum, maximum, weighted values, all fp32) in the
// workspace, and a second kernel joins them in the order of the keys: results do not depend on timing.
//
// Inside a warp nothing is shared and nothing synchronised: a lane asks for exactly the 16-byte vectors of codes that its
// fragments need and waits for its own copies only (cp.async ring, kStages steps deep).
//   S = Q K^T   mma m16n8k16: lane (g, t) holds of key g the elements 16 t .. 16 t + 15 of each 64; the order of the elements in the
//               sum is free, so a 4-byte word of codes is one B fragment and Q's fragments follow the same order
//   O = P V     lane (g, t) holds of the keys 2t, 2t+1, 2t+8, 2t+9 the D / 8 elements from g D / 8 on; byte permutes pair
//               two keys of one element, and the accumulator's columns 2t, 2t+1 are then D / 4 neighbouring elements of the result
// Every e4m3 value is an fp16 value (one cvt for two); q is brought into fp16 by a power of two per row, exactly for bf16, in two
// terms of 11 bits for fp32.  The scale of a block of K multiplies its scores; that of V is added, as a logarithm, to the exponent, so
// that the weights handed to the tensor cores have the size of what they contribute, and the sum takes it off again.
// Weights are at most 2^15 (fp16 normal down to 2^-29 of a row's largest): the reference of a row moves only when a score is
// 2^8 over the weight it gave its largest, and then everything is rescaled.
// What bounds it: the codes, 2 D bytes per (key, key / value head), from HBM.
#include "kv_cache.cuh"

namespace molora {
namespace {

constexpr int kWarpsPerCta = 4, kThreads = kWarpsPerCta * 32;
constexpr int kCtasPerSm = 3;
constexpr int kStages = 4;
constexpr int kRows = 16, kStepKeys = 16;
constexpr int kMinShare = 4;                 // steps: shorter shares cost more in joining than they save
constexpr float kNone = -1e30f;              // reference of a row that has seen nothing
constexpr float kTop = 7.f;                  // weight of a row's largest score when the reference is set: 2^7

// What a cut unit leaves behind.
struct CutUnit {
    int32_t b, row_tile, head, pieces;       // pieces 0: no unit begins in this share and goes on in the next
};
__host__ __device__ constexpr int slot_floats(int dim) { return 2 * kRows + kRows * dim; }
__host__ __device__ inline size_t cut_bytes(int64_t workers) { return (size_t)((workers * (int64_t)sizeof(CutUnit) + 255) / 256 * 256); }

__device__ __forceinline__ void mma_f16(float* d, const uint32_t* a, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// the rest that fp16 leaves of two values, as fp16
__device__ __forceinline__ uint32_t pack_f16_rest(float lo, float hi, uint32_t top)
{
    const float2 t = f16x2_to_f32x2(top);
    return pack_f16(lo - t.x, hi - t.y);
}
__device__ __forceinline__ void cp_async_8(uint32_t dst, const void* src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}

// steps of every unit of a sequence, and where its keys begin
struct Span {
    int32_t lo;        // first key, a multiple of 16
    int32_t steps;     // of 16 keys, per unit
    int32_t tiles;     // row tiles
};
__device__ __forceinline__ Span span_of(const Sequence& s, int group, int window)
{
    Span r{0, 0, 0};
    if (s.n == 0) return r;
    r.lo = window > 0 ? max(0, s.first_pos() - window + 1) & ~(kStepKeys - 1) : 0;
    r.steps = max(1, (s.len - r.lo + kStepKeys - 1) / kStepKeys);
    r.tiles = (int32_t)(((int64_t)s.n * group + kRows - 1) / kRows);
    return r;
}

template <typename T>
__device__ __forceinline__ void load16(const T* p, float* x)
{
    constexpr int E = VecTraits<T>::kElems;
#pragma unroll
    for (int i = 0; i < 16 / E; ++i) unpack<T>(ld128_rw_stream(p + i * E), x + i * E);
}

template <typename T, int D>
__device__ __forceinline__ void store_run(T* p, const float* x)          // D / 4 neighbouring elements
{
    constexpr int E = VecTraits<T>::kElems;
#pragma unroll
    for (int i = 0; i < D / 4 / E; ++i) stg128(p + i * E, pack<T>(x + i * E));
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, sizeof(T) == 2 ? kCtasPerSm : 2)
    attend_rows_kernel(const __grid_constant__ AttendArgs a, CutUnit* __restrict__ cuts, float* __restrict__ slots)
{
    constexpr bool kTwo = sizeof(T) == 4;               // q and the weights in two fp16 terms
    constexpr int kTerms = kTwo ? 2 : 1;
    constexpr int HF = D / 64;                          // 64-element parts of a key
    constexpr int kVBytes = D / 8;                      // of a value, per lane
    constexpr int kStageBytes = 32 * (2 * HF * 16 + 4 * kVBytes);
    __shared__ int64_t s_upto[kThreads];                // steps of the sequences up to the end of thread i's part
    __shared__ float2 s_scales[kWarpsPerCta][kStages];
    extern __shared__ __align__(16) uint8_t ring_all[];
    ptx::grid_dependency_sync();

    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int group = a.heads / a.c.kv_heads;
    const int plog = a.c.page_log2;
    const uint32_t ring = ptx::smem_u32(ring_all) + (uint32_t)(warp * kStages * kStageBytes);

    // ---- the shares
    const int part = (a.c.B + kThreads - 1) / kThreads;
    int64_t mine = 0;
    for (int b = tid * part; b < min(a.c.B, (tid + 1) * part); ++b) {
        const Sequence sq = sequence_of(a.c, b, a.N);
        const Span sp = span_of(sq, group, a.window);
        mine += (int64_t)sp.steps * sp.tiles * a.c.kv_heads;
        if (sq.bad && blockIdx.x == 0 && a.dev_status != nullptr) atomicOr(a.dev_status, MOLORA_DEV_BAD_SEQUENCE);
    }
    s_upto[tid] = mine;
    __syncthreads();
    for (int o = 1; o < kThreads; o <<= 1) {
        const int64_t add = tid >= o ? s_upto[tid - o] : 0;
        __syncthreads();
        s_upto[tid] += add;
        __syncthreads();
    }
    const int64_t total = s_upto[kThreads - 1];
    const int64_t workers = (int64_t)gridDim.x * kWarpsPerCta, w = (int64_t)blockIdx.x * kWarpsPerCta + warp;
    const int64_t share = max((total + workers - 1) / workers, (int64_t)kMinShare);
    int64_t at = w * share;
    const int64_t stop = min(total, at + share);
    CutUnit cut{0, 0, 0, 0};
    if (at < stop) {
        // the sequence in which the share begins
        int lo = 0, hi = kThreads - 1;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (s_upto[mid] > at) hi = mid;
            else lo = mid + 1;
        }
        int b = lo * part;
        int64_t base = lo > 0 ? s_upto[lo - 1] : 0;      // first step of sequence b
        Sequence sq = sequence_of(a.c, b, a.N);
        Span sp = span_of(sq, group, a.window);
        while (at < stop) {
            while (base + (int64_t)sp.steps * sp.tiles * a.c.kv_heads <= at) {
                base += (int64_t)sp.steps * sp.tiles * a.c.kv_heads;
                sq = sequence_of(a.c, ++b, a.N);
                sp = span_of(sq, group, a.window);
            }
            const int64_t unit = (at - base) / sp.steps;
            const int64_t unit_at = base + unit * sp.steps;                 // its first step
            const int first = (int)(at - unit_at), last = (int)min((int64_t)sp.steps, stop - unit_at);
            const int head = (int)(unit % a.c.kv_heads), tile = (int)(unit / a.c.kv_heads);
            at = unit_at + last;

            // ---- the rows of the unit
            const int n_rows = (int)min((int64_t)kRows, (int64_t)sq.n * group - (int64_t)tile * kRows);
            const int64_t tile_row = (int64_t)tile * kRows;
            auto token_of = [&](int r) { return (int)((tile_row + r) / group); };
            auto upper = [&](int token) { return a.causal ? max(0, min(sq.first_pos() + token + 1, sq.len)) : sq.len; };
            auto lower = [&](int token) { return a.window > 0 ? max(0, sq.first_pos() + token - a.window + 1) : 0; };
            const int tok_lo = token_of(0), tok_hi = token_of(n_rows - 1);
            const int hi_min = upper(tok_lo), hi_max = upper(tok_hi), lo_min = lower(tok_lo), lo_max = lower(tok_hi);
            int hi_row[2], lo_row[2];
            float rowf[2], m[2] = {kNone, kNone}, l[2] = {0.f, 0.f};
            uint32_t qa[kTerms][4 * HF][4];
            int64_t out_row[2];
            int out_head[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = min(g + 8 * i, n_rows - 1);
                const int token = token_of(r);
                const int qh = head * group + (int)((tile_row + r) - (int64_t)token * group);
                hi_row[i] = upper(token), lo_row[i] = lower(token);
                out_row[i] = (int64_t)sq.row0 + token, out_head[i] = qh;
                float x[HF][16], amax = 0.f;
                const T* q = static_cast<const T*>(a.q) + out_row[i] * a.ldq + (int64_t)qh * D;
#pragma unroll
                for (int f = 0; f < HF; ++f) {
                    load16(q + f * 64 + t * 16, x[f]);
#pragma unroll
                    for (int e = 0; e < 16; ++e) amax = fmaxf(amax, fabsf(x[f][e]));
                }
                amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
                amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
                // the row's largest element to [2^14, 2^15)
                const int e = amax > 0.f ? min(100, 14 - ((int)(__float_as_uint(amax) >> 23) - 127)) : 0;
                const float up = __uint_as_float((uint32_t)(e + 127) << 23);
                rowf[i] = a.scale_log2 * __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
                for (int f = 0; f < HF; ++f)
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            const float p0 = x[f][4 * c + 2 * z] * up, p1 = x[f][4 * c + 2 * z + 1] * up;
                            const uint32_t top = pack_f16(p0, p1);
                            qa[0][4 * f + c][2 * z + i] = top;
                            if constexpr (kTwo) qa[kTerms - 1][4 * f + c][2 * z + i] = pack_f16_rest(p0, p1, top);
                        }
            }
            float o[D / 8][4];
#pragma unroll
            for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;

            // ---- its steps that some row sees
            const int s0 = max(first, (lo_min - sp.lo) / kStepKeys);
            const int s1 = min(last, hi_max > sp.lo ? (hi_max - sp.lo + kStepKeys - 1) / kStepKeys : 0);
            const int32_t* table = a.c.table + (int64_t)b * a.c.ld_table;
            int group0 = -1;                              // first of the 32 pages whose ids and scales the lanes hold
            int32_t page_id = -1;
            float page_ks = 0.f, page_vs = 0.f;
            auto issue = [&](int s) {
                if (s < s1) {
                    const int key = sp.lo + s * kStepKeys, page = key >> plog;
                    if (group0 < 0 || page >= group0 + 32) {
                        group0 = page;
                        page_id = -1;
                        if (((int64_t)(page + lane) << plog) < hi_max) {
                            page_id = ptx::ld_dependent(table + page + lane);
                            if (page_id < 0 || page_id >= a.c.n_pages) {
                                page_id = -1;
                                if (a.dev_status != nullptr) atomicOr(a.dev_status, MOLORA_DEV_BAD_SEQUENCE);
                            } else {
                                const int64_t block = (int64_t)page_id * a.c.kv_heads + head;
                                page_ks = ptx::ld_dependent(a.c.k_scale + block);
                                page_vs = fminf(fmaxf(ptx::ld_dependent(a.c.v_scale + block), 7.8886090522e-31f), 1.2676506002e30f);      // 2^-100, 2^100
                            }
                        }
                    }
                    const int32_t id = __shfl_sync(0xFFFFFFFFu, page_id, page - group0);
                    const float ks = __shfl_sync(0xFFFFFFFFu, page_ks, page - group0), vs = __shfl_sync(0xFFFFFFFFu, page_vs, page - group0);
                    if (lane == 0) s_scales[warp][s % kStages] = make_float2(ks, id >= 0 ? vs : -1.f);
                    if (id >= 0) {
                        const int64_t row = (((int64_t)id * a.c.kv_heads + head) << plog) + (key & ((1 << plog) - 1));
                        const uint32_t dst = ring + (uint32_t)((s % kStages) * kStageBytes);
                        const uint8_t* k = a.c.k + (row + g) * D + t * 16;
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int f = 0; f < HF; ++f)
                                ptx::cp_async_16(dst + (uint32_t)(((j * HF + f) * 32 + lane) * 16), k + j * 8 * D + f * 64);
                        const uint8_t* v = a.c.v + row * D + g * kVBytes;
                        const uint32_t vdst = dst + 2 * HF * 512;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint8_t* src = v + (2 * t + (j & 1) + 8 * (j >> 1)) * D;
                            if constexpr (kVBytes == 16) ptx::cp_async_16(vdst + (uint32_t)((j * 32 + lane) * 16), src);
                            else cp_async_8(vdst + (uint32_t)((j * 32 + lane) * 8), src);
                        }
                    }
                }
                ptx::cp_async_commit();                   // (empty groups keep the count)
            };
            __syncwarp();
            for (int s = s0; s < s0 + kStages - 1; ++s) issue(s);
            for (int s = s0; s < s1; ++s) {
                issue(s + kStages - 1);
                ptx::cp_async_wait<kStages - 1>();
                __syncwarp();                             // (the scales)
                const float2 sc = s_scales[warp][s % kStages];
                if (sc.y < 0.f) continue;                 // a page outside the pool
                const uint8_t* stage = ring_all + (warp * kStages + s % kStages) * kStageBytes;
                uint32_t kw[2][HF][4], vw[4][kVBytes / 4];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int f = 0; f < HF; ++f) {
                        const uint4 x = *reinterpret_cast<const uint4*>(stage + ((j * HF + f) * 32 + lane) * 16);
                        kw[j][f][0] = x.x, kw[j][f][1] = x.y, kw[j][f][2] = x.z, kw[j][f][3] = x.w;
                    }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (kVBytes == 16) {
                        const uint4 x = *reinterpret_cast<const uint4*>(stage + 2 * HF * 512 + (j * 32 + lane) * 16);
                        vw[j][0] = x.x, vw[j][1] = x.y, vw[j][2] = x.z, vw[j][3] = x.w;
                    } else {
                        const uint2 x = *reinterpret_cast<const uint2*>(stage + 2 * HF * 512 + (j * 32 + lane) * 8);
                        vw[j][0] = x.x, vw[j][1] = x.y;
                    }
                }
                float x[2][4];
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    x[j][0] = x[j][1] = x[j][2] = x[j][3] = 0.f;
#pragma unroll
                    for (int f = 0; f < HF; ++f)
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const uint32_t b0 = e4m3x2_to_f16x2(kw[j][f][c]), b1 = e4m3x2_to_f16x2_high(kw[j][f][c]);
#pragma unroll
                            for (int z = 0; z < kTerms; ++z) mma_f16(x[j], qa[z][4 * f + c], b0, b1);
                        }
                }
                const int key0 = sp.lo + s * kStepKeys;
                if (key0 + kStepKeys > hi_min || key0 < lo_max) {
                    // Some row does not see some key of this step.  Values that no row sees count as zero; a NaN among the codes of a value
                    // becomes a NaN in the scores of the rows that see it and a zero here, so that it cannot reach the others through
                    // their weight of zero.
                    unsigned nan = 0;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int key = key0 + 2 * t + (j & 1) + 8 * (j >> 1);
                        const bool none = key >= hi_max || key < lo_min;
#pragma unroll
                        for (int i = 0; i < kVBytes / 4; ++i) {
                            const uint32_t bits = e4m3x4_nan_bits(vw[j][i]);
                            if (bits != 0 && !none) nan |= 1u << j;
                            vw[j][i] = none ? 0u : vw[j][i] & ~((bits >> 7) * 0xFFu);
                        }
                    }
                    nan |= __shfl_xor_sync(0xFFFFFFFFu, nan, 4);
                    nan |= __shfl_xor_sync(0xFFFFFFFFu, nan, 8);
                    nan |= __shfl_xor_sync(0xFFFFFFFFu, nan, 16);
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const int key = key0 + 8 * j + 2 * t + (c & 1), i = c >> 1;
                            const bool poisoned = (nan >> (2 * j + (c & 1))) & 1u;
                            x[j][c] = key >= hi_row[i] || key < lo_row[i] ? -INFINITY : poisoned ? __int_as_float(0x7FC00000) : x[j][c];
                        }
                }
                const float lvs = __log2f(sc.y), inv_vs = 1.f / sc.y;
                float c[2], off[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) c[i] = fmaxf(rowf[i] * sc.x, 1.17549435e-38f), off[i] = lvs - m[i];      // (never 0: a hidden score is -infinity times it)
                float y[2][4];
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        y[j][e] = fmaf(x[j][e], c[e >> 1], off[e >> 1]);
                        top = fmaxf(top, y[j][e]);
                    }
                if (__any_sync(0xFFFFFFFFu, top > kTop + 8.f)) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float r = fmaxf(fmaxf(y[0][2 * i], y[0][2 * i + 1]), fmaxf(y[1][2 * i], y[1][2 * i + 1]));
                        r = fmaxf(r, __shfl_xor_sync(0xFFFFFFFFu, r, 1));
                        r = fmaxf(r, __shfl_xor_sync(0xFFFFFFFFu, r, 2));
                        // (against the new reference from the scores themselves: m may be the one of a row that has seen nothing)
                        float raw = fmaxf(fmaxf(x[0][2 * i] * c[i], x[0][2 * i + 1] * c[i]), fmaxf(x[1][2 * i] * c[i], x[1][2 * i + 1] * c[i]));
                        raw = fmaxf(raw, __shfl_xor_sync(0xFFFFFFFFu, raw, 1));
                        raw = fmaxf(raw, __shfl_xor_sync(0xFFFFFFFFu, raw, 2));
                        const float next = r > kTop ? raw + lvs - kTop : m[i];
                        const float shrink = ex2(m[i] - next);
                        m[i] = next;
                        off[i] = lvs - next;
                        l[i] *= shrink;
#pragma unroll
                        for (int d = 0; d < D / 8; ++d) o[d][2 * i] *= shrink, o[d][2 * i + 1] *= shrink;
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            y[j][2 * i] = fmaf(x[j][2 * i], c[i], off[i]);
                            y[j][2 * i + 1] = fmaf(x[j][2 * i + 1], c[i], off[i]);
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[j][e] = ex2(y[j][e]);
                l[0] = fmaf((y[0][0] + y[0][1]) + (y[1][0] + y[1][1]), inv_vs, l[0]);
                l[1] = fmaf((y[0][2] + y[0][3]) + (y[1][2] + y[1][3]), inv_vs, l[1]);
                uint32_t pa[kTerms][4];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        pa[0][2 * j + i] = pack_f16(y[j][2 * i], y[j][2 * i + 1]);
                        if constexpr (kTwo) pa[kTerms - 1][2 * j + i] = pack_f16_rest(y[j][2 * i], y[j][2 * i + 1], pa[0][2 * j + i]);
                    }
#pragma unroll
                for (int i = 0; i < kVBytes / 4; ++i)
#pragma unroll
                    for (int z = 0; z < 2; ++z) {                    // elements 4 i + 2 z and the next of each key
                        const uint32_t sel = z == 0 ? 0x5140u : 0x7362u;
                        const uint32_t p0 = __byte_perm(vw[0][i], vw[1][i], sel), p1 = __byte_perm(vw[2][i], vw[3][i], sel);
                        const uint32_t a0 = e4m3x2_to_f16x2(p0), a1 = e4m3x2_to_f16x2(p1);
                        const uint32_t b0 = e4m3x2_to_f16x2_high(p0), b1 = e4m3x2_to_f16x2_high(p1);
#pragma unroll
                        for (int y2 = 0; y2 < kTerms; ++y2) {
                            mma_f16(o[4 * i + 2 * z], pa[y2], a0, a1);
                            mma_f16(o[4 * i + 2 * z + 1], pa[y2], b0, b1);
                        }
                    }
            }
            ptx::cp_async_wait<0>();

            // ---- the result, or a piece of it
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 1);
                l[i] += __shfl_xor_sync(0xFFFFFFFFu, l[i], 2);
            }
            const bool begins = first == 0, ends = last == sp.steps;
            if (begins && ends) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (g + 8 * i >= n_rows) continue;
                    const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
                    float r[D / 4];
#pragma unroll
                    for (int d = 0; d < D / 8; ++d) r[d] = o[d][2 * i] * inv, r[D / 8 + d] = o[d][2 * i + 1] * inv;
                    store_run<T, D>(static_cast<T*>(a.out) + out_row[i] * a.ldo + (int64_t)out_head[i] * D + t * (D / 4), r);
                    if (a.lse != nullptr && t == 0)
                        a.lse[out_row[i] * a.heads + out_head[i]] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * 0.69314718056f;
                }
            } else {
                float* slot = slots + (2 * w + (begins ? 1 : 0)) * (int64_t)slot_floats(D);
                if (begins) {
                    cut.b = b, cut.row_tile = tile, cut.head = head;
                    cut.pieces = (int32_t)((unit_at + sp.steps - 1) / share - w + 1);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int row = g + 8 * i;
                    if (row >= n_rows) continue;
                    float r[D / 4];
#pragma unroll
                    for (int d = 0; d < D / 8; ++d) r[d] = o[d][2 * i], r[D / 8 + d] = o[d][2 * i + 1];
                    store_run<float, D>(slot + 2 * kRows + row * D + t * (D / 4), r);
                    if (t == 0) slot[row] = m[i], slot[kRows + row] = l[i];
                }
            }
        }
    }
    if (lane == 0) cuts[w] = cut;
}

// Joins the pieces of the unit that begins in share blockIdx.x and goes on behind it: with M the largest reference, the sum of
// 2^(m - M) (values, sum) over the pieces.  A warp takes a row, or a row's every k-th piece where there are fewer rows than warps.
constexpr int kJoinWarps = 8;
template <typename T, int D>
__global__ void __launch_bounds__(kJoinWarps * 32) attend_join_kernel(const __grid_constant__ AttendArgs a, const CutUnit* __restrict__ cuts,
                                                                     const float* __restrict__ slots)
{
    constexpr int E = D / 32;                              // elements per lane
    __shared__ float part[kJoinWarps][D];
    ptx::grid_dependency_sync();
    const int4 c4 = __ldcg(reinterpret_cast<const int4*>(cuts + blockIdx.x));
    const CutUnit cut{c4.x, c4.y, c4.z, c4.w};
    if (cut.pieces == 0) return;
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    const int group = a.heads / a.c.kv_heads;
    const Sequence sq = sequence_of(a.c, cut.b, a.N);
    const int rows = (int)min((int64_t)kRows, (int64_t)sq.n * group - (int64_t)cut.row_tile * kRows);
    const int split = rows >= kJoinWarps ? 1 : kJoinWarps / rows;              // warps per row
    const int64_t w0 = blockIdx.x;
    auto slot = [&](int p) { return slots + (p == 0 ? 2 * w0 + 1 : 2 * (w0 + p)) * (int64_t)slot_floats(D); };
    for (int r0 = 0; r0 < rows; r0 += kJoinWarps / split) {
        const int row = r0 + warp / split, sub = warp % split;
        const bool on = row < rows && warp < kJoinWarps / split * split;
        float M = kNone, L = 0.f, acc[E];
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
        if (on) {
            for (int p = lane; p < cut.pieces; p += 32) M = fmaxf(M, __ldcg(slot(p) + row));
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
            for (int p = lane; p < cut.pieces; p += 32) L += __ldcg(slot(p) + kRows + row) * ex2(__ldcg(slot(p) + row) - M);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) L += __shfl_xor_sync(0xFFFFFFFFu, L, o);
#pragma unroll 8
            for (int p = sub; p < cut.pieces; p += split) {
                const float f = ex2(__ldcg(slot(p) + row) - M);
                const float* v = slot(p) + 2 * kRows + row * D + lane * E;
                if constexpr (E == 4) {
                    const float4 x = __ldcg(reinterpret_cast<const float4*>(v));
                    acc[0] = fmaf(x.x, f, acc[0]), acc[1] = fmaf(x.y, f, acc[1]), acc[2] = fmaf(x.z, f, acc[2]), acc[3] = fmaf(x.w, f, acc[3]);
                } else {
                    const float2 x = __ldcg(reinterpret_cast<const float2*>(v));
                    acc[0] = fmaf(x.x, f, acc[0]), acc[1] = fmaf(x.y, f, acc[1]);
                }
            }
        }
        if (split > 1) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < E; ++e) part[warp][lane * E + e] = acc[e];
            __syncthreads();
            if (on && sub == 0)
                for (int z = 1; z < split; ++z)
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] += part[warp + z][lane * E + e];
        }
        if (on && sub == 0) {
            const int64_t r = (int64_t)cut.row_tile * kRows + row, token = r / group;
            const int64_t orow = sq.row0 + token;
            const int oh = cut.head * group + (int)(r - token * group);
            const float inv = L == 0.f ? 0.f : 1.f / L;
            T* out = static_cast<T*>(a.out) + orow * a.ldo + (int64_t)oh * D + lane * E;
            if constexpr (sizeof(T) == 4) {
                if constexpr (E == 4) *reinterpret_cast<float4*>(out) = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
                else *reinterpret_cast<float2*>(out) = make_float2(acc[0] * inv, acc[1] * inv);
            } else {
                if constexpr (E == 4)
                    *reinterpret_cast<uint2*>(out) = make_uint2(f32x2_to_bf16x2(acc[0] * inv, acc[1] * inv), f32x2_to_bf16x2(acc[2] * inv, acc[3] * inv));
                else *reinterpret_cast<uint32_t*>(out) = f32x2_to_bf16x2(acc[0] * inv, acc[1] * inv);
            }
            if (a.lse != nullptr && lane == 0) a.lse[orow * a.heads + oh] = L == 0.f ? -INFINITY : (M + log2f(L)) * 0.69314718056f;
        }
    }
}

int64_t worker_count() { return (int64_t)sm_count() * kCtasPerSm * kWarpsPerCta; }

template <typename T, int D>
molora_status_t launch(const AttendArgs& a, void* ws, cudaStream_t s)
{
    constexpr int kStageBytes = 32 * (2 * (D / 64) * 16 + 4 * (D / 8));
    constexpr size_t smem = (size_t)kWarpsPerCta * kStages * kStageBytes;
    static bool ready[kMaxDevices] = {};
    bool& done = ready[device_slot()];
    if (!done) {
        if (cudaFuncSetAttribute(attend_rows_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return MOLORA_ERR_CUDA;
        done = true;
    }
    const int ctas = sm_count() * (sizeof(T) == 2 ? kCtasPerSm : 2);
    const int workers = ctas * kWarpsPerCta;
    CutUnit* cuts = static_cast<CutUnit*>(ws);
    float* slots = reinterpret_cast<float*>(static_cast<char*>(ws) + cut_bytes(worker_count()));
    cudaError_t e = launch_kernel(attend_rows_kernel<T, D>, dim3((unsigned)ctas), dim3(kThreads), smem, s, 1, true, a, cuts, slots);
    if (e != cudaSuccess) return MOLORA_ERR_CUDA;
    return cuda_ok(launch_kernel(attend_join_kernel<T, D>, dim3((unsigned)workers), dim3(kJoinWarps * 32), 0, s, 1, true, a,
                                 static_cast<const CutUnit*>(cuts), static_cast<const float*>(slots)));
}

}  // namespace

size_t attend_rows_workspace_bytes(int32_t dim) { return cut_bytes(worker_count()) + (size_t)(2 * worker_count() * slot_floats(dim)) * sizeof(float); }

molora_status_t launch_attend_rows(const AttendArgs& a, molora_dtype_t dt, void* ws, cudaStream_t s)
{
    if (a.c.dim == 64) return dt == MOLORA_F32 ? launch<float, 64>(a, ws, s) : launch<__nv_bfloat16, 64>(a, ws, s);
    return dt == MOLORA_F32 ? launch<float, 128>(a, ws, s) : launch<__nv_bfloat16, 128>(a, ws, s);
}

}  // namespace molora
