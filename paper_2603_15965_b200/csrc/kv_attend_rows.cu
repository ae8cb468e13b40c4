// Attention over the paged 8-bit cache for fp32 rows, and for bf16 rows with heads of 64 (molora_kv_attend), in tiles of 8 to 32 rows.
//
// A row of a sequence is (new token, query head of the group that shares a key / value head); 8 NT consecutive rows, one
// key / value head and the keys that they see are a UNIT.  The units' keys, cut into steps of 32, form one long list; every CTA
// of the grid takes an equal, contiguous share of it, whatever the lengths of the sequences, and its four warps a
// quarter each of what the share has of a unit.  A unit that lies inside one share is written at once; one that is cut leaves its
// pieces (sum, maximum, weighted values, all fp32) in the workspace, and a second kernel joins them in the order of the
// keys: results do not depend on timing.  There are twice as many shares as resident CTAs, since SMs do not get equal shares of the
// memory's bandwidth.
//
// On its keys a warp shares nothing and synchronises with nobody: a lane asks for exactly the 16-byte vectors of codes that its
// fragments need and waits for its own copies only (cp.async ring).  Keys and elements of the values are the 16 rows of the
// tensor instruction (mma m16n8k16), query rows its 8 columns, so that a single token's few heads waste little:
//   S^T = K Q^T   lane (g, t) holds of the keys g and g + 8 the elements 16 t .. 16 t + 15 of each 64; the order of the elements
//                 in the sum is free, so a 4-byte word of codes is half an A fragment and Q's fragments follow the same order
//   O^T = V^T P^T lane (g, t) holds of the keys 2t, 2t+1, 2t+8, 2t+9 the D / 8 elements from g D / 8 on; byte permutes pair
//                 two keys of one element; the weights come into place by movmatrix, and a lane ends with D / 8 neighbouring
//                 elements of two rows
// Every e4m3 value is an fp16 value (one cvt for two); q is brought into fp16 by a power of two per row, exactly for bf16, in two
// terms of 11 bits for fp32.  The scale of a block of K multiplies its scores; that of V multiplies its weights once the sum has them
// (kv_attend.cuh), so that the weights handed to the tensor cores have the size of what they contribute.
// Weights are at most 2^15: the reference of a row moves only when a score is 2^8 over the weight it gave its largest, 2^7, and then everything
// is rescaled.  So fp16 has all 11 bits down to 2^-21 of a row's largest weight, and steps of 2^-31 of it below (22 bits down to 2^-10 in two terms).
// What bounds it: the codes, 2 D bytes per (key, key / value head), from HBM: 256 sequences of 3 to 4095 tokens, 16 heads over 8 of 64, take 122 to 126 us
// in bf16 and 130 to 136 in fp32 (4.2 and 4.0 TB/s), of 128 in fp32 271 to 286 us; for prompts the tensor instruction (8 of 1024 tokens, 32 heads
// of 64: 521 and 724 us, of 128 in fp32 1354), which reaches a quarter of what tcgen05 would give.
#include <algorithm>
#include <type_traits>

#include "kv_attend.cuh"

namespace molora {
namespace {

constexpr int kWarpsPerCta = 4, kThreads = kWarpsPerCta * 32;
constexpr int kHalfKeys = 16, kStepKeys = 32;  // keys of a tensor instruction, and of a step: two of them, in one page or in two of 16
constexpr int kUnitCost = 4;                 // steps that a unit's rows and results cost
constexpr int kMinShare = 4;                 // steps of a CTA: shorter shares cost more in joining than they save
constexpr int kWaves = 2;                    // shares per resident CTA
constexpr int kMaxTiles = 4;                 // 8-row tiles of a unit
constexpr float kTop = 7.f;                  // weight of a row's largest score when the reference is set: 2^7

// CTAs per SM by what a thread holds (accumulators D / 4 NT, fragments of q D / 8 NT per term), and copies in flight per warp
template <typename T, int D, int NT>
struct Shape {
    static constexpr int kTerms = sizeof(T) == 4 ? 2 : 1;
    static constexpr int kWork = (D / 4 + D / 8 * kTerms) * NT;          // registers
    static constexpr int kCtas = kWork <= 48 ? 3 : 2;
    static constexpr bool kPairs = kWork <= 96;                           // two steps at a time
    static constexpr int kStages = 2;                                     // steps in the ring of a warp
    static constexpr int kHalfBytes = kHalfKeys * 2 * D;
    static constexpr size_t kSmem = (size_t)kWarpsPerCta * kStages * 2 * kHalfBytes;      // (and 8 NT rows of fp32 values per warp fit it)
    static_assert(kStages * 2 * kHalfBytes >= 8 * NT * D * 4, "a warp's share of the ring holds its rows");
};

__device__ __forceinline__ void mma_f16(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// 8 x 8 matrix of 16-bit elements, transposed across the warp
__device__ __forceinline__ uint32_t transposed(uint32_t v)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
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
template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src)
{
    if constexpr (BYTES == 16) ptx::cp_async_16(dst, src);
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}

template <typename T>
__device__ __forceinline__ void load16(const T* p, float* x)
{
    constexpr int E = VecTraits<T>::kElems;
#pragma unroll
    for (int i = 0; i < 16 / E; ++i) unpack<T>(ld128_rw_stream(p + i * E), x + i * E);
}

template <typename T, int N>
__device__ __forceinline__ void store_run(T* p, const float* x)          // N neighbouring elements
{
    constexpr int E = VecTraits<T>::kElems;
#pragma unroll
    for (int i = 0; i < N / E; ++i) stg128(p + i * E, pack<T>(x + i * E));
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kThreads, Shape<T, D, NT>::kCtas)
    attend_rows_kernel(const __grid_constant__ AttendArgs a, CutUnit* __restrict__ cuts, float* __restrict__ slots)
{
    using Sh = Shape<T, D, NT>;
    constexpr int kTerms = Sh::kTerms;                  // fp16 terms of q and of the weights
    constexpr int kStages = Sh::kStages;
    constexpr int kRows = 8 * NT;
    constexpr int HF = D / 64;                          // 64-element parts of a key
    constexpr int kVBytes = D / 8;                      // of a value, per lane
    constexpr int kMT = D / 16;                         // 16-element tiles of the values
    constexpr bool kPairs = Sh::kPairs;
    __shared__ ShareStart s_start;
    __shared__ float4 s_scales[kWarpsPerCta][kStages][2];  // of a half: scale of K, logarithm of V's, V's, whether its page can be used
    __shared__ float s_m[kWarpsPerCta][kRows], s_l[kWarpsPerCta][kRows];
    extern __shared__ __align__(16) uint8_t ring_all[];
    ptx::grid_dependency_sync();

    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int group = a.group;
    const int plog = a.c.page_log2;
    uint8_t* const ring = ring_all + warp * kStages * 2 * Sh::kHalfBytes;
    const uint32_t ring_at = ptx::smem_u32(ring);

    const int64_t w = blockIdx.x;
    Walk<kRows, kStepKeys, kUnitCost> walk(a);
    cut_shares<kThreads, 1>(a, w, gridDim.x, kMinShare, &s_start, [&](const Sequence& sq) { return steps_of<kRows, kStepKeys, kUnitCost>(a, sq, group); });
    walk.begin(s_start, w, kThreads);
    CutUnit cut{};
    Unit un;
    while (walk.next(un)) {
        const Sequence& sq = un.sq;
        const int lo0 = un.sp.lo, head = un.head, n_rows = un.n_rows, tile_row = un.tile_row;
        const int hi_min = un.hi_min, hi_max = un.hi_max, lo_min = un.lo_min, lo_max = un.lo_max;
        auto token_of = [&](int r) { return (tile_row + min(r, n_rows - 1)) / group; };

        // ---- its steps that some row sees, a contiguous part of them for each warp; the first come in while q does
        const int u0 = un.u0, u1 = un.u1;
        const int per_warp = (max(u1 - u0, 0) + kWarpsPerCta - 1) / kWarpsPerCta;
        const int s0 = u0 + warp * per_warp, s1 = min(u1, s0 + per_warp);
        const int32_t* table = a.c.table + (int64_t)un.b * a.c.ld_table;
        int group0 = -1;                              // first of the 32 pages whose ids and scales the lanes hold
        int32_t page_id = -1;
        float page_ks = 0.f, page_lvs = 0.f, page_vs = 0.f;
        auto load_pages = [&](int page) {
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
                    page_vs = read_v_scale(ptx::ld_dependent(a.c.v_scale + block));
                    page_lvs = log2f(page_vs);
                }
            }
        };
        // 16 keys from `row` (of all tokens of the pool) on
        auto copy_half = [&](int64_t row, uint32_t dst) {
            const uint8_t* k = a.c.k + row * D + (g * D + t * 16);
            const uint32_t kdst = dst + (uint32_t)(lane * 16);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int f = 0; f < HF; ++f) copy_async<16>(kdst + (uint32_t)((j * HF + f) * 512), k + j * 8 * D + f * 64);
            const uint8_t* v = a.c.v + row * D + (2 * t * D + g * kVBytes);
            const uint32_t vdst = dst + 2 * HF * 512 + (uint32_t)(lane * kVBytes);
#pragma unroll
            for (int j = 0; j < 4; ++j) copy_async<kVBytes>(vdst + (uint32_t)(j * 32 * kVBytes), v + ((j & 1) + 8 * (j >> 1)) * D);
        };
        auto issue = [&](int s) {
            if (s < s1) {
                const int key = lo0 + s * kStepKeys, page = key >> plog, put = (s - s0) & (kStages - 1);
                if (group0 < 0 || page >= group0 + 32 || (plog == 4 && page + 1 >= group0 + 32)) load_pages(page);
                const uint32_t dst = ring_at + (uint32_t)(put * 2 * Sh::kHalfBytes);
                const int32_t id = __shfl_sync(0xFFFFFFFFu, page_id, page - group0);
                const float4 sc = make_float4(page_ks, page_lvs, page_vs, page_id >= 0 ? 1.f : 0.f);
                const int64_t row = (((int64_t)id * a.c.kv_heads + head) << plog) + (key & ((1 << plog) - 1));
                if (lane == page - group0) s_scales[warp][put][0] = sc;
                if (id >= 0) copy_half(row, dst);
                if (plog > 4) {
                    if (lane == page - group0) s_scales[warp][put][1] = sc;
                    if (id >= 0) copy_half(row + kHalfKeys, dst + Sh::kHalfBytes);
                } else {
                    const int32_t id1 = __shfl_sync(0xFFFFFFFFu, page_id, page + 1 - group0);
                    if (lane == page + 1 - group0) s_scales[warp][put][1] = sc;
                    if (id1 >= 0) copy_half(((int64_t)id1 * a.c.kv_heads + head) << plog, dst + Sh::kHalfBytes);
                }
            }
            ptx::cp_async_commit();                   // (empty groups keep the count)
        };
        issue(s0);

        float rowf[NT][2], m[NT][2], l[NT][2];        // rows 8 n + 2 t and the next
        uint32_t qb[kTerms][NT][4 * HF][2];           // row 8 n + g
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = min(8 * n + g, n_rows - 1);
            const int token = token_of(r), qh = head * group + (tile_row + r - token * group);
            float x[HF][16], amax = 0.f;
            const T* q = static_cast<const T*>(a.q) + ((int64_t)sq.row0 + token) * a.ldq + (int64_t)qh * D;
#pragma unroll
            for (int f = 0; f < HF; ++f) {
                load16(q + f * 64 + t * 16, x[f]);
#pragma unroll
                for (int e = 0; e < 16; ++e) amax = fmaxf(amax, fabsf(x[f][e]));
            }
            amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
            amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
            const RowScale by = row_scale<14>(amax);
            const float up = by.up, down = a.scale_log2 * by.down;
#pragma unroll
            for (int f = 0; f < HF; ++f)
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        const float p0 = x[f][4 * c + 2 * z] * up, p1 = x[f][4 * c + 2 * z + 1] * up;
                        const uint32_t top = pack_f16(p0, p1);
                        qb[0][n][4 * f + c][z] = top;
                        if constexpr (kTerms == 2) qb[kTerms - 1][n][4 * f + c][z] = pack_f16_rest(p0, p1, top);
                    }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                rowf[n][i] = __shfl_sync(0xFFFFFFFFu, down, (2 * t + i) * 4);
                m[n][i] = kNone, l[n][i] = 0.f;
            }
        }
        float o[NT][kMT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < kMT; ++i) o[n][i][0] = o[n][i][1] = o[n][i][2] = o[n][i][3] = 0.f;

        // SUBS halves from key0 on, in ring position `at_step` from half `half` on
        auto work = [&](int key0, int at_step, int half, auto subs) {
            constexpr int SUBS = decltype(subs)::value;
            float4 sc[SUBS];
            float x[SUBS][NT][4];                     // keys g (0, 1) and g + 8 (2, 3), rows 2 t and 2 t + 1
#pragma unroll
            for (int u = 0; u < SUBS; ++u) {
                const uint8_t* stage = ring + (2 * at_step + half + u) * Sh::kHalfBytes;
                sc[u] = s_scales[warp][at_step][half + u];
                uint32_t kw[2][HF][4];
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int f = 0; f < HF; ++f) {
                        const uint4 w4 = *reinterpret_cast<const uint4*>(stage + ((j * HF + f) * 32 + lane) * 16);
                        kw[j][f][0] = w4.x, kw[j][f][1] = w4.y, kw[j][f][2] = w4.z, kw[j][f][3] = w4.w;
                    }
                float part[HF][NT][4];                // (a chain of sums per half: each waits for its predecessor)
#pragma unroll
                for (int f = 0; f < HF; ++f)
#pragma unroll
                    for (int n = 0; n < NT; ++n) part[f][n][0] = part[f][n][1] = part[f][n][2] = part[f][n][3] = 0.f;
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int f = 0; f < HF; ++f) {
                        const uint32_t a0 = e4m3x2_to_f16x2(kw[0][f][c]), a2 = e4m3x2_to_f16x2_high(kw[0][f][c]);
                        const uint32_t a1 = e4m3x2_to_f16x2(kw[1][f][c]), a3 = e4m3x2_to_f16x2_high(kw[1][f][c]);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int z = 0; z < kTerms; ++z) mma_f16(part[f][n], a0, a1, a2, a3, qb[z][n][4 * f + c][0], qb[z][n][4 * f + c][1]);
                    }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[u][n][e] = HF == 2 ? part[0][n][e] + part[HF - 1][n][e] : part[0][n][e];
            }
            const bool border = key0 + SUBS * kHalfKeys > hi_min || key0 < lo_max;
            uint32_t vw[SUBS][4][kVBytes / 4];
#pragma unroll
            for (int u = 0; u < SUBS; ++u) {
                const uint8_t* stage = ring + (2 * at_step + half + u) * Sh::kHalfBytes + 2 * HF * 512;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if constexpr (kVBytes == 16) {
                        const uint4 w4 = *reinterpret_cast<const uint4*>(stage + (j * 32 + lane) * 16);
                        vw[u][j][0] = w4.x, vw[u][j][1] = w4.y, vw[u][j][2] = w4.z, vw[u][j][3] = w4.w;
                    } else {
                        const uint2 w2 = *reinterpret_cast<const uint2*>(stage + (j * 32 + lane) * 8);
                        vw[u][j][0] = w2.x, vw[u][j][1] = w2.y;
                    }
                }
            }
            if (border) {
                // Some row does not see some key of these steps.  Values that no row sees count as zero; a NaN among the codes of a value
                // becomes a NaN in the scores of the rows that see it and a zero here, so that it cannot reach the others through
                // their weight of zero.
                unsigned nan = 0;
#pragma unroll
                for (int u = 0; u < SUBS; ++u)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int k16 = 16 * u + 2 * t + (j & 1) + 8 * (j >> 1), key = key0 + k16;
                        const bool none = key >= hi_max || key < lo_min;
#pragma unroll
                        for (int i = 0; i < kVBytes / 4; ++i) {
                            const uint32_t bits = e4m3x4_nan_bits(vw[u][j][i]);
                            if (bits != 0 && !none) nan |= 1u << k16;
                            vw[u][j][i] = none ? 0u : vw[u][j][i] & ~((bits >> 7) * 0xFFu);
                        }
                    }
                nan = __reduce_or_sync(0xFFFFFFFFu, nan);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int token = token_of(8 * n + 2 * t + i), hi_row = upper_key(a, sq, token), lo_row = lower_key(a, sq, token);
#pragma unroll
                        for (int u = 0; u < SUBS; ++u)
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                const int k16 = 16 * u + g + 8 * j, key = key0 + k16;
                                float& v = x[u][n][2 * j + i];
                                v = key >= hi_row || key < lo_row ? -INFINITY : (nan >> k16) & 1u ? __int_as_float(0x7FC00000) : v;
                            }
                    }
            }
            // sc: scale of K, logarithm of V's, V's
            float c[SUBS][NT][2], top = -INFINITY, y[SUBS][NT][4];
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int i = 0; i < 2; ++i) c[u][n][i] = fmaxf(rowf[n][i] * sc[u].x, 1.17549435e-38f);      // (never 0: a hidden score is -infinity times it)
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        const float2 z = fma2(make_float2(x[u][n][e], x[u][n][e + 1]), make_float2(c[u][n][0], c[u][n][1]), make_float2(-m[n][0], -m[n][1]));
                        y[u][n][e] = z.x, y[u][n][e + 1] = z.y;
                    }
                    top = fmaxf(top, fmaxf(fmaxf(y[u][n][0], y[u][n][1]), fmaxf(y[u][n][2], y[u][n][3])) + sc[u].y);
                }
            if (__any_sync(0xFFFFFFFFu, top > kTop + 8.f)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float raw = -INFINITY;
#pragma unroll
                        for (int u = 0; u < SUBS; ++u) raw = fmaxf(raw, fmaxf(x[u][n][i] * c[u][n][i], x[u][n][2 + i] * c[u][n][i]) + sc[u].y);
#pragma unroll
                        for (int z = 4; z < 32; z <<= 1) raw = fmaxf(raw, __shfl_xor_sync(0xFFFFFFFFu, raw, z));
                        const float next = raw - m[n][i] > kTop ? raw - kTop : m[n][i];
                        const Shrink by(m[n][i] - next);
                        const float shrink = by.both();
                        m[n][i] = next;
                        l[n][i] = by.of(l[n][i]);
#pragma unroll
                        for (int d = 0; d < kMT; ++d) o[n][d][i] *= shrink, o[n][d][2 + i] *= shrink;
#pragma unroll
                        for (int u = 0; u < SUBS; ++u) {
                            y[u][n][i] = fmaf(x[u][n][i], c[u][n][i], -next);
                            y[u][n][2 + i] = fmaf(x[u][n][2 + i], c[u][n][i], -next);
                        }
                    }
            }
            uint32_t pb[SUBS][kTerms][NT][2];
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[u][n][e] = ex2(y[u][n][e]);
                    const float2 sum = add2(make_float2(l[n][0], l[n][1]), add2(make_float2(y[u][n][0], y[u][n][1]), make_float2(y[u][n][2], y[u][n][3])));
                    l[n][0] = sum.x, l[n][1] = sum.y;
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        const float2 z = mul2(make_float2(y[u][n][e], y[u][n][e + 1]), make_float2(sc[u].z, sc[u].z));
                        y[u][n][e] = z.x, y[u][n][e + 1] = z.y;
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t p = pack_f16(y[u][n][2 * j], y[u][n][2 * j + 1]);
                        pb[u][0][n][j] = transposed(p);
                        if constexpr (kTerms == 2) pb[u][kTerms - 1][n][j] = transposed(pack_f16_rest(y[u][n][2 * j], y[u][n][2 * j + 1], p));
                    }
                }
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int i = 0; i < kVBytes / 4; ++i)
#pragma unroll
                    for (int z = 0; z < 2; ++z) {                    // elements 4 i + 2 z and the next of each key
                        const uint32_t sel = z == 0 ? 0x5140u : 0x7362u;
                        const uint32_t p0 = __byte_perm(vw[u][0][i], vw[u][1][i], sel), p1 = __byte_perm(vw[u][2][i], vw[u][3][i], sel);
                        const uint32_t a0 = e4m3x2_to_f16x2(p0), a1 = e4m3x2_to_f16x2_high(p0);
                        const uint32_t a2 = e4m3x2_to_f16x2(p1), a3 = e4m3x2_to_f16x2_high(p1);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int y2 = 0; y2 < kTerms; ++y2) mma_f16(o[n][2 * i + z], a0, a1, a2, a3, pb[u][y2][n][0], pb[u][y2][n][1]);
                    }
        };
        // both halves at a time: their chains of dependent instructions overlap
        for (int s = s0; s < s1; ++s) {
            issue(s + 1);
            ptx::cp_async_wait<1>();
            __syncwarp();                             // (the scales)
            const int get = (s - s0) & (kStages - 1), key0 = lo0 + s * kStepKeys;
            const bool one = s_scales[warp][get][0].w != 0.f, two = s_scales[warp][get][1].w != 0.f;
            if (kPairs && one && two) {
                work(key0, get, 0, std::integral_constant<int, kPairs ? 2 : 1>{});
            } else {
                if (one) work(key0, get, 0, std::integral_constant<int, 1>{});
                if (two) work(key0 + kHalfKeys, get, 1, std::integral_constant<int, 1>{});
            }
            __syncwarp();
        }
        ptx::cp_async_wait<0>();

        // ---- the four warps' parts become one: everybody's values by the largest reference, through the ring
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int z = 4; z < 32; z <<= 1) l[n][i] += __shfl_xor_sync(0xFFFFFFFFu, l[n][i], z);
                if (g == 0) s_m[warp][8 * n + 2 * t + i] = m[n][i], s_l[warp][8 * n + 2 * t + i] = l[n][i];
            }
        __syncthreads();
        float* const rows = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = 8 * n + 2 * t + i;
                if (row >= n_rows) continue;
                float top = s_m[0][row];
#pragma unroll
                for (int z = 1; z < kWarpsPerCta; ++z) top = fmaxf(top, s_m[z][row]);
                const float f = Shrink(m[n][i] - top).both();
                float r[kVBytes];
#pragma unroll
                for (int d = 0; d < kMT; ++d) r[2 * d] = o[n][d][i] * f, r[2 * d + 1] = o[n][d][2 + i] * f;
                store_run<float, kVBytes>(rows + row * D + g * kVBytes, r);
            }
        __syncthreads();
        const bool begins = un.first == 0, ends = un.last == un.sp.steps, whole = begins && ends;
        float* slot = slots + (2 * w + (begins ? 1 : 0)) * (int64_t)slot_floats(kRows, D);
        if (begins && !ends) {
            cut.row0 = un.sq.row0, cut.tile_row = tile_row, cut.rows = n_rows, cut.head = head;
            cut.pieces = walk.pieces(un, w);
        }
        for (int i = tid; i < n_rows * (D / 4); i += kThreads) {
            const int row = i / (D / 4), d = i % (D / 4) * 4;
            float top = s_m[0][row], sum = 0.f;
#pragma unroll
            for (int z = 1; z < kWarpsPerCta; ++z) top = fmaxf(top, s_m[z][row]);
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int z = 0; z < kWarpsPerCta; ++z) {
                sum += Shrink(s_m[z][row] - top).of(s_l[z][row]);
                const float4 x = *reinterpret_cast<const float4*>(ring_all + z * kStages * 2 * Sh::kHalfBytes + (row * D + d) * 4);
                v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
            }
            if (whole) {
                const float inv = sum == 0.f ? 0.f : 1.f / sum;
                const int token = token_of(row), qh = head * group + (tile_row + row - token * group);
                const int64_t orow = (int64_t)sq.row0 + token;
                store4(static_cast<T*>(a.out) + orow * a.ldo + (int64_t)qh * D + d, v, inv);
                if (a.lse != nullptr && d == 0) a.lse[orow * a.heads + qh] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718056f;
            } else {
                *reinterpret_cast<float4*>(slot + 2 * kRows + row * D + d) = v;
                if (d == 0) slot[row] = top, slot[kRows + row] = sum;
            }
        }
        __syncthreads();
    }
    if (tid == 0) cuts[w] = cut;
}

template <typename T, int D, int NT>
int64_t worker_count() { return (int64_t)sm_count() * Shape<T, D, NT>::kCtas * kWaves; }

template <typename T, int D, int NT>
size_t bytes_needed()
{
    const int64_t n = worker_count<T, D, NT>();
    return cut_bytes(n) + (size_t)(2 * n * slot_floats(8 * NT, D)) * sizeof(float);
}

template <typename T, int D, int NT>
molora_status_t launch(const AttendArgs& a, void* ws, cudaStream_t s)
{
    using Sh = Shape<T, D, NT>;
    static bool ready[kMaxDevices] = {};
    bool& done = ready[device_slot()];
    if (!done) {
        if (cudaFuncSetAttribute(attend_rows_kernel<T, D, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Sh::kSmem) != cudaSuccess) return MOLORA_ERR_CUDA;
        done = true;
    }
    const int workers = (int)worker_count<T, D, NT>();
    CutUnit* cuts = static_cast<CutUnit*>(ws);
    float* slots = reinterpret_cast<float*>(static_cast<char*>(ws) + cut_bytes(workers));
    if (launch_kernel(attend_rows_kernel<T, D, NT>, dim3((unsigned)workers), dim3(kThreads), Sh::kSmem, s, 1, true, a, cuts, slots) != cudaSuccess)
        return MOLORA_ERR_CUDA;
    return cuda_ok(launch_kernel(attend_join_kernel<T, D, 8 * NT>, dim3((unsigned)workers, join_groups(8 * NT)), dim3(kJoinWarps * 32), 0, s, 1, true, a,
                                 static_cast<const CutUnit*>(cuts), static_cast<const float*>(slots)));
}

// f<T, D, NT>() of the variant for these rows: as few 8-row tiles as hold the rows that share a key / value head in the longest sequence, at most 4
// (2 for fp32, whose terms take the registers)
template <typename T, int D, typename F>
auto for_tiles(int64_t rows, F f)
{
    if (rows <= 8) return f.template operator()<T, D, 1>();
    if (rows <= 16 || sizeof(T) == 4) return f.template operator()<T, D, 2>();
    if constexpr (sizeof(T) == 2) {
        if (rows <= 24) return f.template operator()<T, D, 3>();
        return f.template operator()<T, D, kMaxTiles>();
    }
    return f.template operator()<T, D, 2>();
}
template <typename F>
auto for_variant(molora_dtype_t dt, int32_t dim, int64_t rows, F f)
{
    if (dt == MOLORA_F32) return dim == 64 ? for_tiles<float, 64>(rows, f) : for_tiles<float, 128>(rows, f);
    return for_tiles<__nv_bfloat16, 64>(rows, f);
}
struct BytesNeeded {
    template <typename T, int D, int NT>
    size_t operator()() const { return bytes_needed<T, D, NT>(); }
};
struct Launch {
    const AttendArgs& a;
    void* ws;
    cudaStream_t s;
    template <typename T, int D, int NT>
    molora_status_t operator()() const { return launch<T, D, NT>(a, ws, s); }
};

}  // namespace

// the most that any number of rows up to this needs (24 rows of bf16, with fewer CTAs, need less than 16)
size_t attend_rows_workspace_bytes(molora_dtype_t dt, int32_t dim, int64_t rows)
{
    size_t most = 0;
    for (int64_t r = 8; r < 8 * kMaxTiles; r += 8)
        if (r < rows) most = std::max(most, for_variant(dt, dim, r, BytesNeeded{}));
    return std::max(most, for_variant(dt, dim, rows, BytesNeeded{}));
}

molora_status_t launch_attend_rows(const AttendArgs& a, molora_dtype_t dt, int64_t rows, void* ws, cudaStream_t s)
{
    return for_variant(dt, a.c.dim, rows, Launch{a, ws, s});
}

}  // namespace molora
