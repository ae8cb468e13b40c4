// Attention over the paged 8-bit cache for up to 32 query rows, bf16, heads of 128 (molora_kv_attend): decode and drafted tokens.
//
// The codes of keys and values go from memory to the tensor cores as they are: TMA brings blocks of the cache into shared
// memory, tcgen05.mma (kind::f8f6f4) reads them there, and no thread ever touches them.  What is not 8 bits wide is
// written as a sum of e4m3 terms, each in columns of its own:
//   q (8 significant bits) = t1 + t2 / 32, exactly: the rest that rounding to 4 bits leaves of 8 fits 4; a power of two per row brings the largest
//       element to [2^7, 2^8), so elements below 2^-14 of it are off by at most 2^-23 of it
//   a weight = t1 + t2 / 32 + t3 / 1024, to 2^-12 of it (and 2^-20 where a row's largest is 2^4 or more)
//   S^T [128 keys x 2 rows]   = K Q^T     A = K tile, keys the 128 lanes of TMEM; B = q's terms
//   O^T [128 elements x 3 rows] += V^T P^T  A = V tile read across (MN-major); B = the weights' terms
// with the key as the lane a thread owns one key: the scales of its block, its mask and its weights are its own, and reductions
// over keys are needed only when a row's reference moves (a score 2^4 over the reference) and at the end of a unit.
//   warp 0    page table, scales, TMA (kStages tiles of 128 keys = 32 KB each in flight)
//   warp 1    the MMAs of S one tile ahead of those of O
//   warps 2-5 a key per thread: weights and their terms into shared memory; at the end of a unit an element per thread
// Weights are at most 2^8; the scale of a block of K multiplies its scores, that of V is added to the exponent as a logarithm and taken off
// the sum again, so that weights have the size of what they contribute.
// What bounds it: 32 KB a tile from HBM; the chain of a tile (S, weights, O) takes about half of what the bytes do.
#include "kv_attend.cuh"
#include "pipeline.cuh"
#include "tensor_map.cuh"

namespace molora {
namespace {

constexpr int kDim = 128, kKeys = 128;
constexpr int kThreads = 192, kKeyThreads = 128;
constexpr int kStages = 5;
constexpr int kTileBytes = kKeys * kDim, kStageBytes = 2 * kTileBytes;
constexpr int kMinShare = 2;                 // tiles
constexpr int kWaves = 1;
constexpr int kTermsQ = 2, kTermsP = 3;
constexpr float kTermStep = 32.f;            // a term's weight against the next
constexpr float kTop = 4.f, kSlack = 4.f;    // a row's largest weight when its reference is set: 2^4; it may grow by 2^4 before the reference moves
constexpr float kNan = __builtin_nanf("");

template <int ROWS>
struct Cfg {
    static constexpr int kNS = kTermsQ * ROWS;                            // columns of S: a multiple of 16
    static constexpr int kNP = (kTermsP * ROWS + 15) / 16 * 16;           // columns of O, the last ones unused
    static constexpr int kQBytes = (kNS + 7) / 8 * 1024, kPBytes = (kNP + 7) / 8 * 1024;
    static constexpr uint32_t kSCol0 = 0, kSCol1 = 64, kOCol = 128, kTmemCols = 256;
    static_assert(kNS <= 64 && kNP <= 128, "TMEM columns");
    static constexpr size_t kSmem = 1024 + (size_t)kStages * kStageBytes + kQBytes + 2 * kPBytes;
};

struct Control {
    uint64_t full[kStages], empty[kStages], s_full[2], s_empty[2], p_full[2], p_empty[2], q_full, o_empty, drained;
    uint32_t tmem_base;
    int abort_flag;
};

__device__ __forceinline__ void key_threads_sync() { asm volatile("barrier.cta.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ bool key_threads_any(bool v)
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred P, Q;\n\tsetp.ne.b32 P, %1, 0;\n\tbarrier.cta.red.or.pred Q, 1, 128, P;\n\tselp.u32 %0, 1, 0, Q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)v)
        : "memory");
    return r != 0;
}
__device__ __forceinline__ float warp_max(float v)
{
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
// two values -> their e4m3 codes (low byte: a) and what the codes leave of them, times 32
__device__ __forceinline__ uint32_t split_pair(float& a, float& b)
{
    const uint32_t c = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const float2 f = f16x2_to_f32x2(e4m3x2_to_f16x2(c));
    a = (a - f.x) * kTermStep, b = (b - f.y) * kTermStep;
    return c;
}
// byte `b` of line `line` of a K-major operand of 128-byte lines, 128-byte swizzle
__device__ __forceinline__ uint32_t line_offset(int line, int b) { return (uint32_t)(line * 128 + ((((b >> 4) ^ line) & 7) << 4) + (b & 15)); }

template <int N>
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t* v)          // N columns, a multiple of 8
{
#pragma unroll
    for (int i = 0; i + 16 <= N; i += 16) ptx::tmem_ld_x16(addr + i, v + i);
    if constexpr (N % 16 != 0) ptx::tmem_ld_x8(addr + N / 16 * 16, v + N / 16 * 16);
    ptx::tmem_wait_ld();
}

template <int ROWS>
__global__ void __launch_bounds__(kThreads, 1)
    attend_stream_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                         CutUnit* __restrict__ cuts, float* __restrict__ slots)
{
    using C = Cfg<ROWS>;
    using namespace ptx;
    __shared__ Control ctrl;
    __shared__ int64_t s_upto[kThreads];
    __shared__ float4 s_scales[kStages][8];          // of 16 keys: scale of K, logarithm and reciprocal of V's, whether their page can be used
    __shared__ float s_row[ROWS], s_part[4][ROWS];
    extern __shared__ uint8_t smem_raw[];
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - raw);
    const uint32_t q_at = base + kStages * kStageBytes, p_at = q_at + C::kQBytes;
    volatile int* abort_flag = &ctrl.abort_flag;
    auto bar = [](const uint64_t* b) { return smem_u32(b); };

    grid_dependency_wait();
    if (tid == 0) {
        prefetch_tensormap(&tm_k);
        prefetch_tensormap(&tm_v);
        for (int s = 0; s < kStages; ++s) mbar_init(bar(&ctrl.full[s]), 1), mbar_init(bar(&ctrl.empty[s]), 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(&ctrl.s_full[i]), 1), mbar_init(bar(&ctrl.s_empty[i]), kKeyThreads);
            mbar_init(bar(&ctrl.p_full[i]), kKeyThreads), mbar_init(bar(&ctrl.p_empty[i]), 1);
        }
        mbar_init(bar(&ctrl.q_full), kKeyThreads);
        mbar_init(bar(&ctrl.o_empty), kKeyThreads);
        mbar_init(bar(&ctrl.drained), 1);
        ctrl.abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(&ctrl.tmem_base), C::kTmemCols);
        tmem_relinquish();
    }
    // operand lines of no row are zero for good
    for (int i = tid; i < (C::kQBytes + 2 * C::kPBytes) / 16; i += kThreads) *reinterpret_cast<uint4*>(smem + kStages * kStageBytes + i * 16) = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    Walk<ROWS, kKeys> walk(a);
    begin_share<kThreads>(walk, blockIdx.x, gridDim.x, kMinShare, s_upto);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_dependency_trigger();                        // (not before TMEM is mine)
    const uint32_t tmem = ctrl.tmem_base;
    const int group = walk.group, plog = a.c.page_log2;
    Unit u;

    if (warp == 0) {
        // ============================================================ pages, scales, copies
        const int box_log2 = min(plog, 7), boxes = kKeys >> box_log2;      // copies of a tile, each of one page (or of a part of 128)
        const uint32_t box_bytes = (uint32_t)kDim << box_log2;
        int s = 0, tiles = 0;
        uint32_t ph = 1;
        while (walk.next(u)) {
            const int32_t* table = a.c.table + (int64_t)u.b * a.c.ld_table;
            int group0 = -1;
            int32_t page_id = -1;
            float4 sc = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int i = u.u0; i < u.u1; ++i) {
                const int key0 = u.sp.lo + i * kKeys, page = key0 >> plog;
                if (group0 < 0 || page + boxes > group0 + 32) {
                    group0 = page;
                    page_id = -1;
                    sc = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (((int64_t)(page + lane) << plog) < u.hi_max) {
                        page_id = ld_dependent(table + page + lane);
                        if (page_id < 0 || page_id >= a.c.n_pages) {
                            page_id = -1;
                            if (a.dev_status != nullptr) atomicOr(a.dev_status, MOLORA_DEV_BAD_SEQUENCE);
                        } else {
                            const int64_t block = (int64_t)page_id * a.c.kv_heads + u.head;
                            const float vs = clamped_scale(ld_dependent(a.c.v_scale + block));
                            sc = make_float4(ld_dependent(a.c.k_scale + block), log2f(vs), 1.f / vs, 1.f);
                        }
                    }
                }
                if (tiles >= kStages) wait_bar(bar(&ctrl.empty[s]), ph, abort_flag, a.dev_status);
                if (*abort_flag) break;
                const int mine = page - group0 + (((lane & 7) * 16) >> plog);           // the page of 16 keys
                float4 g;
                g.x = __shfl_sync(0xFFFFFFFFu, sc.x, mine & 31), g.y = __shfl_sync(0xFFFFFFFFu, sc.y, mine & 31);
                g.z = __shfl_sync(0xFFFFFFFFu, sc.z, mine & 31), g.w = __shfl_sync(0xFFFFFFFFu, sc.w, mine & 31);
                if (lane < 8) s_scales[s][lane] = g;
                const int32_t id = __shfl_sync(0xFFFFFFFFu, page_id, (page - group0 + lane) & 31);
                const bool copies = lane < boxes && id >= 0;
                const uint32_t bytes = 2u * box_bytes * (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, copies));
                const uint32_t fb = bar(&ctrl.full[s]);
                if (lane == 0) mbar_arrive_expect_tx(fb, bytes);
                __syncwarp();
                if (copies) {
                    const int row = (int)((((int64_t)id * a.c.kv_heads + u.head) << plog) + (key0 & ((1 << plog) - 1)));
                    const uint32_t dst = base + (uint32_t)(s * kStageBytes) + (uint32_t)lane * box_bytes;
                    tma_load_2d(dst, &tm_k, 0, row, fb);
                    tma_load_2d(dst + kTileBytes, &tm_v, 0, row, fb);
                }
                __syncwarp();
                ++tiles;
                if (++s == kStages) s = 0, ph ^= 1u;
            }
            if (*abort_flag) break;
        }
        // every copy has landed before the memory is given up (an abort may come with copies in flight; this wait has its own limit)
        for (int i = 0; i < min(tiles, kStages); ++i) {
            const int t = tiles - 1 - i;
            const long long t0 = clock64();
            while (!mbar_try_wait(bar(&ctrl.full[t % kStages]), (uint32_t)(t / kStages) & 1u))
                if (clock64() - t0 > kTimeoutCycles) break;
        }
    } else if (warp == 1) {
        // ============================================================ MMAs
        const bool leader = elect_one();
        const uint32_t tm = __shfl_sync(0xFFFFFFFFu, tmem, 0);
        constexpr uint32_t idesc_s = idesc_e4m3_f32(kKeys, C::kNS, 0, 0), idesc_o = idesc_e4m3_f32(kDim, C::kNP, 1, 0);
        constexpr uint32_t kL128 = swizzle_layout_type(Swizzle::B128);
        const uint64_t k_desc = smem_desc(base, 16, 1024, kL128), v_desc = smem_desc(base + kTileBytes, 0, 1024, kL128);
        const uint64_t q_desc = smem_desc(q_at, 16, 1024, kL128), p_desc = smem_desc(p_at, 16, 1024, kL128);
        bool live = true;
        int tiles = 0, units = 0;                     // tiles whose S has been asked for, units with tiles begun
        auto issue_s = [&](bool first) {              // S of tile `tiles`
            const int s = tiles % kStages, b = tiles & 1;
            if (first) live = wait_bar(bar(&ctrl.q_full), (uint32_t)units & 1u, abort_flag, a.dev_status) && live, ++units;
            live = wait_bar(bar(&ctrl.full[s]), (uint32_t)(tiles / kStages) & 1u, abort_flag, a.dev_status) && live;
            if (tiles >= 2) live = wait_bar(bar(&ctrl.s_empty[b]), ((uint32_t)(tiles >> 1) & 1u) ^ 1u, abort_flag, a.dev_status) && live;
            tc_fence_after();
            if (leader && live) {
                const uint64_t at = (uint64_t)(s * (kStageBytes >> 4));
                const uint32_t d = tm + (b ? C::kSCol1 : C::kSCol0);
#pragma unroll
                for (int j = 0; j < 4; ++j) umma_f8(d, k_desc + at + j * 2, q_desc + j * 2, idesc_s, j > 0);      // 32 elements a step
                umma_commit(bar(&ctrl.s_full[b]));
            }
            ++tiles;
        };
        auto issue_o = [&](int t, bool first, int unit) {
            const int s = t % kStages, b = t & 1;
            live = wait_bar(bar(&ctrl.p_full[b]), (uint32_t)(t >> 1) & 1u, abort_flag, a.dev_status) && live;
            if (first && unit > 0) live = wait_bar(bar(&ctrl.o_empty), ((uint32_t)unit & 1u) ^ 1u, abort_flag, a.dev_status) && live;
            tc_fence_after();
            if (leader && live) {
                const uint64_t at = (uint64_t)(s * (kStageBytes >> 4)), pa = (uint64_t)(b * (C::kPBytes >> 4));
#pragma unroll
                for (int j = 0; j < 4; ++j)           // 32 keys a step: 4 groups of 8 lines of V
                    umma_f8(tm + C::kOCol, v_desc + at + j * (4096 >> 4), p_desc + pa + j * 2, idesc_o, !first || j > 0);
                umma_commit(bar(&ctrl.p_empty[b]));
                umma_commit(bar(&ctrl.empty[s]));
            }
        };
        while (live && walk.next(u)) {
            const int n = u.u1 - u.u0;
            if (n <= 0) continue;
            const int t0 = tiles, unit = units;
            issue_s(true);
            for (int i = 0; i < n && live; ++i) {
                if (i + 1 < n) issue_s(false);        // one ahead, but not into the next unit: its rows are made ready when this one is done
                issue_o(t0 + i, i == 0, unit);
            }
        }
        if (leader) umma_commit(bar(&ctrl.drained));  // nothing of the tensor cores' is in flight when TMEM and shared memory are given up
        const long long c0 = clock64();
        while (!mbar_try_wait(bar(&ctrl.drained), 0))
            if (clock64() - c0 > kTimeoutCycles) break;
        __syncwarp();
    } else {
        // ============================================================ a key per thread
        const int q4 = warp & 3, key_lane = q4 * 32 + lane;      // the quarter of TMEM's lanes that this warp may access
        const int kt = tid - 64;                                 // 0 .. 127
        const uint32_t lane_addr = (uint32_t)(q4 * 32) << 16;
        const int64_t w = blockIdx.x;
        CutUnit cut{0, 0, 0, 0};
        int tiles = 0;
        // (after an abort the waits fall through and everybody goes on to the end together: nobody is left at a barrier)
        while (walk.next(u)) {
            const int n = max(u.u1 - u.u0, 0);
            auto token_of = [&](int r) { return (u.tile_row + min(r, u.n_rows - 1)) / group; };
            float m[ROWS], l[ROWS], rowf[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) m[r] = kNone, l[r] = 0.f;
            if (n > 0) {
                // ---- q's terms: four threads a row, 32 elements each
                const int row = kt >> 2, part = kt & 3;
                const bool have = row < u.n_rows;
                float x[32], amax = 0.f;
                if (have) {
                    const int token = token_of(row), qh = u.head * group + (u.tile_row + row - token * group);
                    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + ((int64_t)u.sq.row0 + token) * a.ldq + (int64_t)qh * kDim + part * 32;
#pragma unroll
                    for (int i = 0; i < 4; ++i) unpack<__nv_bfloat16>(ld128_rw_stream(q + i * 8), x + i * 8);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] = 0.f;
                }
#pragma unroll
                for (int i = 0; i < 32; ++i) amax = fmaxf(amax, fabsf(x[i]));
                amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
                amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
                const int e = amax > 0.f ? min(100, 7 - ((int)(__float_as_uint(amax) >> 23) - 127)) : 0;
                const float up = __uint_as_float((uint32_t)(e + 127) << 23);
                if (row < ROWS) {
                    if (part == 0) s_row[row] = a.scale_log2 * __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
                    for (int i = 0; i < 32; ++i) x[i] *= up;
#pragma unroll
                    for (int t = 0; t < kTermsQ; ++t)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t c[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t lo = split_pair(x[16 * h + 4 * i], x[16 * h + 4 * i + 1]);
                                c[i] = lo | (split_pair(x[16 * h + 4 * i + 2], x[16 * h + 4 * i + 3]) << 16);
                            }
                            *reinterpret_cast<uint4*>(smem + (q_at - base) + line_offset(t * ROWS + row, part * 32 + h * 16)) = make_uint4(c[0], c[1], c[2], c[3]);
                        }
                }
                fence_proxy_async_smem();
                mbar_arrive(bar(&ctrl.q_full));
                key_threads_sync();
#pragma unroll
                for (int r = 0; r < ROWS; ++r) rowf[r] = s_row[r];
            }
            for (int i = 0; i < n; ++i, ++tiles) {
                const int s = tiles % kStages, b = tiles & 1;
                wait_bar(bar(&ctrl.s_full[b]), (uint32_t)(tiles >> 1) & 1u, abort_flag, a.dev_status);
                wait_bar(bar(&ctrl.full[s]), (uint32_t)(tiles / kStages) & 1u, abort_flag, a.dev_status);      // (long complete: for the scales and V in shared memory)
                __syncwarp();
                tc_fence_after();
                float y[ROWS];
                {
                    uint32_t v[C::kNS];
                    tmem_load<C::kNS>(tmem + lane_addr + (b ? C::kSCol1 : C::kSCol0), v);
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) y[r] = fmaf(__uint_as_float(v[ROWS + r]), 1.f / kTermStep, __uint_as_float(v[r]));
                }
                tc_fence_before();
                mbar_arrive(bar(&ctrl.s_empty[b]));
                const float4 sc = s_scales[s][key_lane >> 4];
                const int key = u.sp.lo + (u.u0 + i) * kKeys + key_lane;
                // (the bounds of a tile are the same for all threads; whether a page is missing is not known to all, but matters to its keys only)
                const int key0 = key - key_lane;
                const bool border = key0 + kKeys > u.hi_min || key0 < u.lo_max;
                float ks = fmaxf(sc.x, 1.17549435e-38f);
                bool hidden = false, poisoned = false;
                if (border || sc.w == 0.f) {
                    // A value that no row sees counts as zero; a NaN among the codes of one becomes a NaN in the scores of the rows that see it and a
                    // zero here, so that it cannot reach the others through their weight of zero.
                    hidden = sc.w == 0.f || key >= u.hi_max || key < u.lo_min;
                    uint8_t* line = smem + s * kStageBytes + kTileBytes + key_lane * 128;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        uint4* at = reinterpret_cast<uint4*>(line + ((c ^ key_lane) & 7) * 16);
                        uint4 x = hidden ? make_uint4(0, 0, 0, 0) : *at;
                        const uint32_t n0 = e4m3x4_nan_bits(x.x), n1 = e4m3x4_nan_bits(x.y), n2 = e4m3x4_nan_bits(x.z), n3 = e4m3x4_nan_bits(x.w);
                        const bool nan = (n0 | n1 | n2 | n3) != 0;
                        poisoned |= nan;
                        if (hidden || nan)
                            *at = make_uint4(x.x & ~((n0 >> 7) * 0xFFu), x.y & ~((n1 >> 7) * 0xFFu), x.z & ~((n2 >> 7) * 0xFFu), x.w & ~((n3 >> 7) * 0xFFu));
                    }
                    if (hidden) ks = 1.f;
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) {
                        const int token = token_of(r);
                        const bool sees = !hidden && key < upper_key(a, u.sq, token) && key >= lower_key(a, u.sq, token);
                        y[r] = !sees ? -INFINITY : poisoned ? kNan : y[r];
                    }
                }
                // y: the weight's exponent over the row's reference
                bool over = false;
#pragma unroll
                for (int r = 0; r < ROWS; ++r) {
                    y[r] = fmaf(y[r], fmaxf(rowf[r] * ks, 1.17549435e-38f), sc.y);
                    over |= y[r] - m[r] > kTop + kSlack;
                }
                if (key_threads_any(over)) {
                    float shrink[ROWS];
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) {
                        const float top = warp_max(y[r]);
                        if (lane == 0) s_part[q4][r] = top;
                    }
                    key_threads_sync();
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) {
                        const float top = fmaxf(fmaxf(s_part[0][r], s_part[1][r]), fmaxf(s_part[2][r], s_part[3][r]));
                        const float next = top - m[r] > kTop ? top - kTop : m[r];
                        shrink[r] = ex2(m[r] - next);
                        m[r] = next;
                        l[r] *= shrink[r];
                    }
                    if (i > 0) {                      // what is in O already: the MMAs of the tile before are done, those of this one wait for its weights
                        wait_bar(bar(&ctrl.p_empty[b ^ 1]), (uint32_t)((tiles - 1) >> 1) & 1u, abort_flag, a.dev_status);
                        __syncwarp();
                        tc_fence_after();
#pragma unroll
                        for (int t = 0; t < kTermsP; ++t) {
                            uint32_t v[ROWS];
                            tmem_load<ROWS>(tmem + lane_addr + C::kOCol + t * ROWS, v);
#pragma unroll
                            for (int r = 0; r < ROWS; ++r) v[r] = __float_as_uint(__uint_as_float(v[r]) * shrink[r]);
#pragma unroll
                            for (int r = 0; r < ROWS; r += 8) tmem_st<8>(tmem + lane_addr + C::kOCol + t * ROWS + r, v + r);
                        }
                        tmem_wait_st();
                        tc_fence_before();
                    }
                    key_threads_sync();               // (s_part is free again)
                }
                if (tiles >= 2) wait_bar(bar(&ctrl.p_empty[b]), ((uint32_t)(tiles >> 1) & 1u) ^ 1u, abort_flag, a.dev_status);
                uint8_t* const p = smem + (p_at - base) + b * C::kPBytes;
#pragma unroll
                for (int r = 0; r < ROWS; r += 2) {
                    float w0 = ex2(y[r] - m[r]), w1 = ex2(y[r + 1] - m[r + 1]);
                    l[r] = fmaf(w0, sc.z, l[r]), l[r + 1] = fmaf(w1, sc.z, l[r + 1]);
#pragma unroll
                    for (int t = 0; t < kTermsP; ++t) {
                        const uint32_t c = split_pair(w0, w1);
                        p[line_offset(t * ROWS + r, key_lane)] = (uint8_t)c;
                        p[line_offset(t * ROWS + r + 1, key_lane)] = (uint8_t)(c >> 8);
                    }
                }
                fence_proxy_async_smem();
                tc_fence_before();
                mbar_arrive(bar(&ctrl.p_full[b]));
            }
            // ---- the unit's result, or a piece of it: an element per thread
            const bool begins = u.first == 0, ends = u.last == u.sp.steps, whole = begins && ends;
            if (begins && !ends) {
                cut.b = u.b, cut.row_tile = u.tile, cut.head = u.head;
                cut.pieces = walk.pieces(u, w);
            }
            float o[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) o[r] = 0.f;
            if (n > 0) {
                const int t = tiles - 1;
                wait_bar(bar(&ctrl.p_empty[t & 1]), (uint32_t)(t >> 1) & 1u, abort_flag, a.dev_status);
                __syncwarp();
                tc_fence_after();
                float f = 1.f;
#pragma unroll
                for (int z = 0; z < kTermsP; ++z, f /= kTermStep) {
                    uint32_t v[ROWS];
                    tmem_load<ROWS>(tmem + lane_addr + C::kOCol + z * ROWS, v);
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) o[r] = fmaf(__uint_as_float(v[r]), f, o[r]);
                }
                tc_fence_before();
                mbar_arrive(bar(&ctrl.o_empty));
            }
            const bool live = *abort_flag == 0;       // (nothing of an aborted call is stored)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
#pragma unroll
                for (int z = 16; z > 0; z >>= 1) l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], z);
                if (lane == 0) s_part[q4][r] = l[r];
            }
            key_threads_sync();
            float* slot = slots + (2 * w + (begins ? 1 : 0)) * (int64_t)slot_floats(ROWS, kDim);
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                if (r >= u.n_rows || !live) continue;
                const float sum = (s_part[0][r] + s_part[1][r]) + (s_part[2][r] + s_part[3][r]);
                if (whole) {
                    const int token = token_of(r), qh = u.head * group + (u.tile_row + r - token * group);
                    const int64_t orow = (int64_t)u.sq.row0 + token;
                    static_cast<__nv_bfloat16*>(a.out)[orow * a.ldo + (int64_t)qh * kDim + key_lane] = __float2bfloat16(sum == 0.f ? 0.f : o[r] / sum);
                    if (a.lse != nullptr && kt == 0) a.lse[orow * a.heads + qh] = sum == 0.f ? -INFINITY : (m[r] + log2f(sum)) * 0.69314718056f;
                } else {
                    slot[2 * ROWS + r * kDim + key_lane] = o[r];
                    if (kt == 0) slot[r] = m[r], slot[ROWS + r] = sum;
                }
            }
            key_threads_sync();                       // (s_part, s_row)
        }
        if (kt == 0) cuts[w] = *abort_flag == 0 ? cut : CutUnit{0, 0, 0, 0};
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem, C::kTmemCols);
}

template <int ROWS>
int64_t share_count() { return (int64_t)sm_count() * kWaves; }

template <int ROWS>
size_t bytes_needed() { return cut_bytes(share_count<ROWS>()) + (size_t)(2 * share_count<ROWS>() * slot_floats(ROWS, kDim)) * sizeof(float); }

template <int ROWS>
molora_status_t launch(const AttendArgs& a, void* ws, cudaStream_t s)
{
    using C = Cfg<ROWS>;
    static bool ready[kMaxDevices] = {};
    bool& done = ready[device_slot()];
    if (!done) {
        if (cudaFuncSetAttribute(attend_stream_kernel<ROWS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmem) != cudaSuccess) return MOLORA_ERR_CUDA;
        done = true;
    }
    CUtensorMap tm_k, tm_v;
    const uint64_t rows = ((uint64_t)a.c.n_pages * (uint64_t)a.c.kv_heads) << a.c.page_log2;
    const uint32_t box = 1u << a.c.page_log2;
    if (!make_tensor_map_bytes_2d(&tm_k, a.c.k, kDim, rows, kDim, box, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_tensor_map_bytes_2d(&tm_v, a.c.v, kDim, rows, kDim, box, CU_TENSOR_MAP_SWIZZLE_128B))
        return MOLORA_ERR_CUDA;
    const int64_t shares = share_count<ROWS>();
    CutUnit* cuts = static_cast<CutUnit*>(ws);
    float* slots = reinterpret_cast<float*>(static_cast<char*>(ws) + cut_bytes(shares));
    if (launch_kernel(attend_stream_kernel<ROWS>, dim3((unsigned)shares), dim3(kThreads), C::kSmem, s, 1, true, a, tm_k, tm_v, cuts, slots) != cudaSuccess)
        return MOLORA_ERR_CUDA;
    return cuda_ok(launch_kernel(attend_join_kernel<__nv_bfloat16, kDim, ROWS>, dim3((unsigned)shares, ROWS / 8), dim3(kJoinWarps * 32), 0, s, 1, true, a,
                                 static_cast<const CutUnit*>(cuts), static_cast<const float*>(slots)));
}

}  // namespace

// bf16, heads of 128, up to 32 rows; a pool that TMA's coordinates reach (and that there is)
bool attend_stream_eligible(const KvView& c, molora_dtype_t dt, int64_t rows)
{
    return dt == MOLORA_BF16 && c.dim == kDim && rows <= 32 && c.n_pages > 0 && (((int64_t)c.n_pages * c.kv_heads) << c.page_log2) <= INT32_MAX;
}

size_t attend_stream_workspace_bytes(int64_t rows)
{
    return rows <= 8 ? bytes_needed<8>() : rows <= 16 ? bytes_needed<16>() : rows <= 24 ? bytes_needed<24>() : bytes_needed<32>();
}

molora_status_t launch_attend_stream(const AttendArgs& a, int64_t rows, void* ws, cudaStream_t s)
{
    return rows <= 8 ? launch<8>(a, ws, s) : rows <= 16 ? launch<16>(a, ws, s) : rows <= 24 ? launch<24>(a, ws, s) : launch<32>(a, ws, s);
}

}  // namespace molora
