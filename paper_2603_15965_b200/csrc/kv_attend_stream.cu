// Attention over the paged 8-bit cache for up to 32 query rows, bf16, heads of 128 (molora_kv_attend): decode and drafted tokens.
//
// The codes of keys and values go from memory to the tensor cores as they are: TMA brings blocks of the cache into shared
// memory, tcgen05.mma (kind::f8f6f4) reads them there, and no thread ever touches them.  What is not 8 bits wide is
// written as a sum of e4m3 terms, each in columns of its own:
//   q (8 significant bits) = t1 + t2 / 32, exactly: the rest that rounding to 4 bits leaves of 8 fits 4; a power of two per row brings the largest
//       element to [2^7, 2^8), so elements below 2^-14 of it are off by at most 2^-22 of it
//   a weight, rounded to fp16 (11 bits), = t1 + t2 / 32 + t3 / 1024, exactly (to 2^-20 where a row's largest is 32 or more)
//   S^T [128 keys x 2 rows]   = K Q^T     A = K tile, keys the 128 lanes of TMEM; B = q's terms
//   O^T [128 elements x 3 rows] += V^T P^T  A = V tile read across (MN-major); B = the weights' terms
// with the key as the lane a thread owns one key: the scales of its block, its mask and its weights are its own, and reductions
// over keys are needed only when a row's reference moves (a score 2^8 over the weight of one) and at the end of a unit.
// A CTA is two workers (one for 32 rows), each with a share of the units, a ring, operands, TMEM columns and warps of its own, so that the
// latencies of one -- a chain of S, weights, O per tile, and the end of one unit before the next -- are filled by the other:
//   copies    pages, scales and TMA: 2 to 5 tiles of 128 keys, 32 KB each, in flight or in use
//   MMAs      those of S one tile ahead of those of O
//   rows      two warps: the rows of the units, one or two units ahead: q's terms, factors, bounds, places of the results
//   groups    of four warps, each with 4 or 8 of the rows: a key per thread, weights and their terms into shared memory; at the end of a unit an
//             element per thread.  Code that runs once a unit is kept short and the state of a unit in shared memory: instructions that are not in the
//             cache cost more than what they do.
// (One worker whose groups took alternate units: 196 us against 172 for 256 sequences of 3 to 4095 tokens and two rows, 81 against 68 for 64
// sequences of 100 to 2043 tokens and 20 rows.)
// Weights are at most 2^8; the scale of a block of K multiplies its scores, that of V its weights once the sum has them (kv_attend.cuh), so that
// weights have the size of what they contribute.
// What bounds it: for few rows 32 KB a tile from HBM (1.06 GB in 166 to 170 us, 6.2 to 6.4 TB/s, 95 to 97 % of a copy's rate); for 20 rows the instructions, 6500 of
// all warps a tile, at 51 % of the schedulers' slots (158 MB in 68 us); for a single short sequence (776 tokens: 10.6 to 11.2 us with the join) the
// chain of first reads -- lengths, page, scales, codes -- and two launches.
#include <algorithm>

#include "kv_attend.cuh"
#include "pipeline.cuh"
#include "tensor_map.cuh"

namespace molora {
namespace {

constexpr int kDim = 128, kKeys = 128;
constexpr int kRoleWarps = 4;                // of a worker: copies, MMAs, rows (two)
constexpr int kMaxStages = 5;                // tiles in flight or in use
constexpr int kTileBytes = kKeys * kDim, kStageBytes = 2 * kTileBytes;      // K, then V
constexpr int kMinShare = 2;                 // tiles
constexpr int kTermsQ = 2, kTermsP = 3;
constexpr float kTermStep = 32.f;            // a term's weight against the next
constexpr float kTop = 5.f, kSlack = 3.f;    // a row's largest weight when its reference is set: 2^5; it may grow by 2^3 before the reference moves
constexpr float kNan = __builtin_nanf("");

template <int ROWS>
struct Cfg {
    static constexpr int kRowsPerGroup = ROWS >= 16 ? 8 : 4, kGroups = ROWS / kRowsPerGroup;
    static constexpr int kWorkers = ROWS <= 24 ? 2 : 1;
    static constexpr int kUnitCost = ROWS < 16 ? 2 : 3;                                   // tiles that a unit's rows and results cost
    static constexpr int kKeyThreads = 128 * kGroups, kFirstGroupWarp = kRoleWarps * kWorkers;      // (kKeyThreads: of a worker)
    static constexpr int kThreads = 32 * kFirstGroupWarp + kWorkers * kKeyThreads;
    static_assert(kThreads <= 1024, "threads");
    static constexpr int kNS = (kTermsQ * ROWS + 15) / 16 * 16;           // columns of S and of O: multiples of 16, the last ones unused
    static constexpr int kNP = (kTermsP * ROWS + 15) / 16 * 16;
    static constexpr int kQBytes = kNS / 8 * 1024, kPBytes = kNP / 8 * 1024;
    static constexpr uint32_t kSCol1 = 64, kOCol = 128, kWorkerCols = 256, kTmemCols = kWorkers * kWorkerCols;      // S of even tiles, of odd tiles, O
    static_assert(kNS <= 64 && kNP <= 128, "TMEM columns");
    static constexpr int kStages = kWorkers == 1 ? 5 : ROWS <= 16 ? 3 : 2;
    static constexpr int kQAt = kStages * kStageBytes, kPAt = kQAt + 2 * kQBytes, kWorkerBytes = kPAt + kPBytes;
    static constexpr size_t kSmem = 1024 + (size_t)kWorkers * kWorkerBytes;
    static_assert(kStages <= kMaxStages, "stages");
};

// A warp arrives as one: arrivals of single threads at a barrier follow one another.  A thread that waits for a phase by its parity must have seen
// the phase before it; hence q_ready (for the MMAs) beside q_full, since units without tiles pass the MMAs by.
struct Control {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t s_full[2], s_empty[2], p_full, p_empty;
    uint64_t q_full[2], q_ready[2], q_empty[2];
    uint64_t drained;
};
// A tile in the ring: the scales of every 16 keys (of K, logarithm of V's, V's, whether their page can be used), and where in its unit it stands.
struct Tile {
    float4 scale[8];
    int32_t kind;                             // kFirst: begins a unit, kOdd: of an odd one; kLast: no tile, there are no more
};
enum : int32_t { kFirst = 1, kOdd = 2, kLast = 4 };
// A unit and its rows.
template <int ROWS>
struct Rows {
    float factor[ROWS];                       // of a score: scale, powers of two
    int32_t lower[ROWS], upper[ROWS];         // keys that the row sees
    int64_t out[ROWS], lse[ROWS];             // places in out and lse
    int32_t tiles;                            // -1: there are no more units
    int32_t key0, n_rows;                     // first key of the first tile
    int32_t hi_min, hi_max, lo_min, lo_max;
    int32_t slot;                             // where a piece goes; -1: the unit is whole
};

// barriers of a group (1 + group) and of a worker (14 + worker)
template <int THREADS>
__device__ __forceinline__ void sync_threads_of(int id) { asm volatile("barrier.cta.sync %0, %1;" ::"r"(id), "n"(THREADS) : "memory"); }
template <int THREADS>
__device__ __forceinline__ bool threads_any(int id, bool v)
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred P, Q;\n\tsetp.ne.b32 P, %1, 0;\n\tbarrier.cta.red.or.pred Q, %2, %3, P;\n\tselp.u32 %0, 1, 0, Q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)v), "r"(id), "n"(THREADS)
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

// N = 4 or 8 neighbouring columns
template <int N>
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t* v)
{
    if constexpr (N == 4) ptx::tmem_ld_x4(addr, v);
    else ptx::tmem_ld_x8(addr, v);
}

template <int ROWS>
__global__ void __launch_bounds__(Cfg<ROWS>::kThreads, 1)
    attend_stream_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                         CutUnit* __restrict__ cuts, float* __restrict__ slots)
{
    using C = Cfg<ROWS>;
    constexpr int RPG = C::kRowsPerGroup, W = C::kWorkers;
    using namespace ptx;
    __shared__ Control ctrls[W];
    __shared__ uint32_t s_tmem_base;
    __shared__ int s_abort;
    __shared__ ShareStart s_start[W];
    __shared__ Tile s_tiles_all[W][C::kStages];
    __shared__ Rows<ROWS> s_rows_all[W][2];
    __shared__ float s_part[W * C::kGroups][4][RPG];
    extern __shared__ uint8_t smem_raw[];
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // which worker the warp belongs to
    const int worker = warp < C::kFirstGroupWarp ? warp / kRoleWarps : (warp - C::kFirstGroupWarp) / (4 * C::kGroups);
    const uint32_t raw = smem_u32(smem_raw), first = (raw + 1023u) & ~1023u, base = first + (uint32_t)(worker * C::kWorkerBytes);
    uint8_t* const smem = smem_raw + (base - raw);
    const uint32_t q_at = base + C::kQAt, p_at = base + C::kPAt;
    volatile int* abort_flag = &s_abort;
    Control& ctrl = ctrls[worker];
    Tile* const s_tiles = s_tiles_all[worker];
    Rows<ROWS>* const s_rows = s_rows_all[worker];
    auto bar = [](const uint64_t* b) { return smem_u32(b); };

    if (tid < W) {
        Control& c = ctrls[tid];
        for (int s = 0; s < C::kStages; ++s) mbar_init(bar(&c.full[s]), 1), mbar_init(bar(&c.empty[s]), 1);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(&c.s_full[i]), 1), mbar_init(bar(&c.s_empty[i]), C::kKeyThreads / 32);
            mbar_init(bar(&c.q_full[i]), 2), mbar_init(bar(&c.q_ready[i]), 2), mbar_init(bar(&c.q_empty[i]), C::kKeyThreads / 32);
        }
        mbar_init(bar(&c.p_full), C::kKeyThreads / 32), mbar_init(bar(&c.p_empty), 1);
        mbar_init(bar(&c.drained), 1);
        if (tid == 0) {
            prefetch_tensormap(&tm_k);
            prefetch_tensormap(&tm_v);
            s_abort = 0;
        }
        fence_mbar_init();
    }
    // operand lines of no row are zero for good
    constexpr int kLines = (2 * C::kQBytes + C::kPBytes) / 16;
#pragma unroll
    for (int w = 0; w < W; ++w)
        for (int i = tid; i < kLines; i += C::kThreads)
            *reinterpret_cast<uint4*>(smem_raw + (first - raw) + w * C::kWorkerBytes + C::kQAt + i * 16) = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
    grid_dependency_wait();
    if (warp == 1) take_tmem(&s_tmem_base, C::kTmemCols);
    const int group = a.group, plog = a.c.page_log2;
    cut_shares<C::kThreads, W>(a, (int64_t)blockIdx.x * W, (int64_t)gridDim.x * W, kMinShare, s_start,
                               [&](const Sequence& sq) { return steps_of<ROWS, kKeys, C::kUnitCost>(a, sq, group); });
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_dependency_trigger();                        // (not before TMEM is mine)
    const uint32_t tmem = s_tmem_base + (uint32_t)worker * C::kWorkerCols;
    const int64_t share = (int64_t)blockIdx.x * W + worker;
    Walk<ROWS, kKeys, C::kUnitCost> walk(a);
    const int role = warp < C::kFirstGroupWarp ? warp % kRoleWarps : kRoleWarps;
    if (role < kRoleWarps && role != 1) walk.begin(s_start[worker], share, C::kThreads);

    if (role == 0) {
        // ============================================================ pages, scales, copies
        const uint32_t page_bytes = (uint32_t)kDim << plog;
        const int step = kKeys >> plog;                       // pages of a tile, a copy of K and one of V each
        int tiles = 0, units = 0;
        Unit u;
        // the place of the next tile, when it is free
        auto claim = [&]() {
            const int s = tiles % C::kStages;
            if (tiles >= C::kStages) wait_bar(bar(&ctrl.empty[s]), ((uint32_t)(tiles / C::kStages) & 1u) ^ 1u, abort_flag, a.dev_status);
            __syncwarp();
            return s;
        };
        for (; *abort_flag == 0 && walk.next(u); ++units) {
            int group0 = 0;                                   // first of the 32 pages whose ids and scales the lanes hold
            int32_t page_id = -1;
            float ks = 0.f, vs = 0.f;
            float4 sc = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int i = u.u0; i < u.u1; ++i) {
                const int key0 = u.sp.lo + i * kKeys, page = key0 >> plog;
                const bool fresh = i == u.u0 || page + step > group0 + 32;
                if (fresh) {
                    group0 = page;
                    page_id = -1;
                    if (((int64_t)(page + lane) << plog) < u.hi_max) {
                        page_id = ld_dependent(a.c.table + (int64_t)u.b * a.c.ld_table + page + lane);
                        if (page_id < 0 || page_id >= a.c.n_pages) {
                            page_id = -1;
                            if (a.dev_status != nullptr) atomicOr(a.dev_status, MOLORA_DEV_BAD_SEQUENCE);
                        } else {
                            const int64_t block = (int64_t)page_id * a.c.kv_heads + u.head;
                            ks = ld_dependent(a.c.k_scale + block), vs = ld_dependent(a.c.v_scale + block);
                        }
                    }
                    __syncwarp();
                }
                const int32_t id = __shfl_sync(0xFFFFFFFFu, page_id, (page - group0 + lane) & 31);
                const bool copies = lane < step && id >= 0;
                const uint32_t bytes = 2u * page_bytes * (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, copies));
                const int row = (int)((((int64_t)id * a.c.kv_heads + u.head) << plog) + (key0 & ((1 << plog) - 1)));
                const int s = claim();
                if (*abort_flag) break;
                // the copies go out while the scales are on their way: the phase does not end before lane 0's arrival, which tells how many bytes they are
                if (copies) {
                    const uint32_t dst = base + (uint32_t)(s * kStageBytes) + (uint32_t)lane * page_bytes;
                    tma_load_2d(dst, &tm_k, 0, row, bar(&ctrl.full[s]));
                    tma_load_2d(dst + kTileBytes, &tm_v, 0, row, bar(&ctrl.full[s]));
                }
                __syncwarp();
                if (fresh) {
                    const float v = read_v_scale(vs);
                    sc = page_id >= 0 ? make_float4(ks, log2f(v), v, 1.f) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
                const int mine = (page - group0 + (((lane & 7) * 16) >> plog)) & 31;           // the page of 16 keys
                float4 g;
                g.x = __shfl_sync(0xFFFFFFFFu, sc.x, mine), g.y = __shfl_sync(0xFFFFFFFFu, sc.y, mine);
                g.z = __shfl_sync(0xFFFFFFFFu, sc.z, mine), g.w = __shfl_sync(0xFFFFFFFFu, sc.w, mine);
                if (lane < 8) s_tiles[s].scale[lane] = g;
                if (lane == 0) s_tiles[s].kind = (i == u.u0 ? kFirst : 0) | ((units & 1) ? kOdd : 0);
                __syncwarp();
                if (lane == 0) mbar_arrive_expect_tx(bar(&ctrl.full[s]), bytes);
                ++tiles;
            }
        }
        const int last = claim();
        if (*abort_flag == 0 && lane == 0) {
            s_tiles[last].kind = kLast;
            mbar_arrive(bar(&ctrl.full[last]));
        }
        // every copy has landed before the memory is given up: otherwise they have been worked on, but an abort may come with some in flight
        // (this wait has its own limit)
        if (*abort_flag)
            for (int i = 0; i < min(tiles, C::kStages); ++i) {
                const int z = tiles - 1 - i;
                const long long t0 = clock64();
                while (!mbar_try_wait(bar(&ctrl.full[z % C::kStages]), (uint32_t)(z / C::kStages) & 1u))
                    if (clock64() - t0 > kTimeoutCycles) break;
            }
    } else if (role == 1) {
        // ============================================================ MMAs
        const bool leader = elect_one();
        const uint32_t tm = __shfl_sync(0xFFFFFFFFu, tmem, 0);
        constexpr uint32_t idesc_s = idesc_e4m3_f32(kKeys, C::kNS, 0, 0), idesc_o = idesc_e4m3_f32(kDim, C::kNP, 1, 0);
        constexpr uint32_t kL128 = swizzle_layout_type(Swizzle::B128);
        const uint64_t k_desc = smem_desc(base, 16, 1024, kL128), v_desc = smem_desc(base + kTileBytes, 0, 1024, kL128);
        const uint64_t q_desc = smem_desc(q_at, 16, 1024, kL128), p_desc = smem_desc(p_at, 16, 1024, kL128);
        bool live = true;
        int ahead = 0, done = 0;                      // tiles whose S, whose O has been asked for
        int ready0 = 0, ready1 = 0;                   // units with tiles whose rows have been waited for, per buffer
        // S of a tile goes out before O of the one before it, but nothing that is not there yet is waited for while an O is due.
        bool end = false;                             // no more tiles
        bool first_a = false, first_b = false;        // of the tiles in between, in order: whether they begin a unit
        auto there = [&](const uint64_t* b, uint32_t parity, bool wait) {
            if (wait) return live = wait_bar(bar(b), parity, abort_flag, a.dev_status) && live;
            return __shfl_sync(0xFFFFFFFFu, (int)mbar_test_wait(bar(b), parity), 0) != 0;
        };
        while (live) {
            const bool due = ahead != done;
            const int s = ahead % C::kStages;
            bool go = !end && ahead - done < 2 && there(&ctrl.full[s], (uint32_t)(ahead / C::kStages) & 1u, !due);
            const int kind = go ? *const_cast<volatile int32_t*>(&s_tiles[s].kind) : 0, qb = (kind & kOdd) ? 1 : 0;
            if (kind & kLast) end = true, go = false;
            if (go && (kind & kFirst) && !there(&ctrl.q_ready[qb], (uint32_t)(qb == 0 ? ready0 : ready1) & 1u, !due)) go = false;
            if (go && live) {
                const int b = ahead & 1;
                if (kind & kFirst) ++(qb == 0 ? ready0 : ready1);
                if (ahead >= 2) live = wait_bar(bar(&ctrl.s_empty[b]), ((uint32_t)(ahead >> 1) & 1u) ^ 1u, abort_flag, a.dev_status) && live;
                tc_fence_after();
                if (leader && live) {
                    const uint64_t at = (uint64_t)(s * (kStageBytes >> 4)), qa = (uint64_t)(qb * (C::kQBytes >> 4));
#pragma unroll
                    for (int j = 0; j < 4; ++j) umma_f8(tm + (b ? C::kSCol1 : 0u), k_desc + at + j * 2, q_desc + qa + j * 2, idesc_s, j > 0);      // 32 elements a step
                    umma_commit(bar(&ctrl.s_full[b]));
                }
                __syncwarp();
                if (ahead == done) first_a = (kind & kFirst) != 0;
                else first_b = (kind & kFirst) != 0;
                ++ahead;
                if (ahead - done < 2) continue;
            }
            if (ahead == done) {
                if (end) break;
                continue;
            }
            const int so = done % C::kStages;
            live = wait_bar(bar(&ctrl.p_full), (uint32_t)done & 1u, abort_flag, a.dev_status) && live;
            tc_fence_after();
            if (leader && live) {
                const uint64_t at = (uint64_t)(so * (kStageBytes >> 4));
#pragma unroll
                for (int j = 0; j < 4; ++j)           // 32 keys a step: 4 groups of 8 lines of V
                    umma_f8(tm + C::kOCol, v_desc + at + j * (4096 >> 4), p_desc + j * 2, idesc_o, !first_a || j > 0);
                umma_commit(bar(&ctrl.p_empty));
                umma_commit(bar(&ctrl.empty[so]));
            }
            __syncwarp();
            ++done;
            first_a = first_b;
        }
        if (leader) umma_commit(bar(&ctrl.drained));  // nothing of the tensor cores' is in flight when TMEM and shared memory are given up
        const long long c0 = clock64();
        while (!mbar_try_wait(bar(&ctrl.drained), 0))
            if (clock64() - c0 > kTimeoutCycles) break;
        __syncwarp();
    } else if (role < kRoleWarps) {
        // ============================================================ the rows of the units, one unit ahead: pairs of rows in turn
        Unit u;
        CutUnit cut{};
        const int turn = role - 2;
        for (int k = 0;; ++k) {
            const bool more = walk.next(u);
            if (k >= 2) wait_bar(bar(&ctrl.q_empty[k & 1]), ((uint32_t)(k >> 1) & 1u) ^ 1u, abort_flag, a.dev_status);
            if (*abort_flag) break;
            __syncwarp();
            Rows<ROWS>& rows = s_rows[k & 1];
            if (!more) {
                if (lane == 0) {
                    if (turn == 0) rows.tiles = -1;
                    mbar_arrive(bar(&ctrl.q_full[k & 1]));
                }
                break;
            }
            const bool begins = u.first == 0, whole = begins && u.last == u.sp.steps;
            if (begins && !whole) cut.row0 = u.sq.row0, cut.tile_row = u.tile_row, cut.rows = u.n_rows, cut.head = u.head, cut.pieces = walk.pieces(u, share);
            const int n = max(u.u1 - u.u0, 0);
            if (turn == 0 && lane == 0) {
                rows.tiles = n, rows.key0 = u.sp.lo + u.u0 * kKeys, rows.n_rows = u.n_rows;
                rows.hi_min = u.hi_min, rows.hi_max = u.hi_max, rows.lo_min = u.lo_min, rows.lo_max = u.lo_max;
                rows.slot = whole ? -1 : (int)(2 * share + (begins ? 1 : 0));
            }
            const int row = min(lane, u.n_rows - 1);
            const int token = (u.tile_row + row) / group, qh = u.head * group + (u.tile_row + row - token * group);
            const int64_t in = ((int64_t)u.sq.row0 + token) * a.ldq + (int64_t)qh * kDim;
            if (turn == 0 && lane < ROWS) {
                rows.lower[lane] = lower_key(a, u.sq, token);
                rows.upper[lane] = upper_key(a, u.sq, token);
                rows.out[lane] = ((int64_t)u.sq.row0 + token) * a.ldo + (int64_t)qh * kDim;
                rows.lse[lane] = ((int64_t)u.sq.row0 + token) * a.heads + qh;
            }
            uint4 q[ROWS / 4];                        // half a warp a row, eight elements a lane; asked for together
#pragma unroll
            for (int i = 0; i < ROWS / 4; ++i) {
                const int r = 4 * i + 2 * turn + (lane >> 4);
                const int64_t from = __shfl_sync(0xFFFFFFFFu, in, r);
                q[i] = r < u.n_rows ? ld128_rw_stream(static_cast<const __nv_bfloat16*>(a.q) + from + (lane & 15) * 8) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < ROWS / 4; ++i) {
                const int r = 4 * i + 2 * turn + (lane >> 4), chunk = lane & 15;
                float x[8], amax = 0.f;
                unpack<__nv_bfloat16>(q[i], x);
#pragma unroll
                for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, o));
                const RowScale by = row_scale<7>(amax);
                if (chunk == 0) rows.factor[r] = a.scale_log2 * by.down;
#pragma unroll
                for (int z = 0; z < 8; ++z) x[z] *= by.up;
#pragma unroll
                for (int z = 0; z < kTermsQ; ++z) {
                    uint2 c;
                    c.x = split_pair(x[0], x[1]);
                    c.x |= split_pair(x[2], x[3]) << 16;
                    c.y = split_pair(x[4], x[5]);
                    c.y |= split_pair(x[6], x[7]) << 16;
                    *reinterpret_cast<uint2*>(smem + (q_at - base) + (k & 1) * C::kQBytes + line_offset(z * ROWS + r, chunk * 8)) = c;
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(bar(&ctrl.q_full[k & 1]));
                if (n > 0) mbar_arrive(bar(&ctrl.q_ready[k & 1]));
            }
        }
        if (turn == 0 && lane == 0) cuts[share] = *abort_flag == 0 ? cut : CutUnit{};
    } else {
        // ============================================================ a key per thread
        const int q4 = warp & 3, key_lane = q4 * 32 + lane;      // the quarter of TMEM's lanes that this warp may access
        const int all = (warp - C::kFirstGroupWarp) >> 2, gr = all % C::kGroups, r0 = gr * RPG;
        const uint32_t lane_addr = (uint32_t)(q4 * 32) << 16;
        const uint32_t p_off = (uint32_t)(((((key_lane >> 4) ^ r0) & 7) << 4) + (key_lane & 15));      // of this key in line r0 of the weights; r bits 4.. on
        int tiles = 0;                                // so far
        for (int k = 0;; ++k) {
            wait_bar(bar(&ctrl.q_full[k & 1]), (uint32_t)(k >> 1) & 1u, abort_flag, a.dev_status);
            // after an abort the waits fall through: a worker's groups leave here together, or go on to the end of the unit together, so that
            // nobody is left at a barrier
            if (threads_any<C::kKeyThreads>(14 + worker, *abort_flag != 0)) break;
            const Rows<ROWS>& rows = s_rows[k & 1];
            const int n = rows.tiles, n_rows = rows.n_rows, hi_min = rows.hi_min, hi_max = rows.hi_max, lo_min = rows.lo_min, lo_max = rows.lo_max;
            if (n < 0) break;
            int key0 = rows.key0;
            float m[RPG], l[RPG];
#pragma unroll
            for (int r = 0; r < RPG; ++r) m[r] = kNone, l[r] = 0.f;
#pragma unroll 1
            for (int i = 0; i < n; ++i, ++tiles, key0 += kKeys) {
                const int b = tiles & 1;
                wait_bar(bar(&ctrl.s_full[b]), (uint32_t)(tiles >> 1) & 1u, abort_flag, a.dev_status);
                const int s = tiles % C::kStages;
                wait_bar(bar(&ctrl.full[s]), (uint32_t)(tiles / C::kStages) & 1u, abort_flag, a.dev_status);      // (long complete: for what was written there)
                __syncwarp();
                tc_fence_after();
                const float4 sc = s_tiles[s].scale[key_lane >> 4];
                float y[RPG];
                {
                    uint32_t v0[RPG], v1[RPG];
                    const uint32_t at = tmem + lane_addr + (b ? C::kSCol1 : 0u) + r0;
                    tmem_load<RPG>(at, v0);
                    tmem_load<RPG>(at + ROWS, v1);
                    tmem_wait_ld();
#pragma unroll
                    for (int r = 0; r < RPG; ++r) y[r] = fmaf(__uint_as_float(v1[r]), 1.f / kTermStep, __uint_as_float(v0[r]));
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&ctrl.s_empty[b]));
                const int key = key0 + key_lane;
                const bool border = key0 + kKeys > hi_min || key0 < lo_max;
                // e: the logarithm of the key's part of the row's sum, over the row's reference; with V's, that of its weight
                float e[RPG], top = -INFINITY;
#pragma unroll
                for (int r = 0; r < RPG; ++r) {
                    y[r] *= rows.factor[r0 + r] * sc.x;
                    e[r] = y[r] - m[r];
                }
                const bool hidden = sc.w == 0.f || key >= hi_max || key < lo_min;      // no row sees the key, or its page cannot be used
                if (border || hidden) {
                    // A value that no row sees counts as zero; a NaN among the codes of one becomes a NaN in the scores of the rows that see it and a
                    // zero here, so that it cannot reach the others through their weight of zero.
                    uint8_t* line = smem + s * kStageBytes + kTileBytes + key_lane * 128;
                    bool nan = false;
                    if (!hidden)
#pragma unroll 2
                        for (int c = 0; c < 8; ++c) {
                            const uint4 x = *reinterpret_cast<const uint4*>(line + ((c ^ lane) & 7) * 16);
                            nan |= (e4m3x4_nan_bits(x.x) | e4m3x4_nan_bits(x.y) | e4m3x4_nan_bits(x.z) | e4m3x4_nan_bits(x.w)) != 0;
                        }
                    if (border && C::kGroups > 1) sync_threads_of<C::kKeyThreads>(14 + worker);      // every group has looked
                    if (gr == 0 && (hidden || nan))
#pragma unroll 2
                        for (int c = 0; c < 8; ++c) {
                            uint4 x = *reinterpret_cast<const uint4*>(line + ((c ^ lane) & 7) * 16);
                            x.x &= hidden ? 0u : ~((e4m3x4_nan_bits(x.x) >> 7) * 0xFFu), x.y &= hidden ? 0u : ~((e4m3x4_nan_bits(x.y) >> 7) * 0xFFu);
                            x.z &= hidden ? 0u : ~((e4m3x4_nan_bits(x.z) >> 7) * 0xFFu), x.w &= hidden ? 0u : ~((e4m3x4_nan_bits(x.w) >> 7) * 0xFFu);
                            *reinterpret_cast<uint4*>(line + ((c ^ lane) & 7) * 16) = x;
                        }
#pragma unroll
                    for (int r = 0; r < RPG; ++r) {
                        const bool sees = !hidden && key < rows.upper[r0 + r] && key >= rows.lower[r0 + r];
                        if (!sees || nan) y[r] = e[r] = sees ? kNan : -INFINITY;
                    }
                }
#pragma unroll
                for (int r = 0; r < RPG; ++r) top = fmaxf(top, e[r]);
                if (threads_any<128>(1 + all, top + sc.y > kTop + kSlack)) {
                    float shrink[RPG];
#pragma unroll
                    for (int r = 0; r < RPG; ++r) {
                        const float most = warp_max(y[r] + sc.y);
                        if (lane == 0) s_part[all][q4][r] = most;
                    }
                    sync_threads_of<128>(1 + all);
#pragma unroll
                    for (int r = 0; r < RPG; ++r) {
                        const float top = fmaxf(fmaxf(s_part[all][0][r], s_part[all][1][r]), fmaxf(s_part[all][2][r], s_part[all][3][r]));
                        const float next = top - m[r] > kTop ? top - kTop : m[r];
                        const Shrink by(m[r] - next);
                        shrink[r] = by.both();
                        m[r] = next;
                        l[r] = by.of(l[r]);
                        e[r] = y[r] - next;
                    }
                    if (i > 0) {                      // what is in O already: the MMAs of the tile before are done, those of this one wait for its weights
                        wait_bar(bar(&ctrl.p_empty), (uint32_t)(tiles - 1) & 1u, abort_flag, a.dev_status);
                        __syncwarp();
                        tc_fence_after();
#pragma unroll 1
                        for (int z = 0; z < kTermsP; ++z) {
                            uint32_t v[RPG];
                            tmem_load<RPG>(tmem + lane_addr + C::kOCol + z * ROWS + r0, v);
                            tmem_wait_ld();
#pragma unroll
                            for (int r = 0; r < RPG; ++r) v[r] = __float_as_uint(__uint_as_float(v[r]) * shrink[r]);
                            tmem_st<RPG>(tmem + lane_addr + C::kOCol + z * ROWS + r0, v);
                        }
                        tmem_wait_st();
                        tc_fence_before();
                    }
                    sync_threads_of<128>(1 + all);     // (s_part is free again)
                }
                if (tiles >= 1) wait_bar(bar(&ctrl.p_empty), (uint32_t)(tiles - 1) & 1u, abort_flag, a.dev_status);
                uint8_t* const p = smem + (p_at - base) + r0 * 128;
#pragma unroll
                for (int r = 0; r < RPG; r += 2) {
                    float2 w = make_float2(ex2(e[r]), ex2(e[r + 1]));
                    const float2 sum = add2(make_float2(l[r], l[r + 1]), w);
                    l[r] = sum.x, l[r + 1] = sum.y;
                    w = mul2(w, make_float2(sc.z, sc.z));
                    __half2 rest = __floats2half2_rn(w.x, w.y);
#pragma unroll
                    for (int z = 0; z < kTermsP; ++z) {
                        const uint32_t code = __nv_cvt_halfraw2_to_fp8x2(rest, __NV_SATFINITE, __NV_E4M3);
                        const uint32_t back = e4m3x2_to_f16x2(code);
                        rest = __hmul2(__hsub2(rest, *reinterpret_cast<const __half2*>(&back)), __float2half2_rn(kTermStep));
                        // line z ROWS + r0 + r: r0 is a multiple of 4 (and of 8 where groups have 8 rows)
                        p[(z * ROWS + r) * 128 + (p_off ^ (uint32_t)((z * ROWS ^ r) & 7) << 4)] = (uint8_t)code;
                        p[(z * ROWS + r + 1) * 128 + (p_off ^ (uint32_t)((z * ROWS ^ (r + 1)) & 7) << 4)] = (uint8_t)(code >> 8);
                    }
                }
                fence_proxy_async_smem();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(&ctrl.p_full));
            }
            // ---- the unit's result, or a piece of it: an element per thread
#pragma unroll
            for (int r = 0; r < RPG; ++r) {
#pragma unroll
                for (int z = 16; z > 0; z >>= 1) l[r] += __shfl_xor_sync(0xFFFFFFFFu, l[r], z);
                if (lane == 0) s_part[all][q4][r] = l[r];
            }
            float o[RPG];
#pragma unroll
            for (int r = 0; r < RPG; ++r) o[r] = 0.f;
            if (n > 0) {
                wait_bar(bar(&ctrl.p_empty), (uint32_t)(tiles - 1) & 1u, abort_flag, a.dev_status);
                __syncwarp();
                tc_fence_after();
                float f = 1.f;
#pragma unroll
                for (int z = 0; z < kTermsP; ++z, f /= kTermStep) {
                    uint32_t v[RPG];
                    tmem_load<RPG>(tmem + lane_addr + C::kOCol + z * ROWS + r0, v);
                    tmem_wait_ld();
#pragma unroll
                    for (int r = 0; r < RPG; ++r) o[r] = fmaf(__uint_as_float(v[r]), f, o[r]);
                }
                tc_fence_before();
            }
            const bool live = *abort_flag == 0;       // (nothing of an aborted call is stored)
            sync_threads_of<128>(1 + all);
            const int at_slot = rows.slot;
            float* slot = slots + at_slot * (int64_t)slot_floats(ROWS, kDim);
#pragma unroll
            for (int r = 0; r < RPG; ++r) {
                const int row = r0 + r;
                if (row >= n_rows || !live) continue;
                const float sum = (s_part[all][0][r] + s_part[all][1][r]) + (s_part[all][2][r] + s_part[all][3][r]);
                if (at_slot < 0) {
                    static_cast<__nv_bfloat16*>(a.out)[rows.out[row] + key_lane] = __float2bfloat16(sum == 0.f ? 0.f : __fdividef(o[r] * kVScaleDown, sum));
                    if (a.lse != nullptr && key_lane == 0) a.lse[rows.lse[row]] = sum == 0.f ? -INFINITY : (m[r] + log2f(sum)) * 0.69314718056f;
                } else {
                    slot[2 * ROWS + row * kDim + key_lane] = o[r];
                    if (key_lane == 0) slot[row] = m[r], slot[ROWS + row] = sum;
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(&ctrl.q_empty[k & 1]));
            sync_threads_of<128>(1 + all);             // (s_part)
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) tmem_dealloc(s_tmem_base, C::kTmemCols);
}

template <int ROWS>
int64_t share_count() { return (int64_t)sm_count() * Cfg<ROWS>::kWorkers; }

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
    // (of a pool without pages nothing is copied, but a map has to be of something)
    const uint32_t box = 1u << a.c.page_log2;
    const bool none = a.c.n_pages == 0;
    const uint64_t rows = none ? box : ((uint64_t)a.c.n_pages * (uint64_t)a.c.kv_heads) << a.c.page_log2;
    if (!make_tensor_map_bytes_2d(&tm_k, none ? ws : a.c.k, kDim, rows, kDim, box, CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_tensor_map_bytes_2d(&tm_v, none ? ws : a.c.v, kDim, rows, kDim, box, CU_TENSOR_MAP_SWIZZLE_128B))
        return MOLORA_ERR_CUDA;
    const int64_t shares = share_count<ROWS>();
    CutUnit* cuts = static_cast<CutUnit*>(ws);
    float* slots = reinterpret_cast<float*>(static_cast<char*>(ws) + cut_bytes(shares));
    if (launch_kernel(attend_stream_kernel<ROWS>, dim3((unsigned)sm_count()), dim3(C::kThreads), C::kSmem, s, 1, true, a, tm_k, tm_v, cuts, slots) != cudaSuccess)
        return MOLORA_ERR_CUDA;
    return cuda_ok(launch_kernel(attend_join_kernel<__nv_bfloat16, kDim, ROWS>, dim3((unsigned)shares, join_groups(ROWS)), dim3(kJoinWarps * 32), 0, s, 1, true, a,
                                 static_cast<const CutUnit*>(cuts), static_cast<const float*>(slots)));
}

}  // namespace

// the most that any number of rows up to this needs (32 rows, with one worker per CTA, need less than 24 or 16)
size_t attend_stream_workspace_bytes(int64_t rows)
{
    size_t most = bytes_needed<4>();
    if (rows > 4) most = std::max(most, bytes_needed<8>());
    if (rows > 8) most = std::max(most, bytes_needed<16>());
    if (rows > 16) most = std::max(most, bytes_needed<24>());
    if (rows > 24) most = std::max(most, bytes_needed<32>());
    return most;
}

molora_status_t launch_attend_stream(const AttendArgs& a, int64_t rows, void* ws, cudaStream_t s)
{
    return rows <= 4 ? launch<4>(a, ws, s) : rows <= 8 ? launch<8>(a, ws, s) : rows <= 16 ? launch<16>(a, ws, s) : rows <= 24 ? launch<24>(a, ws, s) : launch<32>(a, ws, s);
}

}  // namespace molora
