// Attention over the paged 8-bit cache for more than 32 query rows, bf16, heads of 128 (molora_kv_attend): prompts and chunks of prompts.
//
// A unit is 256 consecutive rows of a sequence (new token, query head of the group that shares a key / value head) in two tiles of 128, one key /
// value head and the keys that they see; here the tensor cores are the bound, so the codes of K and V are brought to fp16 once for both tiles.
//   S_t = Q_t K^T  [128 rows x 64 keys]        A = Q_t in shared memory, B = K in shared memory
//   O_t += P_t V   [128 rows x 128 elements]   A = P_t in TMEM (fp16, in the place of S_t), B = V in shared memory, read across (MN-major)
//   warps 0-7, 8-15 two threads per row of tile 0 and 1, each with 32 of a step's 64 keys: q to fp16 by a power of two, weights (S_t -> P_t),
//                   the sum, the result.  The reference of a row moves when a score is 2^8 over the weight that its largest was given, and then
//                   O_t is rescaled; whether it does is all that the two ask each other, step by step.  (One thread per row, 128 keys one after
//                   the other at the latencies of one warp per scheduler, took 3500 cycles per 128 keys.)
//   warps 16-19     codes -> fp16, two tiles of 128 keys of K and of V ahead, the codes of the next tile on their way in registers
//   warps 20, 21    the MMAs of tile 0 and of tile 1: O of a step, then S of the step after the next, so that the scores of the next step are there
//                   when the weights of this one are done.  (One warp for both took 8 % longer, with steps of 64 keys and with steps of 128, whose S has
//                   to wait for all of the last P; S of 64 keys costs the tensor cores 56 cycles per 16 elements where 128 keys cost 64.)
//   warp 22         units, pages and scales, into queues: what depends on one another there is waited for long before it is needed
// The tensor cores work in the order of issue: O, which reads P, is through before S is written in its place.
// TMEM: S_0 S_1 O_0 O_1, 128 columns each, S for even and odd steps.  Shared memory: Q 64 KB, K and V 2 x 32 KB each.
// Shares, pieces and the join as in kv_attend.cuh, but with the steps that each tile of rows really sees.
// What bounds it, measured with 2048 rows of 32 heads behind 14336 tokens (651 to 659 us, 0.8 PFLOP/s): no unit alone.  Per 128 keys it takes 5300
// cycles, of which the tensor cores are busy 52 %, the special-function units 39 % (256 x 128 exponentials), the schedulers 60 %; taking out the
// exponentials or seven eighths of the MMAs gained 4 % each, both together with the codes 11 %.  With short prompts (8 of 1024 tokens: 174 us) it
// is what a unit costs by itself, 13,000 cycles, 5500 of them for q.
#include "kv_attend.cuh"
#include "pipeline.cuh"

namespace molora {
namespace {

constexpr int kDim = 128, kKeys = 128, kStepKeys = 64, kTileRows = 128, kUnitRows = 256;
constexpr int kThreads = 768;                                 // (the last warp only makes a warpgroup of four)
constexpr int kConvWarp0 = 16, kMmaWarp0 = 20, kMmaWarp1 = 21, kWalkWarp = 22;      // an MMA warp for each tile of rows
// Registers: the converting warps hold 64 words of codes, which the last four give up (6 x 128 threads, 80 registers each at launch)
constexpr int kConvRegs = 104, kOtherRegs = 56;
static_assert(kConvRegs + kOtherRegs <= 2 * 80, "register split");
constexpr int kOperandBytes = 128 * kDim * 2;                 // of a Q tile, of a tile of K or of V, in fp16
constexpr int kQAt = 0, kKAt = 2 * kOperandBytes, kVAt = 4 * kOperandBytes;
constexpr size_t kSmem = 1024 + 6 * (size_t)kOperandBytes;
constexpr uint32_t kTmemCols = 512, kOCol = 256;
constexpr int kTileQueue = 8, kUnitQueue = 4;
constexpr int kUnitCost = 3, kMinShare = 4;                   // tiles of keys
constexpr float kTop = 7.f, kSlack = 8.f;                     // a row's largest weight when its reference is set, and by how much it may grow: fp16

// (a warp arrives as one: arrivals of single threads at a barrier follow one another, 256 of them cost a step as much as its weights)
struct Control {
    uint64_t s_full[2][2], p_full[2][2], o_done[2][2];         // of each tile of rows, for even and odd steps of it
    uint64_t q_full[2], k_full[2], k_empty[2], v_full[2], v_empty[2];
    uint64_t tile_full[kTileQueue], tile_empty[kTileQueue], unit_full[kUnitQueue], unit_empty[kUnitQueue], drained[2];
    uint32_t tmem_base;
    int abort_flag;
};
constexpr int kUnitReaders = kConvWarp0 + 2;                  // the warps of rows, those of the MMAs

// A tile of keys in the queue.
struct KeyTile {
    float4 scale[8];                           // of 16 keys: scale of K, logarithm of V's, V's, whether their page can be used
    int64_t line[8];                           // of 16 keys: the first one's line in the pool, -1: none
    uint32_t nan[4];                           // keys with a NaN among the codes of V, where not every row sees every key
    int32_t key0, hi_max, lo_min;
    int32_t kind;                              // 0: every row sees every key, 1: not so, 2: no tile, there are no more
};
// A unit in the queue.
struct UnitInfo {
    int32_t row0, pos0, len;                   // of its sequence
    int32_t tile_row, n_rows, head;
    int32_t key0, n;                           // first key, tiles of keys; n -1: there are no more units
    int32_t steps;                             // of 64 keys: 2 n, or one less where no row sees the last
    int32_t slot;                              // where its piece goes, -1: it is whole
};

// A unit's key range belongs to its tile of rows.
struct TileUnit {
    Sequence sq;
    int64_t at;                                // its first step in the list
    int32_t b, head, tile, n_rows, tile_row;
    int32_t lo, steps, first, last;            // first key (a multiple of 128); steps [first, last) are in this share
    int32_t hi_min, hi_max, lo_min, lo_max;
    int32_t u0, u1;                            // tiles of keys, counted from lo
};
struct TileSpan {
    int32_t lo, steps;
};
__device__ __forceinline__ int row_tiles(const Sequence& s, int group) { return (int)(((int64_t)s.n * group + kUnitRows - 1) / kUnitRows); }
__device__ __forceinline__ TileSpan tile_span(const AttendArgs& a, const Sequence& s, int tile, int group)
{
    const int r0 = tile * kUnitRows, r1 = min((int64_t)r0 + kUnitRows, (int64_t)s.n * group) - 1;
    TileSpan t;
    t.lo = lower_key(a, s, r0 / group) & ~(kKeys - 1);
    t.steps = kUnitCost + max(1, (upper_key(a, s, r1 / group) - t.lo + kKeys - 1) / kKeys);
    return t;
}

struct TileWalk {
    const AttendArgs& a;
    int64_t at = 0, stop = 0, base = 0, share = 1;      // next step, end of the share, first step of the tile of rows
    // A share that would end so near to an end of a unit ends there instead: a piece costs its 128 KB in the workspace twice, about as much as
    // three steps (8 prompts of 1024 tokens, shares of 52 steps: 181 us without, 174 so; more than that costs balance).
    __device__ int64_t near() const { return min(share >> 3, (int64_t)6); }
    int b = 0, tile = 0, tiles = 0, group;
    Sequence sq;
    TileSpan sp{0, 1};
    __device__ explicit TileWalk(const AttendArgs& args) : a(args), group(args.group) {}
    __device__ void load(const Sequence& s)
    {
        sq = s;
        tiles = row_tiles(sq, group);
        tile = 0;
        if (tiles > 0) sp = tile_span(a, sq, 0, group);
    }
    __device__ void skip_to(int64_t to)                 // the tile of rows that step `to` belongs to
    {
        for (;;) {
            if (tile < tiles) {
                const int64_t end = base + (int64_t)sp.steps * a.c.kv_heads;
                if (to < end) return;
                base = end;
                if (++tile < tiles) sp = tile_span(a, sq, tile, group);
            } else {
                ++b;
                load(sequence_of(a.c, b, a.N));
            }
        }
    }
    __device__ void begin(const ShareStart& from, int64_t w)
    {
        share = from.share;
        at = w * share;
        stop = min(from.total, at + share);
        if (at >= stop) return;
        b = from.part * ((a.c.B + kThreads - 1) / kThreads);
        base = from.base;
        load(from.sq);
        skip_to(at);
        const int64_t in_unit = (at - base) % sp.steps;
        if (in_unit <= near()) at -= in_unit;           // (its beginning counts first)
        else if (sp.steps - in_unit <= near()) at += sp.steps - in_unit;
    }
    __device__ bool next(TileUnit& u)
    {
        if (at >= stop) return false;
        skip_to(at);
        u.sq = sq, u.b = b, u.tile = tile;
        u.head = (int)quotient(at - base, sp.steps);
        u.at = base + (int64_t)u.head * sp.steps;
        u.lo = sp.lo, u.steps = sp.steps;
        const int64_t cut = stop - u.at;                // (a share that ends inside the unit, as begin() of the next one sees it)
        if (cut < sp.steps && cut <= near()) return false;
        u.first = (int)(at - u.at), u.last = cut >= sp.steps - near() ? sp.steps : (int)cut;
        at = u.at + u.last;
        u.tile_row = tile * kUnitRows;
        u.n_rows = (int)min((int64_t)kUnitRows, (int64_t)sq.n * group - u.tile_row);
        const int t0 = u.tile_row / group, t1 = (u.tile_row + u.n_rows - 1) / group;
        u.hi_min = upper_key(a, sq, t0), u.hi_max = upper_key(a, sq, t1);
        u.lo_min = lower_key(a, sq, t0), u.lo_max = lower_key(a, sq, t1);
        u.u0 = max(0, u.first - kUnitCost);
        u.u1 = min(u.last - kUnitCost, u.hi_max > u.lo ? (u.hi_max - u.lo + kKeys - 1) / kKeys : 0);
        return true;
    }
    __device__ int32_t pieces(const TileUnit& u, int64_t w) const { return (int32_t)((u.at + u.steps - near() - 1) / share - w + 1); }
};

// fp16 operands of kind::f16, fp32 accumulation
__host__ __device__ constexpr uint32_t idesc_f16_f32(int M, int N, int b_mn_major)
{
    return (1u << 4) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// 16 codes of element chunk c (of 16) of line r of a [2][128][64] fp16 operand with 128-byte swizzle
__device__ __forceinline__ void store_codes_f16(uint8_t* operand, int r, int c, uint4 w)
{
    uint8_t* line = operand + (c >> 2) * (kOperandBytes / 2) + r * 128;
    const int x = (2 * c) & 7;
    const uint4 lo = make_uint4(e4m3x2_to_f16x2(w.x), e4m3x2_to_f16x2_high(w.x), e4m3x2_to_f16x2(w.y), e4m3x2_to_f16x2_high(w.y));
    const uint4 hi = make_uint4(e4m3x2_to_f16x2(w.z), e4m3x2_to_f16x2_high(w.z), e4m3x2_to_f16x2(w.w), e4m3x2_to_f16x2_high(w.w));
    // (the two parts of a line lie in the same banks: half of the lanes begin with the second of their pieces)
    const int odd = c >> 2;
    *reinterpret_cast<uint4*>(line + (((x + odd) ^ (r & 7)) << 4)) = odd ? hi : lo;
    *reinterpret_cast<uint4*>(line + (((x + 1 - odd) ^ (r & 7)) << 4)) = odd ? lo : hi;
}

__global__ void __launch_bounds__(kThreads, 1)
    attend_tiles_kernel(const __grid_constant__ AttendArgs a, CutUnit* __restrict__ cuts, float* __restrict__ slots)
{
    using namespace ptx;
    __shared__ Control ctrl;
    __shared__ ShareStart s_start;
    __shared__ KeyTile s_tiles[kTileQueue];
    __shared__ UnitInfo s_units[kUnitQueue];
    __shared__ float s_pair[2][2][kTileRows];         // what the two threads of a row tell each other
    extern __shared__ uint8_t smem_raw[];
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - raw);
    volatile int* abort_flag = &ctrl.abort_flag;
    auto bar = [](const uint64_t* b) { return smem_u32(b); };
    const int group = a.group;

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            for (int z = 0; z < 2; ++z)
                mbar_init(bar(&ctrl.s_full[i][z]), 1), mbar_init(bar(&ctrl.p_full[i][z]), 8), mbar_init(bar(&ctrl.o_done[i][z]), 1);
            mbar_init(bar(&ctrl.q_full[i]), 8);
            mbar_init(bar(&ctrl.k_full[i]), 4), mbar_init(bar(&ctrl.k_empty[i]), 2);
            mbar_init(bar(&ctrl.v_full[i]), 4), mbar_init(bar(&ctrl.v_empty[i]), 2);
            mbar_init(bar(&ctrl.drained[i]), 1);
        }
        for (int i = 0; i < kTileQueue; ++i) mbar_init(bar(&ctrl.tile_full[i]), 1), mbar_init(bar(&ctrl.tile_empty[i]), 2);
        for (int i = 0; i < kUnitQueue; ++i) mbar_init(bar(&ctrl.unit_full[i]), 1), mbar_init(bar(&ctrl.unit_empty[i]), kUnitReaders);
        ctrl.abort_flag = 0;
        fence_mbar_init();
    }
    grid_dependency_wait();
    if (warp == kMmaWarp0) take_tmem(&ctrl.tmem_base, kTmemCols);
    cut_shares<kThreads, 1>(a, blockIdx.x, gridDim.x, kMinShare, &s_start, [&](const Sequence& sq) {
        int64_t steps = 0;
        const int tiles = row_tiles(sq, group);
        for (int t = 0; t < tiles; ++t) steps += (int64_t)tile_span(a, sq, t, group).steps * a.c.kv_heads;
        return steps;
    });
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_dependency_trigger();                        // (not before TMEM is mine)
    const uint32_t tmem = ctrl.tmem_base;
    // unit k of the share, for a warp that reads them all in turn; given back by done_with
    auto unit = [&](int k) {
        wait_bar(bar(&ctrl.unit_full[k % kUnitQueue]), (uint32_t)(k / kUnitQueue) & 1u, abort_flag, a.dev_status);
        UnitInfo u = s_units[k % kUnitQueue];
        if (*abort_flag) u.n = -1;
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(&ctrl.unit_empty[k % kUnitQueue]));
        return u;
    };

    if (warp < kConvWarp0) {
        // ============================================================ half a row per thread
        const int t = warp >> 3, half = (warp >> 2) & 1, row = (warp & 3) * 32 + lane;       // tile, half of the keys, row of the tile = lane of TMEM
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + lane_addr + (uint32_t)(t * 128 + half * 32), o_at = tmem + lane_addr + kOCol + (uint32_t)(t * 128 + half * 64);
        uint8_t* const q_tile = smem + kQAt + t * kOperandBytes;
        const int pair = 1 + t * 4 + (warp & 3);      // barrier of the two warps that share 32 rows
        auto pair_sync = [&]() { asm volatile("barrier.cta.sync %0, 64;" ::"r"(pair) : "memory"); };
        auto pair_any = [&](bool v) {
            uint32_t r;
            asm volatile(
                "{\n\t.reg .pred P, Q;\n\tsetp.ne.b32 P, %1, 0;\n\tbarrier.cta.red.or.pred Q, %2, 64, P;\n\tselp.u32 %0, 1, 0, Q;\n\t}"
                : "=r"(r)
                : "r"((uint32_t)v), "r"(pair)
                : "memory");
            return r != 0;
        };
        int tiles = 0, own = 0;                       // key tiles of the share so far; steps that this tile of rows took part in
        float rowf = 0.f;
        int64_t out_at = 0, lse_at = 0;
        int hi_row = 0, lo_row = 0;
        bool real = false;
        auto takes_part = [&](const UnitInfo& u) { return t * kTileRows < u.n_rows; };
        // This thread's row of unit u, and q of the warp's 32 rows as lines of the A operand (the MMAs of S that read the last ones are done):
        // half a warp a row, eight elements a lane.
        auto begin_unit = [&](const UnitInfo& u) {
            const int mine = t * kTileRows + row, r = u.tile_row + min(mine, u.n_rows - 1);
            const int token = r / group, qh = u.head * group + (r - token * group);
            real = mine < u.n_rows;
            const int p = u.pos0 + token;
            hi_row = a.causal ? max(0, min(p + 1, u.len)) : u.len;
            lo_row = a.window > 0 && p >= a.window ? p - a.window + 1 : 0;
            const int64_t at = (int64_t)u.row0 + token, in = at * a.ldq + (int64_t)qh * kDim;
            out_at = at * a.ldo + (int64_t)qh * kDim, lse_at = at * a.heads + qh;
            if (u.n <= 0) return;
            uint4 w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t from = __shfl_sync(0xFFFFFFFFu, in, half * 16 + 2 * i + (lane >> 4));
                w[i] = ld128_rw_stream(static_cast<const __nv_bfloat16*>(a.q) + from + (lane & 15) * 8);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float x[8], amax = 0.f;
                unpack<__nv_bfloat16>(w[i], x);
#pragma unroll
                for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, o));
                const RowScale by = row_scale<14>(amax);
                uint32_t h[4];
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    const __half2 p = __floats2half2_rn(x[2 * z] * by.up, x[2 * z + 1] * by.up);
                    h[z] = *reinterpret_cast<const uint32_t*>(&p);
                }
                const int line = (warp & 3) * 32 + half * 16 + 2 * i + (lane >> 4), chunk = lane & 15;
                if (chunk == 0) s_pair[t][0][line] = a.scale_log2 * by.down;
                *reinterpret_cast<uint4*>(q_tile + (chunk >> 3) * (kOperandBytes / 2) + line * 128 + (((chunk ^ line) & 7) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
            }
            pair_sync();
            rowf = s_pair[t][0][row];
            pair_sync();                              // (s_pair is free again)
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(&ctrl.q_full[t]));
        };
        // (after an abort the waits fall through: the two warps of a pair leave together, so that neither is left at a barrier)
        auto next_unit = [&](int k) {
            UnitInfo u = unit(k);
            if (pair_any(u.n < 0)) u.n = -1;
            return u;
        };
        UnitInfo u = next_unit(0);
        if (u.n >= 0 && takes_part(u)) begin_unit(u);
        for (int k = 1; u.n >= 0; ++k) {
            const int n = u.n, steps = u.steps, slot_at = u.slot, mine = t * kTileRows + row;
            const bool part = takes_part(u);
            float m = kNone, l = 0.f;
            if (part) {
#pragma unroll 1
                for (int i = 0; i < steps; ++i, ++own) {
                    const int kt = tiles + (i >> 1), b = own & 1;
                    const uint32_t parity = (uint32_t)(own >> 1) & 1u;
                    wait_bar(bar(&ctrl.s_full[t][b]), parity, abort_flag, a.dev_status);
                    __syncwarp();
                    tc_fence_after();
                    uint32_t v[32];
                    tmem_ld_x32(s_at + b * kStepKeys, v);
                    // for the scales and what is known of V (its place is not filled again before this thread has handed over its weights, so that this
                    // phase cannot be missed)
                    if ((i & 1) == 0) wait_bar(bar(&ctrl.v_full[kt & 1]), (uint32_t)(kt >> 1) & 1u, abort_flag, a.dev_status);
                    // (done before S of this step; waited for so that no phase is missed)
                    if (own >= 2) wait_bar(bar(&ctrl.o_done[t][b]), parity ^ 1u, abort_flag, a.dev_status);
                    __syncwarp();
                    const KeyTile& tile = s_tiles[kt % kTileQueue];
                    const int at = (i & 1) * kStepKeys + half * 32;      // this thread's 32 keys of the tile
                    const float4* scales = tile.scale + (at >> 4);
                    const float4 sc0 = scales[0], sc1 = scales[1];
                    bool seen = true;                                    // some row of the warp sees some of these keys
                    tmem_wait_ld();
                    if (tile.kind != 0) {
                        const int first = max(lo_row - tile.key0 - at, 0), behind = hi_row - tile.key0 - at;      // the row sees [first, behind)
                        uint32_t sees = first > 31 || behind <= 0 ? 0u : (0xFFFFFFFFu << first) & (0xFFFFFFFFu >> (32 - min(behind, 32)));
                        if (sc0.w == 0.f) sees &= 0xFFFF0000u;
                        if (sc1.w == 0.f) sees &= 0x0000FFFFu;
                        const uint32_t nan = tile.nan[at >> 5];
                        seen = __any_sync(0xFFFFFFFFu, sees != 0);
                        if (nan != 0)
#pragma unroll
                            for (int z = 0; z < 32; ++z)
                                if ((nan >> z) & 1u) v[z] = 0x7FC00000u;
#pragma unroll
                        for (int z = 0; z < 32; ++z)
                            if (!((sees >> z) & 1u)) v[z] = 0xFF800000u;
                    }
                    // ---- the largest exponent (a factor is never 0: a hidden score is -infinity times it)
                    const float f0 = fmaxf(rowf * sc0.x, 1.17549435e-38f), f1 = fmaxf(rowf * sc1.x, 1.17549435e-38f);
                    auto top_of = [](const uint32_t* w) {
                        float x = max3(__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]));
                        float y = max3(__uint_as_float(w[3]), __uint_as_float(w[4]), __uint_as_float(w[5]));
#pragma unroll
                        for (int z = 6; z < 14; z += 4) {
                            x = max3(x, __uint_as_float(w[z]), __uint_as_float(w[z + 1]));
                            y = max3(y, __uint_as_float(w[z + 2]), __uint_as_float(w[z + 3]));
                        }
                        return fmaxf(max3(x, __uint_as_float(w[14]), __uint_as_float(w[15])), y);
                    };
                    float top = -INFINITY;
                    if (seen) top = fmaxf(fmaf(top_of(v), f0, sc0.y), fmaf(top_of(v + 16), f1, sc1.y));
                    if (pair_any(top - m > kTop + kSlack)) {
                        s_pair[t][half][row] = top;
                        pair_sync();
                        top = fmaxf(top, s_pair[t][half ^ 1][row]);
                        const float next = top - m > kTop + kSlack ? top - kTop : m;
                        const Shrink by(m - next);
                        const float shrink = by.both();
                        m = next;
                        l = by.of(l);
                        if (i > 0) {
                            wait_bar(bar(&ctrl.o_done[t][b ^ 1]), (uint32_t)((own - 1) >> 1) & 1u, abort_flag, a.dev_status);
                            __syncwarp();
                            tc_fence_after();
#pragma unroll 1
                            for (int g = 0; g < 8; ++g) {
                                uint32_t o[8];
                                tmem_ld_x8(o_at + g * 8, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int z = 0; z < 8; ++z) o[z] = __float_as_uint(__uint_as_float(o[z]) * shrink);
                                tmem_st<8>(o_at + g * 8, o);
                            }
                        }
                        pair_sync();                  // (s_pair is free again)
                    }
                    // ---- the weights, two to a column, over scores that have been read
                    uint32_t p[16];
                    if (seen) {
                        float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            const float f = g == 0 ? f0 : f1, vs = g == 0 ? sc0.z : sc1.z;
#pragma unroll
                            for (int z = 0; z < 8; ++z) {
                                float2 x = make_float2(__uint_as_float(v[16 * g + 2 * z]), __uint_as_float(v[16 * g + 2 * z + 1]));
                                x = fma2(x, make_float2(f, f), make_float2(-m, -m));
                                x = make_float2(ex2(x.x), ex2(x.y));
                                sum = add2(sum, x);
                                x = mul2(x, make_float2(vs, vs));
                                const __half2 w2 = __floats2half2_rn(x.x, x.y);
                                p[8 * g + z] = *reinterpret_cast<const uint32_t*>(&w2);
                            }
                        }
                        l += sum.x + sum.y;
                    } else {
#pragma unroll
                        for (int z = 0; z < 16; ++z) p[z] = 0;
                    }
                    tmem_st<16>(s_at + b * kStepKeys, p);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(&ctrl.p_full[t][b]));
                }
            }
            tiles += n;
            const int64_t out_was = out_at, lse_was = lse_at;
            const bool real_was = real;
            // ---- the next unit's q while the last O is on its way
            u = next_unit(k);
            if (u.n >= 0 && takes_part(u)) begin_unit(u);
            if (!part) continue;
            if (n > 0) {
                wait_bar(bar(&ctrl.o_done[t][(own - 1) & 1]), (uint32_t)((own - 1) >> 1) & 1u, abort_flag, a.dev_status);
                __syncwarp();
                tc_fence_after();
            }
            s_pair[t][half][row] = l;
            pair_sync();
            l += s_pair[t][half ^ 1][row];
            const bool whole = slot_at < 0, store = real_was && *abort_flag == 0;       // (nothing of an aborted call is stored)
            const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l, down = whole ? kVScaleDown : 1.f;
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + out_was;
            float* slot = slots + max(slot_at, 0) * (int64_t)slot_floats(kUnitRows, kDim);
#pragma unroll 1
            for (int g = 0; g < 4; ++g) {             // 16 elements of this half
                uint32_t v[16];
                if (n > 0) {
                    tmem_ld_x16(o_at + g * 16, v);
                    tmem_wait_ld();
                } else {
#pragma unroll
                    for (int z = 0; z < 16; ++z) v[z] = 0;
                }
                float x[16];
#pragma unroll
                for (int z = 0; z < 16; ++z) x[z] = __uint_as_float(v[z]) * down * inv;
                if (!store) continue;
                const int at = half * 64 + g * 16;
                if (whole) {
#pragma unroll
                    for (int z = 0; z < 2; ++z) stg128(out + at + z * 8, pack<__nv_bfloat16>(x + 8 * z));
                } else {
#pragma unroll
                    for (int z = 0; z < 4; ++z) stg128(slot + 2 * kUnitRows + mine * kDim + at + z * 4, pack<float>(x + 4 * z));
                }
            }
            tc_fence_before();                        // (the next O begins behind this thread's next weights)
            if (store && half == 0) {
                if (!whole) slot[mine] = m, slot[kUnitRows + mine] = l;
                else if (a.lse != nullptr) a.lse[lse_was] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718056f;
            }
            pair_sync();                              // (s_pair is free again)
        }
    } else if (warp < kMmaWarp0) {
        // ============================================================ codes -> fp16
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kConvRegs));
        const int ct = tid - kConvWarp0 * 32, chunk = ct & 7, r0 = ct >> 3;      // chunk of 16 elements, lines r0 + 16 j
        const int64_t lane_at = (int64_t)r0 * kDim + chunk * 16;
        uint4 k[8], v[8];
        auto load = [&](const KeyTile& tile, const uint8_t* codes, uint4* w) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t line = tile.line[j];
                w[j] = line >= 0 ? ld128_rw_stream(codes + line * kDim + lane_at) : make_uint4(0, 0, 0, 0);
            }
        };
        // (after an abort the queue is not looked at any more)
        auto there = [&](int kt) {
            const bool ok = wait_bar(bar(&ctrl.tile_full[kt % kTileQueue]), (uint32_t)(kt / kTileQueue) & 1u, abort_flag, a.dev_status);
            return ok && *const_cast<volatile int32_t*>(&s_tiles[kt % kTileQueue].kind) != 2;
        };
        bool more = there(0);
        if (more) load(s_tiles[0], a.c.k, k), load(s_tiles[0], a.c.v, v);
        for (int kt = 0; more; ++kt) {
            KeyTile& tile = s_tiles[kt % kTileQueue];
            const KeyTile& next = s_tiles[(kt + 1) % kTileQueue];
            const int st = kt & 1;
            const uint32_t again = ((uint32_t)(kt >> 1) & 1u) ^ 1u;
            if (kt >= 2) wait_bar(bar(&ctrl.k_empty[st]), again, abort_flag, a.dev_status);
#pragma unroll
            for (int j = 0; j < 8; ++j) store_codes_f16(smem + kKAt + st * kOperandBytes, 16 * j + r0, chunk, k[j]);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(&ctrl.k_full[st]));
            more = there(kt + 1);
            if (more) load(next, a.c.k, k);
            if (tile.kind == 1) {
                // Some row does not see some key: values that no row sees count as zero; a NaN among the codes of one becomes a NaN in the scores of
                // the rows that see it and a zero here, so that it cannot reach the others through their weight of zero.
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int at = 16 * j + r0, key = tile.key0 + at;
                    const bool none = key >= tile.hi_max || key < tile.lo_min;
                    uint32_t* w[4] = {&v[j].x, &v[j].y, &v[j].z, &v[j].w};
                    bool nan = false;
#pragma unroll
                    for (int z = 0; z < 4; ++z) {
                        const uint32_t bits = e4m3x4_nan_bits(*w[z]);
                        nan |= bits != 0;
                        *w[z] = none ? 0u : *w[z] & ~((bits >> 7) * 0xFFu);
                    }
                    if (nan && !none) atomicOr(&tile.nan[at >> 5], 1u << (at & 31));
                }
            }
            if (kt >= 2) wait_bar(bar(&ctrl.v_empty[st]), again, abort_flag, a.dev_status);
#pragma unroll
            for (int j = 0; j < 8; ++j) store_codes_f16(smem + kVAt + st * kOperandBytes, 16 * j + r0, chunk, v[j]);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(&ctrl.v_full[st]));
            if (more) load(next, a.c.v, v);
        }
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
      if (warp == kMmaWarp0 || warp == kMmaWarp1) {
        // ============================================================ MMAs of a tile of rows
        const bool leader = elect_one();
        const int t = warp - kMmaWarp0;
        const uint32_t tm = __shfl_sync(0xFFFFFFFFu, tmem, 0), s_col = tm + (uint32_t)(t * 128), o_col = tm + kOCol + (uint32_t)(t * 128);
        constexpr uint32_t idesc_s = idesc_f16_f32(kTileRows, kStepKeys, 0), idesc_o = idesc_f16_f32(kTileRows, kDim, 1);
        constexpr uint32_t kL128 = swizzle_layout_type(Swizzle::B128);
        const uint64_t q_desc = smem_desc(base + kQAt + t * kOperandBytes, 16, 1024, kL128), k_desc = smem_desc(base + kKAt, 16, 1024, kL128);
        const uint64_t v_desc = smem_desc(base + kVAt, kOperandBytes / 2, 1024, kL128);      // 64 elements a group, 8 keys a group
        bool live = true;
        int units = 0, begun = 0, tiles = 0, steps = 0;              // units with rows here, steps of earlier ones; tiles of keys; steps of the unit
        // S and O of step i of the unit; the last step of a tile gives back what was read
        auto issue_s = [&](int i) {
            const int kt = tiles + (i >> 1), b = (begun + i) & 1;
            if (leader && live) {
                const uint64_t ka = k_desc + (uint64_t)((kt & 1) * (kOperandBytes >> 4) + (i & 1) * (kStepKeys * 128 >> 4));
                const uint32_t d = s_col + (uint32_t)(b * kStepKeys);
#pragma unroll
                for (int j = 0; j < 8; ++j) {         // 16 elements a step, 64 a part
                    const uint64_t off = (uint64_t)((j >> 2) * (kOperandBytes / 2 >> 4) + (j & 3) * 2);
                    umma_bf16(d, q_desc + off, ka + off, idesc_s, j > 0);
                }
                umma_commit(bar(&ctrl.s_full[t][b]));
                if ((i & 1) || i + 1 == steps) umma_commit(bar(&ctrl.k_empty[kt & 1]));
            }
            __syncwarp();
        };
        auto issue_o = [&](int i) {
            const int kt = tiles + (i >> 1), own = begun + i, b = own & 1;
            live = wait_bar(bar(&ctrl.p_full[t][b]), (uint32_t)(own >> 1) & 1u, abort_flag, a.dev_status) && live;
            if ((i & 1) == 0) live = wait_bar(bar(&ctrl.v_full[kt & 1]), (uint32_t)(kt >> 1) & 1u, abort_flag, a.dev_status) && live;
            tc_fence_after();
            if (leader && live) {
                const uint64_t va = v_desc + (uint64_t)((kt & 1) * (kOperandBytes >> 4) + (i & 1) * (kStepKeys * 128 >> 4));
                const uint32_t p = s_col + (uint32_t)(b * kStepKeys);
#pragma unroll
                for (int j = 0; j < 4; ++j)           // 16 keys a step: two groups of 8 lines
                    umma_bf16_ts(o_col, p + (j >> 1) * 32 + (j & 1) * 8, va + j * (2048 >> 4), idesc_o, i > 0 || j > 0);
                umma_commit(bar(&ctrl.o_done[t][b]));
                if ((i & 1) || i + 1 == steps) {
                    umma_commit(bar(&ctrl.v_empty[kt & 1]));
                    umma_commit(bar(&ctrl.tile_empty[kt % kTileQueue]));
                }
            }
            __syncwarp();
        };
        auto wait_k = [&](int kt) {
            live = wait_bar(bar(&ctrl.k_full[kt & 1]), (uint32_t)(kt >> 1) & 1u, abort_flag, a.dev_status) && live;
            tc_fence_after();
        };
        for (int z = 0; live; ++z) {
            const UnitInfo u = unit(z);
            if (u.n < 0) break;
            if (u.n == 0) continue;
            steps = u.steps;
            if (t * kTileRows >= u.n_rows) {          // no rows here: the tiles are given back as they come
                for (int i = 0; i < u.n && live; ++i) {
                    const int kt = tiles + i;
                    wait_k(kt);
                    live = wait_bar(bar(&ctrl.v_full[kt & 1]), (uint32_t)(kt >> 1) & 1u, abort_flag, a.dev_status) && live;
                    if (leader && live) mbar_arrive(bar(&ctrl.k_empty[kt & 1])), mbar_arrive(bar(&ctrl.v_empty[kt & 1])), mbar_arrive(bar(&ctrl.tile_empty[kt % kTileQueue]));
                    __syncwarp();
                }
                tiles += u.n;
                continue;
            }
            live = wait_bar(bar(&ctrl.q_full[t]), (uint32_t)(units++) & 1u, abort_flag, a.dev_status) && live;
            wait_k(tiles);
            issue_s(0);
            if (steps > 1) issue_s(1);
            for (int i = 0; i < steps && live; ++i) {
                issue_o(i);
                if (i + 2 < steps) {
                    if ((i & 1) == 0) wait_k(tiles + (i >> 1) + 1);
                    issue_s(i + 2);
                }
            }
            tiles += u.n;
            begun += steps;
        }
        if (leader) umma_commit(bar(&ctrl.drained[t]));   // nothing of the tensor cores' is in flight when TMEM and shared memory are given up
        const long long c0 = clock64();
        while (!mbar_try_wait(bar(&ctrl.drained[t]), 0))
            if (clock64() - c0 > kTimeoutCycles) break;
        __syncwarp();
      } else if (warp == kWalkWarp) {
        // ============================================================ units, pages, scales
        const int plog = a.c.page_log2;
        TileWalk walk(a);
        walk.begin(s_start, blockIdx.x);
        CutUnit cut{};
        int tiles = 0, units = 0;
        auto push_unit = [&](const UnitInfo& info) {
            const int slot = units % kUnitQueue;
            if (units >= kUnitQueue) wait_bar(bar(&ctrl.unit_empty[slot]), ((uint32_t)(units / kUnitQueue) & 1u) ^ 1u, abort_flag, a.dev_status);
            if (lane == 0) {
                s_units[slot] = info;
                mbar_arrive(bar(&ctrl.unit_full[slot]));
            }
            __syncwarp();
            ++units;
        };
        auto claim_tile = [&]() -> KeyTile& {
            const int slot = tiles % kTileQueue;
            if (tiles >= kTileQueue) wait_bar(bar(&ctrl.tile_empty[slot]), ((uint32_t)(tiles / kTileQueue) & 1u) ^ 1u, abort_flag, a.dev_status);
            __syncwarp();
            return s_tiles[slot];
        };
        auto hand_over = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(&ctrl.tile_full[tiles % kTileQueue]));
            ++tiles;
        };
        TileUnit u{};
        while (*abort_flag == 0 && walk.next(u)) {
            const bool begins = u.first == 0, whole = begins && u.last == u.steps;
            if (begins && !whole) cut.row0 = u.sq.row0, cut.tile_row = u.tile_row, cut.rows = u.n_rows, cut.head = u.head, cut.pieces = walk.pieces(u, blockIdx.x);
            UnitInfo info;
            info.row0 = u.sq.row0, info.pos0 = u.sq.pos0, info.len = u.sq.len;
            info.tile_row = u.tile_row, info.n_rows = u.n_rows, info.head = u.head;
            info.key0 = u.lo + u.u0 * kKeys, info.n = max(u.u1 - u.u0, 0);
            info.steps = 2 * info.n - (info.n > 0 && u.lo + u.u1 * kKeys - kStepKeys >= u.hi_max ? 1 : 0);
            info.slot = whole ? -1 : 2 * (int)blockIdx.x + (begins ? 1 : 0);
            push_unit(info);
            // lanes hold 32 sixteens of keys: four tiles
            int32_t id = -1;
            float4 sc = make_float4(0.f, 0.f, 0.f, 0.f);
            int64_t line = -1;
            for (int i = u.u0; i < u.u1; ++i) {
                const int key0 = u.lo + i * kKeys, from = (i - u.u0) & 3;
                if (from == 0) {
                    const int key = key0 + lane * 16;
                    id = -1, line = -1;
                    sc = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (((key >> plog) << plog) < u.hi_max) {
                        id = ld_dependent(a.c.table + (int64_t)u.b * a.c.ld_table + (key >> plog));
                        if (id < 0 || id >= a.c.n_pages) {
                            if (a.dev_status != nullptr) atomicOr(a.dev_status, MOLORA_DEV_BAD_SEQUENCE);
                        } else {
                            const int64_t block = (int64_t)id * a.c.kv_heads + u.head;
                            const float vs = read_v_scale(ld_dependent(a.c.v_scale + block));
                            sc = make_float4(ld_dependent(a.c.k_scale + block), log2f(vs), vs, 1.f);
                            line = (block << plog) + (key & ((1 << plog) - 1));
                        }
                    }
                    __syncwarp();
                }
                const bool missing = __any_sync(0xFFFFFFFFu, lane >> 3 == from && line < 0);
                KeyTile& tile = claim_tile();
                if (*abort_flag) break;
                if (lane >> 3 == from) tile.scale[lane & 7] = sc, tile.line[lane & 7] = line;
                if (lane < 4) tile.nan[lane] = 0;
                if (lane == 0) {
                    tile.key0 = key0, tile.hi_max = u.hi_max, tile.lo_min = u.lo_min;
                    tile.kind = missing || key0 + kKeys > u.hi_min || key0 < u.lo_max ? 1 : 0;
                }
                hand_over();
            }
        }
        UnitInfo end{};
        end.n = -1;
        push_unit(end);
        KeyTile& tile = claim_tile();
        if (lane == 0) tile.kind = 2;
        hand_over();
        if (lane == 0) cuts[blockIdx.x] = *abort_flag == 0 ? cut : CutUnit{};
      }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp0) tmem_dealloc(tmem, kTmemCols);
}

int64_t share_count() { return sm_count(); }

}  // namespace

size_t attend_tiles_workspace_bytes() { return cut_bytes(share_count()) + (size_t)(2 * share_count() * slot_floats(kUnitRows, kDim)) * sizeof(float); }

molora_status_t launch_attend_tiles(const AttendArgs& a, void* ws, cudaStream_t s)
{
    static bool ready[kMaxDevices] = {};
    bool& done = ready[device_slot()];
    if (!done) {
        if (cudaFuncSetAttribute(attend_tiles_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem) != cudaSuccess) return MOLORA_ERR_CUDA;
        done = true;
    }
    const int64_t shares = share_count();
    CutUnit* cuts = static_cast<CutUnit*>(ws);
    float* slots = reinterpret_cast<float*>(static_cast<char*>(ws) + cut_bytes(shares));
    if (launch_kernel(attend_tiles_kernel, dim3((unsigned)shares), dim3(kThreads), kSmem, s, 1, true, a, cuts, slots) != cudaSuccess) return MOLORA_ERR_CUDA;
    return cuda_ok(launch_kernel(attend_join_kernel<__nv_bfloat16, kDim, kUnitRows>, dim3((unsigned)shares, join_groups(kUnitRows)), dim3(kJoinWarps * 32), 0, s,
                                 1, true, a, static_cast<const CutUnit*>(cuts), static_cast<const float*>(slots)));
}

}  // namespace molora
