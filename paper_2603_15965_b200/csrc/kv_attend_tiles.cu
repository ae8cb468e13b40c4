// Attention over the paged 8-bit cache for more than 32 query rows, bf16, heads of 128 (molora_kv_attend): prompts and chunks of prompts.
//
// A unit is 256 consecutive rows of a sequence (new token, query head of the group that shares a key / value head) in two tiles of 128, one key /
// value head and the keys that they see; here the tensor cores are the bound, so the codes of K and V are brought to fp16 once for both tiles.
//   S_t = Q_t K^T  [128 rows x 128 keys]       A = Q_t in shared memory, B = K in shared memory
//   O_t += P_t V   [128 rows x 128 elements]   A = P_t in TMEM (fp16, in the place of S_t), B = V in shared memory, read across (MN-major)
//   warps 0-3, 4-7  a row per thread of tile 0 and 1: q to fp16 by a power of two, weights of a tile (S_t -> P_t), the sum, the result.  Nothing
//                   is shared between rows, so nothing is synchronised; the reference of a row moves when a score is 2^8 over the weight that its
//                   largest was given, and then O_t is rescaled (by warps: TMEM is read and written by whole warps)
//   warps 8-11      codes -> fp16, two tiles of 128 keys of K and of V ahead
//   warp 12         the MMAs: O_0 S_0 O_1 S_1 ... -- while the weights of one tile are worked out, the other has the tensor cores
// S_t of the next keys is asked for right behind O_t of the last, which is the last to read P_t: the tensor cores work in the order of issue.
// TMEM: S_0 S_1 O_0 O_1, 128 columns each.  Shared memory: Q 64 KB, K and V 2 x 32 KB each.
// Shares, pieces and the join as in kv_attend.cuh, but with the steps that each tile of rows really sees.
// What bounds it: per 128 keys 4 x 512 cycles of the tensor cores, and as many of the special-function units (256 x 128 exponentials).
#include "kv_attend.cuh"
#include "pipeline.cuh"

namespace molora {
namespace {

constexpr int kDim = 128, kKeys = 128, kTileRows = 128, kUnitRows = 256;
constexpr int kThreads = 416;
constexpr int kConvWarp0 = 8, kMmaWarp = 12;
constexpr int kOperandBytes = 128 * kDim * 2;                 // of a Q tile, of a tile of K or of V, in fp16
constexpr int kQAt = 0, kKAt = 2 * kOperandBytes, kVAt = 4 * kOperandBytes;
constexpr size_t kSmem = 1024 + 6 * (size_t)kOperandBytes;
constexpr uint32_t kTmemCols = 512, kOCol = 256;
constexpr int kScaleRing = 4;
constexpr int kUnitCost = 1, kMinShare = 2;                   // tiles of keys
constexpr float kTop = 7.f, kSlack = 8.f;                     // a row's largest weight when its reference is set, and by how much it may grow: fp16

struct Control {
    uint64_t q_full[2], s_full[2], p_full[2], o_full[2], k_full[2], k_empty[2], v_full[2], v_empty[2], drained;
    uint32_t tmem_base;
    int abort_flag;
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
    int b = 0, tile = 0, tiles = 0, group;
    Sequence sq;
    TileSpan sp{0, 1};
    __device__ explicit TileWalk(const AttendArgs& args) : a(args), group(args.heads / args.c.kv_heads) {}
    __device__ void load()
    {
        sq = sequence_of(a.c, b, a.N);
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
                load();
            }
        }
    }
    __device__ void begin(const int64_t* s_upto, int64_t w)
    {
        const int64_t total = s_upto[kThreads - 1];
        share = max((total + gridDim.x - 1) / gridDim.x, (int64_t)kMinShare);
        at = w * share;
        stop = min(total, at + share);
        if (at >= stop) return;
        int lo = 0, hi = kThreads - 1;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (s_upto[mid] > at) hi = mid;
            else lo = mid + 1;
        }
        b = lo * ((a.c.B + kThreads - 1) / kThreads);
        base = lo > 0 ? s_upto[lo - 1] : 0;
        load();
    }
    __device__ bool next(TileUnit& u)
    {
        if (at >= stop) return false;
        skip_to(at);
        u.sq = sq, u.b = b, u.tile = tile;
        u.head = (int)((at - base) / sp.steps);
        u.at = base + (int64_t)u.head * sp.steps;
        u.lo = sp.lo, u.steps = sp.steps;
        u.first = (int)(at - u.at), u.last = (int)min((int64_t)sp.steps, stop - u.at);
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
    __device__ int32_t pieces(const TileUnit& u, int64_t w) const { return (int32_t)((u.at + u.steps - 1) / share - w + 1); }
};

__device__ __forceinline__ void umma_f16(uint32_t d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, bool accumulate) { ptx::umma_bf16(d, a_desc, b_desc, idesc, accumulate); }

// fp16 operands of kind::f16, fp32 accumulation
__host__ __device__ constexpr uint32_t idesc_f16_f32(int M, int N, int b_mn_major)
{
    return (1u << 4) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

// 16 codes of element chunk c (of 16) of line r of a [2][128][64] fp16 operand with 128-byte swizzle
__device__ __forceinline__ void store_codes_f16(uint8_t* operand, int r, int c, uint4 w)
{
    uint8_t* line = operand + (c >> 2) * (kOperandBytes / 2) + r * 128;
    const int x = (2 * c) & 7;
    const uint4 lo = make_uint4(e4m3x2_to_f16x2(w.x), e4m3x2_to_f16x2_high(w.x), e4m3x2_to_f16x2(w.y), e4m3x2_to_f16x2_high(w.y));
    const uint4 hi = make_uint4(e4m3x2_to_f16x2(w.z), e4m3x2_to_f16x2_high(w.z), e4m3x2_to_f16x2(w.w), e4m3x2_to_f16x2_high(w.w));
    *reinterpret_cast<uint4*>(line + ((x ^ (r & 7)) << 4)) = lo;
    *reinterpret_cast<uint4*>(line + (((x + 1) ^ (r & 7)) << 4)) = hi;
}

__global__ void __launch_bounds__(kThreads, 1)
    attend_tiles_kernel(const __grid_constant__ AttendArgs a, CutUnit* __restrict__ cuts, float* __restrict__ slots)
{
    using namespace ptx;
    __shared__ Control ctrl;
    __shared__ int64_t s_upto[kThreads];
    __shared__ float4 s_scales[kScaleRing][8];        // of 16 keys: scale of K, logarithm and reciprocal of V's, whether their page can be used
    __shared__ int32_t s_pages[kScaleRing][8];
    __shared__ uint32_t s_nan[kScaleRing][4];         // keys with a NaN among the codes of V that not every row sees
    extern __shared__ uint8_t smem_raw[];
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - raw);
    volatile int* abort_flag = &ctrl.abort_flag;
    auto bar = [](const uint64_t* b) { return smem_u32(b); };
    const int group = a.heads / a.c.kv_heads;

    grid_dependency_wait();
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(&ctrl.q_full[i]), kTileRows), mbar_init(bar(&ctrl.s_full[i]), 1);
            mbar_init(bar(&ctrl.p_full[i]), kTileRows), mbar_init(bar(&ctrl.o_full[i]), 1);
            mbar_init(bar(&ctrl.k_full[i]), 128), mbar_init(bar(&ctrl.k_empty[i]), 1);
            mbar_init(bar(&ctrl.v_full[i]), 128), mbar_init(bar(&ctrl.v_empty[i]), 1);
        }
        mbar_init(bar(&ctrl.drained), 1);
        ctrl.abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(&ctrl.tmem_base), kTmemCols);
        tmem_relinquish();
    }
    {
        const int part = (a.c.B + kThreads - 1) / kThreads;
        int64_t incl = 0;
        for (int b = tid * part; b < min(a.c.B, (tid + 1) * part); ++b) {
            const Sequence sq = sequence_of(a.c, b, a.N);
            const int tiles = row_tiles(sq, group);
            for (int t = 0; t < tiles; ++t) incl += (int64_t)tile_span(a, sq, t, group).steps * a.c.kv_heads;
            if (sq.bad && blockIdx.x == 0 && a.dev_status != nullptr) atomicOr(a.dev_status, MOLORA_DEV_BAD_SEQUENCE);
        }
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
            if (lane >= o) incl += up;
        }
        if (lane == 31) s_upto[tid] = incl;
        __syncthreads();
        for (int z = 0; z < warp; ++z) incl += s_upto[32 * z + 31];
        __syncthreads();
        s_upto[tid] = incl;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_dependency_trigger();                        // (not before TMEM is mine)
    const uint32_t tmem = ctrl.tmem_base;
    TileWalk walk(a);
    walk.begin(s_upto, blockIdx.x);
    TileUnit u{};

    if (warp < kConvWarp0) {
        // ============================================================ a row per thread
        const int t = warp >> 2, row = (warp & 3) * 32 + lane;       // tile, and row of the tile = lane of TMEM
        const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at = tmem + lane_addr + (uint32_t)(t * 128), o_at = tmem + lane_addr + kOCol + (uint32_t)(t * 128);
        uint8_t* const q_tile = smem + kQAt + t * kOperandBytes;
        int tiles = 0, units = 0;                     // key tiles of the share so far, and of this tile of rows units with any
        int own = 0;                                  // key tiles that this tile of rows took part in
        float rowf = 0.f;
        int token = 0, qh = 0;
        // q of this row of unit u, as the A operand; the MMAs of S that read the last one are done
        auto load_q = [&]() {
            const int r = min(u.tile_row + t * kTileRows + row, u.tile_row + u.n_rows - 1);
            token = r / group, qh = u.head * group + (r - token * group);
            const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q) + ((int64_t)u.sq.row0 + token) * a.ldq + (int64_t)qh * kDim;
            uint4 w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = ld128_rw_stream(q + 8 * i);
            float amax = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float x[8];
                unpack<__nv_bfloat16>(w[i], x);
#pragma unroll
                for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(x[e]));
            }
            // the row's largest element to [2^14, 2^15)
            const int e = amax > 0.f ? min(100, 14 - ((int)(__float_as_uint(amax) >> 23) - 127)) : 0;
            const float up = __uint_as_float((uint32_t)(e + 127) << 23);
            rowf = a.scale_log2 * __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float x[8];
                unpack<__nv_bfloat16>(w[i], x);
                uint32_t h[4];
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    const __half2 p = __floats2half2_rn(x[2 * z] * up, x[2 * z + 1] * up);
                    h[z] = *reinterpret_cast<const uint32_t*>(&p);
                }
                *reinterpret_cast<uint4*>(q_tile + (i >> 3) * (kOperandBytes / 2) + row * 128 + (((i & 7) ^ (row & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
            }
            fence_proxy_async_smem();
            mbar_arrive(bar(&ctrl.q_full[t]));
        };
        bool more = walk.next(u);
        auto takes_part = [&]() { return u.u0 < u.u1 && t * kTileRows < u.n_rows; };
        if (more && takes_part()) load_q();
        while (more) {
            const TileUnit c = u;                     // the unit in hand; u becomes the next one before it is finished
            const int n = max(c.u1 - c.u0, 0);
            const bool part = t * kTileRows < c.n_rows;
            const int row_at = c.tile_row + t * kTileRows + row;
            const bool real = t * kTileRows + row < c.n_rows;
            const int my_token = part && n > 0 ? token : min(row_at, c.tile_row + c.n_rows - 1) / group;
            const int my_head = part && n > 0 ? qh : c.head * group + (min(row_at, c.tile_row + c.n_rows - 1) - my_token * group);
            const int hi_row = upper_key(a, c.sq, my_token), lo_row = lower_key(a, c.sq, my_token);
            float m = kNone, l = 0.f;
            if (part) {
                for (int i = 0; i < n; ++i, ++own) {
                    const int key0 = c.lo + (c.u0 + i) * kKeys, kt = tiles + i;
                    wait_bar(bar(&ctrl.s_full[t]), (uint32_t)own & 1u, abort_flag, a.dev_status);
                    // for the scales and what is known of V (its place is not filled again before this thread has handed over its weights, so that this
                    // phase cannot be missed)
                    wait_bar(bar(&ctrl.v_full[kt & 1]), (uint32_t)(kt >> 1) & 1u, abort_flag, a.dev_status);
                    const float4* scales = s_scales[kt % kScaleRing];
                    bool border = key0 + kKeys > c.hi_min || key0 < c.lo_max;
                    uint32_t nan[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int g = 0; g < 8; ++g) border |= scales[g].w == 0.f;
                    if (border) {
#pragma unroll
                        for (int z = 0; z < 4; ++z) nan[z] = s_nan[kt % kScaleRing][z];
                    }
                    __syncwarp();
                    tc_fence_after();
                    // 32 scores, with what hides them; y: the raw score
                    auto scores = [&](int c32, float* y) {
                        uint32_t v[32];
                        tmem_ld_x16(s_at + c32 * 32, v);
                        tmem_ld_x16(s_at + c32 * 32 + 16, v + 16);
                        tmem_wait_ld();
#pragma unroll
                        for (int z = 0; z < 32; ++z) y[z] = __uint_as_float(v[z]);
                        if (border) {
#pragma unroll
                            for (int z = 0; z < 32; ++z) {
                                const int key = key0 + c32 * 32 + z;
                                const bool sees = key < hi_row && key >= lo_row && scales[2 * c32 + (z >> 4)].w != 0.f;
                                y[z] = !sees ? -INFINITY : (nan[c32] >> z) & 1u ? __int_as_float(0x7FC00000) : y[z];
                            }
                        }
                    };
                    float top = -INFINITY;
#pragma unroll 1
                    for (int c32 = 0; c32 < 4; ++c32) {
                        float y[32];
                        scores(c32, y);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float raw = y[16 * h];
#pragma unroll
                            for (int z = 1; z < 16; ++z) raw = fmaxf(raw, y[16 * h + z]);
                            const float4 sc = scales[2 * c32 + h];
                            top = fmaxf(top, fmaf(raw, fmaxf(rowf * sc.x, 1.17549435e-38f), sc.y));      // (never 0: a hidden score is -infinity times it)
                        }
                    }
                    const bool moves = top - m > kTop + kSlack;
                    if (__any_sync(0xFFFFFFFFu, moves)) {
                        const float next = moves ? top - kTop : m, shrink = ex2(m - next);
                        m = next;
                        l *= shrink;
                        if (i > 0) {                  // (S of this tile was asked for behind O of the last, which is therefore done)
#pragma unroll 1
                            for (int c16 = 0; c16 < 8; ++c16) {
                                uint32_t v[16];
                                tmem_ld_x16(o_at + c16 * 16, v);
                                tmem_wait_ld();
#pragma unroll
                                for (int z = 0; z < 16; ++z) v[z] = __float_as_uint(__uint_as_float(v[z]) * shrink);
                                tmem_st<16>(o_at + c16 * 16, v);
                            }
                        }
                    }
#pragma unroll 1
                    for (int c32 = 0; c32 < 4; ++c32) {
                        float y[32];
                        scores(c32, y);
                        uint32_t p[16];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float4 sc = scales[2 * c32 + h];
                            const float f = fmaxf(rowf * sc.x, 1.17549435e-38f), off = sc.y - m;
                            float sum = 0.f;
#pragma unroll
                            for (int z = 0; z < 16; z += 2) {
                                const float w0 = ex2(fmaf(y[16 * h + z], f, off)), w1 = ex2(fmaf(y[16 * h + z + 1], f, off));
                                sum += w0 + w1;
                                const __half2 w = __floats2half2_rn(w0, w1);
                                p[8 * h + z / 2] = *reinterpret_cast<const uint32_t*>(&w);
                            }
                            l = fmaf(sum, sc.z, l);
                        }
                        tmem_st<16>(s_at + c32 * 16, p);
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(bar(&ctrl.p_full[t]));
                }
            }
            tiles += n;
            // ---- the next unit's q while the last O is on its way
            more = walk.next(u);
            if (more && takes_part()) load_q();
            if (!part) continue;
            const bool begins = c.first == 0, whole = begins && c.last == c.steps;
            float* slot = slots + (2 * (int64_t)blockIdx.x + (begins ? 1 : 0)) * (int64_t)slot_floats(kUnitRows, kDim);
            const int r = t * kTileRows + row;
            if (n > 0) {
                wait_bar(bar(&ctrl.o_full[t]), (uint32_t)units & 1u, abort_flag, a.dev_status);
                ++units;
                __syncwarp();
                tc_fence_after();
            }
            const bool store = real && *abort_flag == 0;       // (nothing of an aborted call is stored)
            const float inv = !whole ? 1.f : l == 0.f ? 0.f : 1.f / l;
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + ((int64_t)c.sq.row0 + my_token) * a.ldo + (int64_t)my_head * kDim;
#pragma unroll 1
            for (int c32 = 0; c32 < 4; ++c32) {
                uint32_t v[32];
                if (n > 0) {
                    tmem_ld_x16(o_at + c32 * 32, v);
                    tmem_ld_x16(o_at + c32 * 32 + 16, v + 16);
                    tmem_wait_ld();
                } else {
#pragma unroll
                    for (int z = 0; z < 32; ++z) v[z] = 0;
                }
                float x[32];
#pragma unroll
                for (int z = 0; z < 32; ++z) x[z] = __uint_as_float(v[z]) * inv;
                if (!store) continue;
                if (whole) {
#pragma unroll
                    for (int z = 0; z < 4; ++z) stg128(out + c32 * 32 + z * 8, pack<__nv_bfloat16>(x + 8 * z));
                } else {
#pragma unroll
                    for (int z = 0; z < 8; ++z) stg128(slot + 2 * kUnitRows + r * kDim + c32 * 32 + z * 4, pack<float>(x + 4 * z));
                }
            }
            tc_fence_before();                        // (the next O begins behind this thread's next weights)
            if (store) {
                if (!whole) slot[r] = m, slot[kUnitRows + r] = l;
                else if (a.lse != nullptr) a.lse[((int64_t)c.sq.row0 + my_token) * a.heads + my_head] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718056f;
            }
        }
    } else if (warp < kMmaWarp) {
        // ============================================================ codes -> fp16
        const int ct = tid - kConvWarp0 * 32, chunk = ct & 7, r0 = ct >> 3;      // chunk of 16 elements, lines r0 + 16 i
        const int plog = a.c.page_log2;
        CutUnit cut{0, 0, 0, 0};
        int tiles = 0;
        auto sync = [] { asm volatile("barrier.cta.sync 1, 128;" ::: "memory"); };
        while (walk.next(u)) {
            if (u.first == 0 && u.last < u.steps) cut.b = u.b, cut.row_tile = u.tile, cut.head = u.head, cut.pieces = walk.pieces(u, blockIdx.x);
            const int32_t* table = a.c.table + (int64_t)u.b * a.c.ld_table;
            // page and scales of the ct-th 16 keys of tile i, ct < 8: asked for one tile ahead
            int32_t id = -1;
            float4 sc = make_float4(0.f, 0.f, 0.f, 0.f);
            auto look_up = [&](int i) {
                if (ct >= 8) return;
                id = -1;
                sc = make_float4(0.f, 0.f, 0.f, 0.f);
                const int key = u.lo + i * kKeys + ct * 16;
                if (i < u.u1 && ((key >> plog) << plog) < u.hi_max) {
                    id = ld_dependent(table + (key >> plog));
                    if (id < 0 || id >= a.c.n_pages) {
                        id = -1;
                        if (a.dev_status != nullptr) atomicOr(a.dev_status, MOLORA_DEV_BAD_SEQUENCE);
                    } else {
                        const int64_t block = (int64_t)id * a.c.kv_heads + u.head;
                        const float vs = clamped_scale(ld_dependent(a.c.v_scale + block));
                        sc = make_float4(ld_dependent(a.c.k_scale + block), log2f(vs), 1.f / vs, 1.f);
                    }
                }
            };
            look_up(u.u0);
            for (int i = u.u0; i < u.u1; ++i, ++tiles) {
                const int slot = tiles % kScaleRing, st = tiles & 1;
                const uint32_t again = ((uint32_t)(tiles >> 1) & 1u) ^ 1u;
                const int key0 = u.lo + i * kKeys;
                // (the slot's last tile was four tiles ago: its weights went into an O before the place of V two tiles ago was given back)
                if (ct < 8) s_scales[slot][ct] = sc, s_pages[slot][ct] = id;
                if (ct < 4) s_nan[slot][ct] = 0;
                sync();
                uint4 k[8], v[8];
                auto load = [&](const uint8_t* codes, uint4* w) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int32_t page = s_pages[slot][j];
                        const int64_t line = (((int64_t)page * a.c.kv_heads + u.head) << plog) + ((key0 + 16 * j + r0) & ((1 << plog) - 1));
                        w[j] = page >= 0 ? ld128_rw_stream(codes + line * kDim + chunk * 16) : make_uint4(0, 0, 0, 0);
                    }
                };
                load(a.c.k, k);
                load(a.c.v, v);
                look_up(i + 1);
                if (tiles >= 2) wait_bar(bar(&ctrl.k_empty[st]), again, abort_flag, a.dev_status);
#pragma unroll
                for (int j = 0; j < 8; ++j) store_codes_f16(smem + kKAt + st * kOperandBytes, 16 * j + r0, chunk, k[j]);
                fence_proxy_async_smem();
                mbar_arrive(bar(&ctrl.k_full[st]));
                if (key0 + kKeys > u.hi_min || key0 < u.lo_max) {
                    // Some row does not see some key: values that no row sees count as zero; a NaN among the codes of one becomes a NaN in the scores of
                    // the rows that see it and a zero here, so that it cannot reach the others through their weight of zero.
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int key = key0 + 16 * j + r0;
                        const bool none = key >= u.hi_max || key < u.lo_min;
                        uint32_t* w[4] = {&v[j].x, &v[j].y, &v[j].z, &v[j].w};
                        bool nan = false;
#pragma unroll
                        for (int z = 0; z < 4; ++z) {
                            const uint32_t bits = e4m3x4_nan_bits(*w[z]);
                            nan |= bits != 0;
                            *w[z] = none ? 0u : *w[z] & ~((bits >> 7) * 0xFFu);
                        }
                        if (nan && !none) atomicOr(&s_nan[slot][(16 * j + r0) >> 5], 1u << ((16 * j + r0) & 31));
                    }
                }
                if (tiles >= 2) wait_bar(bar(&ctrl.v_empty[st]), again, abort_flag, a.dev_status);
#pragma unroll
                for (int j = 0; j < 8; ++j) store_codes_f16(smem + kVAt + st * kOperandBytes, 16 * j + r0, chunk, v[j]);
                fence_proxy_async_smem();
                mbar_arrive(bar(&ctrl.v_full[st]));
            }
        }
        if (ct == 0) cuts[blockIdx.x] = *abort_flag == 0 ? cut : CutUnit{0, 0, 0, 0};
    } else {
        // ============================================================ MMAs
        const bool leader = elect_one();
        const uint32_t tm = __shfl_sync(0xFFFFFFFFu, tmem, 0);
        constexpr uint32_t idesc_s = idesc_f16_f32(kTileRows, kKeys, 0), idesc_o = idesc_f16_f32(kTileRows, kDim, 1);
        constexpr uint32_t kL128 = swizzle_layout_type(Swizzle::B128);
        const uint64_t q_desc = smem_desc(base + kQAt, 16, 1024, kL128), k_desc = smem_desc(base + kKAt, 16, 1024, kL128);
        const uint64_t v_desc = smem_desc(base + kVAt, kOperandBytes / 2, 1024, kL128);      // 64 elements a group, 8 keys a group
        bool live = true;
        int units[2] = {0, 0}, ps[2] = {0, 0};        // of each tile of rows: units with keys, weights waited for
        int tiles = 0;
        auto issue_s = [&](int t, int kt, bool last) {
            if (leader && live) {
                const uint64_t qa = (uint64_t)(t * (kOperandBytes >> 4)), ka = (uint64_t)((kt & 1) * (kOperandBytes >> 4));
#pragma unroll
                for (int j = 0; j < 8; ++j) {         // 16 elements a step, 64 a part
                    const uint64_t off = (uint64_t)((j >> 2) * (kOperandBytes / 2 >> 4) + (j & 3) * 2);
                    umma_f16(tm + (uint32_t)(t * 128), q_desc + qa + off, k_desc + ka + off, idesc_s, j > 0);
                }
                umma_commit(bar(&ctrl.s_full[t]));
                if (last) umma_commit(bar(&ctrl.k_empty[kt & 1]));
            }
            __syncwarp();
        };
        auto issue_o = [&](int t, int kt, bool begins, bool ends, bool last) {
            live = wait_bar(bar(&ctrl.p_full[t]), (uint32_t)(t == 0 ? ps[0]++ : ps[1]++) & 1u, abort_flag, a.dev_status) && live;
            live = wait_bar(bar(&ctrl.v_full[kt & 1]), (uint32_t)(kt >> 1) & 1u, abort_flag, a.dev_status) && live;
            tc_fence_after();
            if (leader && live) {
                const uint64_t va = (uint64_t)((kt & 1) * (kOperandBytes >> 4));
#pragma unroll
                for (int j = 0; j < 8; ++j)           // 16 keys a step: two groups of 8 lines
                    umma_bf16_ts(tm + kOCol + (uint32_t)(t * 128), tm + (uint32_t)(t * 128 + j * 8), v_desc + va + j * (2048 >> 4), idesc_o, !begins || j > 0);
                if (last) umma_commit(bar(&ctrl.v_empty[kt & 1]));
                if (ends) umma_commit(bar(&ctrl.o_full[t]));
            }
            __syncwarp();
        };
        auto wait_k = [&](int kt) {
            live = wait_bar(bar(&ctrl.k_full[kt & 1]), (uint32_t)(kt >> 1) & 1u, abort_flag, a.dev_status) && live;
            tc_fence_after();
        };
        while (live && walk.next(u)) {
            const int n = u.u1 - u.u0;
            if (n <= 0) continue;
            const bool two = u.n_rows > kTileRows;
            for (int t = 0; t < 1 + two; ++t) {
                live = wait_bar(bar(&ctrl.q_full[t]), (uint32_t)(t == 0 ? units[0]++ : units[1]++) & 1u, abort_flag, a.dev_status) && live;
                if (t == 0) wait_k(tiles);
                tc_fence_after();
                issue_s(t, tiles, t == (int)two);
            }
            for (int i = 0; i < n && live; ++i) {
                const int kt = tiles + i;
                const bool ends = i + 1 == n;
                issue_o(0, kt, i == 0, ends, !two);
                if (!ends) wait_k(kt + 1), issue_s(0, kt + 1, !two);
                if (two) {
                    issue_o(1, kt, i == 0, ends, true);
                    if (!ends) issue_s(1, kt + 1, true);
                }
            }
            tiles += n;
        }
        if (leader) umma_commit(bar(&ctrl.drained));  // nothing of the tensor cores' is in flight when TMEM and shared memory are given up
        const long long c0 = clock64();
        while (!mbar_try_wait(bar(&ctrl.drained), 0))
            if (clock64() - c0 > kTimeoutCycles) break;
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) tmem_dealloc(tmem, kTmemCols);
}

int64_t share_count() { return sm_count(); }

}  // namespace

// bf16, heads of 128
bool attend_tiles_eligible(const KvView& c, molora_dtype_t dt) { return dt == MOLORA_BF16 && c.dim == kDim && c.n_pages > 0; }

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
    return cuda_ok(launch_kernel(attend_join_kernel<__nv_bfloat16, kDim, kUnitRows>, dim3((unsigned)shares, kUnitRows / kJoinRows), dim3(kJoinWarps * 32), 0, s,
                                 1, true, a, static_cast<const CutUnit*>(cuts), static_cast<const float*>(slots)));
}

}  // namespace molora
