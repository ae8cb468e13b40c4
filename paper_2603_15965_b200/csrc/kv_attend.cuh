// What the attention kernels over the paged cache share: units, their equal shares, what a cut unit leaves behind, the join.
//
// A row of a sequence is (new token, query head of the group that shares a key / value head); ROWS consecutive rows, one key /
// value head and the keys that they see are a UNIT.  The units' keys, cut into steps of KEYS, form one long list; every CTA of the
// grid (or each of its workers) takes an equal, contiguous share of it, whatever the lengths of the sequences.  A unit that lies inside one share is written at
// once; one that is cut leaves its pieces (sum, reference, weighted values, all fp32) in the workspace, and a second kernel joins
// them in the order of the keys: results do not depend on timing.
#pragma once
#include "kv_cache.cuh"

namespace molora {
namespace {

constexpr float kNone = -1e30f;              // reference of a row that has seen nothing

// What a cut unit leaves behind.
struct alignas(16) CutUnit {
    int32_t row0, tile_row, rows, head;      // first row of its sequence; of its tile: the first row and how many there are; key / value head
    int32_t pieces, unused[3];               // 0: no unit begins in this share and goes on in the next
};
__host__ __device__ constexpr int slot_floats(int rows, int dim) { return 2 * rows + rows * dim; }
__host__ __device__ inline size_t cut_bytes(int64_t workers) { return (size_t)((workers * (int64_t)sizeof(CutUnit) + 255) / 256 * 256); }

// steps of every unit of a sequence, and where its keys begin.  In front of its keys a unit has COST steps without any, so that shares are
// equal in time where short sequences come with their units' fixed costs.
struct Span {
    int32_t lo;        // first key, a multiple of KEYS
    int32_t steps;     // per unit
    int32_t tiles;     // of rows
};
template <int ROWS, int KEYS, int COST>
__device__ __forceinline__ Span span_of(const Sequence& s, int group, int window)
{
    Span r{0, 0, 0};
    if (s.n == 0) return r;
    r.lo = window > 0 && s.pos0 >= window ? (s.pos0 - window + 1) & ~(KEYS - 1) : 0;
    r.steps = COST + max(1, (s.len - r.lo + KEYS - 1) / KEYS);
    r.tiles = (int32_t)(((int64_t)s.n * group + ROWS - 1) / ROWS);
    return r;
}
// steps of all units of a sequence
template <int ROWS, int KEYS, int COST>
__device__ __forceinline__ int64_t steps_of(const AttendArgs& a, const Sequence& s, int group)
{
    const Span sp = span_of<ROWS, KEYS, COST>(s, group, a.window);
    return (int64_t)sp.steps * sp.tiles * a.c.kv_heads;
}

// A unit, and what of its keys lies in this share.
struct Unit {
    Sequence sq;
    Span sp;
    int64_t at;                             // its first step in the list
    int32_t b, head, tile, first, last;     // its steps [first, last) are in this share
    int32_t n_rows, tile_row;
    int32_t hi_min, hi_max, lo_min, lo_max; // keys below hi_min and from lo_max on are seen by every row, [lo_min, hi_max) by some
    int32_t u0, u1;                         // its steps of keys, counted from lo, that some row sees
};
__device__ __forceinline__ int upper_key(const AttendArgs& a, const Sequence& sq, int token)
{
    return a.causal ? max(0, min(sq.pos0 + token + 1, sq.len)) : sq.len;
}
__device__ __forceinline__ int lower_key(const AttendArgs& a, const Sequence& sq, int token)
{
    const int p = sq.pos0 + token;
    return a.window > 0 && p >= a.window ? p - a.window + 1 : 0;      // (p may be far below 0)
}

// a / b of numbers that are not negative; most a are below 2^32, where it is a fifth of the instructions
__device__ __forceinline__ int64_t quotient(int64_t a, int32_t b)
{
    return (uint64_t)a >> 32 == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// Where a share begins: which part of the sequences (see cut_shares), the first step of it, how many steps there are and how many a share has.
struct ShareStart {
    int64_t base, total, share;
    int32_t part;
    Sequence sq;                            // the part's first sequence
};

// The units of a share, in order; every thread (or warp) that asks gets the same.
template <int ROWS, int KEYS, int COST>
struct Walk {
    const AttendArgs& a;
    int64_t at, stop, base;                 // next step, end of the share, first step of sequence b
    int64_t share = 1;
    int b, group;
    Sequence sq;
    Span sp;
    __device__ explicit Walk(const AttendArgs& args) : a(args), at(0), stop(0), base(0), b(0), group(args.group) {}

    __device__ void load()
    {
        sq = sequence_of(a.c, b, a.N);
        sp = span_of<ROWS, KEYS, COST>(sq, group, a.window);
    }
    __device__ bool next(Unit& u)
    {
        if (at >= stop) return false;
        while (base + (int64_t)sp.steps * sp.tiles * a.c.kv_heads <= at) {
            base += (int64_t)sp.steps * sp.tiles * a.c.kv_heads;
            ++b;
            load();
        }
        const int64_t unit = quotient(at - base, sp.steps);
        u.sq = sq, u.sp = sp, u.b = b;
        u.at = base + unit * sp.steps;
        u.first = (int)(at - u.at), u.last = (int)min((int64_t)sp.steps, stop - u.at);
        u.tile = (int)quotient(unit, a.c.kv_heads), u.head = (int)(unit - (int64_t)u.tile * a.c.kv_heads);
        u.tile_row = u.tile * ROWS;
        u.n_rows = (int)min((int64_t)ROWS, (int64_t)sq.n * group - u.tile_row);
        at = u.at + u.last;
        const bool one = sq.n == 1;         // (nothing to divide)
        const int t0 = one ? 0 : u.tile_row / group, t1 = one ? 0 : (u.tile_row + u.n_rows - 1) / group;
        u.hi_min = upper_key(a, sq, t0), u.hi_max = upper_key(a, sq, t1);
        u.lo_min = lower_key(a, sq, t0), u.lo_max = lower_key(a, sq, t1);
        u.u0 = max(u.first - COST, (u.lo_min - sp.lo) / KEYS);
        u.u1 = min(u.last - COST, u.hi_max > sp.lo ? (u.hi_max - sp.lo + KEYS - 1) / KEYS : 0);
        return true;
    }
    // the shares in which the unit lies, from this one (w), where it begins, on
    __device__ int32_t pieces(const Unit& u, int64_t w) const { return (int32_t)((u.at + u.sp.steps - 1) / share - w + 1); }
    // Puts the walk at the beginning of share w; `parts`: into how many parts the sequences are divided.
    __device__ void begin(const ShareStart& from, int64_t w, int parts)
    {
        share = from.share;
        at = w * share;
        stop = min(from.total, at + share);
        if (at >= stop) return;
        b = from.part * ((a.c.B + parts - 1) / parts);
        base = from.base;
        sq = from.sq;
        sp = span_of<ROWS, KEYS, COST>(sq, group, a.window);
    }
};

// Equal shares of all steps, none shorter than min_share: where the W shares from first_share on begin, into s_start.  All THREADS threads of
// the CTA; each looks after a part of the sequences, steps_of tells the steps of one.
template <int THREADS, int W, typename StepsOf>
__device__ __forceinline__ void cut_shares(const AttendArgs& a, int64_t first_share, int64_t shares, int min_share, ShareStart* s_start, StepsOf steps_of)
{
    __shared__ int64_t s_warp[32];
    const int tid = (int)threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int part = (a.c.B + THREADS - 1) / THREADS;
    int64_t own = 0;
    Sequence first{};
    for (int b = tid * part; b < min(a.c.B, (tid + 1) * part); ++b) {
        const Sequence sq = sequence_of(a.c, b, a.N);
        if (b == tid * part) first = sq;
        own += steps_of(sq);
        if (sq.bad && blockIdx.x == 0 && a.dev_status != nullptr) atomicOr(a.dev_status, MOLORA_DEV_BAD_SEQUENCE);
    }
    auto scan = [lane](int64_t v) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t up = __shfl_up_sync(0xFFFFFFFFu, v, o);
            if (lane >= o) v += up;
        }
        return v;
    };
    int64_t upto = scan(own);
    if (lane == 31) s_warp[warp] = upto;
    __syncthreads();
    const int64_t warps = scan(lane < THREADS / 32 ? s_warp[lane] : 0);
    const int64_t before = __shfl_sync(0xFFFFFFFFu, warps, (warp - 1) & 31), total = __shfl_sync(0xFFFFFFFFu, warps, 31);
    if (warp > 0) upto += before;
    const int64_t share = max(quotient(total + shares - 1, (int32_t)shares), (int64_t)min_share);
#pragma unroll
    for (int w = 0; w < W; ++w) {
        const int64_t at = (first_share + w) * share;
        if (at >= upto - own && at < upto) s_start[w].base = upto - own, s_start[w].part = tid, s_start[w].sq = first;
        if (tid == 0) s_start[w].total = total, s_start[w].share = share;
    }
    __syncthreads();
}

// The power of two that brings a row of q, of largest magnitude amax (NaN aside), to [2^TOP, 2^(TOP + 1)), and its reciprocal.  A row with an infinity
// in it becomes NaN throughout, as its softmax is (scores of both signs, or all of them one infinity): 8-bit terms would saturate instead, and a row
// whose scores are all -infinity would look like one that sees nothing.
struct RowScale {
    float up, down;
};
template <int TOP>
__device__ __forceinline__ RowScale row_scale(float amax)
{
    const int e = amax > 0.f ? min(100, TOP - ((int)(__float_as_uint(amax) >> 23) - 127)) : 0;
    return {amax > 3.402823466e38f ? __int_as_float(0x7FC00000) : __uint_as_float((uint32_t)(e + 127) << 23), __uint_as_float((uint32_t)(127 - e) << 23)};
}

// A kernel's columns of TMEM, by one warp: after the wait for its predecessor, which may hold them, and before its successor may start.
__device__ __forceinline__ void take_tmem(uint32_t* base, uint32_t columns)
{
    ptx::tmem_alloc(ptx::smem_u32(base), columns);
    ptx::tmem_relinquish();
}

// Scales of V, and the softmax's sum.  With s a score in powers of two, vs the scale of its key's block and m the row's reference, a key adds 2^(s - m) to
// the sum and is handed to the tensor cores with the weight 2^(s - m) vs, which has the size of what it contributes; m goes by the largest
// weight, the sum goes by the scores alone.  So fp32 has to hold both ends at once: where the reference was set, a weight was 2^5 or more, and its
// part of the sum 2^5 / vs; no weight is ever above 2^15, and no part above 2^15 / vs.  Scales are read as if they lay in [2^-100, 2^90], times 2^18
// (taken off the result): parts reach from 2^-103 to 2^97, sums of 2^30 of them stay below 2^128, and what is flushed, below 2^-126, is 2^-23 of
// its row's sum at most, at the far ends only.  (2^(s - m) as the weight over vs lost whole blocks where scales lay 2^126 apart.)
constexpr float kVScaleUp = 262144.f, kVScaleDown = 1.f / 262144.f;
__device__ __forceinline__ float read_v_scale(float v) { return fminf(fmaxf(v, 7.8886090522e-31f), 1.2379400393e27f) * kVScaleUp; }

// 2^d, d <= 0, as half * half: a sum may move between references that lie further apart than one factor can say.  (A factor and a constant that is
// 2^-120 where d is below: 2 % slower for prompts with heads of 64.)
struct Shrink {
    float half;
    __device__ __forceinline__ explicit Shrink(float d) : half(ex2(0.5f * d)) {}
    __device__ __forceinline__ float both() const { return half * half; }
    __device__ __forceinline__ float of(float sum) const { return sum * half * half; }
};

// two sums, two products, two products and sums in one instruction each
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 r;
    asm("{\n\t.reg .b64 A, B, C;\n\tmov.b64 A, {%2, %3};\n\tmov.b64 B, {%4, %5};\n\tadd.rn.f32x2 C, A, B;\n\tmov.b64 {%0, %1}, C;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 r;
    asm("{\n\t.reg .b64 A, B, C;\n\tmov.b64 A, {%2, %3};\n\tmov.b64 B, {%4, %5};\n\tmul.rn.f32x2 C, A, B;\n\tmov.b64 {%0, %1}, C;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 r;
    asm("{\n\t.reg .b64 A, B, C, D;\n\tmov.b64 A, {%2, %3};\n\tmov.b64 B, {%4, %5};\n\tmov.b64 C, {%6, %7};\n\tfma.rn.f32x2 D, A, B, C;\n\tmov.b64 {%0, %1}, D;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}

// four elements of a row's result: values over sum
__device__ __forceinline__ float4 over(float4 v, float f)
{
    return make_float4(v.x * kVScaleDown * f, v.y * kVScaleDown * f, v.z * kVScaleDown * f, v.w * kVScaleDown * f);
}
__device__ __forceinline__ void store4(float* p, float4 v, float f) { *reinterpret_cast<float4*>(p) = over(v, f); }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 v, float f)
{
    const float4 r = over(v, f);
    *reinterpret_cast<uint2*>(p) = make_uint2(f32x2_to_bf16x2(r.x, r.y), f32x2_to_bf16x2(r.z, r.w));
}

// Joins the pieces of the units that are cut: with M the largest reference, the sums of 2^(m - M) (values, sum) over the pieces,
// always in the same order.  A CTA looks after rows of the unit that begins in share blockIdx.x and goes on behind it, four rows at a time.
// Units of few rows come in many pieces: four rows a CTA, whose warps take every fourth piece each and are added up in order (asked for row by row,
// the pieces of a unit cut into 55 took 32 us).  Units of many rows come in few: four rows a warp, all of their pieces (four rows a CTA, a chunk's
// 148 cut units of 256 rows took 20 us).
constexpr int kJoinWarps = 4, kJoinRows = 4;
__host__ __device__ constexpr bool join_by_warp(int rows) { return rows > 32; }
__host__ constexpr unsigned join_groups(int rows) { return (unsigned)(rows / (join_by_warp(rows) ? kJoinWarps * kJoinRows : kJoinRows)); }
template <typename T, int D, int ROWS>
__global__ void __launch_bounds__(kJoinWarps * 32) attend_join_kernel(const __grid_constant__ AttendArgs a, const CutUnit* __restrict__ cuts,
                                                                     const float* __restrict__ slots)
{
    constexpr int kLanes = D / 4;                          // lanes of four elements
    constexpr bool kAlone = join_by_warp(ROWS);
    __shared__ float4 part[kAlone ? 1 : kJoinWarps][kJoinRows][kLanes];
    __shared__ float part_l[kJoinWarps][kJoinRows];
    ptx::grid_dependency_sync();
    const int4 cut = __ldcg(reinterpret_cast<const int4*>(cuts + blockIdx.x));
    const int pieces = __ldcg(&cuts[blockIdx.x].pieces);
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    const int r0 = kJoinRows * (kAlone ? (int)blockIdx.y * kJoinWarps + warp : (int)blockIdx.y), rows = cut.z - r0;
    if (pieces == 0 || rows <= 0) return;
    const int64_t w0 = blockIdx.x;
    auto slot = [&](int p) { return slots + (p == 0 ? 2 * w0 + 1 : 2 * (w0 + p)) * (int64_t)slot_floats(ROWS, D) + r0; };
    // row `row` of the unit: its sum, its values and the reference that they are in
    auto write = [&](int row, float4 v, float sum, float top) {
        const int r = cut.y + row, token = r / a.group;
        const int64_t orow = (int64_t)cut.x + token;
        const int oh = cut.w * a.group + (r - token * a.group);
        if (lane < kLanes) store4(static_cast<T*>(a.out) + orow * a.ldo + (int64_t)oh * D + lane * 4, v, sum == 0.f ? 0.f : 1.f / sum);
        if (a.lse != nullptr && lane == 0) a.lse[orow * a.heads + oh] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718056f;
    };
    float M[kJoinRows], L[kJoinRows] = {};
    float4 acc[kJoinRows] = {};
#pragma unroll
    for (int r = 0; r < kJoinRows; ++r) M[r] = kNone;
    for (int p = lane; p < pieces; p += 32) {
        const float4 m = __ldcg(reinterpret_cast<const float4*>(slot(p)));
        M[0] = fmaxf(M[0], m.x), M[1] = fmaxf(M[1], m.y), M[2] = fmaxf(M[2], m.z), M[3] = fmaxf(M[3], m.w);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int r = 0; r < kJoinRows; ++r) M[r] = fmaxf(M[r], __shfl_xor_sync(0xFFFFFFFFu, M[r], o));
    // (rows behind the last hold whatever was there: their M, sums and values are not used)
#pragma unroll 4
    for (int p = kAlone ? 0 : warp; p < pieces; p += kAlone ? 1 : kJoinWarps) {
        const float* s = slot(p);
        const float4 m = __ldcg(reinterpret_cast<const float4*>(s)), l = __ldcg(reinterpret_cast<const float4*>(s + ROWS));
        const Shrink by[kJoinRows] = {Shrink(m.x - M[0]), Shrink(m.y - M[1]), Shrink(m.z - M[2]), Shrink(m.w - M[3])};
        const float f[kJoinRows] = {by[0].both(), by[1].both(), by[2].both(), by[3].both()};
        L[0] += by[0].of(l.x), L[1] += by[1].of(l.y), L[2] += by[2].of(l.z), L[3] += by[3].of(l.w);
#pragma unroll
        for (int r = 0; r < kJoinRows; ++r)
            if (r < rows && lane < kLanes) {
                const float4 x = __ldcg(reinterpret_cast<const float4*>(s + 2 * ROWS - r0 + (r0 + r) * D + lane * 4));
                acc[r].x = fmaf(x.x, f[r], acc[r].x), acc[r].y = fmaf(x.y, f[r], acc[r].y);
                acc[r].z = fmaf(x.z, f[r], acc[r].z), acc[r].w = fmaf(x.w, f[r], acc[r].w);
            }
    }
    if constexpr (kAlone) {
#pragma unroll
        for (int r = 0; r < kJoinRows; ++r)
            if (r < rows) write(r0 + r, acc[r], L[r], M[r]);
    } else {
#pragma unroll
        for (int r = 0; r < kJoinRows; ++r) {
            if (lane < kLanes) part[warp][r][lane] = acc[r];
            if (lane == 0) part_l[warp][r] = L[r];
        }
        __syncthreads();
        if (warp >= rows) return;                          // a row per warp from here on
        float sum = 0.f;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int z = 0; z < kJoinWarps; ++z) {
            const float4 x = part[z][warp][lane % kLanes];
            v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
            sum += part_l[z][warp];
        }
        write(r0 + warp, v, sum, warp == 0 ? M[0] : warp == 1 ? M[1] : warp == 2 ? M[2] : M[3]);
    }
}

}  // namespace
}  // namespace molora
