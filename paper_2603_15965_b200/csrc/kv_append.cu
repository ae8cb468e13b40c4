// Position rotation and append to the paged 8-bit cache (molora_kv_append).
//
// A block of the cache (one page of one head) has one scale, so what a call adds to a block is handled by one CTA (or, a few
// tokens only, by one warp): it holds the rotated values in registers, reduces their largest magnitude, and writes codes and
// scale.  Nothing is read twice; older tokens of the block are touched only when the scale has to grow, which a power of two
// does seldom and, for e4m3 codes, without rounding anything but values that become subnormal.
//   grid.x   runs of `run` consecutive rows; a CTA takes the pieces (rows of one sequence inside one page) that begin in its run
//   grid.y   groups of kHeadsPerCta heads of k, of v, of q
// A thread's unit is 16 elements of a row -- two 8-element vectors that the rotation pairs, or that lie side by side -- and stays
// the same for every head of the group, so sines and cosines are computed once per CTA, in turns: p * f / 2 pi in 64 bits, reduced
// to half a turn, then sinpi / cospi in fp32.
#include "kv_cache.cuh"

namespace molora {
namespace {

constexpr int kHeadsPerCta = 8;
constexpr int kUnits = 2;              // units per thread: a page of 128 tokens of 128 elements over 512 threads
constexpr int kWarpTokens = 8;         // pieces of up to this many tokens: a warp per head

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* x);
template <>
__device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float* x)
{
    unpack<__nv_bfloat16>(ld128_rw_stream(p), x);
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float* x)
{
    unpack<float>(ld128_rw_stream(p), x);
    unpack<float>(ld128_rw_stream(p + 4), x + 4);
}
template <typename T>
__device__ __forceinline__ void store8(T* p, const float* x)
{
    stg128(p, pack<T>(x));
    if constexpr (sizeof(T) == 4) stg128(p + 4, pack<T>(x + 4));
}

struct AppendArgs {
    KvView c;
    int64_t N;
    const void *k, *v, *q;
    void* q_out;
    int64_t ldk, ldv, ldq, ldqo;
    int32_t heads, rotary, interleaved, run, k_groups, dim;
    const float* inv_freq;
    uint32_t* dev_status;
};

// the smallest 2^e with amax <= 448 * 2^e (448 = 1.75 * 2^8, the largest e4m3 value), e in [-64, 64]
__device__ __forceinline__ float scale_for(float amax)
{
    const uint32_t u = __float_as_uint(amax);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return __uint_as_float((uint32_t)(max(-64, min(64, e)) + 127) << 23);
}

// One unit of a thread: where its two vectors lie in a row, and its eight pairs' cosines and sines.
struct Unit {
    int token;                 // within the piece; past its end: no unit
    int off0, off1;
    int kind;                  // 0: not rotated, 1: pairs across the two vectors, 2: neighbours inside each
    float c[8], s[8];
};

__device__ __forceinline__ void make_unit(Unit& u, int id, int count, int pos0, const AppendArgs& a, bool rotate)
{
    const int per_token = a.dim >> 4, j = id % per_token;
    u.token = id / per_token;
    const int rotary = rotate ? a.rotary : 0;
    u.off0 = j * 16, u.off1 = j * 16 + 8, u.kind = 0;
    if (j * 16 < rotary) {
        u.kind = a.interleaved ? 2 : 1;
        if (!a.interleaved) u.off0 = j * 8, u.off1 = j * 8 + rotary / 2;
    }
    if (u.kind == 0 || u.token >= count) return;
    const double pos = (double)(pos0 + u.token);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double turns = pos * (double)ptx::ld_dependent(a.inv_freq + j * 8 + i) * 0.15915494309189533577;      // 1 / 2 pi
        const float half_turns = (float)((turns - rint(turns)) * 2.0);
        sincospif(half_turns, &u.s[i], &u.c[i]);
    }
}

__device__ __forceinline__ void rotate_unit(const Unit& u, float* x)
{
    if (u.kind == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = x[i], b = x[8 + i];
            x[i] = a * u.c[i] - b * u.s[i];
            x[8 + i] = b * u.c[i] + a * u.s[i];
        }
    } else if (u.kind == 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = x[2 * i], b = x[2 * i + 1];
            x[2 * i] = a * u.c[i] - b * u.s[i];
            x[2 * i + 1] = b * u.c[i] + a * u.s[i];
        }
    }
}

__device__ __forceinline__ float finite_amax(const float* x, float m)
{
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float v = fabsf(x[i]);
        m = fmaxf(m, v <= 3.402823466e38f ? v : 0.f);        // infinities and NaN have no say
    }
    return m;
}

__device__ __forceinline__ void store_codes(uint8_t* row, const Unit& u, const float* x, float inv)
{
    const uint2 a = make_uint2(f32x4_to_e4m3x4(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv),
                               f32x4_to_e4m3x4(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv));
    const uint2 b = make_uint2(f32x4_to_e4m3x4(x[8] * inv, x[9] * inv, x[10] * inv, x[11] * inv),
                               f32x4_to_e4m3x4(x[12] * inv, x[13] * inv, x[14] * inv, x[15] * inv));
    if (u.off1 == u.off0 + 8) {
        *reinterpret_cast<uint4*>(row + u.off0) = make_uint4(a.x, a.y, b.x, b.y);
    } else {
        *reinterpret_cast<uint2*>(row + u.off0) = a;
        *reinterpret_cast<uint2*>(row + u.off1) = b;
    }
}

// 16 older codes divided by the growth of their block's scale
__device__ __forceinline__ void regrow16(uint8_t* p, float ratio)
{
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 a = f16x2_to_f32x2(e4m3x2_to_f16x2(w[i])), b = f16x2_to_f32x2(e4m3x2_to_f16x2_high(w[i]));
        r[i] = f32x4_to_e4m3x4(a.x * ratio, a.y * ratio, b.x * ratio, b.y * ratio);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(r[0], r[1], r[2], r[3]);
}

// The sequence that row i belongs to: the number of cu[1..B] that are <= i (32 probes a round); B if none
__device__ __forceinline__ int sequence_of_row(const int32_t* cu, int B, int64_t i)
{
    const int lane = threadIdx.x & 31;
    int base = 0, span = B;                                // the answer is in [base, base + span]
    while (span > 0) {
        const int step = (span + 31) / 32;
        const int at = min(base + (lane + 1) * step, base + span);
        const unsigned le = __ballot_sync(0xFFFFFFFFu, (int64_t)ptx::ld_dependent(cu + at) <= i);
        const int k = __popc(le);                          // (a prefix of the lanes, cu being sorted)
        const int next = min(base + k * step, base + span);
        span = k == 32 ? 0 : min(step - 1, base + span - next);
        base = next;
    }
    return base;
}

template <typename T>
__global__ void __launch_bounds__(512) kv_append_kernel(const __grid_constant__ AppendArgs a)
{
    __shared__ float warp_max[16];
    ptx::grid_dependency_sync();
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31, threads = (int)blockDim.x, warps = threads >> 5;
    // the group of heads
    const int g = (int)blockIdx.y;
    const int kind = g < a.k_groups ? 0 : g < 2 * a.k_groups ? 1 : 2;                  // k, v, q
    const int h0 = (kind == 0 ? g : kind == 1 ? g - a.k_groups : g - 2 * a.k_groups) * kHeadsPerCta;
    const int h1 = min(h0 + kHeadsPerCta, kind == 2 ? a.heads : a.c.kv_heads);
    const T* src = static_cast<const T*>(kind == 0 ? a.k : kind == 1 ? a.v : a.q);
    const int64_t ld = kind == 0 ? a.ldk : kind == 1 ? a.ldv : a.ldq;
    uint8_t* codes = kind == 0 ? a.c.k : a.c.v;
    float* scales = kind == 0 ? a.c.k_scale : a.c.v_scale;
    const int page = 1 << a.c.page_log2, units = a.dim >> 4;

    const int64_t run_end = min(a.N, ((int64_t)blockIdx.x + 1) * a.run);
    int64_t i = (int64_t)blockIdx.x * a.run;
    int b = sequence_of_row(a.c.cu, a.c.B, i);
    while (i < run_end && b < a.c.B) {
        const Sequence sq = sequence_of(a.c, b, a.N);
        const int64_t end = (int64_t)sq.row0 + sq.n;
        if (i >= end) {                                    // an empty sequence, or the end of this one
            ++b;
            continue;
        }
        const int64_t j = i - sq.row0;
        if (j < 0) break;                                  // (rows of no sequence: cu does not start at 0)
        const int pos = sq.first_pos() + (int)j;
        const bool report = sq.bad && tid == 0 && g == 0 && a.dev_status != nullptr;
        if (report) atomicOr(a.dev_status, MOLORA_DEV_BAD_SEQUENCE);
        if (pos < 0) {                                     // in front of the sequence's beginning: left out
            i = min(end, i - pos);
            continue;
        }
        const int row0 = pos & (page - 1);
        const int count = (int)min(end - i, (int64_t)(page - row0));
        if (row0 != 0 && j != 0) {                         // begins in an earlier run, whose CTA takes it whole
            i += count;
            continue;
        }
        const int at = pos >> a.c.page_log2;
        const int32_t id = at < a.c.max_pages ? ptx::ld_dependent(a.c.table + b * a.c.ld_table + at) : -1;
        const bool usable = id >= 0 && id < a.c.n_pages;
        if (!usable && kind != 2) {
            if (tid == 0 && a.dev_status != nullptr) atomicOr(a.dev_status, MOLORA_DEV_BAD_SEQUENCE);
            i += count;
            continue;
        }
        const bool by_warp = count <= kWarpTokens;
        const int id0 = by_warp ? lane : tid, stride = by_warp ? 32 : threads;
        Unit u[kUnits];
#pragma unroll
        for (int n = 0; n < kUnits; ++n) make_unit(u[n], id0 + n * stride, count, pos, a, kind != 1);
        if (kind == 2) {
            const int ahead = by_warp ? warps : 1;
            for (int h = h0 + (by_warp ? warp : 0); h < h1; h += ahead) {
                float x[kUnits][16];
#pragma unroll
                for (int n = 0; n < kUnits; ++n) {
                    if (u[n].token >= count) continue;
                    const T* p = src + (i + u[n].token) * ld + h * a.dim;
                    load8(p + u[n].off0, x[n]);
                    load8(p + u[n].off1, x[n] + 8);
                }
#pragma unroll
                for (int n = 0; n < kUnits; ++n) {
                    if (u[n].token >= count) continue;
                    rotate_unit(u[n], x[n]);
                    T* p = static_cast<T*>(a.q_out) + (i + u[n].token) * a.ldqo + h * a.dim;
                    store8(p + u[n].off0, x[n]);
                    store8(p + u[n].off1, x[n] + 8);
                }
            }
        } else {
            for (int h = h0 + (by_warp ? warp : 0); h < h1; h += by_warp ? warps : 1) {
                const int64_t block = (int64_t)id * a.c.kv_heads + h;
                uint8_t* rows = codes + ((block << a.c.page_log2) * a.dim);
                const float old = row0 > 0 ? scales[block] : 0.f;
                float x[kUnits][16], m = 0.f;
#pragma unroll
                for (int n = 0; n < kUnits; ++n) {
                    if (u[n].token >= count) continue;
                    const T* p = src + (i + u[n].token) * ld + h * a.dim;
                    load8(p + u[n].off0, x[n]);
                    load8(p + u[n].off1, x[n] + 8);
                }
#pragma unroll
                for (int n = 0; n < kUnits; ++n) {
                    if (u[n].token >= count) continue;
                    rotate_unit(u[n], x[n]);
                    m = finite_amax(x[n], m);
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
                if (!by_warp) {
                    if (lane == 0) warp_max[warp] = m;
                    __syncthreads();
                    for (int w = 0; w < warps; ++w) m = fmaxf(m, warp_max[w]);
                    __syncthreads();                       // (everybody has read it, and the old scale, before either is written again)
                }
                __syncwarp();
                const float scale = row0 > 0 ? fmaxf(old, scale_for(m)) : scale_for(m);
                if (id0 == 0) scales[block] = scale;
                const float inv = 1.f / scale;
#pragma unroll
                for (int n = 0; n < kUnits; ++n)
                    if (u[n].token < count) store_codes(rows + (int64_t)(row0 + u[n].token) * a.dim, u[n], x[n], inv);
                if (row0 > 0 && scale != old) {
                    const float ratio = old * inv;
                    for (int w = id0; w < row0 * units; w += stride) regrow16(rows + (int64_t)w * 16, ratio);
                }
            }
        }
        i += count;
    }
}

template <typename T>
molora_status_t launch(const AppendArgs& a, cudaStream_t s)
{
    const int page = 1 << a.c.page_log2;
    const int threads = max(256, page * (a.dim >> 4) / kUnits);
    const int groups = 2 * a.k_groups + ceil_div(a.heads, kHeadsPerCta);
    const dim3 grid((unsigned)ceil_div64(a.N, a.run), (unsigned)groups);
    return cuda_ok(launch_kernel(kv_append_kernel<T>, grid, dim3((unsigned)threads), 0, s, 1, true, a));
}

}  // namespace

molora_status_t launch_kv_append(const KvView& c, molora_dtype_t dt, int64_t N, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                 const void* q, int64_t ldq, void* q_out, int64_t ldqo, int32_t heads, const float* inv_freq,
                                 int32_t rotary, int32_t interleaved, uint32_t* dev_status, cudaStream_t s)
{
    AppendArgs a;
    a.c = c;
    a.N = N;
    a.k = k, a.v = v, a.q = q, a.q_out = q_out;
    a.ldk = ldk, a.ldv = ldv, a.ldq = ldq, a.ldqo = ldqo;
    a.heads = heads, a.rotary = rotary, a.interleaved = interleaved, a.dim = c.dim;
    a.inv_freq = inv_freq;
    a.dev_status = dev_status;
    a.k_groups = ceil_div(c.kv_heads, kHeadsPerCta);
    // rows per CTA: one while that is a few waves, else as many as the smallest page, so that most CTAs begin a piece
    a.run = N <= 1024 ? 1 : 16;
    return dt == MOLORA_F32 ? launch<float>(a, s) : launch<__nv_bfloat16>(a, s);
}

}  // namespace molora
