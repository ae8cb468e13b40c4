// Position rotation and append to the paged 8-bit cache (molora_kv_append).
//
// A block of the cache (one page of one head) has one scale, so what a call adds to a block is handled by one CTA, or, a few
// tokens only, by a part of a warp: it holds the rotated values in registers, reduces their largest magnitude, and writes codes and
// scale.  Older tokens of the block are touched only when the scale has to grow, which a power of two does seldom and, for e4m3
// codes, without rounding anything but values that become subnormal.
//   grid.x   runs of `run` consecutive rows; a CTA takes the pieces (rows of one sequence inside one page) that begin in its run
//   grid.y   groups of heads of k, of v, of q
// Sines and cosines are computed once per piece, into shared memory, in turns: p * f / 2 pi in 64 bits, reduced to half a turn, then
// sinpi / cospi in fp32, turned by what fp32 leaves of the reduced angle.  A thread's unit is 16 elements of a row -- two 8-element vectors that the rotation pairs, or that lie side by
// side -- and stays the same for every head of the group; the next head's vectors are on their way while a head is worked on (asked
// for when its turn came, two units a thread, sines in registers: 71 us against 45 for 8192 tokens of 32 + 2 x 8 heads of 128, 185 MB; 45.6 now, 4.05 TB/s).
// What bounds it there: instructions (66 % of the issue slots, conversions and packing above all) and 16 warps per SM; a token each: the chain
// of dependent reads.
#include "kv_cache.cuh"

namespace molora {
namespace {

constexpr int kMaxThreads = 1024;      // a page of 128 tokens of 128 elements

// the two vectors of a unit as they lie in memory
template <typename T>
struct Raw {
    static constexpr int kWords = 16 / VecTraits<T>::kElems;
    uint4 w[kWords];
    __device__ __forceinline__ void load(const T* row, int off0, int off1)
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            w[i] = ld128_rw_stream(row + (i < kWords / 2 ? off0 : off1) + i % (kWords / 2) * VecTraits<T>::kElems);
    }
    __device__ __forceinline__ void values(float* x) const
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) unpack<T>(w[i], x + i * VecTraits<T>::kElems);
    }
};
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
    int32_t heads, rotary, interleaved, run, per_cta, k_groups, dim;      // (per_cta, k_groups: heads of a group, groups of k)
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

// One unit of a thread: where its two vectors lie in a row, and its eight pairs' cosines and sines (in shared memory).
struct Unit {
    int token;                 // within the piece
    int off0, off1;
    int kind;                  // 0: not rotated, 1: pairs across the two vectors, 2: neighbours inside each
    const float4* turn;        // cos, sin, cos, sin of two pairs each, `next` apart
    __device__ __forceinline__ Unit(int id, const AppendArgs& a, bool rotate, const float2* turns)
    {
        const int per_token = a.dim >> 4, j = id % per_token;
        token = id / per_token;
        const int rotary = rotate ? a.rotary : 0;
        off0 = j * 16, off1 = j * 16 + 8, kind = 0, turn = nullptr;
        if (j * 16 < rotary) {
            kind = a.interleaved ? 2 : 1;
            if (!a.interleaved) off0 = j * 8, off1 = j * 8 + rotary / 2;
            turn = reinterpret_cast<const float4*>(turns + token * (rotary / 2)) + j;
        }
    }
    __device__ __forceinline__ void rotate(float* x, int next) const
    {
        if (kind == 0) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 t = turn[i * next];
            if (kind == 1) {
                turn_pair(x[2 * i], x[8 + 2 * i], t.x, t.y);
                turn_pair(x[2 * i + 1], x[8 + 2 * i + 1], t.z, t.w);
            } else {
                turn_pair(x[4 * i], x[4 * i + 1], t.x, t.y);
                turn_pair(x[4 * i + 2], x[4 * i + 3], t.z, t.w);
            }
        }
    }
    static __device__ __forceinline__ void turn_pair(float& p, float& q, float c, float s)
    {
        const float a = p, b = q;
        p = a * c - b * s;
        q = b * c + a * s;
    }
};

__device__ __forceinline__ float finite_amax(const float* x, float m)
{
    float t = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) t = fmaxf(t, fabsf(x[i]));  // (NaN has no say)
    if (t > 3.402823466e38f) {                               // nor have infinities
        t = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float v = fabsf(x[i]);
            t = fmaxf(t, v <= 3.402823466e38f ? v : 0.f);
        }
    }
    return fmaxf(m, t);
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

// WHOLE: there are as many threads as the largest piece has units
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(kMaxThreads) kv_append_kernel(const __grid_constant__ AppendArgs a)
{
    __shared__ float warp_max[kMaxThreads / 32];
    extern __shared__ __align__(16) float2 turns[];        // cosines, sines: [token of the piece][two pairs of a unit][unit][pair], so that neighbours read neighbours
    ptx::grid_dependency_sync();
    const int tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31, threads = (int)blockDim.x;
    // the group of heads
    const int g = (int)blockIdx.y;
    const int kind = g < a.k_groups ? 0 : g < 2 * a.k_groups ? 1 : 2;                  // k, v, q
    const int h0 = (kind == 0 ? g : kind == 1 ? g - a.k_groups : g - 2 * a.k_groups) * a.per_cta;
    const int h1 = min(h0 + a.per_cta, kind == 2 ? a.heads : a.c.kv_heads);
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
        if (j < 0) {                                       // rows of no sequence, in front of the first one's
            i = sq.row0;
            continue;
        }
        const int pos = sq.pos0 + (int)j;
        if (sq.bad && tid == 0 && g == 0 && a.dev_status != nullptr) atomicOr(a.dev_status, MOLORA_DEV_BAD_SEQUENCE);
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
        const int32_t id = at < a.c.max_pages && pos < kMaxTokens ? ptx::ld_dependent(a.c.table + b * a.c.ld_table + at) : -1;
        if ((id < 0 || id >= a.c.n_pages) && kind != 2) {
            if (tid == 0 && a.dev_status != nullptr) atomicOr(a.dev_status, MOLORA_DEV_BAD_SEQUENCE);
            i += count;
            continue;
        }
        // Threads per head, a power of two: as many as the piece has units, so that several heads are in hand at a time where it is short
        // (what lies inside a warp needs no barrier); a piece of more units than there are threads is gone through twice.
        const int total = count * units;
        const bool small = WHOLE || total <= threads;
        const int sub = small ? 1 << (32 - __clz(max(total - 1, 1))) : threads;
        const bool by_warp = sub <= 32;
        const int mine = tid & (sub - 1), first = h0 + tid / sub, step = threads / sub;
        if (kind != 1 && a.rotary > 0) {
            const int pairs = a.rotary >> 1;
            __syncthreads();                               // (the last piece's are done with)
            for (int z = tid; z < count * pairs; z += threads) {
                const int token = z / pairs, w = z - token * pairs;
                const double angle = (double)(pos + token) * (double)ptx::ld_dependent(a.inv_freq + w) * 0.15915494309189533577;      // 1 / 2 pi
                const double half_turns = (angle - rint(angle)) * 2.0;
                const float near = (float)half_turns, rest = (float)(half_turns - (double)near) * 3.14159265f;
                float sn, cs;
                sincospif(near, &sn, &cs);
                const float2 t = make_float2(fmaf(-sn, rest, cs), fmaf(cs, rest, sn));
                turns[token * pairs + ((((w & 7) >> 1) * (pairs >> 3) + (w >> 3)) << 1) + (w & 1)] = t;
            }
            __syncthreads();
        }
        const Unit u(min(mine, total - 1), a, kind != 1, turns);
        // (whole warps stay together: heads past the last and lanes without a unit go along)
        const int rounds = (h1 - h0 + step - 1) / step;
        const bool have = mine < total;
        Raw<T> raw;
        auto row_of = [&](int h, const Unit& v) { return src + (i + v.token) * ld + h * a.dim; };
        if (have && first < h1) raw.load(row_of(first, u), u.off0, u.off1);
        for (int r = 0; r < rounds; ++r) {
            const int h = first + r * step;
            const bool on = have && h < h1;
            float x[16];
            raw.values(x);
            if (have && h + step < h1) raw.load(row_of(h + step, u), u.off0, u.off1);
            u.rotate(x, a.rotary >> 4);
            if (kind == 2) {
                auto put = [&](const Unit& v) {
                    T* p = static_cast<T*>(a.q_out) + (i + v.token) * a.ldqo + h * a.dim;
                    store8(p + v.off0, x);
                    store8(p + v.off1, x + 8);
                };
                if (on) put(u);
                if (!small)
                    for (int z = tid + threads; z < total; z += threads) {
                        const Unit v(z, a, true, turns);
                        Raw<T> w;
                        w.load(row_of(h, v), v.off0, v.off1);
                        w.values(x);
                        v.rotate(x, a.rotary >> 4);
                        put(v);
                    }
                continue;
            }
            const int64_t block = (int64_t)id * a.c.kv_heads + min(h, h1 - 1);
            uint8_t* rows = codes + ((block << a.c.page_log2) * a.dim);
            const float old = row0 > 0 ? scales[block] : 0.f;
            float m = on ? finite_amax(x, 0.f) : 0.f;
            if (!small)                                    // more units than threads: the others are read twice
                for (int z = tid + threads; z < total; z += threads) {
                    const Unit v(z, a, kind == 0, turns);
                    Raw<T> w;
                    float y[16];
                    w.load(row_of(h, v), v.off0, v.off1);
                    w.values(y);
                    v.rotate(y, a.rotary >> 4);
                    m = finite_amax(y, m);
                }
            for (int o = min(sub, 32) >> 1; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            if (!by_warp) {
                if (lane == 0) warp_max[warp] = m;
                __syncthreads();
                const int per = sub >> 5;                  // warps of this head
                m = warp_max[(warp & ~(per - 1)) + (lane & (per - 1))];
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
                __syncthreads();                           // (everybody has read it, and the old scale, before either is written again)
            }
            __syncwarp();
            const float scale = row0 > 0 ? fmaxf(old, scale_for(m)) : scale_for(m);
            if (h >= h1) continue;
            if (mine == 0) scales[block] = scale;
            const float inv = 1.f / scale;
            if (have) store_codes(rows + (int64_t)(row0 + u.token) * a.dim, u, x, inv);
            if (!small)
                for (int z = tid + threads; z < total; z += threads) {
                    const Unit v(z, a, kind == 0, turns);
                    Raw<T> w;
                    w.load(row_of(h, v), v.off0, v.off1);
                    w.values(x);
                    v.rotate(x, a.rotary >> 4);
                    store_codes(rows + (int64_t)(row0 + v.token) * a.dim, v, x, inv);
                }
            if (row0 > 0 && scale != old) {
                const float ratio = old * inv;
                for (int w = mine; w < row0 * units; w += sub) regrow16(rows + (int64_t)w * 16, ratio);
            }
        }
        i += count;
    }
}

template <typename T>
molora_status_t launch(const AppendArgs& a, cudaStream_t s)
{
    // powers of two: single tokens, a warp for four heads of 128; drafts; one unit per thread of the largest piece there can be
    const int most = (1 << a.c.page_log2) * (a.dim >> 4);
    const int threads = a.run == 1 ? 128 : a.run < 16 ? 256 : max(512, min(kMaxThreads, most));
    const int groups = 2 * a.k_groups + ceil_div(a.heads, a.per_cta);
    const dim3 grid((unsigned)ceil_div64(a.N, a.run), (unsigned)groups);
    const size_t turns = (size_t)min((int64_t)(1 << a.c.page_log2), a.N) * (a.rotary >> 1) * sizeof(float2);      // at most 64 KB
    static bool ready[kMaxDevices] = {};
    bool& done = ready[device_slot()];
    if (!done) {
        if (cudaFuncSetAttribute(kv_append_kernel<T, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, 65536) != cudaSuccess ||
            cudaFuncSetAttribute(kv_append_kernel<T, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, 65536) != cudaSuccess)
            return MOLORA_ERR_CUDA;
        done = true;
    }
    return cuda_ok(launch_kernel(threads >= most ? kv_append_kernel<T, true> : kv_append_kernel<T, false>, grid, dim3((unsigned)threads), turns, s, 1, true, a));
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
    // Rows per CTA: as many as a sequence has on average, a page at most.  A CTA in whose run no piece begins costs its search (2 us, and
    // with runs of 16 rows three of four have none where whole pages of 64 are written), one in whose run many begin takes them in turn.
    a.run = (int32_t)max((int64_t)1, min((int64_t)(1 << c.page_log2), N / c.B));
    // Heads per CTA: sines and cosines are computed anew by every group, which costs about as much as two heads of 8, so 16 where there are
    // CTAs enough all the same.
    a.per_cta = 8;
    if (ceil_div64(N, a.run) * (2 * ceil_div(c.kv_heads, 16) + ceil_div(heads, 16)) >= 2 * sm_count()) a.per_cta = 16;
    a.k_groups = ceil_div(c.kv_heads, a.per_cta);
    return dt == MOLORA_F32 ? launch<float>(a, s) : launch<__nv_bfloat16>(a, s);
}

}  // namespace molora
