// Verification of drafted tokens (molora_verify_drafts).
//
// A cluster of CTAs works on one sequence.  Every CTA finds the number of accepted drafts by itself (one warp, one lane per
// draft: three dependent gathers).  That names the one row of p, and after a refusal the one row of q, that have to be
// read: max(p - q, 0) is summed in 64 bits, each warp over a contiguous piece of the CTA's contiguous slice, the slices' sums are
// exchanged through distributed shared memory, and the CTA in which the running sum passes u * total looks at the piece
// of the warp in which it does once more (from L2), a short run per thread.  So the vocabulary is read once, and the order of
// summation does not matter to more than the last bits of 64.
// What bounds it: the two rows, 8 bytes per word of the vocabulary in fp32 (64 sequences, 160,000 words, five drafts: 21.5 us, 11 of
// them for the 68 MB that these acceptances ask for, at 6.2 TB/s); the dependent reads in front, the exchange and the second look take the
// rest.  (Differences in 32 bits with what their rounding leaves, to spare the conversions: 20.5 us, not worth sums that are no longer 64 bits.)
#include "common.cuh"
#include "kv_cache.cuh"

namespace molora {
namespace {

constexpr int kMaxThreads = 512, kMaxWarps = kMaxThreads / 32;
constexpr int kMaxCluster = 8;

__device__ __forceinline__ float load_prob(const float* p) { return ptx::ld_dependent(p); }
__device__ __forceinline__ float load_prob(const __nv_bfloat16* p)
{
    uint16_t v;
    asm volatile("ld.global.u16 %0, [%1];" : "=h"(v) : "l"(p) : "memory");
    return __uint_as_float((uint32_t)v << 16);
}

// one term of the distribution that the next token is drawn from; q may be null
template <typename T>
struct Residual {
    const T* p;
    const T* q;
    int32_t certain;          // the drafted token where the drafter gives no distribution (-1: none)
    __device__ double at(int t) const
    {
        const float a = load_prob(p + t);
        return term(a, q != nullptr ? load_prob(q + t) : 0.f, t);
    }
    __device__ double term(float a, float b, int t) const { return a > b && t != certain ? (double)a - (double)b : 0.0; }
};

__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// sum of the terms [lo, hi) by one warp, 16 bytes a load where p and q allow it
template <typename T>
__device__ double piece_sum(const Residual<T>& r, int lo, int hi)
{
    constexpr int E = VecTraits<T>::kElems;
    const int lane = threadIdx.x & 31;
    double acc = 0.0;
    const uintptr_t ap = reinterpret_cast<uintptr_t>(r.p + lo) & 15u;
    const bool vec = r.q == nullptr || ap == (reinterpret_cast<uintptr_t>(r.q + lo) & 15u);
    if (!vec) {
        for (int t = lo + lane; t < hi; t += 32) acc += r.at(t);
        return warp_sum(acc);
    }
    const int body = min(hi, lo + (int)(((16u - ap) & 15u) / sizeof(T)));      // first 16-byte boundary
    const int end = body + (hi - body) / E * E;
    if (lo + lane < body) acc += r.at(lo + lane);
    if (end + lane < hi) acc += r.at(end + lane);
    int t = body + lane * E;
    for (; t + 3 * 32 * E < end; t += 4 * 32 * E) {                             // four loads of each row in flight
        uint4 a[4], b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[j] = ld128_rw_stream(r.p + t + j * 32 * E);
            b[j] = r.q != nullptr ? ld128_rw_stream(r.q + t + j * 32 * E) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float x[E], y[E];
            unpack<T>(a[j], x);
            unpack<T>(b[j], y);
#pragma unroll
            for (int e = 0; e < E; ++e) acc += r.term(x[e], y[e], t + j * 32 * E + e);
        }
    }
    for (; t < end; t += 32 * E) {
        float x[E], y[E];
        unpack<T>(ld128_rw_stream(r.p + t), x);
        unpack<T>(r.q != nullptr ? ld128_rw_stream(r.q + t) : make_uint4(0, 0, 0, 0), y);
#pragma unroll
        for (int e = 0; e < E; ++e) acc += r.term(x[e], y[e], t + e);
    }
    return warp_sum(acc);
}

template <typename T>
__global__ void __launch_bounds__(kMaxThreads, 2) verify_drafts_kernel(const T* __restrict__ target, int64_t tls, int64_t tl,
                                                                 const T* __restrict__ draft, int64_t dls, int64_t dl,
                                                                 const int32_t* __restrict__ drafted,
                                                                 const int32_t* __restrict__ n_drafted,
                                                                 const float* __restrict__ uniform, int32_t S, int32_t V,
                                                                 int32_t* __restrict__ tokens, int32_t* __restrict__ accepted,
                                                                 uint32_t* dev_status)
{
    __shared__ double slice_sum[2];                    // this CTA's, read by its peers: with q, and without (the second only where needed)
    __shared__ double piece[kMaxWarps], run[kMaxWarps];
    __shared__ int s_accepted, s_n, s_bad, s_last;
    ptx::grid_dependency_sync();
    const int ctas = (int)ptx::cluster_nctarank(), rank = (int)ptx::cluster_ctarank();
    const int b = (int)blockIdx.x / ctas, tid = (int)threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int threads = (int)blockDim.x, warps = threads >> 5;

    if (warp == 0) {
        const int n = n_drafted != nullptr ? max(0, min(S, ptx::ld_dependent(n_drafted + b))) : S;
        bool ok = false, bad = false;
        if (lane < n) {
            const int x = ptx::ld_dependent(drafted + (int64_t)b * S + lane);
            bad = x < 0 || x >= V;
            if (!bad) {
                const double p = load_prob(target + b * tls + lane * tl + x);
                const double q = draft != nullptr ? (double)load_prob(draft + b * dls + lane * dl + x) : 1.0;
                ok = (double)ptx::ld_dependent(uniform + (int64_t)b * (S + 1) + lane) * q < p;
            }
        }
        const int a = __ffs(~__ballot_sync(0xFFFFFFFFu, ok)) - 1;      // (n <= 31: some lane says no)
        if (lane == 0) s_accepted = a, s_n = n;
        if (lane == a) s_bad = bad;
    }
    __syncthreads();
    const int a = s_accepted;
    const bool refused = a < s_n;
    if (s_bad && tid == 0 && rank == 0 && dev_status != nullptr) atomicOr(dev_status, MOLORA_DEV_BAD_DRAFT);
    Residual<T> r;
    r.p = target + b * tls + a * tl;
    r.q = refused && draft != nullptr ? draft + b * dls + a * dl : nullptr;
    r.certain = refused && draft == nullptr ? ptx::ld_dependent(drafted + (int64_t)b * S + a) : -1;

    // slices of whole 32-byte sectors, pieces of the slices likewise
    const int slice = ceil_div(ceil_div(V, ctas), 16) * 16;
    const int lo = min(V, rank * slice), hi = min(V, lo + slice);
    const int per = ceil_div(ceil_div(slice, warps), 16) * 16;
    double sums[kMaxCluster], total = 0.0;                // the slices' sums, the same bits in every CTA
    for (int round = 0;; ++round) {
        const double s = piece_sum(r, min(hi, lo + warp * per), min(hi, lo + (warp + 1) * per));
        if (lane == 0) piece[warp] = s;
        __syncthreads();
        double own = 0.0;
        for (int w = 0; w < warps; ++w) own += piece[w];
        if (ctas > 1) {
            if (tid == 0) slice_sum[round] = own;
            ptx::cluster_sync_all();
        }
        total = 0.0;
#pragma unroll
        for (int c = 0; c < kMaxCluster; ++c) {
            sums[c] = 0.0;
            if (c >= ctas) continue;
            if (ctas > 1) {
                const uint32_t at = ptx::map_to_cta(ptx::smem_u32(&slice_sum[round]), (uint32_t)c);
                asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(sums[c]) : "r"(at) : "memory");
            } else {
                sums[c] = own;
            }
            total += sums[c];
        }
        if (round == 1 || total > 0.0 || (r.q == nullptr && r.certain < 0)) break;      // the same in every CTA
        r.q = nullptr;                                    // max(p - q, 0) has no mass: p itself
        r.certain = -1;
        __syncthreads();
    }
    const double goal = (double)ptx::ld_dependent(uniform + (int64_t)b * (S + 1) + S) * total;
    const bool mass = total > 0.0;
    // the first slice in which the running sum passes the goal; where none does (u not below 1), the last one with mass
    int chosen = -1;
    double before = 0.0, cum_slices = 0.0;
    bool passed = false;
#pragma unroll
    for (int c = 0; c < kMaxCluster; ++c) {
        if (sums[c] > 0.0 && !passed) {
            chosen = c;
            before = cum_slices;
            passed = cum_slices + sums[c] > goal;
        }
        cum_slices += sums[c];
    }
    if (rank == (mass ? chosen : 0)) {
        if (tid == 0) s_last = -1;
        __syncthreads();
        if (mass) {
            double at = before;
            int w = 0, held = -1;
            double held_at = before;
            for (; w < warps; ++w) {                     // (every thread walks the same few sums)
                if (piece[w] > 0.0) held = w, held_at = at;
                if (at + piece[w] > goal && piece[w] > 0.0) break;
                at += piece[w];
            }
            w = held, at = held_at;
            const int p0 = min(hi, lo + w * per), p1 = min(hi, lo + (w + 1) * per);
            const int len = ceil_div(max(p1 - p0, 1), threads);
            const int t0 = min(p1, p0 + tid * len), t1 = min(p1, t0 + len);
            double mine_sum = 0.0;
            for (int t = t0; t < t1; ++t) mine_sum += r.at(t);
            double incl = mine_sum;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double up = __shfl_up_sync(0xFFFFFFFFu, incl, o);
                if (lane >= o) incl += up;
            }
            if (lane == 31) run[warp] = incl;
            __syncthreads();
            double base = at;
            for (int i = 0; i < warp; ++i) base += run[i];
            // first run that passes the goal; where rounding lets none pass, the last token with mass (both by atomicMax on reversed order)
            const bool passes = base + incl > goal && mine_sum > 0.0;
            const unsigned first = __ballot_sync(0xFFFFFFFFu, passes);
            if (passes && lane == __ffs(first) - 1) {
                double cum = base + incl - mine_sum;
                int found = -1;
                for (int t = t0; t < t1; ++t) {
                    const double v = r.at(t);
                    if (v > 0.0) {
                        cum += v;
                        found = t;
                        if (cum > goal) break;
                    }
                }
                atomicMax(&s_last, INT32_MAX - found);
            }
            __syncthreads();
            if (s_last < 0) {                             // nothing passed: the last token with mass
                int last = -1;
                for (int t = t0; t < t1; ++t)
                    if (r.at(t) > 0.0) last = t;
                __syncthreads();
                atomicMax(&s_last, last);
                __syncthreads();
                if (tid == 0) s_last = INT32_MAX - s_last;
                __syncthreads();
            }
        } else {
            if (tid == 0) {
                s_last = INT32_MIN;                       // (INT32_MAX - s_last below must give -1)
                if (dev_status != nullptr) atomicOr(dev_status, MOLORA_DEV_BAD_DRAFT);
            }
            __syncthreads();
        }
        const int token = mass ? INT32_MAX - s_last : -1;
        if (tid <= S) tokens[(int64_t)b * (S + 1) + tid] = tid < a ? ptx::ld_dependent(drafted + (int64_t)b * S + tid) : tid == a ? token : -1;
        if (tid == 0) accepted[b] = a;
    }
    if (ctas > 1) ptx::cluster_sync_all();                // a peer may still read slice_sum
}

template <typename T>
molora_status_t launch(const void* target, int64_t tls, int64_t tl, const void* draft, int64_t dls, int64_t dl, const int32_t* drafted,
                       const int32_t* n_drafted, const float* uniform, int32_t B, int32_t S, int32_t V, int32_t* tokens, int32_t* accepted,
                       uint32_t* dev_status, cudaStream_t s)
{
    // CTAs per sequence: enough for the SMs (four CTAs of 256 threads each, 64 registers a thread), none with less than 2048 words; 512
    // threads where two such CTAs per SM take them all.  What is past the SMs' room waits for a whole CTA's time: 64 sequences of 160,000
    // words in clusters of eight CTAs of 512 threads took 29 us.
    int ctas = 1;
    while (ctas < kMaxCluster && (int64_t)B * ctas < 2 * sm_count() && V >= ctas * 2 * 2048) ctas *= 2;
    const int threads = (int64_t)B * ctas <= 2 * sm_count() ? kMaxThreads : kMaxThreads / 2;
    const dim3 grid((unsigned)(B * (int64_t)ctas));
    return cuda_ok(launch_kernel(verify_drafts_kernel<T>, grid, dim3((unsigned)threads), 0, s, (unsigned)ctas, true, static_cast<const T*>(target), tls, tl,
                                 static_cast<const T*>(draft), dls, dl, drafted, n_drafted, uniform, S, V, tokens, accepted, dev_status));
}

}  // namespace

molora_status_t launch_verify_drafts(const void* target, int64_t tls, int64_t tl, const void* draft, int64_t dls, int64_t dl, molora_dtype_t dt,
                                     const int32_t* drafted, const int32_t* n_drafted, const float* uniform, int32_t B, int32_t S, int32_t V,
                                     int32_t* tokens, int32_t* accepted, uint32_t* dev_status, cudaStream_t s)
{
    return dt == MOLORA_F32 ? launch<float>(target, tls, tl, draft, dls, dl, drafted, n_drafted, uniform, B, S, V, tokens, accepted, dev_status, s)
                            : launch<__nv_bfloat16>(target, tls, tl, draft, dls, dl, drafted, n_drafted, uniform, B, S, V, tokens, accepted, dev_status, s);
}

}  // namespace molora
