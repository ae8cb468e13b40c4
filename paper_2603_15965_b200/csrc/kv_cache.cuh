// The paged 8-bit key / value cache: device view, sequence lookup and e4m3 conversions shared by its kernels.
#pragma once
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "common.cuh"

namespace molora {

// What the kernels need of molora_kv_cache_t and molora_sequences_t.
struct KvView {
    uint8_t* k;
    uint8_t* v;
    float* k_scale;
    float* v_scale;
    int32_t n_pages, kv_heads, page_log2, dim;
    const int32_t* table;
    int64_t ld_table;
    const int32_t* cu;
    const int32_t* kv_lens;
    int32_t B, max_pages;
};

// Sequence b of the call, with what cannot be true of it put right: rows inside [0, N], tokens inside the page table.  What is cut off is left out;
// the tokens that stay keep the positions that the sequence's length as it was given and its rows as they were given make.
constexpr int32_t kMaxTokens = 1 << 30;      // of a sequence: sums of keys, windows and tiles stay within 32 bits
struct Sequence {
    int32_t row0;     // first of its rows
    int32_t n;        // its rows
    int32_t pos0;     // position of the first; the last one's is below 2^31 - 1
    int32_t len;      // tokens that can be in the cache
    bool bad;         // something had to be put right
};
__device__ __forceinline__ Sequence sequence_of(const KvView& c, int b, int64_t N)
{
    Sequence s;
    const int32_t a = ptx::ld_dependent(c.cu + b), e = ptx::ld_dependent(c.cu + b + 1), l = ptx::ld_dependent(c.kv_lens + b);
    const int64_t room = min((int64_t)c.max_pages << c.page_log2, (int64_t)kMaxTokens);
    const int32_t top = (int32_t)min(N, (int64_t)INT32_MAX);
    s.row0 = max(0, min(a, top));
    s.n = max(0, min(e, top) - s.row0);
    const int32_t given = max(l, 0);
    s.pos0 = s.n > 0 ? (int32_t)((int64_t)given - e + s.row0) : 0;      // (e > row0: between -2^31 and given - 1)
    s.len = (int32_t)min((int64_t)given, room);
    s.bad = s.row0 != a || (int64_t)e - a != s.n || s.len != l || (int64_t)e - a > l;
    return s;
}

// ---- e4m3 <-> fp16 / fp32 (every e4m3 value is an fp16 value)
// two codes in the low half of w -> two fp16 (low byte in the low half)
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t w)
{
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2_high(uint32_t w)
{
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
// four fp32 -> four codes, nearest even, infinities and what is too large saturate at +-448, NaN stays NaN
__device__ __forceinline__ uint32_t f32x4_to_e4m3x4(float a, float b, float c, float d)
{
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}
__device__ __forceinline__ float2 f16x2_to_f32x2(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }
// 0x80 in every byte that is a NaN code (0x7F or 0xFF)
__device__ __forceinline__ uint32_t e4m3x4_nan_bits(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Host launchers.
molora_status_t launch_kv_append(const KvView& c, molora_dtype_t dt, int64_t N, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                 const void* q, int64_t ldq, void* q_out, int64_t ldqo, int32_t heads, const float* inv_freq,
                                 int32_t rotary, int32_t interleaved, uint32_t* dev_status, cudaStream_t s);
struct AttendArgs {
    KvView c;
    int64_t N;
    const void* q;
    int64_t ldq;
    void* out;
    int64_t ldo;
    float* lse;
    int32_t heads, group, causal, window;      // group: query heads that share a key / value head
    float scale_log2;      // scale * log2(e): the softmax runs in powers of two
    uint32_t* dev_status;
};
// rows: of the longest sequence, per key / value head.  fp32, or heads of 64:
size_t attend_rows_workspace_bytes(molora_dtype_t dt, int32_t dim, int64_t rows);
molora_status_t launch_attend_rows(const AttendArgs& a, molora_dtype_t dt, int64_t rows, void* ws, cudaStream_t s);
// bf16, heads of 128; in units of up to kMaxStreamRows rows, and of 256:
constexpr int64_t kMaxStreamRows = 32;
size_t attend_stream_workspace_bytes(int64_t rows);
molora_status_t launch_attend_stream(const AttendArgs& a, int64_t rows, void* ws, cudaStream_t s);
size_t attend_tiles_workspace_bytes();
molora_status_t launch_attend_tiles(const AttendArgs& a, void* ws, cudaStream_t s);
molora_status_t launch_verify_drafts(const void* target, int64_t tls, int64_t tl, const void* draft, int64_t dls, int64_t dl, molora_dtype_t dt,
                                     const int32_t* drafted, const int32_t* n_drafted, const float* uniform, int32_t B, int32_t S, int32_t V,
                                     int32_t* tokens, int32_t* accepted, uint32_t* dev_status, cudaStream_t s);

}  // namespace molora
