// The 4-bit K/V cache: format and device helpers shared by the kernels that fill and read it.
//
// A row of C channels is C/8 32-bit words of codes and C/32 scales. Each group of 32 channels shares a scale
// s: its largest magnitude over 7, rounded up to five significant bits (so no code is clipped), held as bf16. A channel is
// a code in [-7, 7] times s. Three bits times five: every decoded value is exact in bf16, so what the tensor core multiplies
// is the value the cache stands for. Neither rounding leaves a doubt: x / s of a bf16 x is either exactly half way between two
// codes or at least 2^-10 from it, and the largest magnitude over 7 is either a number of five bits or at least 2^-11 (relative)
// from one.
// A word holds the codes plus 8 of eight channels c..c+7: channel c+2i in bits 4i..4i+3, c+2i+1 in bits 16+4i..19+4i, so that
// one shift and one logical operation give a pair of neighbouring channels as two bf16 numbers 128 + 8 (code + 8), and one
// fused multiply-add by s/8 and -24 s the two values: (128 + 8 u) s/8 - 24 s = (u - 8) s with all operands and the result exact.
// A group with an infinity, a NaN or a magnitude of 2^120 or more has scale NaN and reads as NaN; a group of zeros, or of
// magnitudes below 2^-121, reads as zeros or the nearest multiples of 2^-120.
#pragma once

#include "tc_common.cuh"

namespace c4 {

constexpr int kGroup = 32;             // channels that share a scale

// A pair of neighbouring channels of a word as 128 + 8 (code + 8), two bf16. I in 0..3.
template <int I>
__device__ __forceinline__ uint32_t raw_pair(uint32_t w)
{
    const uint32_t sh = I == 0 ? w << 3 : w >> (4 * I - 3);
    return (sh & 0x00780078u) | 0x43004300u;
}
__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c)
{
    uint32_t r;
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Two scales (one per half) as the multiply-add's operands.
struct Scale2 {
    uint32_t eighth, offset;           // s / 8 and -24 s, exact: s has five significant bits and is 0 or in [2^-120, 2^118)
    __device__ __forceinline__ explicit Scale2(uint32_t s2)
        : eighth(mul_bf16x2(s2, 0x3e003e00u)), offset(mul_bf16x2(s2, 0xc1c0c1c0u)) {}
};
__device__ __forceinline__ uint32_t both(uint16_t s) { return (uint32_t)s * 0x10001u; }
template <int I>
__device__ __forceinline__ uint32_t value_pair(uint32_t w, const Scale2& s) { return fma_bf16x2(raw_pair<I>(w), s.eighth, s.offset); }
// The eight values of a word, in channel order.
__device__ __forceinline__ void decode8(uint32_t w, const Scale2& s, uint32_t (&out)[4])
{
    out[0] = value_pair<0>(w, s);
    out[1] = value_pair<1>(w, s);
    out[2] = value_pair<2>(w, s);
    out[3] = value_pair<3>(w, s);
}

// Keys of an image of a call that brings `rows` rows of it. own: the rows have been appended without advancing the length, and count
// too, unless they did not fit (the append left them out then, and what lies behind the length is nobody's).
__device__ __forceinline__ bool rows_fit(int kv_len, int rows, int Lmax) { return kv_len >= 0 && (long)kv_len + rows <= Lmax; }
__device__ __forceinline__ int keys_of(int kv_len, int rows, bool own, int Lmax)
{
    return own && rows_fit(kv_len, rows, Lmax) ? kv_len + rows : min(max(kv_len, 0), Lmax);
}

// Image of compacted row r: the largest b with cu[b] <= r (B >= 1).
__device__ __forceinline__ int image_of(const int32_t* cu, int B, int r)
{
    int lo = 0, hi = B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu[mid] <= r) lo = mid; else hi = mid;
    }
    return lo;
}

}  // namespace c4

// Argument checks that the calls on such a cache share. Returns NOVA_OK, or the status that the call returns.
nova_status nova_cache4_check(nova_ctx* ctx, const char* who, const nova_cache4* c);
// And of the rows of a call: cu_rows, and row strides in elements.
nova_status nova_cache4_check_rows(nova_ctx* ctx, const char* who, const nova_cache4* c, const void* a, const void* b,
                                   const int32_t* cu_rows, int M, int64_t ld);

nova_status nova_launch_cache4_append(nova_ctx* ctx, const nova_cache4* c, const void* k, const void* v, int64_t ld, const int32_t* cu,
                                      int M, int advance, cudaStream_t st);

// Attention over the cache. own_rows: the keys of image b are its kv_len[b] rows and the cu[b+1] - cu[b] behind them (appended
// without advancing the lengths; an image whose rows did not fit has only the former), else the kv_len[b] rows alone.
struct nova_cache4_attn_args {
    const nova_cache4* cache;
    const __nv_bfloat16* q;        // [M, C], row stride ldq elements
    int64_t ldq;
    const int32_t* cu;             // [B+1]
    int M;
    __nv_bfloat16* o;              // [M, C]
    float* lse;                    // [n_heads, M] or NULL
    bool own_rows;
    void* scratch;
    size_t scratch_bytes;
};
size_t nova_cache4_attention_scratch(int num_sms, int dh, int M);
nova_status nova_launch_cache4_attention(nova_ctx* ctx, const nova_cache4_attn_args& a, cudaStream_t st);
// The same on the tensor cores' 128-row tiles (attention.cu).
size_t nova_cache4_tiles_scratch(int num_sms, int dh);
nova_status nova_launch_cache4_tiles(nova_ctx* ctx, const nova_cache4_attn_args& a, cudaStream_t st);
size_t nova_cache4_weights_scratch(int num_sms);
nova_status nova_launch_cache4_weights(nova_ctx* ctx, const nova_cache4* c, const __nv_bfloat16* q, int64_t ldq, const float* lse, const int32_t* cu,
                                       int M, const float* in, float* out, bool own_rows, void* scratch, size_t scratch_bytes, cudaStream_t st);
