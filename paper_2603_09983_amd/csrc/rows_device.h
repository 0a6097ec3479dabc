// What the calls that move, sum, quantise and multiply rows share: their launch, 16-byte words of bf16 or fp32 as floats, the 8-bit blocks.
#pragma once
#include "moe_internal.h"

namespace moe {

// Launch of one of the calls on rows (permute.hip, fp8.hip, fp8_matmul.hip): `args` is the kernel's one argument; returns a status code.
int launch_rows(const void *fn, dim3 grid, int threads, void *args, size_t lds, void *stream, int kind);
int launch_failed(hipError_t e);   // keeps the error's text for moe_status_string, returns MOE_ERR_LAUNCH
static inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

namespace rows {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;

// Elements of a 16-byte word, and the word as floats and back (to bf16: to nearest, ties to even, NaN stays NaN).
template <bool BF16>
constexpr int kPerWord = BF16 ? 8 : 4;

template <bool BF16>
__device__ __forceinline__ void to_floats(u32x4 w, float *f)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BF16) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            f[i] = __uint_as_float(w[i]);
        }
    }
}

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}

template <bool BF16>
__device__ __forceinline__ u32x4 to_word(const float *f)
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = BF16 ? pack_bf16(f[2 * i], f[2 * i + 1]) : __float_as_uint(f[i]);
    return w;
}

// Results beyond what the L2s can keep for the next call (half of their 32 MB) are stored without a place in them: 98304 rows of 2048
// bytes written from 16384 tokens 42 against 58 us, 8192 tokens summed from six rows each 46 against 50.5 us, a gradient of 8192 rows of
// 4096 31 against 38 us.  Followed by the product that reads them the rows cost the same in all.
constexpr size_t kStreamBytes = (size_t)16 << 20;
__device__ __forceinline__ void put(u32x4 *to, u32x4 v, int stream)
{
    if (stream) {
        asm volatile("");   // (on both sides: or the compiler makes one store of the two, an ordinary one)
        __builtin_nontemporal_store(v, to);
        asm volatile("");
    } else {
        *to = v;
    }
}

// ---- values in 8 bits (e4m3) with a scale for each block of 128 ----
// m = max(|x|, 2^-100) over the block, scale = m / 448, q = x * (448 / m) to nearest, ties to even.  The bound of 2^-100 keeps
// both quotients normal numbers (a block of zeros: q = 0).  Magnitudes are compared as integers, in which order NaN comes behind
// infinity: a block with NaN has scale NaN, one with infinity scale infinity, and their products are not numbers either.
constexpr int kBlock = 128;
constexpr unsigned kLeastBits = 0x0d800000u;   // 2^-100
constexpr float kTop = 448.f;

__device__ __forceinline__ unsigned magnitude(float f) { return __float_as_uint(f) & 0x7fffffffu; }
__device__ __forceinline__ unsigned larger(unsigned a, unsigned b) { return a > b ? a : b; }

// Largest of eight neighbouring lanes, in each of them: in pairs, in fours, then with the lane mirrored in the eight.
__device__ __forceinline__ unsigned largest_of_8(unsigned m)
{
    m = larger(m, (unsigned)__builtin_amdgcn_mov_dpp((int)m, 0xb1, 0xf, 0xf, false));    // quad_perm 1,0,3,2
    m = larger(m, (unsigned)__builtin_amdgcn_mov_dpp((int)m, 0x4e, 0xf, 0xf, false));    // quad_perm 2,3,0,1
    return larger(m, (unsigned)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xf, 0xf, false));   // row_half_mirror
}

// Sixteen values times `by`, in 8 bits.
__device__ __forceinline__ u32x4 sixteen_fp8(const float *f, float by)
{
    u32x4 q;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        int v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i] * by, f[4 * i + 1] * by, 0, false);
        v = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2] * by, f[4 * i + 3] * by, v, true);
        q[i] = (uint32_t)v;
    }
    return q;
}

// n / d for 0 <= n < 2^31 by one multiplication: rcp = floor(2^32 / d) (0xffffffff for d = 1) is never too large and at most one short.
__device__ __forceinline__ unsigned quotient(unsigned n, unsigned d, unsigned rcp)
{
    unsigned q = __umulhi(n, rcp);
    if (n - q * d >= d) ++q;
    return q;
}

}  // namespace rows

}  // namespace moe
