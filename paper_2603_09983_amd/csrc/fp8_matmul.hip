// The experts' products in 8 bits: rows sorted by expert times that expert's weights,
//      out[r,n] = sum over blocks b of 128:  sa[r,b] sw[e,n/128,b]  sum over i in b:  a[r,i] w[e,n,i],    offsets[e] <= r < offsets[e+1].
// The products of a block are summed by the matrix cores (fp32), the blocks' sums times their scales in fp32.
//
// Weight rows are the MFMA's rows and tokens its columns, so that a lane's four results belong to one token and take one scale.
#include "../../include/moe_spac.h"
#include "rows_device.h"

namespace moe {

namespace {

using namespace rows;

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;

constexpr int kThreads = 256, kWaves = kThreads / kWave;

struct MatmulArgs {
    const uint8_t *a, *w;        // [M,K], [E,N,K]
    const float *a_scale, *w_scale;   // [M,K/128], [E,ceil(N/128),K/128]
    const int32_t *offsets;      // [E+1]
    void *out;                   // [M,N]
    int M, N, K;
};

// 128 columns' products of sixteen weight rows and sixteen tokens (each lane: 32 columns of one row of both).
//
// The 8-bit matrix instruction adds its products in groups of eight consecutive columns, every product of a group cut toward zero at
// 2^-13 of the group's largest (of the power of two that its operands' exponents make; found with single products, each position and
// size).  On normal values that puts 1.6e-5 of their norm into the results, less than a hundredth of what rounding them to bf16 does
// (1.7e-3), so bf16 results are made that way.  EXACT, for fp32 results: both operands converted to bf16, in which every e4m3 value
// is exact, and multiplied by the bf16 instruction, which keeps 32-bit sums (1e-8 of the norm on the same values).
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;

__device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi)
{
    const bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true),
                         __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true)};
    return bf16x8{v[0][0], v[0][1], v[1][0], v[1][1], v[2][0], v[2][1], v[3][0], v[3][1]};
}

template <bool EXACT>
struct Operand;
template <>
struct Operand<false> {
    i32x8 v;
    __device__ __forceinline__ Operand(u32x4 a, u32x4 b)
        : v{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]}
    {
    }
};
template <>
struct Operand<true> {
    bf16x8 v[4];
    __device__ __forceinline__ Operand(u32x4 a, u32x4 b)
        : v{widen8(a[0], a[1]), widen8(a[2], a[3]), widen8(b[0], b[1]), widen8(b[2], b[3])}
    {
    }
};

__device__ __forceinline__ f32x4 mfma128(const Operand<false> &a, const Operand<false> &b)
{
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a.v, b.v, zero, 0, 0, 0, 0, 0, 0);   // (no scales of its own, both operands e4m3)
}
__device__ __forceinline__ f32x4 mfma128(const Operand<true> &a, const Operand<true> &b)
{
    f32x4 p = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; ++i) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v[i], b.v[i], p, 0, 0, 0);
    return p;
}

// A workgroup has 32 weight rows of one expert against its tokens, sixteen at a time; its four wavefronts share the columns,
// block by block, and their sums meet in LDS.
template <bool OUT16>
__global__ __launch_bounds__(kThreads) void grouped_matmul_kernel(MatmulArgs a)
{
    __shared__ f32x4 part[kWaves][2][kWave];
    const int e = blockIdx.y, n0 = blockIdx.x * 32;
    int lo = a.offsets[e], hi = a.offsets[e + 1];
    lo = lo < 0 ? 0 : lo;
    hi = hi > a.M ? a.M : hi;
    if (lo >= hi) return;
    const int lane = threadIdx.x & (kWave - 1), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int col = lane & 15, grp = lane >> 4, kb = a.K / kBlock;
    const uint8_t *wrow[2];
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const int n = n0 + 16 * m + col < a.N ? n0 + 16 * m + col : a.N - 1;
        wrow[m] = a.w + ((size_t)e * a.N + n) * a.K + grp * 32;
    }
    const float *sw = a.w_scale + ((size_t)e * ((a.N + kBlock - 1) / kBlock) + n0 / kBlock) * kb;
    for (int r0 = lo; r0 < hi; r0 += 16) {
        const int r = r0 + col < hi ? r0 + col : hi - 1;
        const uint8_t *arow = a.a + (size_t)r * a.K + grp * 32;
        const float *sa = a.a_scale + (size_t)r * kb;
        f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        for (int b = w; b < kb; b += kWaves) {
            const u32x4 *x = (const u32x4 *)(arow + (size_t)b * kBlock);
            const Operand<!OUT16> xo(x[0], x[1]);
            const float s = sa[b] * sw[b];
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                const u32x4 *y = (const u32x4 *)(wrow[m] + (size_t)b * kBlock);
                const f32x4 p = mfma128(Operand<!OUT16>(y[0], y[1]), xo);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][i] = __builtin_fmaf(p[i], s, acc[m][i]);
            }
        }
        part[w][0][lane] = acc[0];
        part[w][1][lane] = acc[1];
        __syncthreads();
        if (w < 2) {
            f32x4 sum = part[0][w][lane];
            for (int v = 1; v < kWaves; ++v) sum += part[v][w][lane];
            const int n = n0 + 16 * w + 4 * grp;   // (N is a multiple of 8)
            if (r0 + col < hi && n < a.N) {
                const size_t at = (size_t)r * a.N + n;
                if (OUT16) {
                    const u32x2 v = {pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
                    *(u32x2 *)((uint16_t *)a.out + at) = v;
                } else {
                    *(f32x4 *)((float *)a.out + at) = sum;
                }
            }
        }
        __syncthreads();
    }
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" int moe_grouped_matmul_fp8(const void *x, const float *x_scale, const void *w, const float *w_scale, const int32_t *offsets,
                                      int M, int N, int K, int E, void *out, int out_bf16, void *stream)
{
    if (!x || !x_scale || !w || !w_scale || !offsets || !out) return MOE_ERR_NULL;
    if (M < 1 || N < 1 || K < 1 || E < 1 || E > kMaxC || M > 1 << 30 || N > 1 << 24 || K > 1 << 24) return MOE_ERR_SHAPE;
    if (N % 8 || K % kBlock || !aligned16(x) || !aligned16(w) || !aligned16(out)) return MOE_ERR_ALIGN;
    MatmulArgs a = {(const uint8_t *)x, (const uint8_t *)w, x_scale, w_scale, offsets, out, M, N, K};
    return launch_rows(out_bf16 ? (const void *)grouped_matmul_kernel<true> : (const void *)grouped_matmul_kernel<false>,
                       dim3((N + 31) / 32, E), kThreads, &a, 0, stream, MOE_KERNEL_MATMUL);
}
