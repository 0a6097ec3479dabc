// Values in 8 bits (e4m3) with a scale for each block of 128: rows as they are or behind SiLU(gate) * up, and weight matrices
// (one scale for 128 x 128).  A row of K values takes Kp = 128 ceil(K / 128) bytes, zeros behind the K-th: the product
// (fp8_matmul.hip) reads whole blocks.  Bound by memory: every value is read once, 16 or 32 bytes a lane.
#include "../../include/moe_spac.h"
#include "rows_device.h"

namespace moe {

namespace {

using namespace rows;

constexpr int kQuantThreads = 256;
constexpr unsigned kMostGroups = 1u << 20;

struct QuantArgs {
    const void *x;              // [M,K], or [M,2K] (gate | up)
    const int32_t *n_rows;      // [1] or null: rows from *n_rows on are left as they are
    u32x4 *q;                   // [M,Kp]
    float *scale;               // [M,Kb]
    int M, K, stream;
    unsigned blocks, rcp_blocks, items;
};

// Sixteen values of a row from column c on, zeros from column K on (c < Kp, K a multiple of 8).
template <bool BF16>
__device__ __forceinline__ void load16(const void *x, size_t row, int c, int K, float *f)
{
    constexpr int n = kPerWord<BF16>;
#pragma unroll
    for (int i = 0; i < 16 / n; ++i) {
        u32x4 v = {0u, 0u, 0u, 0u};
        if (c + i * n < K) v = ((const u32x4 *)x)[(row + c) / n + i];
        to_floats<BF16>(v, f + i * n);
    }
}

// e^x as 2^t, t = x log2(e), by the instruction, which is one step off at most.  What the roundings of t and of log2(e) have left out of the
// exponent, up to 6e-6 at |x| = 87, comes back as a factor (the rounding of a product is a fused multiply-add).  Within four roundings of
// 2^-24 where the result is a normal number; without the factor it was 59.  (With expf and a division the call below takes 39 us instead of 31.)
__device__ __forceinline__ float exponential(float x)
{
    constexpr double log2e = 1.4426950408889634, ln2 = 0.69314718055994531;
    constexpr float hi = (float)log2e, rest = (float)((log2e - hi) * ln2);
    x = fminf(fmaxf(x, -104.f), 104.f);   // (0 and infinity from here on)
    const float t = x * hi;
    return __builtin_amdgcn_exp2f(t) * __builtin_fmaf(__builtin_fmaf(x, hi, -t), (float)ln2, __builtin_fmaf(x, rest, 1.f));
}
// g / (1 + e^-g) by the reciprocal instruction, one step off at most; both sides of the quotient are quartered, so that the reciprocal of a
// finite number is a normal one.
__device__ __forceinline__ float silu(float g)
{
    return g * 0.25f * __builtin_amdgcn_rcpf(__builtin_fmaf(exponential(-g), 0.25f, 0.25f));
}

// Eight lanes have a block, sixteen values a lane: the block's largest magnitude comes from three exchanges in registers, and a row is read
// once.  24576 rows of SiLU(gate) * up, 1408 of each in bf16: 31 us, 5.6 TB/s.  (SiLU * up within nine roundings of 2^-24; the
// only rounding to fewer bits is that to e4m3.)
template <bool BF16, bool SWIGLU>
__global__ __launch_bounds__(kQuantThreads) void quantize_kernel(QuantArgs a)
{
    unsigned items = a.items;
    if (a.n_rows) {
        const int n = *a.n_rows;
        items = (unsigned)(n < 0 ? 0 : n < a.M ? n : a.M) * a.blocks;
    }
    const int sub = threadIdx.x & 7;
    for (unsigned g = (blockIdx.x * kQuantThreads + threadIdx.x) / 8; g < items; g += gridDim.x * (kQuantThreads / 8)) {
        const unsigned r = quotient(g, a.blocks, a.rcp_blocks), b = g - r * a.blocks;
        const int c = (int)b * kBlock + sub * 16;
        float f[16];
        if (SWIGLU) {
            float up[16];
            const size_t row = (size_t)r * 2 * a.K;
            load16<BF16>(a.x, row, c, a.K, f);
            load16<BF16>(a.x, row + a.K, c, a.K, up);
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] = silu(f[i]) * up[i];
        } else {
            load16<BF16>(a.x, (size_t)r * a.K, c, a.K, f);
        }
        unsigned m = kLeastBits;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = larger(m, magnitude(f[i]));
        const float top = __uint_as_float(largest_of_8(m));
        put(a.q + (size_t)g * 8 + sub, sixteen_fp8(f, kTop / top), a.stream);
        if (sub == 0) a.scale[g] = top / kTop;
    }
}

struct QuantWeightArgs {
    const void *w;              // [E,N,K]
    u32x4 *q;                   // [E,N,Kp]
    float *scale;               // [E,Nb,Kb]
    int N, K, stream;
    unsigned nb, kb, rcp_nb, rcp_kb, items;
};

// A workgroup has 128 x 128 weights: eight lanes a row, 32 rows at a time, all in registers until the largest is known.  Eight matrices of
// 14336 x 4096 in bf16: 256 us, 5.5 TB/s.
template <bool BF16>
__global__ __launch_bounds__(kQuantThreads) void quantize_weights_kernel(QuantWeightArgs a)
{
    __shared__ unsigned most[kQuantThreads / kWave];
    const int tid = threadIdx.x, sub = tid & 7;
    for (unsigned item = blockIdx.x; item < a.items; item += gridDim.x) {
        const unsigned en = quotient(item, a.kb, a.rcp_kb), b = item - en * a.kb;   // (expert, block row), block column
        const unsigned e = quotient(en, a.nb, a.rcp_nb), nb = en - e * a.nb;
        const int c = (int)b * kBlock + sub * 16;
        float f[4][16];
        unsigned m = kLeastBits;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = (int)nb * kBlock + i * 32 + tid / 8;
            if (n < a.N) {
                load16<BF16>(a.w, ((size_t)e * a.N + n) * a.K, c, a.K, f[i]);
            } else {
#pragma unroll
                for (int v = 0; v < 16; ++v) f[i][v] = 0.f;
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) m = larger(m, magnitude(f[i][v]));
        }
        for (int s = kWave / 2; s > 0; s >>= 1) m = larger(m, (unsigned)__shfl_xor((int)m, s));
        if ((tid & (kWave - 1)) == 0) most[tid / kWave] = m;
        __syncthreads();
        const float top = __uint_as_float(larger(larger(most[0], most[1]), larger(most[2], most[3])));
        __syncthreads();
        const float by = kTop / top;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = (int)nb * kBlock + i * 32 + tid / 8;
            if (n < a.N) put(a.q + (((size_t)e * a.N + n) * a.kb + b) * 8 + sub, sixteen_fp8(f[i], by), a.stream);
        }
        if (tid == 0) a.scale[item] = top / kTop;
    }
}

int quantize_rows(const void *x, int x_bf16, const int32_t *n_rows, int M, int K, void *q, float *scale, bool swiglu, void *stream)
{
    if (!x || !q || !scale) return MOE_ERR_NULL;
    if (M < 1 || K < 1 || M > 1 << 30 || K > 1 << 24) return MOE_ERR_SHAPE;
    if (K % 8 || !aligned16(x) || !aligned16(q)) return MOE_ERR_ALIGN;
    QuantArgs a = {x, n_rows, (u32x4 *)q, scale, M, K, 0, (unsigned)((K + kBlock - 1) / kBlock), 0, 0};
    a.stream = (size_t)M * a.blocks * kBlock > kStreamBytes;
    const size_t items = (size_t)M * a.blocks;
    if (items >= (size_t)1 << 31) return MOE_ERR_SHAPE;
    a.rcp_blocks = rcp32(a.blocks);
    a.items = (unsigned)items;
    const size_t groups = (items + kQuantThreads / 8 - 1) / (kQuantThreads / 8);
    const void *fn = swiglu ? (x_bf16 ? (const void *)quantize_kernel<true, true> : (const void *)quantize_kernel<false, true>)
                            : (x_bf16 ? (const void *)quantize_kernel<true, false> : (const void *)quantize_kernel<false, false>);
    return launch_rows(fn, groups < kMostGroups ? (unsigned)groups : kMostGroups, kQuantThreads, &a, 0, stream, MOE_KERNEL_QUANTIZE);
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" int moe_quantize_fp8(const void *x, int x_bf16, const int32_t *n_rows, int M, int K, void *q, float *scale, void *stream)
{
    return quantize_rows(x, x_bf16, n_rows, M, K, q, scale, false, stream);
}

extern "C" int moe_swiglu_fp8(const void *gate_up, int x_bf16, const int32_t *n_rows, int M, int F, void *q, float *scale, void *stream)
{
    return quantize_rows(gate_up, x_bf16, n_rows, M, F, q, scale, true, stream);
}

extern "C" int moe_quantize_weights_fp8(const void *w, int w_bf16, int E, int N, int K, void *q, float *scale, void *stream)
{
    if (!w || !q || !scale) return MOE_ERR_NULL;
    if (E < 1 || N < 1 || K < 1 || E > kMaxC || N > 1 << 24 || K > 1 << 24) return MOE_ERR_SHAPE;
    if (K % 8 || !aligned16(w) || !aligned16(q)) return MOE_ERR_ALIGN;
    QuantWeightArgs a = {w, (u32x4 *)q, scale, N, K, 0, (unsigned)((N + kBlock - 1) / kBlock), (unsigned)((K + kBlock - 1) / kBlock), 0, 0, 0};
    a.stream = (size_t)E * N * a.kb * kBlock > kStreamBytes;
    const size_t items = (size_t)E * a.nb * a.kb;
    if (items >= (size_t)1 << 31) return MOE_ERR_SHAPE;
    a.rcp_nb = rcp32(a.nb);
    a.rcp_kb = rcp32(a.kb);
    a.items = (unsigned)items;
    return launch_rows(w_bf16 ? (const void *)quantize_weights_kernel<true> : (const void *)quantize_weights_kernel<false>,
                    items < kMostGroups ? a.items : kMostGroups, kQuantThreads, &a, 0, stream, MOE_KERNEL_QUANTIZE);
}
