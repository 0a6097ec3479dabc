// The experts' products in 8 bits: rows sorted by expert times that expert's weights,
//      out[r,n] = sum over blocks b of 128:  sa[r,b] sw[e,n/128,b]  sum over i in b:  a[r,i] w[e,n,i],    offsets[e] <= r < offsets[e+1].
// The products of a block are summed by the matrix cores (fp32), the blocks' sums times their scales in fp32.
//
// Weight rows are the MFMA's rows and tokens its columns, so that a lane's four results belong to one token and take one scale.
#include "../../include/moe_spac.h"
#include "rows_device.h"
#include <math.h>
#include <type_traits>

namespace moe {

namespace {

using namespace rows;

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(8))) int i32x8;

struct MatmulArgs {
    const uint8_t *a, *w;        // [M,K], [E,N,K]
    const float *a_scale, *w_scale;   // [M,K/128], [E,ceil(N/128),K/128]
    const int32_t *offsets;      // [E+1]
    void *out;                   // [M,N]
    int M, N, K, E;
    int scale_words;             // the rows' scales are whole 16-byte words
    int by_row;                  // (stream_matmul_kernel) workgroups for each row instead of for each expert's groups
};

__device__ __forceinline__ int clamped(int v, int most) { return v < 0 ? 0 : v > most ? most : v; }

// 128 columns' products of sixteen weight rows and sixteen tokens (each lane: 32 columns of one row of both).
//
// EXACT: both operands converted to bf16, in which every e4m3 value is exact, and multiplied by the bf16 instruction, which keeps 32-bit
// sums (1e-8 of the norm on normal values).  Otherwise, and only where the caller asks for it (MOE_BF16_SHORT_SUMS), the 8-bit
// instruction, at twice the rate: it adds its products in groups of eight consecutive columns, every product of a group cut toward zero at
// 2^-13 of the group's largest (of the power of two that its operands' exponents make; found with single products, each position and
// size).  On normal values that puts 1.6e-5 of their norm into the results; beside a wide column the other seven products keep a few bits.
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
    Operand() = default;
    __device__ __forceinline__ Operand(u32x4 a, u32x4 b)
        : v{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]}
    {
    }
};
template <>
struct Operand<true> {
    bf16x8 v[4];
    Operand() = default;
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

// ---- few rows to an expert: its weights streamed past them ----
// Bound by the weights' bytes.  A workgroup has 32 weight rows of one expert against up to 32 of its rows; its wavefronts share the
// columns, block by block (neighbouring wavefronts have neighbouring blocks: together they read consecutive columns), and their sums
// meet in LDS in a fixed order.  Up to 16 rows take one product for each 16 weight rows and two blocks in flight, more of them two and
// one (rows come from L2, where all workgroups of the expert read them, but through the same load unit: 24 rows on each of 64 experts of
// 2816 x 2048 in one pass 96 us, in two 145; 6 rows 58, as if there were 32 65).
// Each 32 rows of an expert have workgroups of their own, so that one that has many (routing is uneven, and the host does not know how)
// keeps nobody waiting: those of the first 32 go by the expert, the others are found from all counts.  (All of them found so: 128 rows
// on 256 experts of 2048 x 1024 46 instead of 34 us.  Workgroups by the mean count, in turn over an expert's rows: 650 skewed rows on
// 256 experts of 384 x 1088 33 instead of 13 us.)
// 27 rows on 18 of 64 experts of 2816 x 2048: 21 us, 5.1 TB/s; 2 rows on 8 of 4096 x 14336: 20 us, 5.8 TB/s, launch included.  (The
// 8-bit instruction would take 7 % off the first and 1 % off the second: its sums are not offered here.)
constexpr int kMostWaves = 8;

// A load instruction takes eight rows' whole 128 columns (16 rows x 64 columns, as the matrix instruction has them, reach 5.8 TB/s, and
// without the hint that they are read once only, or each line would come twice; eight rows 6.2 TB/s with it): lanes 0 to 7 of sixteen
// have the even 16-byte words, 8 to 15 the odd ones, of rows 0 to 7 in v[0] and of rows 8 to 15 in v[1].  Afterwards a lane has both
// words of its own row.
__device__ __forceinline__ void exchange(u32x4 *v, bool upper)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t keep = upper ? v[1][i] : v[0][i];
        const uint32_t other = (uint32_t)__builtin_amdgcn_mov_dpp((int)(upper ? v[0][i] : v[1][i]), 0x128, 0xf, 0xf, false);
        v[0][i] = upper ? other : keep;
        v[1][i] = upper ? keep : other;
    }
}

// The i-th group of ROWS rows behind the experts' first groups: expert and first row; all wavefronts work out the same.  Sums over the
// lanes by register rotations.
struct Group {
    int e, r0, end;   // e < 0: there are not so many
};
template <int ROWS>
__device__ __forceinline__ Group later_group(const int32_t *offsets, int M, int E, int i)
{
    constexpr int n = 4;   // experts of a lane
    const int lane = threadIdx.x & (kWave - 1);
    for (int e = 0; e < E; e += n * kWave) {
        int at[n + 1], up = 0;
#pragma unroll
        for (int k = 0; k <= n; ++k) at[k] = clamped(offsets[e + n * lane + k < E ? e + n * lane + k : E], M);
#pragma unroll
        for (int k = 0; k < n; ++k) up += at[k] < at[k + 1] ? (at[k + 1] - at[k] - 1) / ROWS : 0;
        const int mine = up;   // (and up: with those of the lanes before)
        up += __builtin_amdgcn_update_dpp(0, up, 0x111, 0xf, 0xf, false);   // one to the right in each row of sixteen lanes, two, four, eight
        up += __builtin_amdgcn_update_dpp(0, up, 0x112, 0xf, 0xf, false);
        up += __builtin_amdgcn_update_dpp(0, up, 0x114, 0xf, 0xf, false);
        up += __builtin_amdgcn_update_dpp(0, up, 0x118, 0xf, 0xf, false);
        up += __builtin_amdgcn_update_dpp(0, up, 0x142, 0xa, 0xf, false);   // a row's last lane to the next row, the second's to the upper half
        up += __builtin_amdgcn_update_dpp(0, up, 0x143, 0xc, 0xf, false);
        const unsigned long long behind = __ballot(up > i);
        if (behind) {
            const int l = __builtin_ctzll(behind);
            i -= __builtin_amdgcn_readlane(up - mine, l);
#pragma unroll
            for (int k = 0; k < n; ++k) {
                const int lo = __builtin_amdgcn_readlane(at[k], l), hi = __builtin_amdgcn_readlane(at[k + 1], l);
                const int groups = lo < hi ? (hi - lo - 1) / ROWS : 0;
                if (i < groups) return Group{e + n * l + k, lo + (i + 1) * ROWS, hi};
                i -= groups;
            }
        }
        i -= __builtin_amdgcn_readlane(up, kWave - 1);
    }
    return Group{-1, 0, 0};
}

// Up to 16 T rows of expert e, from r0 on and below hi, U blocks in flight.
template <bool OUT16, int T, int U>
__device__ __forceinline__ void stream_rows(const MatmulArgs &a, f32x4 *part, int e, int r0, int hi)   // part: [wavefront][2 T][lane]
{
    const int lane = threadIdx.x & (kWave - 1), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), waves = blockDim.x / kWave;
    const int col = lane & 15, grp = lane >> 4, kb = a.K / kBlock, n0 = blockIdx.x * 32;
    const bool upper = col >= 8;
    const uint8_t *wrow[4];
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const int n = n0 + 8 * m + (col & 7) < a.N ? n0 + 8 * m + (col & 7) : a.N - 1;
        wrow[m] = a.w + ((size_t)e * a.N + n) * a.K + grp * 32 + (col >> 3) * 16;
    }
    const float *const sw = a.w_scale + ((size_t)e * ((a.N + kBlock - 1) / kBlock) + n0 / kBlock) * kb;
    const uint8_t *xrow[T];
    const float *sx[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int r = r0 + 16 * t + col < hi ? r0 + 16 * t + col : hi - 1;
        xrow[t] = a.a + (size_t)r * a.K + grp * 32;
        sx[t] = a.a_scale + (size_t)r * kb;
    }
    f32x4 acc[2][T];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < T; ++t) acc[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    // Blocks b0, b0 + waves, .. (count of them): all their loads are on their way before the first is used.
    auto blocks = [&](auto count, int b0) {
        constexpr int n = decltype(count)::value;
        u32x4 y[n][2][2], x[n][T][2];
        float sx_of[n][T], sw_of[n];
#pragma unroll
        for (int u = 0; u < n; ++u) {
            const size_t at = (size_t)(b0 + u * waves) * kBlock;
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                y[u][m][0] = __builtin_nontemporal_load((const u32x4 *)(wrow[2 * m] + at));
                y[u][m][1] = __builtin_nontemporal_load((const u32x4 *)(wrow[2 * m + 1] + at));
            }
#pragma unroll
            for (int t = 0; t < T; ++t) {
                x[u][t][0] = *(const u32x4 *)(xrow[t] + at);
                x[u][t][1] = *(const u32x4 *)(xrow[t] + at + 16);
                sx_of[u][t] = sx[t][b0 + u * waves];
            }
            sw_of[u] = sw[b0 + u * waves];
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < n; ++u) {
            exchange(y[u][0], upper);
            exchange(y[u][1], upper);
            const Operand<true> w0(y[u][0][0], y[u][0][1]), w1(y[u][1][0], y[u][1][1]);
#pragma unroll
            for (int t = 0; t < T; ++t) {
                const Operand<true> xo(x[u][t][0], x[u][t][1]);
                const f32x4 p0 = mfma128(w0, xo), p1 = mfma128(w1, xo);
                const float s = sx_of[u][t] * sw_of[u];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    acc[0][t][i] = __builtin_fmaf(p0[i], s, acc[0][t][i]);
                    acc[1][t][i] = __builtin_fmaf(p1[i], s, acc[1][t][i]);
                }
            }
        }
    };
    int b0 = w;
    for (; b0 + (U - 1) * waves < kb; b0 += U * waves) blocks(std::integral_constant<int, U>(), b0);
    if (U > 1)
        for (; b0 < kb; b0 += waves) blocks(std::integral_constant<int, 1>(), b0);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < T; ++t) part[(w * 2 * T + 2 * t + m) * kWave + lane] = acc[m][t];
    __syncthreads();
    for (int i = w; i < 2 * T; i += waves) {
        f32x4 sum = part[i * kWave + lane];
        for (int v = 1; v < waves; ++v) sum += part[(v * 2 * T + i) * kWave + lane];
        const int r = r0 + 16 * (i >> 1) + col, n = n0 + 16 * (i & 1) + 4 * grp;   // (N is a multiple of 8)
        if (r < hi && n < a.N) {
            const size_t at = (size_t)r * a.N + n;
            if (OUT16) {
                const u32x2 v = {pack_bf16(sum[0], sum[1]), pack_bf16(sum[2], sum[3])};
                *(u32x2 *)((uint16_t *)a.out + at) = v;
            } else {
                *(f32x4 *)((float *)a.out + at) = sum;
            }
        }
    }
}

constexpr int kGroup = 32;   // rows of a workgroup

template <bool OUT16>
__global__ __launch_bounds__(kMostWaves *kWave) void stream_matmul_kernel(MatmulArgs a)
{
    extern __shared__ __align__(16) uint8_t lds[];
    Group g = {(int)(blockIdx.z * gridDim.y + blockIdx.y), 0, 0};
    if (a.by_row) {   // workgroups for the rows, of which those of a group's first row are the group's
        int *const found = (int *)lds;   // (its place is part's afterwards)
        const int row = g.e;
        if (threadIdx.x == 0) *found = -1;
        __syncthreads();
        for (int i = threadIdx.x; i < a.E; i += blockDim.x) {
            const int lo = clamped(a.offsets[i], a.M);
            if (lo <= row && row < clamped(a.offsets[i + 1], a.M) && (row - lo) % kGroup == 0) *found = i;
        }
        __syncthreads();
        g = Group{*found, row, *found < 0 ? 0 : clamped(a.offsets[*found + 1], a.M)};
        __syncthreads();
    } else if (g.e >= a.E) {
        g = later_group<kGroup>(a.offsets, a.M, a.E, g.e - a.E);
    } else {
        g.r0 = clamped(a.offsets[g.e], a.M), g.end = clamped(a.offsets[g.e + 1], a.M);
    }
    const int e = __builtin_amdgcn_readfirstlane(g.e), r0 = __builtin_amdgcn_readfirstlane(g.r0), hi = __builtin_amdgcn_readfirstlane(g.end);
    if (e < 0 || r0 >= hi) return;
    if (hi - r0 > 16) stream_rows<OUT16, 2, 1>(a, (f32x4 *)lds, e, r0, hi);
    else stream_rows<OUT16, 1, 2>(a, (f32x4 *)lds, e, r0, hi);
}

// ---- many rows to an expert: tiles of 256 weight rows x 256 tokens (or 128) through LDS ----
// One workgroup of eight wavefronts per CU walks the tiles; a step is one block of 128 columns, 32 KB of weights and 32 (16) KB of rows.
// A wavefront has 64 weight rows x 128 (64) tokens: for each 16 x 16 x 128 product (32 cycles of the matrix core, 64 with 32-bit
// sums) four multiply-adds (16 cycles of the vector ALU) bring the block's sum, times its scales, into the tile's.
//
// 49152 rows on 64 experts of 2816 x 2048, bf16 results: 600 us, 0.95 PFLOP/s, in tiles of 256 x 128; with short sums 340 us, 1.7 PFLOP/s,
// in tiles of 256 x 256.  There the products and multiply-adds alone, on random values, run at 3.1 (2.1 GHz); with the loads and stores
// the clock is 1.7 GHz and the matrix cores are busy 43 % of the cycles (42 % at 1.9 GHz with 32-bit sums), so that most of what is lost is
// waiting: two barriers a step keep the wavefronts together.  One tile in seven has few rows.
//
// LDS holds two steps.  A wavefront reads its weights of a step at its beginning and keeps them; once all have (a second barrier), the
// weights of the step after next are requested into their place.  The rows of the next step are requested when everybody is through
// with the step before.  So the weights, most of which come from HBM, have two steps' time to arrive, the rows, which other workgroups
// of the XCD have mostly brought into its L2, one.
//
// A row's eight 16-byte words are permuted by a key of the row, so that the eight lanes that a read serves at a time find eight
// different words.  Weight rows go to the matrix rows so that a lane's results of two products are eight consecutive columns of `out`.
constexpr int kTile = 256, kTileThreads = 512;             // weight rows of a tile
constexpr int kTileBytes = kTile * kBlock;
constexpr int kChunk = 4;                                  // blocks whose scales are fetched together
constexpr int kChunkBytes = kChunk * (kTile + kWave) * 4;  // of the tokens, then of the two blocks of weight rows (and padding)
constexpr int kTableInts = 2 * (kMaxC + 1) + kTileThreads / kWave;   // count_tiles: experts' first tiles and rows, the wavefronts' sums
template <int J>   // tokens of a tile: 32 J
struct TileSize {
    static constexpr int kTokens = 32 * J, kStage = kTileBytes + kTokens * kBlock;
    static constexpr int kScales = 2 * kStage, kTable = kScales + 2 * kChunkBytes, kLds = kTable + kTableInts * 4;
    static_assert(kLds <= kLdsBytes, "two stages, their scales, the experts' tiles and rows");
};

// 16 (or 4) bytes a lane from base + at to LDS, lane after lane from `to` on.  Not waited for by the compiler: the loop counts.
__device__ __forceinline__ void fetch16(uint32_t to, uint32_t at, const void *base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(at), "s"(base) : "memory");
}
__device__ __forceinline__ void fetch4(uint32_t to, uint32_t at, const void *base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(at), "s"(base) : "memory");
}

// table[e] = tiles of `tokens` rows of the experts before e, e = 0..E (all threads of a workgroup; E <= 2 * threads): no more than
// there can be where no expert's rows are another's too.  Behind these, from kMaxC + 1 on, the experts' first rows: place_of reads them here,
// for a read from memory would be waited for together with all that the tile kernels have on its way there.
__device__ __forceinline__ void count_tiles(int tokens, const int32_t *offsets, int M, int E, int32_t *table)
{
    int32_t *const rows = table + kMaxC + 1, *const wave_sum = rows + kMaxC + 1;
    const int most = (M + tokens - 1) / tokens + (E < M ? E : M);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = tid / kWave;
    int at[3], n[2];
#pragma unroll
    for (int i = 0; i < 3; ++i) at[i] = 2 * tid + i <= E ? clamped(offsets[2 * tid + i], M) : 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) n[i] = 2 * tid + i < E && at[i + 1] > at[i] ? (at[i + 1] - at[i] + tokens - 1) / tokens : 0;
    int up = n[0] + n[1];
    for (int d = 1; d < kWave; d <<= 1) {
        const int o = __shfl_up(up, d);
        if (lane >= d) up += o;
    }
    if (lane == kWave - 1) wave_sum[w] = up;
    __syncthreads();
    int before = up - n[0] - n[1];
    for (int v = 0; v < w; ++v) before += wave_sum[v];
    auto put = [&](int e, int v, int row) {
        if (e > E) return;
        table[e] = v < most ? v : most;
        rows[e] = row;
    };
    put(2 * tid, before, at[0]);
    put(2 * tid + 1, before + n[0], at[1]);
    if (tid == kTileThreads - 1) put(2 * kTileThreads, before + n[0] + n[1], at[2]);
    __syncthreads();
}

// Where tile t lies.  An expert's tiles: its row tiles (TOKENS rows) first, then the next ROWS weight rows.
struct Place {
    int e, n0, r0, end;
};
template <int ROWS, int TOKENS>
__device__ __forceinline__ Place place_of(int E, const int32_t *table, int tiles_n, int t)
{
    const int lane = threadIdx.x & (kWave - 1);
    int e = -1;   // the last expert whose first tile is not behind t
    for (int i = 0; i < E; i += kWave)
        e += __popcll(__ballot(i + lane < E && table[i + lane < E ? i + lane : 0] * tiles_n <= t));
    auto entry = [&](int i) { return __builtin_amdgcn_readfirstlane(table[i]); };
    const int f = entry(e), m = entry(e + 1) - f, local = t - f * tiles_n, n = local / m;
    return Place{e, n * ROWS, entry(kMaxC + 1 + e) + (local - n * m) * TOKENS, entry(kMaxC + 2 + e)};
}

template <bool OUT16, bool EXACT, int J>
__global__ __launch_bounds__(kTileThreads) void tile_matmul_kernel(MatmulArgs a)
{
    constexpr int kTokens = TileSize<J>::kTokens, kStageBytes = TileSize<J>::kStage, kTileScales = TileSize<J>::kScales;
    extern __shared__ __align__(16) uint8_t lds[];
    int32_t *const table = (int32_t *)(lds + TileSize<J>::kTable);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int col = lane & 15, grp = lane >> 4, kb = a.K / kBlock, tiles_n = (a.N + kTile - 1) / kTile, nb = (a.N + kBlock - 1) / kBlock;
    count_tiles(kTokens, a.offsets, a.M, a.E, table);
    const int total = __builtin_amdgcn_readfirstlane(table[a.E]) * tiles_n;

    auto place = [&](int t) { return place_of<kTile, kTokens>(a.E, table, tiles_n, t); };

    // What this thread fetches of a step: rows tid / 8 + 64 i of both tiles, one 16-byte word each.
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    const int frow = tid / 8, wkey = (frow & 3) | ((frow >> 1) & 4), xkey = frow & 7;
    const uint8_t *wbase, *xbase;
    uint32_t wat[4], xat[J / 2];
    auto start_w = [&](const Place &p) {
        wbase = a.w + ((size_t)p.e * a.N + p.n0) * a.K;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = frow + 64 * i < a.N - p.n0 ? frow + 64 * i : a.N - p.n0 - 1;
            wat[i] = (uint32_t)n * a.K + ((tid & 7) ^ wkey) * 16;
        }
    };
    auto fetch_w = [&](int stage, int i) {   // a quarter of a step's weights
        fetch16(lds0 + stage * kStageBytes + w * 1024 + i * 8192, wat[i], wbase);
        if (i == 3) wbase += kBlock;
    };
    // The rows, and the scales of four blocks at a time: tokens' by wavefronts 0 to 3, the weights' two block rows' by wavefront 4.
    // In LDS [token][block] where a row's scales are whole 16-byte words, else [block][token].
    const int by_word = a.scale_words, s_row = by_word ? kChunk * 4 : 4, s_block = by_word ? 4 : kTile * 4, sw_block = by_word ? 4 : kWave * 4;
    const float *sbase;
    uint32_t sat;
    auto start_x = [&](const Place &p) {
        xbase = a.a + (size_t)p.r0 * a.K;
#pragma unroll
        for (int i = 0; i < J / 2; ++i) {
            const int r = frow + 64 * i < p.end - p.r0 ? frow + 64 * i : p.end - p.r0 - 1;
            xat[i] = (uint32_t)r * a.K + ((tid & 7) ^ xkey) * 16;
        }
        if (w < 4) {
            sbase = a.a_scale + (size_t)p.r0 * kb;
            sat = (uint32_t)(tid < p.end - p.r0 ? tid : p.end - p.r0 - 1) * kb * 4;
        } else {
            const int n = p.n0 / kBlock;
            sbase = a.w_scale + ((size_t)p.e * nb + n) * kb;
            sat = (uint32_t)((lane & 1) < nb - n ? lane & 1 : 0) * kb * 4;
        }
    };
    auto fetch_x = [&](int stage, int i) {
        fetch16(lds0 + stage * kStageBytes + kTileBytes + w * 1024 + i * 8192, xat[i], xbase);
        if (i == J / 2 - 1) xbase += kBlock;
    };
    int chunk = 1;   // which half of the scales' place holds the chunk fetched last
    auto fetch_scales = [&](int b) {   // of blocks b .. b + 3
        chunk ^= 1;
        if (w >= 5) return;
        const uint32_t to = lds0 + kTileScales + chunk * kChunkBytes + (w < 4 ? w * kWave * s_row : kChunk * kTile * 4);
        if (by_word) {
            fetch16(to, sat, sbase + b);
        } else {
            for (int i = 0; i < kChunk && b + i < kb; ++i) fetch4(to + i * (w < 4 ? s_block : sw_block), sat, sbase + b + i);
        }
    };

    // Tiles b, b + G, .. of an order in which the workgroups of one XCD (b % 8) are neighbours.
    const int G = gridDim.x, xcds = G % 8 ? 1 : 8, b0 = (blockIdx.x % xcds) * (G / xcds) + blockIdx.x / xcds;
    if (b0 >= total) return;
    const int wn = w & 3, wm = w >> 2;
    const uint32_t wread = (64 * wn + 8 * (col >> 2) + (col & 3)) * kBlock + ((grp ^ (col & 7)) << 4);   // (that row's key: col & 7)
    const uint32_t xread = kTileBytes + (16 * J * wm + col) * kBlock + ((grp ^ (col & 7)) << 4);
    const uint32_t sread = (16 * J * wm + col) * s_row;
    int stage = 0;
    Place here = place(b0), next = here;
    start_w(here);
    start_x(here);
#pragma unroll
    for (int i = 0; i < 4; ++i) fetch_w(0, i);
    fetch_scales(0);
#pragma unroll
    for (int i = 0; i < J / 2; ++i) fetch_x(0, i);
#pragma unroll
    for (int i = 0; i < 4; ++i) fetch_w(1, i);
    asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
    int read_chunk = 1;
    for (int t = b0; t < total; t += G) {
        const bool mine = here.r0 + 16 * J * wm < here.end && here.n0 + 64 * wn < a.N;
        f32x4 acc[4][J];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int b = 0; b < kb; ++b) {
            // This wavefront's part of the step has arrived (four loads, of weights for the next step, may be on their way; for a tile's
            // first step that was waited for before the stores of the tile before) and its reads of the step before are done; then
            // everybody's.
            if (b == 0) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            else asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (b % kChunk == 0) read_chunk ^= 1;
            const uint8_t *const st = lds + kTileScales + read_chunk * kChunkBytes + (b % kChunk) * s_block;
            const uint8_t *const swt = lds + kTileScales + read_chunk * kChunkBytes + kChunk * kTile * 4 + (b % kChunk) * sw_block;
            // (behind the last tile its own first steps are fetched once more and not read)
            if (b + 1 == kb) start_x(next);
            if (b + 1 == kb || (b + 1) % kChunk == 0) fetch_scales(b + 1 == kb ? 0 : b + 1);
            if (b == 0 && t + G < total) next = place(t + G);
            if (b + 2 == kb) start_w(next);
            const uint8_t *const tile = lds + stage * kStageBytes;
            // The loads go out one at a time between the products: the loads of all wavefronts at once keep the address unit busy
            // for a thousand cycles, in which a wavefront whose turn has not come issues nothing else.  The next step's rows first;
            // then, when everybody has its weights (the products that read them are on their way), those of the step after next.
            auto request = [&](int j) {
                if (j < J / 2) {
                    fetch_x(stage ^ 1, j);
                } else {
                    if (j == J / 2) {
                        __builtin_amdgcn_s_barrier();
                        asm volatile("" ::: "memory");
                    }
#pragma unroll
                    for (int i = 0; i < 8 / J; ++i) fetch_w(stage, (j - J / 2) * (8 / J) + i);
                }
            };
            if (!mine) {
#pragma unroll
                for (int j = 0; j < J; ++j) request(j);
                stage ^= 1;
                continue;
            }
            u32x4 xraw[2], wraw[4][2];
            auto read_x = [&](int j) {
                xraw[0] = *(const u32x4 *)(tile + xread + j * 16 * kBlock);
                xraw[1] = *(const u32x4 *)(tile + (xread ^ 64) + j * 16 * kBlock);
            };
            read_x(0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = (i >> 1) * 32 + (i & 1) * 4;
                wraw[i][0] = *(const u32x4 *)(tile + wread + at * kBlock);
                wraw[i][1] = *(const u32x4 *)(tile + (wread ^ 64) + at * kBlock);
            }
            auto scale = [&](int j) { return *(const float *)(st + sread + j * 16 * s_row); };
            const float sw = *(const float *)(swt + (wn >> 1) * s_row);
            Operand<EXACT> wv[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) wv[i] = Operand<EXACT>(wraw[i][0], wraw[i][1]);
            // sixteen tokens' products while those before are scaled and added (in this order: left to itself the compiler puts
            // every product's multiply-adds right behind it and waits)
            f32x4 sum[2][4];
            float s[2] = {scale(0) * sw, 0.f};
#pragma unroll
            for (int j = 0; j <= J; ++j) {
                if (j < J) request(j);
                const Operand<EXACT> now(xraw[0], xraw[1]);
                float next_scale;
                if (j < J - 1) {
                    read_x(j + 1);
                    next_scale = scale(j + 1);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (j < J) sum[j & 1][i] = mfma128(wv[i], now);
                    if (j > 0) {
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            acc[i][j - 1][c] = __builtin_fmaf(sum[~j & 1][i][c], s[~j & 1], acc[i][j - 1][c]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (j < J - 1) s[~j & 1] = next_scale * sw;
            }
            stage ^= 1;
        }
        asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int r = here.r0 + 16 * J * wm + 16 * j + col;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int n = here.n0 + 64 * wn + 32 * i + 8 * grp;
                if (r < here.end && n < a.N) {
                    const f32x4 u = acc[2 * i][j], v = acc[2 * i + 1][j];
                    if (OUT16) {
                        const u32x4 o = {pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]), pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
                        *(u32x4 *)((uint16_t *)a.out + (size_t)r * a.N + n) = o;
                    } else {
                        f32x4 *o = (f32x4 *)((float *)a.out + (size_t)r * a.N + n);
                        o[0] = u;
                        o[1] = v;
                    }
                }
            }
        }
        here = next;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (nothing is on its way to the LDS of a workgroup that has ended)
}

// ---- the same with smaller tiles: 128 weight rows x 128 tokens, four steps in LDS ----
// For calls of few tiles, where a step's time is the latency of its loads and of LDS.  Loads are four steps ahead of the products, and a
// wavefront (32 weight rows x 64 tokens) reads the next step's operands from LDS while it multiplies this one's: behind a step's one
// barrier the matrix cores have work at once; the halves of 32 tokens that are not there are left out.  A step of 128 columns takes 0.7 us
// (short sums; 0.5 with up to 32 tokens), against 1.2 us of 256 x 128 and 1.7 us of 256 x 256 (2120 rows of 8 experts of 512 x 7168:
// 40 against 57 and 84 us); the larger tiles read and move less.  Wavefronts of 64 weight rows x 32 tokens: up to 32 tokens 20 % slower,
// 32-bit sums of full tiles 5 % faster.
constexpr int kRing = 4, kRingTile = 128;
constexpr int kRingHalf = kRingTile * kBlock, kRingStage = 2 * kRingHalf;
constexpr int kRingChunk = kChunk * (kRingTile + kWave) * 4, kRingScales = kRing * kRingStage;
constexpr int kRingTable = kRingScales + kRing * kRingChunk, kRingLds = kRingTable + kTableInts * 4;
static_assert(kRingLds <= kLdsBytes, "the steps, their scales, the experts' tiles and rows");

template <bool OUT16, bool EXACT>
__global__ __launch_bounds__(kTileThreads) void ring_matmul_kernel(MatmulArgs a)
{
    extern __shared__ __align__(16) uint8_t lds[];
    int32_t *const table = (int32_t *)(lds + kRingTable);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = __builtin_amdgcn_readfirstlane(tid / kWave);
    const int col = lane & 15, grp = lane >> 4, kb = a.K / kBlock, tiles_n = (a.N + kRingTile - 1) / kRingTile;
    count_tiles(kRingTile, a.offsets, a.M, a.E, table);
    const int total = __builtin_amdgcn_readfirstlane(table[a.E]) * tiles_n;
    const int G = gridDim.x, xcds = G % 8 ? 1 : 8, b0 = (blockIdx.x % xcds) * (G / xcds) + blockIdx.x / xcds;
    if (b0 >= total) return;
    auto place = [&](int t) { return place_of<kRingTile, kRingTile>(a.E, table, tiles_n, t); };

    // The loads' walk over the steps of all tiles: two 16-byte words a thread of both operands, rows tid / 8 and 64 further on; the scales
    // of four blocks at a time, tokens' by wavefronts 0 and 1, the weights' by wavefront 2 (every lane the same).
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)lds;
    const int by_word = a.scale_words, s_row = by_word ? kChunk * 4 : 4, s_block = by_word ? 4 : kRingTile * 4, sw_block = by_word ? 4 : kWave * 4;
    const uint8_t *wbase, *xbase;
    const float *sbase;
    uint32_t wat[2], xat[2], sat;
    int fetched = 0, stage_in = 0, chunk_in = -1;   // blocks of the walk's tile, where the next step goes
    auto start = [&](const Place &p) {
        const int row = tid / 8, key = (row & 3) | ((row >> 1) & 4);
        wbase = a.w + ((size_t)p.e * a.N + p.n0) * a.K;
        xbase = a.a + (size_t)p.r0 * a.K;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int n = row + 64 * i < a.N - p.n0 ? row + 64 * i : a.N - p.n0 - 1;
            const int r = row + 64 * i < p.end - p.r0 ? row + 64 * i : p.end - p.r0 - 1;
            wat[i] = (uint32_t)n * a.K + ((tid & 7) ^ key) * 16;
            xat[i] = (uint32_t)r * a.K + ((tid & 7) ^ (row & 7)) * 16;
        }
        if (w < 2) {
            sbase = a.a_scale + (size_t)p.r0 * kb;
            sat = (uint32_t)(tid < p.end - p.r0 ? tid : p.end - p.r0 - 1) * kb * 4;
        } else {
            sbase = a.w_scale + ((size_t)p.e * ((a.N + kBlock - 1) / kBlock) + p.n0 / kBlock) * kb;
            sat = 0;
        }
        fetched = 0;
    };
    auto fetch = [&]() {
        if (fetched % kChunk == 0) {
            chunk_in = (chunk_in + 1) % kRing;
            if (w < 3) {
                const uint32_t to = lds0 + kRingScales + chunk_in * kRingChunk + (w < 2 ? w * kWave * s_row : kChunk * kRingTile * 4);
                if (by_word) {
                    fetch16(to, sat, sbase + fetched);
                } else {
                    for (int i = 0; i < kChunk && fetched + i < kb; ++i) fetch4(to + i * (w < 2 ? s_block : sw_block), sat, sbase + fetched + i);
                }
            }
        }
        const uint32_t to = lds0 + stage_in * kRingStage + w * 1024;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            fetch16(to + i * 8192, wat[i], wbase);
            fetch16(to + kRingHalf + i * 8192, xat[i], xbase);
        }
        wbase += kBlock;
        xbase += kBlock;
        ++fetched;
        stage_in = (stage_in + 1) % kRing;
    };

    const int wn = w & 3, wm = w >> 2;
    const uint32_t wread = (32 * wn + 8 * (col >> 2) + (col & 3)) * kBlock + ((grp ^ (col & 7)) << 4);   // (that row's key: col & 7)
    const uint32_t xread = kRingHalf + (64 * wm + col) * kBlock + ((grp ^ (col & 7)) << 4);
    const uint32_t sread = (64 * wm + col) * s_row;
    int stage = 0, chunk = 0;   // of the operands read last
    struct Step {
        u32x4 w[2][2], x[4][2];
        float s[4];
    };
    auto read = [&](u32x4 *o, uint32_t at) {
        o[0] = *(const u32x4 *)(lds + stage * kRingStage + at);
        o[1] = *(const u32x4 *)(lds + stage * kRingStage + (at ^ 64));
    };
    auto read_w = [&](Step &o) {
#pragma unroll
        for (int i = 0; i < 2; ++i) read(o.w[i], wread + i * 4 * kBlock);
    };
    auto read_x = [&](Step &o, int j, int block) {
        const uint8_t *const st = lds + kRingScales + chunk * kRingChunk;
        const float sw = *(const float *)(st + kChunk * kRingTile * 4 + (block % kChunk) * sw_block);
        read(o.x[j], xread + j * 16 * kBlock);
        o.s[j] = *(const float *)(st + (block % kChunk) * s_block + sread + j * 16 * s_row) * sw;
    };
    // How many of a wavefront's two halves of 32 tokens there are in a tile; without any it only loads.
    auto halves = [&](const Place &p) {
        const int rows = p.end - p.r0 - 64 * wm;
        return p.n0 + 32 * wn >= a.N || rows <= 0 ? 0 : rows <= 32 ? 1 : 2;
    };

    Place now = place(b0), next = now;   // (K has at least four blocks: the walk of the loads is in this tile or the next)
    start(now);
#pragma unroll
    for (int i = 0; i < kRing; ++i) fetch();
    asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    Step step;
    read_w(step);
#pragma unroll
    for (int j = 0; j < 4; ++j) read_x(step, j, 0);
    int work = halves(now), next_work = work;
    f32x4 acc[2][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[0][j] = acc[1][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    bool waited = false;   // the next step's loads have been waited for in front of a tile's stores
    for (int t = b0; t < total; t += G) {
        if (t + G < total) next = place(t + G);
        next_work = halves(next);
        for (int b = 0; b < kb; ++b) {
            // The next step has arrived here (the loads of the two behind it may be on their way), and this one's operands are in
            // registers; then everybody's: its place is free.
            if (waited) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            else asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
            waited = false;
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (fetched == kb) start(next);   // (behind the last tile its own steps once more, not used)
            fetch();
            stage = (stage + 1) % kRing;
            const int after = b + 1 < kb ? b + 1 : 0;
            if (after % kChunk == 0) chunk = (chunk + 1) % kRing;
            const int most = after == 0 && next_work > work ? next_work : work;   // (for this step's products and the next one's operands)
            if (most == 0) continue;
            Step ahead;
            read_w(ahead);
            const Operand<EXACT> y0(step.w[0][0], step.w[0][1]), y1(step.w[1][0], step.w[1][1]);
            f32x4 sum[2][2];
            auto multiply = [&](int j) {
                const Operand<EXACT> x(step.x[j][0], step.x[j][1]);
                sum[j & 1][0] = mfma128(y0, x);
                sum[j & 1][1] = mfma128(y1, x);
                read_x(ahead, j, after);
            };
            auto add = [&](int j) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[i][j][c] = __builtin_fmaf(sum[j & 1][i][c], step.s[j], acc[i][j][c]);
                if (!EXACT) __builtin_amdgcn_sched_barrier(0);   // (32-bit sums are 4 % faster in the compiler's order)
            };
            multiply(0);
            if (!EXACT) __builtin_amdgcn_sched_barrier(0);
            multiply(1);
            add(0);
            if (most == 2) {
                multiply(2);
                add(1);
                multiply(3);
                add(2);
                add(3);
            } else {
                add(1);
            }
            step = ahead;
        }
        asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
        waited = true;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = now.r0 + 64 * wm + 16 * j + col, n = now.n0 + 32 * wn + 8 * grp;
            const f32x4 u = acc[0][j], v = acc[1][j];
            if (r < now.end && n < a.N) {
                if (OUT16) {
                    const u32x4 o = {pack_bf16(u[0], u[1]), pack_bf16(u[2], u[3]), pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
                    *(u32x4 *)((uint16_t *)a.out + (size_t)r * a.N + n) = o;
                } else {
                    f32x4 *o = (f32x4 *)((float *)a.out + (size_t)r * a.N + n);
                    o[0] = u;
                    o[1] = v;
                }
            }
            acc[0][j] = acc[1][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        now = next;
        work = next_work;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (nothing is on its way to the LDS of a workgroup that has ended)
}

// Which kernel takes a call: the one that should be the fastest by what they measured, from the sizes alone.  us, short sums to bf16 / 32-bit
// sums to fp32 (to bf16: 6 % less where results are many; the streaming kernel has 32-bit sums only); r: rows an expert, evenly.  64 experts
// of 2816 x 2048, then one of them, then 8 of 512 x 7168:
//            r = 6         12        24        47        94        187       281       768          64        512       12        265
//      streaming 60        73        97        187       329       622       922       -            9         -         15        83
//      128 x 128 71/73     72/75     74/81     81/93     92/127    144/239   197/330   446/755      13/18     16/26     25/34     40/69
//      256 x 128 69/75     71/78     73/81     78/89     89/119    141/212   177/279   362/616      16/25     22/37     43/68     57/104
//      256 x 256 72/-      73/-      76/-      80/-      90/-      117/-     191/-     335/-        20/-      31/-      55/-      84/-
// (The others than streaming: tiles of weight rows x rows.  256 x 256 with 32-bit sums, whose operands are wider
// than its registers hold at once, was never the fastest by more than 5 %.)  Over 3000 calls of random sizes, short sums and
// fp32 results, the choice took 1.025 times the fastest's time (bf16 results with 32-bit sums, 8388 other calls: 1.03);
// without one of the kernels the fastest took 1.005 (256 x 256) to 1.14 (streaming) times as long as with all.
//
// All: the weights' bytes (at the rate that each reaches), once for each pass over an expert's rows.  The streaming kernel: what a CU
// takes in, weights and rows, at 32 B/ns; or the blocks that a wavefront loads one after the other.  The tiles: rounds of them over the
// CUs, each as many steps as there are blocks, a step's time by how many of its rows there are.
struct Choice {
    enum { kStream, kTiles128, kTiles256x128, kTiles256 } kernel;
    int waves;    // of a workgroup of the streaming kernel
};

Choice choose(int M, int N, int K, int E, bool exact, int cus)
{
    auto up = [](double x) { return (double)(long long)(x + 0.999999); };
    auto least = [](double a, double b) { return a < b ? a : b; };
    auto most = [](double a, double b) { return a > b ? a : b; };
    const double kb = K / kBlock;
    const double experts = E * (1 - exp(-(double)M / E));   // that have rows, where each row is anybody's
    const double r = M / experts, groups = experts * ((N + 31) / 32), megabytes = experts * N * K * 1e-6;
    Choice best = {};
    double least_time = 1e30;
    auto consider = [&](double time, Choice c) {
        if (time < least_time) {
            least_time = time;
            best = c;
        }
    };
    // Wavefronts: eight where four would have many blocks each or leave CUs without enough of them (384 rows on 64 experts of
    // 2816 x 2048: 4 wavefronts 59 us, 8 69; 4 rows on one of 8192 x 4096: 10.7 and 9.2; 308 skewed on 128 of 384 x 7936: 48 and 38)
    const int w = kb >= 32 || (kb >= 16 && groups <= 2 * cus) ? kMostWaves : kMostWaves / 2;
    const double more = r <= 8 ? 0 : r >= 24 ? 1 : (r - 8) / 16;   // of the groups of rows, those of more than sixteen
    const double passes = most(1.0, r / kGroup + 0.2);
    const double taken = groups * passes * 32.0 * K * (1.38 + 1.9 * more) / (32e3 * cus);
    const double chain = 0.75 + (0.6 + 0.25 * more) * up(kb / w);
    consider(1.6 + most(most(passes * megabytes / 6.0, taken), chain) + 0.28 * chain, {Choice::kStream, w});
    auto tiles = [&](int rows, int tokens, double step, double rate, Choice c) {
        const double rounds = up(up(r / tokens) * experts * ((N + rows - 1) / rows) / cus);
        consider(2.3 + most(megabytes / rate, rounds * kb * step), c);
    };
    // (the tiles' loads are four and two steps ahead of them)
    const double half = least(r, 128) / 128, full = least(r, 256) / 256;
    const double wide = r > 32;   // (the second 32 rows of each 64)
    if (kb >= 4) tiles(128, 128, exact ? 0.68 + 0.11 * half + 0.33 * wide : 0.42 + 0.17 * half + 0.25 * wide, exact ? 4.1 : 5.2, {Choice::kTiles128, 0});
    if (kb >= 2) tiles(256, 128, exact ? 1.3 + 0.28 * half : 0.7 + 0.4 * half, exact ? 3.7 : 5.2, {Choice::kTiles256x128, 0});
    if (kb >= 2 && !exact) tiles(256, 256, 1.0 + 0.8 * full, 3.8, {Choice::kTiles256, 0});
    return best;
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" int moe_grouped_matmul_fp8(const void *x, const float *x_scale, const void *w, const float *w_scale, const int32_t *offsets,
                                      int M, int N, int K, int E, void *out, int out_bf16, void *stream)
{
    if (!x || !x_scale || !w || !w_scale || !offsets || !out) return MOE_ERR_NULL;
    if (M < 1 || N < 1 || K < 1 || E < 1 || E > kMaxC || M > 1 << 30 || N > 1 << 24 || K > 1 << 20) return MOE_ERR_SHAPE;
    if ((size_t)((M + 127) / 128 + E) * ((N + 127) / 128) >= (size_t)1 << 30) return MOE_ERR_SHAPE;
    if (N % 8 || K % kBlock || !aligned16(x) || !aligned16(w) || !aligned16(out)) return MOE_ERR_ALIGN;
    MatmulArgs a = {(const uint8_t *)x, (const uint8_t *)w, x_scale, w_scale, offsets, out, M, N, K, E,
                    K / kBlock % 4 == 0 && aligned16(x_scale) && aligned16(w_scale), 0};
    hipError_t err;
    const int cus = device_cus(&err);
    if (err != hipSuccess) return launch_failed(err);
    const bool exact = out_bf16 != MOE_BF16_SHORT_SUMS;
    const Choice c = choose(M, N, K, E, exact, cus);
    auto tiles = [&](const void *fn, int rows, int tokens, int lds) {
        const size_t n = ((size_t)(M + tokens - 1) / tokens + (E < M ? E : M)) * ((N + rows - 1) / rows);   // (at most)
        return launch_rows(fn, dim3(n < (size_t)cus ? (unsigned)n : cus), kTileThreads, &a, lds, stream, MOE_KERNEL_MATMUL);
    };
    switch (c.kernel) {
    case Choice::kTiles128:
        return tiles(!exact ? (const void *)ring_matmul_kernel<true, false> : out_bf16 ? (const void *)ring_matmul_kernel<true, true>
                     : (const void *)ring_matmul_kernel<false, true>, 128, 128, kRingLds);
    case Choice::kTiles256x128:
        return tiles(!exact ? (const void *)tile_matmul_kernel<true, false, 4> : out_bf16 ? (const void *)tile_matmul_kernel<true, true, 4>
                     : (const void *)tile_matmul_kernel<false, true, 4>, 256, 128, TileSize<4>::kLds);
    case Choice::kTiles256:
        return tiles((const void *)tile_matmul_kernel<true, false, 8>, 256, 256, TileSize<8>::kLds);
    default: break;
    }
    // Where most experts have no rows, workgroups for the rows: those of an expert without rows only come and go, but thousands of
    // them take longer than the search of the one for a row does (6 rows on 64 experts of 2816 x 2048: 11.6 against 12.2 us; 54 rows
    // 21.9 against 20.0), and where few stay they leave them two to a CU and others empty (2 rows on 8 of 4096 x 14336: 21 against 32).
    a.by_row = M <= E / 8 || (M < E && (size_t)M * ((N + 31) / 32) <= (size_t)2 * cus);
    const int groups = a.by_row ? M : E + (M - 1) / kGroup;   // (at most)
    const dim3 grid((N + 31) / 32, groups < 32768 ? groups : 32768, (groups + 32767) / 32768);
    return launch_rows(out_bf16 ? (const void *)stream_matmul_kernel<true> : (const void *)stream_matmul_kernel<false>, grid, c.waves * kWave, &a,
                       (size_t)c.waves * 2 * (kGroup / 16) * kWave * 16, stream, MOE_KERNEL_MATMUL);
}
