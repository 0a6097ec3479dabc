// Assignments sorted by expert, the tokens' rows brought into that order and back with the gate weights (Sec. 2.2 last line
// for batches of any length), and the gradient of the way back.
//
// Sort: a counting sort, stable, so that a row's place follows from the routing alone.  Rows of expert e are
// [offsets[e], offsets[e+1]), inside them the flat assignment ids ascend.  Assignments of no expert (-1) come to no row.
// Moving and summing rows: bound by memory; every row is read once and written once, 16 bytes a lane.  (A large copy of this card's
// memory moves 4.95 TB/s, read and written; the rates below that are higher have reads or writes that outweigh the other.)
#include "../../include/moe_spac.h"
#include "rows_device.h"

namespace moe {

namespace {

using namespace rows;

// ---- sort ----
// Bound by latency.  Up to 16384 assignments one launch, back to back 3.4 us for 6 assignments, 4.3 for 4000 on 60 experts (one workgroup
// for them all: 5.6), 5.9 for 16320 on 64 (a count and a place launch: 6.9; 24576: 7.0 either way).  Then the two launches, over up to 128
// workgroups: 8.3 us for 98304 on 64, whose 1.2 MB are 0.2 us of memory.
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / kWave;
constexpr int kSortBlocks = 128;      // most workgroups
constexpr int kSortChunk = 1024;      // least assignments of one of its workgroups (98304 on 64 experts: 8.2 us; 2048 8.4, 4096 8.9)
constexpr int kAhead = 4;             // loads in flight
constexpr int kSortOne = 16384;       // up to so many assignments: one launch

struct SortArgs {
    const int32_t *ids;
    int A, E, bits, chunk, blocks;
    int32_t *offsets, *order, *pos;
    int32_t *counts;                  // [blocks][E] (two-launch form)
};

__device__ __forceinline__ int expert_of(const SortArgs &a, int i, int end)
{
    const int e = i < end ? a.ids[i] : -1;
    return e < a.E ? e : -1;
}

// How many assignments of each expert are in a workgroup's chunk.
__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(SortArgs a)
{
    extern __shared__ int32_t lds[];
    for (int e = threadIdx.x; e < a.E; e += kSortThreads) lds[e] = 0;
    __syncthreads();
    const int begin = blockIdx.x * a.chunk, end = begin + a.chunk < a.A ? begin + a.chunk : a.A;
    for (int i = begin + threadIdx.x; i < end; i += kSortThreads) {
        const int e = expert_of(a, i, end);
        if (e >= 0) atomicAdd(&lds[e], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < a.E; e += kSortThreads) a.counts[(size_t)blockIdx.x * a.E + e] = lds[e];
}

// Places of a workgroup's chunk.  A wavefront has a consecutive part of the chunk: the parts' counts, added up over the parts
// before and the chunks before, say where its first assignment of each expert goes; inside sixty-four assignments the lanes
// with the same expert find one another by a ballot for each bit of its number.
// ONE: the only launch, whose workgroups (1024 assignments each) count the whole batch for themselves, each assignment once: into the
// parts, or as one of the chunks before or behind.
template <bool ONE>
__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(SortArgs a)
{
    extern __shared__ int32_t lds[];
    int32_t *part = lds;                            // [kSortWaves][E]: count, then next place
    int32_t *all = lds + kSortWaves * a.E;          // [E] assignments of the expert in the whole batch (ONE: in the chunks behind)
    int32_t *before = all + a.E;                    // [E] ... in the chunks before
    int32_t *wave_sum = before + a.E;               // [kSortWaves]
    const int tid = threadIdx.x, lane = tid & (kWave - 1), w = tid / kWave;
    for (int i = tid; i < (kSortWaves + 2) * a.E; i += kSortThreads) lds[i] = 0;
    __syncthreads();
    const int begin = blockIdx.x * a.chunk, end = begin + a.chunk < a.A ? begin + a.chunk : a.A;
    const int per_wave = a.chunk / kSortWaves;      // (a multiple of 64)
    const int first = begin + w * per_wave, last = first + per_wave < end ? first + per_wave : end;
    if (ONE) {   // (a chunk is an assignment a thread)
        for (int c = 0; c < a.blocks; c += kAhead) {
            int e[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) e[u] = expert_of(a, (c + u) * kSortThreads + tid, a.A);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                int32_t *const counts = c + u == (int)blockIdx.x ? part + w * a.E : c + u < (int)blockIdx.x ? before : all;
                if (e[u] >= 0) atomicAdd(&counts[e[u]], 1);
            }
        }
    } else {
        for (int i = first; i < last; i += kAhead * kWave) {
            int e[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) e[u] = expert_of(a, i + u * kWave + lane, last);
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (e[u] >= 0) atomicAdd(&part[w * a.E + e[u]], 1);
        }
    }
    if (!ONE) {
        // the counts of all chunks: a wavefront has every sixteenth row of the table
        for (int e0 = lane; e0 < a.E; e0 += kAhead * kWave) {
            int n[kAhead] = {}, m[kAhead] = {};
#pragma unroll 4
            for (int b = w; b < a.blocks; b += kSortWaves)
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    const int e = e0 + u * kWave, c = e < a.E ? a.counts[(size_t)b * a.E + e] : 0;
                    n[u] += c;
                    m[u] += b < (int)blockIdx.x ? c : 0;
                }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (n[u]) atomicAdd(&all[e0 + u * kWave], n[u]);
                if (m[u]) atomicAdd(&before[e0 + u * kWave], m[u]);
            }
        }
    }
    __syncthreads();
    // E <= 1024 = threads: thread e has expert e
    int mine = 0;
    if (tid < a.E) {
        mine = all[tid];
        if (ONE) {
            mine += before[tid];
            for (int v = 0; v < kSortWaves; ++v) mine += part[v * a.E + tid];
        }
    }
    int up = mine;                                  // inclusive sum over the wavefront's lanes
    for (int d = 1; d < kWave; d <<= 1) {
        const int o = __shfl_up(up, d);
        if (lane >= d) up += o;
    }
    if (lane == kWave - 1) wave_sum[w] = up;
    __syncthreads();
    int at = up - mine;
    for (int v = 0; v < w; ++v) at += wave_sum[v];
    int valid = 0;
    for (int v = 0; v < kSortWaves; ++v) valid += wave_sum[v];
    if (tid < a.E) {
        if (blockIdx.x == 0) a.offsets[tid] = at;
        int next = at + before[tid];
        for (int v = 0; v < kSortWaves; ++v) {
            const int n = part[v * a.E + tid];
            part[v * a.E + tid] = next;
            next += n;
        }
    }
    if (blockIdx.x == 0 && tid == 0) a.offsets[a.E] = valid;
    for (int r = valid + blockIdx.x * kSortThreads + tid; r < a.A; r += gridDim.x * kSortThreads) a.order[r] = -1;
    __syncthreads();
    for (int i = first; i < last; i += kAhead * kWave) {
        int e[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) e[u] = expert_of(a, i + u * kWave + lane, last);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int at = i + u * kWave;
            if (at >= last) break;
            unsigned long long same = __ballot(e[u] >= 0);
            for (int b = 0; b < a.bits; ++b) {
                const unsigned long long set = __ballot((e[u] >> b) & 1);
                same &= (e[u] >> b) & 1 ? set : ~set;
            }
            const int rank = __popcll(same & ((1ull << lane) - 1ull));
            int place = -1;
            if (e[u] >= 0) {
                place = part[w * a.E + e[u]] + rank;
                a.order[place] = at + lane;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");   // (every lane has read its place before the first of them moves on)
            __builtin_amdgcn_wave_barrier();
            if (e[u] >= 0 && rank == 0) part[w * a.E + e[u]] += __popcll(same);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (at + lane < last) a.pos[at + lane] = place;
        }
    }
}

int sort_blocks(int A)
{
    const int n = (A + kSortChunk - 1) / kSortChunk;
    return n < kSortBlocks ? n : kSortBlocks;
}

// ---- rows ----
constexpr int kRowThreads = 256, kRowWaves = kRowThreads / kWave;
constexpr unsigned kMostGroups = 1u << 20;   // workgroups of a launch (each walks the work with that step)

struct MoveArgs {
    const u32x4 *x;          // [T] rows of `words` words
    const int32_t *pos;      // [T,k]
    u32x4 *out;              // [R]
    int k, R, words, stream;
    unsigned parts, rcp_parts, items;
};

// out[pos[t,j]] = x[t]: a wavefront has U words a lane of one token's row and stores them k times.  1000 tokens of 2040 floats to some 2600
// rows: 7.4 us, 4.0 TB/s; U = 4 as soon as that leaves a wavefront for each SIMD, else 1, so that few tokens spread over more of them.
template <int U>
__global__ __launch_bounds__(kRowThreads) void permute_kernel(MoveArgs a)
{
    const int lane = threadIdx.x & (kWave - 1), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    for (unsigned item = blockIdx.x * kRowWaves + w; item < a.items; item += gridDim.x * kRowWaves) {
        const unsigned t = quotient(item, a.parts, a.rcp_parts), part = item - t * a.parts;
        const int c0 = (int)part * U * kWave + lane;
        const u32x4 *src = a.x + (size_t)t * a.words;
        u32x4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c0 + u * kWave < a.words) v[u] = src[c0 + u * kWave];
        for (int j = 0; j < a.k; ++j) {
            const int r = a.pos[(size_t)t * a.k + j];
            if ((unsigned)r >= (unsigned)a.R) continue;
            u32x4 *dst = a.out + (size_t)r * a.words;
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (c0 + u * kWave < a.words) put(dst + c0 + u * kWave, v[u], a.stream);
        }
    }
}

struct MoveFp8Args {
    const void *x;           // [T,H] bf16 or fp32
    const int32_t *pos;
    u32x4 *q;                // [R,Hp]
    float *scale;            // [R,Hb]
    int k, R, H, stream;
    unsigned blocks, rcp_blocks, items;   // blocks of a row; T * blocks
};

// The same with the row quantised on the way: eight lanes have a block of 128, sixteen values a lane.  A row is read and quantised once and
// stored k times: 16384 tokens of 2048 bf16 to 98304 rows of 2048 bytes 43.5 us, 6.3 TB/s.
template <bool BF16>
__global__ __launch_bounds__(kRowThreads) void permute_fp8_kernel(MoveFp8Args a)
{
    const unsigned g0 = (blockIdx.x * kRowThreads + threadIdx.x) / 8, step = gridDim.x * (kRowThreads / 8);
    const int sub = threadIdx.x & 7;
    for (unsigned g = g0; g < a.items; g += step) {   // (the eight lanes of a block stay together)
        const unsigned t = quotient(g, a.blocks, a.rcp_blocks), b = g - t * a.blocks;
        const int c = (int)b * kBlock + sub * 16;
        float f[16];
        constexpr int n = kPerWord<BF16>;
#pragma unroll
        for (int i = 0; i < 16 / n; ++i) {
            u32x4 v = {0u, 0u, 0u, 0u};
            if (c + i * n < a.H) v = ((const u32x4 *)a.x)[((size_t)t * a.H + c) / n + i];
            to_floats<BF16>(v, f + i * n);
        }
        unsigned m = kLeastBits;
#pragma unroll
        for (int i = 0; i < 16; ++i) m = larger(m, magnitude(f[i]));
        const float top = __uint_as_float(largest_of_8(m));
        const u32x4 q = sixteen_fp8(f, kTop / top);
        const float scale = top / kTop;
        for (int j = 0; j < a.k; ++j) {
            const int r = a.pos[(size_t)t * a.k + j];
            if ((unsigned)r >= (unsigned)a.R) continue;
            put(a.q + ((size_t)r * a.blocks + b) * 8 + sub, q, a.stream);
            if (sub == 0) a.scale[(size_t)r * a.blocks + b] = scale;
        }
    }
}

struct SumArgs {
    const u32x4 *rows;       // [R,H]
    const int32_t *pos;      // [T,k]
    const float *w;          // [T,k] or null (ones)
    u32x4 *out;              // [T,H]
    int k, R, H, accumulate, stream;
    unsigned parts, rcp_parts, items;
};

// Eight columns of a row: one word of bf16, two of fp32.
template <bool BF16>
__device__ __forceinline__ void load8(const u32x4 *row, int unit, float *f)
{
    if (BF16) {
        to_floats<true>(row[unit], f);
    } else {
        to_floats<false>(row[2 * unit], f);
        to_floats<false>(row[2 * unit + 1], f + 4);
    }
}
template <bool BF16>
__device__ __forceinline__ void store8(u32x4 *row, int unit, const float *f, int stream)
{
    if (BF16) {
        put(row + unit, to_word<true>(f), stream);
    } else {
        put(row + 2 * unit, to_word<false>(f), stream);
        put(row + 2 * unit + 1, to_word<false>(f + 4), stream);
    }
}

// out[t] (+)= sum over j of w[t,j] rows[pos[t,j]], in fp32, j ascending: a wavefront has eight columns a lane of one token, so that a
// result is one lane's sum, in the same order whatever the sizes.  8192 tokens of 2048 from six bf16 rows each, to bf16: 46 us, 5.1 TB/s.
template <bool IN16, bool OUT16>
__global__ __launch_bounds__(kRowThreads) void unpermute_kernel(SumArgs a)
{
    const int lane = threadIdx.x & (kWave - 1), w = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int units = a.H / 8;
    constexpr int nin = kPerWord<IN16>, nout = kPerWord<OUT16>;
    for (unsigned item = blockIdx.x * kRowWaves + w; item < a.items; item += gridDim.x * kRowWaves) {
        const unsigned t = quotient(item, a.parts, a.rcp_parts), part = item - t * a.parts;
        const int unit = (int)part * kWave + lane;
        if (unit >= units) continue;
        u32x4 *out = a.out + (size_t)t * (a.H / nout);
        float sum[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] = 0.f;
        if (a.accumulate) load8<OUT16>(out, unit, sum);
        for (int j = 0; j < a.k; ++j) {
            const int r = a.pos[(size_t)t * a.k + j];
            if ((unsigned)r >= (unsigned)a.R) continue;
            const float by = a.w ? a.w[(size_t)t * a.k + j] : 1.f;
            float f[8];
            load8<IN16>(a.rows + (size_t)r * (a.H / nin), unit, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] = __builtin_fmaf(by, f[i], sum[i]);
        }
        store8<OUT16>(out, unit, sum, a.stream);
    }
}

struct BackArgs {
    const u32x4 *dout;       // [T,H]
    const u32x4 *rows;       // [R,H] or null (no dw)
    const int32_t *pos;
    const float *w;          // [T,k] or null
    u32x4 *drows;            // [R,H] or null
    float *dw;               // [T,k] or null
    int k, R, H, stream;
    unsigned A, rcp_k;
};

// drows[pos[t,j]] = w[t,j] dout[t], dw[t,j] = <dout[t], rows[pos[t,j]]>: a wavefront has one assignment, so that the scalar product needs
// no second pass and no atomics; dout comes k times, all but the first from L2.  4096 tokens of 4096 bf16, k = 2: 34 us, 4.9 TB/s.
template <bool OUT16, bool IN16>
__global__ __launch_bounds__(kRowThreads) void unpermute_backward_kernel(BackArgs a)
{
    const int lane = threadIdx.x & (kWave - 1), wv = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int units = a.H / 8;
    constexpr int nin = kPerWord<IN16>, nout = kPerWord<OUT16>;
    for (unsigned i = blockIdx.x * kRowWaves + wv; i < a.A; i += gridDim.x * kRowWaves) {
        const unsigned t = quotient(i, (unsigned)a.k, a.rcp_k);
        const int r = a.pos[i];
        if ((unsigned)r >= (unsigned)a.R) {
            if (a.dw && lane == 0) a.dw[i] = 0.f;
            continue;
        }
        const float by = a.w ? a.w[i] : 1.f;
        const u32x4 *d = a.dout + (size_t)t * (a.H / nout);
        float dot = 0.f;
        for (int unit = lane; unit < units; unit += kWave) {
            float g[8];
            load8<OUT16>(d, unit, g);
            if (a.dw) {
                float f[8];
                load8<IN16>(a.rows + (size_t)r * (a.H / nin), unit, f);
#pragma unroll
                for (int c = 0; c < 8; ++c) dot = __builtin_fmaf(g[c], f[c], dot);
            }
            if (a.drows) {
#pragma unroll
                for (int c = 0; c < 8; ++c) g[c] *= by;
                store8<IN16>(a.drows + (size_t)r * (a.H / nin), unit, g, a.stream);
            }
        }
        if (a.dw) {
            for (int s = kWave / 2; s > 0; s >>= 1) dot += __shfl_xor(dot, s);
            if (lane == 0) a.dw[i] = dot;
        }
    }
}

// Sizes that the four calls on rows share.
int check_rows(int T, int k, int H, int R)
{
    if (T < 1 || k < 1 || H < 1 || R < 1 || (size_t)T * k > (size_t)1 << 30 || R > 1 << 30) return MOE_ERR_SHAPE;
    return H % 8 ? MOE_ERR_ALIGN : MOE_OK;
}

unsigned groups_for(size_t items, int per_group)
{
    const size_t n = (items + per_group - 1) / per_group;
    return n < kMostGroups ? (unsigned)n : kMostGroups;
}

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" int moe_sort_workspace_bytes(int T, int k, int E, size_t *bytes_out)
{
    if (!bytes_out) return MOE_ERR_NULL;
    if (T < 1 || k < 1 || E < 1 || E > kMaxC || (size_t)T * k > (size_t)1 << 30) return MOE_ERR_SHAPE;
    *bytes_out = align256((size_t)(T * k <= kSortOne ? 1 : sort_blocks(T * k)) * E * 4);
    return MOE_OK;
}

extern "C" int moe_sort_assignments(const int32_t *ids, int T, int k, int E, int32_t *offsets, int32_t *order, int32_t *pos,
                                    void *workspace, size_t workspace_bytes, void *stream)
{
    if (!ids || !offsets || !order || !pos || !workspace) return MOE_ERR_NULL;
    size_t need = 0;
    int rc = moe_sort_workspace_bytes(T, k, E, &need);
    if (rc) return rc;
    if (!aligned16(workspace)) return MOE_ERR_ALIGN;
    if (workspace_bytes < need) return MOE_ERR_WORKSPACE;
    const int A = T * k, blocks = sort_blocks(A);
    int bits = 0;
    while (1 << bits < E) ++bits;
    constexpr int step = kSortThreads;   // (a chunk is whole 64s for each wavefront)
    const int chunk = ((A + blocks - 1) / blocks + step - 1) / step * step;
    SortArgs a = {ids, A, E, bits, chunk, blocks, offsets, order, pos, (int32_t *)workspace};
    const size_t lds = ((size_t)(kSortWaves + 2) * E + kSortWaves) * 4;
    const void *place = A <= kSortOne ? (const void *)sort_place_kernel<true> : (const void *)sort_place_kernel<false>;
    if (A > kSortOne) {
        rc = launch_rows((const void *)sort_count_kernel, blocks, kSortThreads, &a, (size_t)E * 4, stream, MOE_KERNEL_SORT);
        if (rc) return rc;
    }
    return launch_rows(place, blocks, kSortThreads, &a, lds, stream, MOE_KERNEL_SORT);
}

extern "C" int moe_permute(const void *x, int x_bf16, const int32_t *pos, int T, int k, int H, int R, void *out, void *stream)
{
    if (!x || !pos || !out) return MOE_ERR_NULL;
    int rc = check_rows(T, k, H, R);
    if (rc) return rc;
    if (!aligned16(x) || !aligned16(out)) return MOE_ERR_ALIGN;
    MoveArgs a = {(const u32x4 *)x, pos, (u32x4 *)out, k, R, x_bf16 ? H / 8 : H / 4, 0, 0, 0, 0};
    a.stream = (size_t)T * k * a.words * 16 > kStreamBytes;
    auto parts = [&](int U) { return (unsigned)((a.words + U * kWave - 1) / (U * kWave)); };
    const int U = (size_t)T * parts(4) >= 1024 ? 4 : 1;
    a.parts = parts(U);
    const size_t items = (size_t)T * a.parts;
    if (items >= (size_t)1 << 31) return MOE_ERR_SHAPE;
    a.rcp_parts = rcp32(a.parts);
    a.items = (unsigned)items;
    return launch_rows(U == 4 ? (const void *)permute_kernel<4> : (const void *)permute_kernel<1>, groups_for(items, kRowWaves),
                    kRowThreads, &a, 0, stream, MOE_KERNEL_PERMUTE);
}

extern "C" int moe_permute_fp8(const void *x, int x_bf16, const int32_t *pos, int T, int k, int H, int R, void *q, float *scale,
                               void *stream)
{
    if (!x || !pos || !q || !scale) return MOE_ERR_NULL;
    int rc = check_rows(T, k, H, R);
    if (rc) return rc;
    if (H > 1 << 24) return MOE_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(q)) return MOE_ERR_ALIGN;
    MoveFp8Args a = {x, pos, (u32x4 *)q, scale, k, R, H, 0, (unsigned)((H + kBlock - 1) / kBlock), 0, 0};
    a.stream = (size_t)T * k * a.blocks * kBlock > kStreamBytes;
    const size_t items = (size_t)T * a.blocks;
    if (items >= (size_t)1 << 31) return MOE_ERR_SHAPE;
    a.rcp_blocks = rcp32(a.blocks);
    a.items = (unsigned)items;
    return launch_rows(x_bf16 ? (const void *)permute_fp8_kernel<true> : (const void *)permute_fp8_kernel<false>,
                    groups_for(items, kRowThreads / 8), kRowThreads, &a, 0, stream, MOE_KERNEL_PERMUTE);
}

extern "C" int moe_unpermute(const void *rows, int rows_bf16, const int32_t *pos, const float *topk_w, int T, int k, int H, int R,
                             void *out, int out_bf16, int accumulate, void *stream)
{
    if (!rows || !pos || !out) return MOE_ERR_NULL;
    int rc = check_rows(T, k, H, R);
    if (rc) return rc;
    if (!aligned16(rows) || !aligned16(out)) return MOE_ERR_ALIGN;
    SumArgs a = {(const u32x4 *)rows, pos, topk_w, (u32x4 *)out, k, R, H, accumulate,
                 (size_t)T * H * (out_bf16 ? 2 : 4) > kStreamBytes, (unsigned)((H / 8 + kWave - 1) / kWave), 0, 0};
    const size_t items = (size_t)T * a.parts;
    if (items >= (size_t)1 << 31) return MOE_ERR_SHAPE;
    a.rcp_parts = rcp32(a.parts);
    a.items = (unsigned)items;
    const void *fn = rows_bf16 ? (out_bf16 ? (const void *)unpermute_kernel<true, true> : (const void *)unpermute_kernel<true, false>)
                               : (out_bf16 ? (const void *)unpermute_kernel<false, true> : (const void *)unpermute_kernel<false, false>);
    return launch_rows(fn, groups_for(items, kRowWaves), kRowThreads, &a, 0, stream, MOE_KERNEL_UNPERMUTE);
}

extern "C" int moe_unpermute_backward(const void *dout, int dout_bf16, const void *rows, int rows_bf16, const int32_t *pos,
                                      const float *topk_w, int T, int k, int H, int R, void *drows, float *dtopk_w, void *stream)
{
    if (!dout || !pos || (!drows && !dtopk_w) || (dtopk_w && !rows)) return MOE_ERR_NULL;
    int rc = check_rows(T, k, H, R);
    if (rc) return rc;
    if (!aligned16(dout) || !aligned16(rows) || !aligned16(drows)) return MOE_ERR_ALIGN;
    BackArgs a = {(const u32x4 *)dout, (const u32x4 *)rows, pos, topk_w, (u32x4 *)drows, dtopk_w, k, R, H,
                  (size_t)T * k * H * (rows_bf16 ? 2 : 4) > kStreamBytes, (unsigned)T * (unsigned)k,
                  rcp32((unsigned)k)};
    const void *fn = dout_bf16 ? (rows_bf16 ? (const void *)unpermute_backward_kernel<true, true> : (const void *)unpermute_backward_kernel<true, false>)
                               : (rows_bf16 ? (const void *)unpermute_backward_kernel<false, true> : (const void *)unpermute_backward_kernel<false, false>);
    return launch_rows(fn, groups_for(a.A, kRowWaves), kRowThreads, &a, 0, stream, MOE_KERNEL_UNPERMUTE);
}
