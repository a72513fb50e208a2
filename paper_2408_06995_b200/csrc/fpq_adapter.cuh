// What the adapter kernels share: values of three types as they lie in memory, which rows a tile has, and the arguments of a pass
// from rows to t and back.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "fpq_common.cuh"
#include "fpq_kernels.h"
#include "fpq_tensormap.h"

namespace fpq {

__device__ __forceinline__ float as_float(float v) { return v; }
__device__ __forceinline__ float as_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float as_float(__half v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ void unpack(uint32_t w, float* v, __nv_bfloat16)
{
    v[0] = __uint_as_float(w << 16);
    v[1] = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack(uint32_t w, float* v, __half)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    v[0] = f.x;
    v[1] = f.y;
}

// n values that lie side by side (n = 4 or 8), as they lie: 32-bit words of one FP32 or two 16-bit values.  They are
// looked into only where they are used: a conversion behind each load would wait for it.
template <typename T, int n>
struct Raw {
    static constexpr int WORDS = n * (int)sizeof(T) / 4;
    uint32_t w[WORDS];

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
            w[i] = 0;
    }
    __device__ __forceinline__ void values(float (&v)[n]) const
    {
#pragma unroll
        for (int i = 0; i < n; ++i)
            if constexpr (sizeof(T) == 4) {
                v[i] = __uint_as_float(w[i]);
            } else if (i % 2 == 0) {
                unpack(w[i / 2], v + i, T());
            }
    }
};

// Values [col, col + n) of a row of `width`; those behind its end are zeros.  VEC: the row starts at a multiple of 16 bytes
// (of 8, for four 16-bit values) and its width is a multiple of what a vector holds.
template <bool VEC, int n, typename T>
__device__ __forceinline__ void load_cols(const T* row, int64_t col, int64_t width, bool there, Raw<T, n>& r)
{
    if constexpr (VEC) {
        constexpr int PIECE = sizeof(T) == 4 ? 4 : n;
#pragma unroll
        for (int i = 0; i < n; i += PIECE) {
            uint32_t* w = r.w + i * (int)sizeof(T) / 4;
            if (there && col + i < width) {
                if constexpr (PIECE * sizeof(T) == 16) {
                    const uint4 q = *reinterpret_cast<const uint4*>(row + col + i);
                    w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
                } else {
                    const uint2 q = *reinterpret_cast<const uint2*>(row + col + i);
                    w[0] = q.x; w[1] = q.y;
                }
            } else {
#pragma unroll
                for (int k = 0; k < PIECE * (int)sizeof(T) / 4; ++k)
                    w[k] = 0;
            }
        }
    } else {
        r.clear();
        const T* p = row + col;
        if (sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(p) & 3) == 0) {
#pragma unroll
            for (int i = 0; i < n; i += 2)
                if (there && col + i + 1 < width)
                    r.w[i / 2] = *reinterpret_cast<const uint32_t*>(p + i);
                else if (there && col + i < width)
                    r.w[i / 2] = reinterpret_cast<const uint16_t*>(p)[i];
        } else {
#pragma unroll
            for (int i = 0; i < n; ++i)
                if (there && col + i < width) {
                    if constexpr (sizeof(T) == 4)
                        r.w[i] = __float_as_uint(p[i]);
                    else
                        r.w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(p)[i] << (16 * (i % 2));
                }
        }
    }
}

// two values as BF16, and what is left of them
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t& h, uint32_t& l)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    const float2 f = __bfloat1622float2(v);
    const __nv_bfloat162 r = __floats2bfloat162_rn(a - f.x, b - f.y);
    h = *reinterpret_cast<const uint32_t*>(&v);
    l = *reinterpret_cast<const uint32_t*>(&r);
}

template <typename T>
constexpr bool WIDE = sizeof(T) == 4;

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

// ---- which rows a tile has ---------------------------------------------------------------------------------------
// Segment s (rows offsets[s] .. offsets[s + 1]) owns the tiles from offsets[s] / BM + s on: as many as it needs, whatever
// its rows, and the grid of M / BM + S tiles is known without reading the offsets.  All lanes get the same answer.
struct TileRows {
    int64_t row;
    int rows, id;
};

__device__ __forceinline__ TileRows find_tile(int BM, int64_t tile, const int32_t* offsets, const int32_t* ids, int S, int G, int64_t M)
{
    const int lane = threadIdx.x & 31;
    TileRows r = {0, 0, -1};
    int lo = 0, span = S;                                  // the answer is in [lo, lo + span), if there is one
    while (true) {
        const int step = (span + 31) / 32, s = lo + lane * step;
        bool below = false;
        if (s < lo + span) {
            const int64_t o = min(max((int64_t)offsets[s], (int64_t)0), M);
            below = (uint32_t)o / (uint32_t)BM + (int64_t)s <= tile;
        }
        const uint32_t votes = __ballot_sync(0xffffffffu, below);
        if (votes == 0)
            return r;                                      // in front of the first segment
        const int last = 31 - __clz(votes);
        span = min(step, lo + span - (lo + last * step));
        lo += last * step;
        if (step == 1)
            break;
    }
    const int64_t begin = min(max((int64_t)offsets[lo], (int64_t)0), M), end = min(max((int64_t)offsets[lo + 1], (int64_t)0), M);
    r.row = begin + (tile - ((uint32_t)begin / (uint32_t)BM + (int64_t)lo)) * BM;
    r.rows = (int)max(min((int64_t)BM, end - r.row), (int64_t)0);
    const int id = ids[lo];
    r.id = id >= 0 && id < G ? id : -1;
    return r;
}

struct RowsArgs {
    const void* in;                // [M][D1], leading dimension ld_in
    const void* w1;                // reduces:   [G][R][D1]
    const void* w2;                // expands:   [G][D2][R]
    const float* scale;            // [G] or NULL
    const int32_t *offsets, *ids;
    const void* base;              // [M][D2] or NULL
    void* out;                     // [M][D2] or NULL
    float* kept;                   // [M][R] or NULL: t (forward), s t (backward)
    int64_t M, D1, D2, ld_in, ld_base, ld_out;
    int G, R, S;
    int kept_scaled;
    int wr;                        // row groups of a block: 1, 2, 4 or 8
    int64_t ld_w1, ld_w2;          // rows of the weights: adapter g's start g R ld_w1 and g D2 ld_w2 elements behind the first
    int in_by, base_by, out_by;    // bytes at a time that the rows allow: 16, 4 or 2
    int vec_w1, vec_w2;            // the weights' rows allow vectors
};

// The pass on tcgen05 MMAs for requests of many rows (fpq_adapter_tile.cu): whether it applies and is expected to be faster than
// the one by warps, and its launch.
bool adapter_tiles_preferred(const RowsArgs& a, int x_type, int w_type);
fpq_status launch_adapter_tiles(const RowsArgs& a, int x_type, int w_type, cudaStream_t st);

// ---- gradients ---------------------------------------------------------------------------------------------------
struct GradArgs {
    const void *x, *dy;
    const float *t, *u;            // [M][R]
    const float* scale;
    const int32_t *offsets, *ids;
    float *da, *db;                // [G][R][K], [G][N][R]
    int64_t M, N, K, ldx, ld_dy;
    int G, R, S, x_by, dy_by;
    int tiles_k, tiles;            // column tiles of dA; those behind them are dB's
    float* sums;                   // [split][G][tiles][64 RP] where the rows are split
    uint32_t* tickets;             // [G][tiles]: how many of the blocks that share a sum have ended
    int splits;
};

// whether any row is adapter `id`'s
__device__ __forceinline__ bool has_rows(const GradArgs& a, int id)
{
#pragma unroll 1
    for (int sg = 0; sg < a.S; ++sg)
        if (a.ids[sg] == id && min(max(a.offsets[sg + 1], 0), (int)a.M) > min(max(a.offsets[sg], 0), (int)a.M))
            return true;
    return false;
}

template <typename XT>
__device__ __forceinline__ void store_gradient(const GradArgs& a, int id, bool is_b, int64_t col, int j, float v)
{
    if (!finite(v)) {
        const XT* wide = (const XT*)(is_b ? a.dy : a.x) + col;
        const float* thin = (is_b ? a.u : a.t) + j;
        const int64_t ld = is_b ? a.ld_dy : a.ldx;
        v = 0.f;
        for (int sg = 0; sg < a.S; ++sg) {
            if (a.ids[sg] != id)
                continue;
            const int64_t begin = min(max((int64_t)a.offsets[sg], (int64_t)0), a.M), end = min(max((int64_t)a.offsets[sg + 1], (int64_t)0), a.M);
            for (int64_t r = begin; r < end && v == v; ++r)    // (a NaN stays one)
                v = fmaf(as_float(wide[r * ld]), thin[r * a.R], v);
        }
    }
    if (is_b) {
        float scaled = a.scale ? v * a.scale[id] : v;
        if (!finite(scaled) && v == 0.f && !has_rows(a, id))
            scaled = 0.f;                                  // (nothing was added up; a zero sum of some rows times infinity is NaN)
        a.db[((int64_t)id * a.N + col) * a.R + j] = scaled;
    } else
        a.da[((int64_t)id * a.R + j) * a.K + col] = v;
}

// Over how many of the a.splits blocks adapter `id`'s rows are spread: its share of all rows, so that adapters of unequal length end together.
// Called by whole warps.
__device__ __forceinline__ int splits_of(const GradArgs& a, int id)
{
    if (a.splits == 1 || a.G == 1)
        return a.splits;
    int64_t mine = 0, all = 0;
    for (int sg = threadIdx.x & 31; sg < a.S; sg += 32) {
        const int other = a.ids[sg], n = min(max(a.offsets[sg + 1], 0), (int)a.M) - min(max(a.offsets[sg], 0), (int)a.M);
        if (n > 0 && other >= 0 && other < a.G) {
            all += n;
            mine += other == id ? n : 0;
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        all += __shfl_xor_sync(0xffffffffu, all, o);
        mine += __shfl_xor_sync(0xffffffffu, mine, o);
    }
    return all == 0 ? 1 : max((int)((mine * a.splits + all - 1) / all), 1);
}

// Which adapter's rows a block takes, and which of its `splits` shares (negative: none).  Up to 32 adapters: the shares of all of them lie
// side by side in the grid's y, splits + G - 1 at most (a block for every adapter and share, most of which have nothing to do, kept
// the SMs' places: 82 us instead of 72 for a whole backward pass of three adapters).  More: y is the adapter, z its share.
// Called by whole warps.
struct GradShare {
    int id, z, splits;
};
inline dim3 grad_grid(const GradArgs& a) { return a.G <= 32 ? dim3(a.tiles, a.splits + a.G - 1) : dim3(a.tiles, a.G, a.splits); }

__device__ __forceinline__ GradShare share_of(const GradArgs& a)
{
    const int at = blockIdx.y;
    if (a.G == 1)
        return {0, at, a.splits};
    if (a.splits == 1 || a.G > 32) {
        const int splits = splits_of(a, at);
        return {at, (int)blockIdx.z < splits ? (int)blockIdx.z : -1, splits};
    }
    const int lane = threadIdx.x & 31;                     // an adapter for every lane
    int64_t mine = 0;
    for (int s0 = 0; s0 < a.S; s0 += 32) {
        const int sg = s0 + lane;
        int id = -1, n = 0;
        if (sg < a.S) {
            id = a.ids[sg];
            n = max(min(max(a.offsets[sg + 1], 0), (int)a.M) - min(max(a.offsets[sg], 0), (int)a.M), 0);
        }
        for (int k = 0; k < min(a.S - s0, 32); ++k) {
            const int other = __shfl_sync(0xffffffffu, id, k), rows = __shfl_sync(0xffffffffu, n, k);
            mine += other == lane ? rows : 0;
        }
    }
    int64_t all = lane < a.G ? mine : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        all += __shfl_xor_sync(0xffffffffu, all, o);
    const int splits = lane >= a.G ? 0 : all == 0 ? 1 : max((int)((mine * a.splits + all - 1) / all), 1);      // as splits_of
    int behind = splits;                                   // the shares up to and with this lane's
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, behind, o);
        behind += lane >= o ? v : 0;
    }
    const uint32_t votes = __ballot_sync(0xffffffffu, behind > at);
    if (votes == 0)
        return {0, -1, 1};
    const int id = __ffs(votes) - 1, its = __shfl_sync(0xffffffffu, splits, id);
    return {id, at - (__shfl_sync(0xffffffffu, behind, id) - its), its};
}

// The gradients by tcgen05 MMAs, for BF16 rows (fpq_adapter_grad_tile.cu): whether it applies and is expected to be faster, over how many
// blocks the rows are split, how many columns of sums that takes (0: none), and the launch (a.splits is set).
bool adapter_grad_tiles_preferred(const GradArgs& a);
int adapter_grad_tile_splits(int64_t M, int64_t N, int64_t K, int G, int R);
size_t adapter_grad_tile_columns(int64_t M, int64_t N, int64_t K, int G, int R);
cudaError_t launch_adapter_grad_tiles(GradArgs a, cudaStream_t st);

// what TMA reads or writes: rows at multiples of 16 bytes
inline bool mapped(const void* p, int64_t ld, int bytes) { return (uintptr_t)p % 16 == 0 && ld * bytes % 16 == 0 && ld * bytes < ((int64_t)1 << 40); }
// rows x cols of a type (FPQ_FP32, ...), rows ld elements apart: boxes of box_rows x box_cols, zeros outside; 128-byte swizzle for boxes
// of 128 bytes
bool encode_rows(EncodeTiledFn enc, CUtensorMap* tm, const void* base, int64_t rows, int64_t cols, int64_t ld, int type, int box_rows, int box_cols,
                 bool swizzle);

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const void* tmap, uint32_t bar, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(tmap), "r"(bar), "r"(c0), "r"(c1)
                 : "memory");
}

// N consecutive FP32 columns of this thread's lane of tensor memory (not waited for)
template <int N>
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t* r)
{
    if constexpr (N == 32) {
        tmem_ld32(addr, r);
    } else if constexpr (N == 16) {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                       "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                     : "r"(addr)
                     : "memory");
    } else if constexpr (N == 4) {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(addr)
                     : "memory");
    } else {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                     : "r"(addr)
                     : "memory");
    }
}

// 16-byte piece c of row r of an operand tile: rows of 128 bytes, 128-byte swizzle
__device__ __forceinline__ int swizzled(int r, int c) { return r * 128 + ((c ^ (r & 7)) << 4); }

}  // namespace fpq
