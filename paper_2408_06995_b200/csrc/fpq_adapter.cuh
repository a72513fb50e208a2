// What the adapter kernels share: values of three types as they lie in memory, which rows a tile has, and the arguments of a pass
// from rows to t and back.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "fpq_kernels.h"

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

}  // namespace fpq
