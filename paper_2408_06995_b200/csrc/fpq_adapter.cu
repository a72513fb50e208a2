// Low-rank adapters of many requests at once, beside a shared projection: forward and backward.
//
//   forward   t_i = A x_i,      y_i  = base_i + B (s t_i)
//   backward  t_i = s B^T dy_i, dx_i = base_i + A^T t_i,   dA = sum_i t_i x_i^T,   dB = s sum_i dy_i u_i^T   (u_i = A x_i)
//
// A, B and s are those of the adapter that row i's request uses.  With a rank of 16 a row costs 2 R (K + N) operations on
// (K + 2 N) values: bound by memory, so every kernel reads its rows once.  Forward and the first half of backward are one
// kernel with the roles of the matrices exchanged: a block (or a cluster of up to 8, sharing the reduction and the output
// columns) takes a tile of rows of one request, reduces it to t in shared memory and multiplies it out again.
//
// Products run on the tensor cores as TF32 with FP32 operands split in two: x = hi + lo with 11 significant bits each, the
// products hi hi, hi lo and lo hi (16-bit operands are TF32 numbers themselves, one term).  What is left out is 2^-22 of a
// product.  The tensor cores cut their sums off instead of rounding them: at most 64 columns are summed there, the rest in
// registers by FP32 additions.  Operands go from global memory straight into the registers of the MMA: the order of the
// reduction is free, so a thread's share of a row is 8 values that lie side by side.
//
// An infinity, or a number that rounds up to one, has no split: a result that is not finite is worked out again by FP32
// multiply-adds.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>

#include "fpq_kernels.h"

namespace fpq {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;

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

// 8 (or 4) values side by side, 16-byte (8-byte for 4 16-bit values) aligned
__device__ __forceinline__ void load_vec(const float* p, float* v, int n)
{
#pragma unroll
    for (int i = 0; i < n; i += 4) {
        const float4 q = *reinterpret_cast<const float4*>(p + i);
        v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
    }
}
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
template <typename T>
__device__ __forceinline__ void load_vec(const T* p, float* v, int n)
{
    if (n == 8) {
        const uint4 q = *reinterpret_cast<const uint4*>(p);
        unpack(q.x, v, T()); unpack(q.y, v + 2, T()); unpack(q.z, v + 4, T()); unpack(q.w, v + 6, T());
    } else {
        const uint2 q = *reinterpret_cast<const uint2*>(p);
        unpack(q.x, v, T()); unpack(q.y, v + 2, T());
    }
}

// Values [col, col + n) of a row of `width`; those behind its end are zeros.
template <int n, typename T>
__device__ __forceinline__ void load_cols(const T* row, int64_t col, int64_t width, bool vec, float* v)
{
    if (vec && col + n <= width) {
        load_vec(row + col, v, n);
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i)
            v[i] = col + i < width ? as_float(row[col + i]) : 0.f;
    }
}

__device__ __forceinline__ uint32_t high(float x) { return (__float_as_uint(x) + 0x1000u) & 0xffffe000u; }
__device__ __forceinline__ uint32_t low(float x, uint32_t hi) { return __float_as_uint(x - __uint_as_float(hi)); }

__device__ __forceinline__ void mma_tf32(float* c, const uint32_t* a, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// c += a b with FP32 operands in two terms each (SPLIT_A / SPLIT_B: the operand has more bits than TF32)
template <bool SPLIT_A, bool SPLIT_B>
__device__ __forceinline__ void mma_split(float* c, const uint32_t* ah, const uint32_t* al, float b0, float b1)
{
    const uint32_t h0 = SPLIT_B ? high(b0) : __float_as_uint(b0), h1 = SPLIT_B ? high(b1) : __float_as_uint(b1);
    if (SPLIT_B)
        mma_tf32(c, ah, low(b0, h0), low(b1, h1));
    if (SPLIT_A)
        mma_tf32(c, al, h0, h1);
    mma_tf32(c, ah, h0, h1);
}

template <bool SPLIT>
__device__ __forceinline__ void split_four(const float (&v)[4], uint32_t (&h)[4], uint32_t (&l)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[i] = SPLIT ? high(v[i]) : __float_as_uint(v[i]);
        if (SPLIT)
            l[i] = low(v[i], h[i]);
    }
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

template <int BM>
__device__ __forceinline__ TileRows find_tile(int64_t tile, const int32_t* offsets, const int32_t* ids, int S, int G, int64_t M)
{
    const int lane = threadIdx.x & 31;
    TileRows r = {0, 0, -1};
    int lo = 0, span = S;                                  // the answer is in [lo, lo + span), if there is one
    while (true) {
        const int step = (span + 31) / 32, s = lo + lane * step;
        bool below = false;
        if (s < lo + span) {
            const int64_t o = min(max((int64_t)offsets[s], (int64_t)0), M);
            below = o / BM + s <= tile;
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
    r.row = begin + (tile - (begin / BM + lo)) * BM;
    r.rows = (int)min((int64_t)BM, end - r.row);
    const int id = ids[lo];
    r.id = id >= 0 && id < G ? id : -1;
    return r;
}

// ---- rows to t and back ------------------------------------------------------------------------------------------
struct RowsArgs {
    const void* in;                // [M][D1], leading dimension ld_in
    const void* w1;                // reduces:   [G][R][D1], or transposed [G][D1][R]
    const void* w2;                // expands:   [G][D2][R], or transposed [G][R][D2]
    const float* scale;            // [G] or NULL
    const int32_t *offsets, *ids;
    const void* base;              // [M][D2] or NULL
    void* out;                     // [M][D2] or NULL
    float* kept;                   // [M][R] or NULL: t (forward), s t (backward)
    int64_t M, D1, D2, ld_in, ld_base, ld_out;
    int G, R, S;
    int vec_in, vec_out, vec_w1, vec_w2;
    int kept_scaled;
};

// The thread's four values per (n-tile, k-pair) of a weight matrix W(n, k): n = row of the MMA's B operand.  Contiguous in k
// (row pitch ld), or TR: contiguous in n.
template <bool TR, typename WT>
__device__ __forceinline__ void load_weights(const WT* w, int64_t n, int64_t N, int64_t k, int64_t K, int64_t ld, bool vec, float (&v)[8])
{
    if (!TR) {
        if (n < N)
            load_cols<8>(w + n * ld, k, K, vec, v);
        else
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[i] = 0.f;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = n < N && k + i < K ? as_float(w[(k + i) * ld + n]) : 0.f;
    }
}

// MT: row tiles of 16 in a block; RP: the rank, padded.  The warps (of all blocks of the cluster) share the reduction in
// groups of 32 columns, then the output in groups of 32 columns.
template <typename XT, typename WT, int MT, int RP, bool TR>
__global__ void __launch_bounds__(THREADS) adapter_rows_kernel(const RowsArgs a)
{
    constexpr int BM = MT * 16, NT = RP / 8, PITCH = RP == 16 ? 16 : RP + 16;
    extern __shared__ float4 smem4[];
    float* parts = reinterpret_cast<float*>(smem4);        // [WARPS][BM][RP], then the block's sum in the first
    float* t_smem = parts + WARPS * BM * RP;               // [BM][PITCH]
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    uint32_t rank = cluster_rank(), C;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
    const int64_t tile = blockIdx.x / C;
    const TileRows tr = find_tile<BM>(tile, a.offsets, a.ids, a.S, a.G, a.M);
    if (tr.rows <= 0)
        return;                                            // (every block of the cluster leaves)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const float s = a.scale && tr.id >= 0 ? a.scale[tr.id] : 1.f;
    const int64_t D1 = a.D1, D2 = a.D2;
    const int R = a.R, workers = WARPS * (int)C, worker = (int)rank * WARPS + warp;
    const XT* in = (const XT*)a.in + tr.row * a.ld_in;
    const WT* w1 = (const WT*)a.w1 + (int64_t)max(tr.id, 0) * R * D1;
    const WT* w2 = (const WT*)a.w2 + (int64_t)max(tr.id, 0) * R * D2;

    if (tr.id >= 0) {
        float acc[MT][NT][4] = {}, part[MT][NT][4] = {};
        int since = 0;
        for (int64_t k0 = (int64_t)worker * 32; k0 < D1; k0 += (int64_t)workers * 32) {
            const int64_t k = k0 + q * 8;
            float x[MT][2][8];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = m * 16 + h * 8 + g;
                    if (r < tr.rows)
                        load_cols<8>(in + r * a.ld_in, k, D1, a.vec_in, x[m][h]);
                    else
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            x[m][h][i] = 0.f;
                }
            float w[NT][8];
#pragma unroll
            for (int n = 0; n < NT; ++n)
                load_weights<TR>(w1, n * 8 + g, R, k, D1, TR ? R : D1, a.vec_w1, w[n]);
#pragma unroll
            for (int st = 0; st < 4; ++st)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const float v[4] = {x[m][0][2 * st], x[m][1][2 * st], x[m][0][2 * st + 1], x[m][1][2 * st + 1]};
                    uint32_t vh[4], vl[4];
                    split_four<WIDE<XT>>(v, vh, vl);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        mma_split<WIDE<XT>, WIDE<WT>>(part[m][n], vh, vl, w[n][2 * st], w[n][2 * st + 1]);
                }
            if (++since == 2) {                            // 64 columns
                since = 0;
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            acc[m][n][i] += part[m][n][i];
                            part[m][n][i] = 0.f;
                        }
            }
        }
        float* mine = parts + warp * BM * RP;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                *reinterpret_cast<float2*>(mine + (m * 16 + g) * RP + n * 8 + 2 * q) =
                    make_float2(acc[m][n][0] + part[m][n][0], acc[m][n][1] + part[m][n][1]);
                *reinterpret_cast<float2*>(mine + (m * 16 + 8 + g) * RP + n * 8 + 2 * q) =
                    make_float2(acc[m][n][2] + part[m][n][2], acc[m][n][3] + part[m][n][3]);
            }
        __syncthreads();
        if (C > 1) {                                       // the block's own sum first: one array per block to fetch
            for (int i = threadIdx.x; i < BM * RP; i += THREADS) {
                float v = parts[i];
#pragma unroll
                for (int k = 1; k < WARPS; ++k)
                    v += parts[k * BM * RP + i];
                parts[i] = v;
            }
            cluster_sync_all();
        }
        for (int i = threadIdx.x; i < BM * RP; i += THREADS) {
            const int r = i / RP, j = i % RP;
            float v = 0.f;
            if (C > 1) {
                for (uint32_t c = 0; c < C; ++c) {
                    float p;
                    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(p) : "r"(peer_smem_addr(smem_u32(parts + i), c)));
                    v += p;
                }
            } else {
#pragma unroll
                for (int k = 0; k < WARPS; ++k)
                    v += parts[k * BM * RP + i];
            }
            if (!finite(v) && r < tr.rows && j < R) {
                v = 0.f;
                for (int64_t k = 0; k < D1; ++k)
                    v = fmaf(as_float(in[r * a.ld_in + k]), as_float(TR ? w1[k * R + j] : w1[j * D1 + k]), v);
            }
            if (a.kept && rank == 0 && r < tr.rows && j < R)
                a.kept[(tr.row + r) * R + j] = a.kept_scaled ? v * s : v;
            t_smem[r * PITCH + j] = j < R ? v * s : 0.f;   // (an infinite x times a padded rank's zeros is NaN)
        }
        __syncthreads();
        if (C > 1)
            cluster_arrive();                              // this block has fetched what it needs of the others
    } else if (a.kept && rank == 0) {
        for (int i = threadIdx.x; i < tr.rows * R; i += THREADS)
            a.kept[tr.row * R + i] = 0.f;
    }

    if (a.out) {
        const XT* base = (const XT*)a.base + tr.row * a.ld_base;
        XT* out = (XT*)a.out + tr.row * a.ld_out;
        for (int64_t c0 = (int64_t)worker * 32; c0 < D2; c0 += (int64_t)workers * 32) {
            const int64_t col = c0 + q * 8;                // this thread's 8 columns of rows g and g + 8 of every tile
            float y[MT][2][8];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = m * 16 + h * 8 + g;
                    if (a.base && r < tr.rows)
                        load_cols<8>(base + r * a.ld_base, col, D2, a.vec_out, y[m][h]);
                    else
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            y[m][h][i] = 0.f;
                }
            if (tr.id >= 0) {
                float acc[MT][4][4] = {};
                // output column of the MMA's column g in tile e: the two columns 2 q and 2 q + 1 that a thread gets of each
                // of the four tiles are its 8 columns
                const int64_t n = c0 + 8 * (g >> 1) + (g & 1);
                constexpr int KG = RP < 32 ? RP : 32;      // ranks at a time
#pragma unroll
                for (int k0 = 0; k0 < RP; k0 += KG) {
                    constexpr int PER = KG / 4;            // ranks of a thread: 4 or 8 side by side
                    float w[4][8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t row = n + 2 * e;
                        const int k = k0 + q * PER;
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            w[e][i] = 0.f;
                        if (row < D2) {
                            if (!TR)
                                load_cols<PER>(w2 + row * R, k, R, a.vec_w2, w[e]);
                            else
#pragma unroll
                                for (int i = 0; i < PER; ++i)
                                    w[e][i] = k + i < R ? as_float(w2[(int64_t)(k + i) * D2 + row]) : 0.f;
                        }
                    }
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        float t[2][PER];
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            load_vec(t_smem + (m * 16 + h * 8 + g) * PITCH + k0 + q * PER, t[h], PER);
#pragma unroll
                        for (int st = 0; st < PER / 2; ++st) {
                            const float v[4] = {t[0][2 * st], t[1][2 * st], t[0][2 * st + 1], t[1][2 * st + 1]};
                            uint32_t vh[4], vl[4];
                            split_four<true>(v, vh, vl);
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                mma_split<true, WIDE<WT>>(acc[m][e], vh, vl, w[e][2 * st], w[e][2 * st + 1]);
                        }
                    }
                }
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float v = acc[m][i >> 1][2 * h + (i & 1)];
                            const int r = m * 16 + h * 8 + g;
                            if (!finite(v) && r < tr.rows && col + i < D2) {
                                v = 0.f;
                                for (int j = 0; j < R; ++j)
                                    v = fmaf(t_smem[r * PITCH + j], as_float(TR ? w2[j * D2 + col + i] : w2[(col + i) * R + j]), v);
                            }
                            y[m][h][i] += v;
                        }
            }
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = m * 16 + h * 8 + g;
                    if (r >= tr.rows)
                        continue;
                    XT* o = out + r * a.ld_out + col;
                    if (a.vec_out && col + 8 <= D2) {
                        alignas(16) XT v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            v[i] = from_float<XT>(y[m][h][i]);
#pragma unroll
                        for (int i = 0; i < (int)(8 * sizeof(XT) / 16); ++i)
                            reinterpret_cast<uint4*>(o)[i] = reinterpret_cast<const uint4*>(v)[i];
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (col + i < D2)
                                o[i] = from_float<XT>(y[m][h][i]);
                    }
                }
        }
    }
    __syncwarp();
    if (C > 1 && tr.id >= 0)
        cluster_wait();                                    // nobody still reads this block's sums
}

// ---- gradients of the adapters -----------------------------------------------------------------------------------
// out(col, j) = sum over an adapter's rows of wide[i][col] * thin[i][j]: columns of x with t (dA) and of dy with u (dB).  A
// block takes 64 columns; its warps, and the blocks of its cluster, share the rows in runs of 16 and add up in a fixed order.
struct GradArgs {
    const void *x, *dy;
    const float *t, *u;            // [M][R]
    const float* scale;
    const int32_t *offsets, *ids;
    float *da, *db;                // [G][R][K], [G][N][R]
    int64_t M, N, K, ldx, ld_dy;
    int G, R, S, vec_x, vec_dy;
    int tiles_k;                   // column tiles of dA; those behind them are dB's
};

// JT: ranks of a warp; RP / JT warps share a run of rows.
template <typename XT, int RP, int JT>
__global__ void __launch_bounds__(THREADS) adapter_grad_kernel(const GradArgs a)
{
    constexpr int NT = JT / 8, WN = RP / JT, WK = WARPS / WN, RUN = 16;
    extern __shared__ float4 smem4[];
    float* parts = reinterpret_cast<float*>(smem4);        // [WK][64][RP]
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    uint32_t rank = cluster_rank(), C;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
    const int tile = blockIdx.x / C, id = blockIdx.y;
    const bool is_b = tile >= a.tiles_k;
    const int64_t D = is_b ? a.N : a.K, ld = is_b ? a.ld_dy : a.ldx, c0 = (int64_t)(is_b ? tile - a.tiles_k : tile) * 64;
    const XT* wide = (const XT*)(is_b ? a.dy : a.x);
    const float* thin = is_b ? a.u : a.t;
    const bool vec = is_b ? a.vec_dy : a.vec_x;
    const int R = a.R, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int wn = warp % WN, wk = warp / WN, workers = WK * (int)C, worker = (int)rank * WK + wk, j0 = wn * JT;

    float acc[4][NT][4] = {}, part[4][NT][4] = {};
    int since = 0, runs = 0;                               // runs of the segments in front, modulo the workers
    for (int sg = 0; sg < a.S; ++sg) {
        if (a.ids[sg] != id)
            continue;
        const int64_t begin = min(max((int64_t)a.offsets[sg], (int64_t)0), a.M), end = min(max((int64_t)a.offsets[sg + 1], (int64_t)0), a.M);
        if (end <= begin)
            continue;
        const int64_t n_runs = (end - begin + RUN - 1) / RUN;
        for (int64_t i = (worker - runs + workers) % workers; i < n_runs; i += workers) {
#pragma unroll
            for (int st = 0; st < RUN / 8; ++st) {
                // rows of MMA k = q and q + 4; columns 4 g .. of both halves of the tile
                const int64_t r0 = begin + i * RUN + st * 8 + q;
                float v[2][2][4], p[NT][2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int64_t r = r0 + 4 * h;
#pragma unroll
                    for (int e = 0; e < 2; ++e)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            v[h][e][k] = 0.f;
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        p[n][h] = 0.f;
                    if (r < end) {
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            load_cols<4>(wide + r * ld, c0 + e * 32 + g * 4, D, vec, v[h][e]);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            if (j0 + n * 8 + g < R)
                                p[n][h] = thin[r * R + j0 + n * 8 + g];
                    }
                }
#pragma unroll
                for (int m = 0; m < 4; ++m) {              // MMA rows g and g + 8 are columns 4 g + m and 32 + 4 g + m
                    const float w[4] = {v[0][0][m], v[0][1][m], v[1][0][m], v[1][1][m]};
                    uint32_t wh[4], wl[4];
                    split_four<WIDE<XT>>(w, wh, wl);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        mma_split<WIDE<XT>, true>(part[m][n], wh, wl, p[n][0], p[n][1]);
                }
            }
            if (++since == 4) {                            // 64 rows
                since = 0;
#pragma unroll
                for (int m = 0; m < 4; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            acc[m][n][k] += part[m][n][k];
                            part[m][n][k] = 0.f;
                        }
            }
        }
        runs = (int)((runs + n_runs) % workers);
    }
    // parts[wk][column][rank]
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<float2*>(parts + (wk * 64 + h * 32 + g * 4 + m) * RP + j0 + n * 8 + 2 * q) =
                    make_float2(acc[m][n][2 * h] + part[m][n][2 * h], acc[m][n][2 * h + 1] + part[m][n][2 * h + 1]);
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * RP; i += THREADS) {
        float v = parts[i];
#pragma unroll
        for (int k = 1; k < WK; ++k)
            v += parts[k * 64 * RP + i];
        parts[i] = v;
    }
    if (C > 1)
        cluster_sync_all();
    else
        __syncthreads();
    const float s = a.scale && is_b ? a.scale[id] : 1.f;
    // every block of the cluster finishes a share; threads along the output's contiguous side
    for (int i = (int)rank * THREADS + threadIdx.x; i < 64 * RP; i += THREADS * (int)C) {
        const int col = is_b ? i / RP : i % 64, j = is_b ? i % RP : i / 64;
        if (c0 + col >= D || j >= R)
            continue;
        float v = 0.f;
        if (C > 1) {
            for (uint32_t c = 0; c < C; ++c) {
                float p;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(p) : "r"(peer_smem_addr(smem_u32(parts + col * RP + j), c)));
                v += p;
            }
        } else {
            v = parts[col * RP + j];
        }
        if (!finite(v)) {
            v = 0.f;
            for (int sg = 0; sg < a.S; ++sg) {
                if (a.ids[sg] != id)
                    continue;
                const int64_t begin = min(max((int64_t)a.offsets[sg], (int64_t)0), a.M), end = min(max((int64_t)a.offsets[sg + 1], (int64_t)0), a.M);
                for (int64_t r = begin; r < end; ++r)
                    v = fmaf(as_float(wide[r * ld + c0 + col]), thin[r * R + j], v);
            }
        }
        if (is_b)
            a.db[((int64_t)id * a.N + c0 + col) * R + j] = v * s;
        else
            a.da[((int64_t)id * R + j) * a.K + c0 + col] = v;
    }
    if (C > 1)
        cluster_sync_all();
}

// ---- launches ----------------------------------------------------------------------------------------------------
template <typename Args>
cudaError_t launch_cluster(void (*kernel)(const Args), std::atomic<uint64_t>& known, dim3 grid, int cluster, size_t smem, cudaStream_t st,
                           const Args& args)
{
    // shared memory beyond 48 KB is asked for once per kernel and device
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess)
        return e;
    if (smem > 48 * 1024 && (dev >= 64 || !(known.load(std::memory_order_relaxed) >> dev & 1))) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess)
            return e;
        if (dev < 64)
            known.fetch_or((uint64_t)1 << dev);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, args);
}

bool vectors(const void* p, int64_t ld, int bytes) { return (uintptr_t)p % 16 == 0 && ld * bytes % 16 == 0; }

int type_bytes(int t) { return t == FPQ_FP32 ? 4 : 2; }

template <typename XT, typename WT, int MT, int RP, bool TR>
cudaError_t launch_rows_as(const RowsArgs& a, cudaStream_t st)
{
    constexpr int BM = MT * 16, PITCH = RP == 16 ? 16 : RP + 16;
    const size_t smem = (size_t)(WARPS * BM * RP + BM * PITCH) * 4;
    const int64_t tiles = a.M / BM + a.S;
    // clusters until there are two blocks for every SM, while every block has a group of columns for most of its warps
    int c = 1;
    const int64_t groups = (std::max(a.D1, a.out ? a.D2 : 0) + 31) / 32;
    const int64_t busy = (a.M + BM - 1) / BM + std::min<int64_t>(a.S, a.M) - 1;
    while (c < 8 && busy * c * 2 <= 2 * 148 && groups > (int64_t)c * WARPS)
        c *= 2;
    static std::atomic<uint64_t> known{0};
    return launch_cluster<RowsArgs>(adapter_rows_kernel<XT, WT, MT, RP, TR>, known, dim3((unsigned)(tiles * c)), c, smem, st, a);
}

template <typename XT, typename WT, bool TR>
cudaError_t launch_rows_rank(const RowsArgs& a, cudaStream_t st)
{
    // row tiles: 32 rows where requests are long enough to fill them
    const bool tall = a.M >= 24 * (int64_t)a.S;
    if (a.R <= 16)
        return tall ? launch_rows_as<XT, WT, 2, 16, TR>(a, st) : launch_rows_as<XT, WT, 1, 16, TR>(a, st);
    if (a.R <= 32)
        return tall ? launch_rows_as<XT, WT, 2, 32, TR>(a, st) : launch_rows_as<XT, WT, 1, 32, TR>(a, st);
    if (a.R <= 64)
        return launch_rows_as<XT, WT, 1, 64, TR>(a, st);
    return launch_rows_as<XT, WT, 1, 128, TR>(a, st);
}

template <bool TR>
cudaError_t launch_rows(const RowsArgs& a, int x_type, int w_type, cudaStream_t st)
{
    if (x_type == FPQ_BF16)
        return launch_rows_rank<__nv_bfloat16, __nv_bfloat16, TR>(a, st);
    if (x_type == FPQ_FP16)
        return launch_rows_rank<__half, __half, TR>(a, st);
    return w_type == FPQ_FP32   ? launch_rows_rank<float, float, TR>(a, st)
           : w_type == FPQ_BF16 ? launch_rows_rank<float, __nv_bfloat16, TR>(a, st)
                                : launch_rows_rank<float, __half, TR>(a, st);
}

template <typename XT, int RP, int JT>
cudaError_t launch_grad_as(const GradArgs& a, int tiles, cudaStream_t st)
{
    const size_t smem = (size_t)(WARPS / (RP / JT)) * 64 * RP * 4;
    int c = 1;
    while (c < 8 && (int64_t)tiles * a.G * c * 2 <= 3 * 148 && a.M > (int64_t)c * 128)
        c *= 2;
    static std::atomic<uint64_t> known{0};
    return launch_cluster<GradArgs>(adapter_grad_kernel<XT, RP, JT>, known, dim3((unsigned)(tiles * c), (unsigned)a.G), c, smem, st, a);
}

template <typename XT>
cudaError_t launch_grad(const GradArgs& a, int tiles, cudaStream_t st)
{
    return a.R <= 16   ? launch_grad_as<XT, 16, 16>(a, tiles, st)
           : a.R <= 32 ? launch_grad_as<XT, 32, 32>(a, tiles, st)
           : a.R <= 64 ? launch_grad_as<XT, 64, 32>(a, tiles, st)
                       : launch_grad_as<XT, 128, 32>(a, tiles, st);
}

}  // namespace

cudaError_t launch_adapter_forward(const AdapterProblem& p, const void* x, int64_t ldx, const void* base, int64_t ld_base, void* y,
                                   int64_t ldy, float* u, cudaStream_t st)
{
    const int xb = type_bytes(p.x_type), wb = type_bytes(p.w_type);
    RowsArgs a = {};
    a.in = x; a.w1 = p.a; a.w2 = p.b; a.scale = p.scale; a.offsets = p.offsets; a.ids = p.ids;
    a.base = base; a.out = y; a.kept = u;
    a.M = p.M; a.D1 = p.K; a.D2 = p.N; a.ld_in = ldx; a.ld_base = ld_base; a.ld_out = ldy;
    a.G = p.G; a.R = p.R; a.S = p.S;
    a.vec_in = vectors(x, ldx, xb);
    a.vec_out = vectors(y, ldy, xb) && (!base || vectors(base, ld_base, xb));
    a.vec_w1 = vectors(p.a, p.K, wb);
    a.vec_w2 = vectors(p.b, p.R, wb);
    return launch_rows<false>(a, p.x_type, p.w_type, st);
}

cudaError_t launch_adapter_backward(const AdapterProblem& p, const void* dy, int64_t ld_dy, const void* x, int64_t ldx, const float* u,
                                    const void* base, int64_t ld_base, void* dx, int64_t ld_dx, float* da, float* db, float* t,
                                    cudaStream_t st)
{
    const int xb = type_bytes(p.x_type);
    if (p.M > 0 && p.S > 0) {
        RowsArgs a = {};
        a.in = dy; a.w1 = p.b; a.w2 = p.a; a.scale = p.scale; a.offsets = p.offsets; a.ids = p.ids;
        a.base = base; a.out = dx; a.kept = t; a.kept_scaled = 1;
        a.M = p.M; a.D1 = p.N; a.D2 = p.K; a.ld_in = ld_dy; a.ld_base = ld_base; a.ld_out = ld_dx;
        a.G = p.G; a.R = p.R; a.S = p.S;
        a.vec_in = vectors(dy, ld_dy, xb);
        a.vec_out = dx && vectors(dx, ld_dx, xb) && (!base || vectors(base, ld_base, xb));
        const cudaError_t e = launch_rows<true>(a, p.x_type, p.w_type, st);
        if (e != cudaSuccess)
            return e;
    }
    GradArgs b = {};
    b.x = x; b.dy = dy; b.t = t; b.u = u; b.scale = p.scale; b.offsets = p.offsets; b.ids = p.ids; b.da = da; b.db = db;
    b.M = p.M; b.N = p.N; b.K = p.K; b.ldx = ldx; b.ld_dy = ld_dy; b.G = p.G; b.R = p.R; b.S = p.M > 0 ? p.S : 0;
    b.vec_x = vectors(x, ldx, xb);
    b.vec_dy = vectors(dy, ld_dy, xb);
    b.tiles_k = (int)((p.K + 63) / 64);
    const int tiles = b.tiles_k + (int)((p.N + 63) / 64);
    return p.x_type == FPQ_FP32   ? launch_grad<float>(b, tiles, st)
           : p.x_type == FPQ_BF16 ? launch_grad<__nv_bfloat16>(b, tiles, st)
                                  : launch_grad<__half>(b, tiles, st);
}

}  // namespace fpq
