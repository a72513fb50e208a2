// Low-rank adapters of many requests at once, beside a shared projection: forward and backward.
//
//   forward   t_i = A x_i,      y_i  = base_i + B (s t_i)
//   backward  t_i = s B^T dy_i, dx_i = base_i + A^T t_i,   dA = sum_i t_i x_i^T,   dB = s sum_i dy_i u_i^T   (u_i = A x_i)
//
// A, B and s are those of the adapter that row i's request uses.  With a rank of 16 a row costs 2 R (K + N) operations on
// (K + 2 N) values: bound by memory, so every kernel reads its rows once.
//
// Forward and the first half of backward are one kernel with the roles of the matrices exchanged: adapter_rows_kernel, for requests of
// many rows and ranks above 16 the tcgen05 pass of fpq_adapter_tile.cu.  A block (or a cluster of up to 8, sharing the reduction and
// the output columns: single tokens) takes 16 to 128 rows of one request, reduces them to t in shared memory and multiplies t out
// again.  8192 x 1280 -> 320, FP32, rank 16: 20 us, 3.2 TB/s; 64 single tokens with an adapter each, 1280 -> 1280: 7.5 us.  It spends some
// 300 instructions on 16 x 32 values (half of the issue slots with 16 warps on an SM): operand splits, the addresses of the weights'
// fragments, the sums.  That and the latency of a tile bound it, not the memory.
//
// Backward then forms dA and dB (adapter_grad_kernel; from BF16 rows, by tcgen05 MMAs, fpq_adapter_grad_tile.cu): columns of x with t and of
// dy with u, rows split over blocks and added up in a fixed order.  8192 x 640 -> 640, FP32, rank 16: 13 of 38 us.  Three launches that
// overlap (weights transposed, rows, gradients): of a small call's 13 us most is their latency.
//
// Products run on the tensor cores as TF32 with FP32 operands in two terms x = hi + lo of 11 significant bits each: hi hi, hi lo and
// lo hi (16-bit operands are TF32 numbers themselves, one term, or are multiplied as they are).  Up to 2^-20 of a product is left
// out: 2^-22 are lo lo, 2^-21 each what the tensor core does not read of either lo.  The tensor cores cut their sums off instead of
// rounding them: at most 64 columns, 16 rows or 64 ranks (24 MMAs) are summed there, with BF16 rows 128 ranks, the rest in registers by
// FP32 additions.  The order of a reduction is free: a thread's share of a row lies side by side.
//
// An infinity, or a number that rounds up to one, has no split: a result that is not finite is worked out again by FP32
// multiply-adds.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "fpq_adapter.cuh"

namespace fpq {

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;

// The two terms of an FP32 number: rounded to 11 significant bits, and what that leaves off (the tensor core reads 11 bits of it).  (The
// number itself as the first term, which the tensor core cuts off, saves an instruction and no time.)
__device__ __forceinline__ uint32_t high(float x) { return (__float_as_uint(x) + 0x1000u) & 0xffffe000u; }
__device__ __forceinline__ uint32_t low(float x, uint32_t hi) { return __float_as_uint(x - __uint_as_float(hi)); }

__device__ __forceinline__ void mma_tf32(float* c, const uint32_t* a, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1, __nv_bfloat16)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1, __half)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// c = a b
__device__ __forceinline__ void mma_tf32_from_zero(float* c, const uint32_t* a, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_16_from_zero(float* c, const uint32_t* a, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// c[n] += a b[n] for N tiles, FP32 operands in two terms each (SPLIT_A / SPLIT_B: the operand has more bits than TF32).  One
// term after the other over all tiles: an MMA that waits for the one in front takes four times as long.
template <bool SPLIT_A, bool SPLIT_B, int N>
__device__ __forceinline__ void mma_split(float (*c)[4], const uint32_t* ah, const uint32_t* al, const float (&b)[N][2])
{
    uint32_t h[N][2];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int k = 0; k < 2; ++k)
            h[n][k] = SPLIT_B ? high(b[n][k]) : __float_as_uint(b[n][k]);
    if (SPLIT_B)
#pragma unroll
        for (int n = 0; n < N; ++n)
            mma_tf32(c[n], ah, low(b[n][0], h[n][0]), low(b[n][1], h[n][1]));
    if (SPLIT_A)
#pragma unroll
        for (int n = 0; n < N; ++n)
            mma_tf32(c[n], al, h[n][0], h[n][1]);
#pragma unroll
    for (int n = 0; n < N; ++n)
        mma_tf32(c[n], ah, h[n][0], h[n][1]);
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

// ---- rows to t and back ------------------------------------------------------------------------------------------
__device__ __forceinline__ void copy_async16(uint32_t dst, const void* src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_async4(uint32_t dst, const void* src, bool there)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}

// The 16-byte pieces at src of N rows (`every` rows and src_step, dst_step apart; of the first `rows` of them) to shared memory, `there`
// values of each and zeros behind: words asynchronously where the rows allow it, otherwise through registers, all loads in front
// of the stores.  Out of line: the path for rows at multiples of 16 bytes stays in the instruction cache.
template <typename XT, int N>
__device__ __noinline__ void copy_pieces(uint8_t* dst, int dst_step, const XT* src, int64_t src_step, int rows, int every, int there, int by,
                                         const void* anywhere)
{
    constexpr int PER = 16 / (int)sizeof(XT);
    if (by >= 4 && (sizeof(XT) == 4 || there >= PER || (there & 1) == 0)) {
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool some = k * every < rows && i * (4 / (int)sizeof(XT)) < there;
                copy_async4(smem_u32(dst + k * dst_step + 4 * i), some ? src + k * src_step + i * (4 / (int)sizeof(XT)) : (const XT*)anywhere, some);
            }
        return;
    }
    uint32_t w[N][4];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint16_t* p = reinterpret_cast<const uint16_t*>(src + k * src_step);
        const bool some = k * every < rows;
        if (some && there >= PER && (reinterpret_cast<uintptr_t>(p) & 3) == 0) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[k][i] = reinterpret_cast<const uint32_t*>(p)[i];
        } else if (some && there >= PER) {
            // between words: the first value, three words, the last value
            const uint32_t a = p[0], b = *reinterpret_cast<const uint32_t*>(p + 1), c = *reinterpret_cast<const uint32_t*>(p + 3),
                           d = *reinterpret_cast<const uint32_t*>(p + 5), e = p[7];
            w[k][0] = a | b << 16;
            w[k][1] = __funnelshift_l(b, c, 16);
            w[k][2] = __funnelshift_l(c, d, 16);
            w[k][3] = d >> 16 | e << 16;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                w[k][i] = (some && 2 * i < there ? (uint32_t)p[2 * i] : 0u) | (some && 2 * i + 1 < there ? (uint32_t)p[2 * i + 1] << 16 : 0u);
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
        *reinterpret_cast<uint4*>(dst + k * dst_step) = make_uint4(w[k][0], w[k][1], w[k][2], w[k][3]);
}

// A warp's share of 32 columns of a row: for FP32 rows, columns 4 q .. and 16 + 4 q .. (q = lane % 4), for 16-bit rows 8 q ..: a vector per
// lane, the vectors of a row side by side.
template <typename XT>
__device__ __forceinline__ int group_column(int q, int i) { return sizeof(XT) == 4 ? (i >> 2) * 16 + 4 * q + (i & 3) : 8 * q + i; }

template <typename XT, bool VEC, typename T>
__device__ __forceinline__ void load_group(const T* row, int c0, int q, int width, bool there, Raw<T, 8>& r, bool vec = true)
{
    if (!VEC && vec) {
        load_group<XT, true>(row, c0, q, width, there, r);
        return;
    }
    if constexpr (sizeof(XT) == 4) {
        Raw<T, 4> a, b;
        load_cols<VEC>(row, c0 + 4 * q, width, there, a);
        load_cols<VEC>(row, c0 + 16 + 4 * q, width, there, b);
#pragma unroll
        for (int i = 0; i < Raw<T, 4>::WORDS; ++i) {
            r.w[i] = a.w[i];
            r.w[Raw<T, 4>::WORDS + i] = b.w[i];
        }
    } else {
        load_cols<VEC>(row, c0 + 8 * q, width, there, r);
    }
}

// Every warp has a ring of its own in shared memory through which its 16 rows of x come, and behind them those of base, in groups of
// 32 columns: fetched asynchronously STAGES - 1 groups ahead, no warp waits for another.
template <typename XT, int RP>
struct RowsRing {
    static constexpr int SLOT = 16 * 32 * (int)sizeof(XT);
    static constexpr int STAGES = sizeof(XT) == 2 ? (RP <= 32 ? 8 : 4) : RP <= 32 ? 4 : RP == 64 ? 2 : 4;   // two blocks on an SM up to rank 64
};

// A block has 16 * wr rows; each of its warps takes 16 of them and, with the 8 / wr warps (times the blocks of the cluster) that
// have the same rows, shares the reduction in groups of 32 columns, then the output in groups of 32 columns.  RP: the rank, padded.  (Two blocks on an
// SM leave 128 registers: rank 64 spills 180 bytes with FP32 rows and weights, 280 without vectors, 16 to 108 otherwise.)
template <typename XT, typename WT, int RP, bool VEC>
__global__ void __launch_bounds__(THREADS, RP <= 64 ? 2 : 1) adapter_rows_kernel(const RowsArgs a)
{
    using Ring = RowsRing<XT, RP>;
    constexpr int NT = RP / 8, PITCH = RP == 16 ? 16 : RP + 16, STAGES = Ring::STAGES;
    constexpr bool NATIVE = sizeof(XT) == 2;               // x and weights of one 16-bit type, multiplied as they are
    constexpr bool AHEAD = RP * sizeof(WT) <= 64;          // registers for the weights of the next group
    extern __shared__ float4 smem4[];
    uint8_t* rings = reinterpret_cast<uint8_t*>(smem4);
    float* parts = reinterpret_cast<float*>(rings + WARPS * STAGES * Ring::SLOT);   // [8 / wr][16 wr][RP], then the block's sum in the first
    float* t_smem = parts + WARPS * 16 * RP;               // [16 wr][PITCH]
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    uint32_t rank = cluster_rank(), C;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
    const int WR = a.wr, WK = WARPS / WR, BM = 16 * WR;
    const int64_t tile = blockIdx.x / C;
    const TileRows tr = find_tile(BM, tile, a.offsets, a.ids, a.S, a.G, a.M);
    if (tr.rows <= 0)
        return;                                            // (every block of the cluster leaves)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int r0 = (warp & (WR - 1)) * 16, wk = warp / WR, here = tr.rows - r0;
    const float s = a.scale && tr.id >= 0 ? a.scale[tr.id] : 1.f;
    const int D1 = (int)a.D1, D2 = (int)a.D2, R = a.R, step = 32 * WK * (int)C, first = 32 * ((int)rank * WK + wk);
    const int ld1 = (int)a.ld_w1, ld2 = (int)a.ld_w2;
    const WT* w1 = (const WT*)a.w1 + (int64_t)max(tr.id, 0) * R * ld1;
    const WT* w2 = (const WT*)a.w2 + (int64_t)max(tr.id, 0) * D2 * ld2;
    const XT* in = (const XT*)a.in + tr.row * a.ld_in;

    // what comes through the ring: groups of x, then groups of base
    uint8_t* ring = rings + warp * (STAGES * Ring::SLOT);
    constexpr int PER = 16 / (int)sizeof(XT), ACROSS = 32 / PER, EVERY = 32 / ACROSS;       // values of a vector, vectors of a row, rows at a time
    const int cr = lane / ACROSS, cc = lane % ACROSS;
    const int xs = here > 0 && tr.id >= 0 && first < D1 ? (D1 - 1 - first) / step + 1 : 0;
    const int bs = here > 0 && a.out && a.base && first < D2 ? (D2 - 1 - first) / step + 1 : 0;
    const XT* x_from = in + (int64_t)(r0 + cr) * a.ld_in + first + cc * PER;
    const XT* b_from = (const XT*)a.base + (tr.row + r0 + cr) * a.ld_base + first + cc * PER;
    int fetched = 0, put = 0, get = 0;
    auto fetch = [&]() {
        if (fetched < xs + bs) {
            const bool is_x = fetched < xs;
            const int i = is_x ? fetched : fetched - xs, col = first + i * step + cc * PER, width = is_x ? D1 : D2;
            const int64_t ld = is_x ? a.ld_in : a.ld_base;
            const XT* src = (is_x ? x_from : b_from) + (int64_t)i * step;
            // FP32: eight vectors a row; the halves of odd rows are exchanged, so that two rows' vectors lie in different banks
            uint8_t* dst = ring + put * Ring::SLOT + cr * (32 * (int)sizeof(XT)) + (sizeof(XT) == 4 ? cc ^ ((cr & 1) << 2) : cc) * 16;
            if constexpr (VEC) {
#pragma unroll
                for (int k = 0; k < 16; k += EVERY) {
                    const bool there = cr + k < here && col < width;
                    copy_async16(smem_u32(dst + k * (32 * (int)sizeof(XT))), there ? src + k * ld : in, there);
                }
            } else {
                const int by = is_x ? a.in_by : a.base_by;
                const XT* anywhere = (const XT*)(is_x ? a.in : a.base);      // (what is not copied has a source too, aligned like the others)
                if (by == 16) {
#pragma unroll 1
                    for (int k = 0; k < 16; k += EVERY) {
                        const bool there = cr + k < here && col < width;
                        copy_async16(smem_u32(dst + k * (32 * (int)sizeof(XT))), there ? src + k * ld : anywhere, there);
                    }
                } else {
                    copy_pieces<XT, 16 / EVERY>(dst, EVERY * 32 * (int)sizeof(XT), src, EVERY * ld, here - cr, EVERY, width - col, by, anywhere);
                }
            }
        }
        ++fetched;
        put = put + 1 == STAGES ? 0 : put + 1;
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto take = [&](Raw<XT, 8> (&v)[2]) {                  // the next group of rows g and g + 8
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
        __syncwarp();
        fetch();                                           // into the slot that was read last, by all lanes in front of this barrier
        const uint8_t* slot = ring + get * Ring::SLOT;
        get = get + 1 == STAGES ? 0 : get + 1;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint8_t* row = slot + (g + 8 * h) * (32 * (int)sizeof(XT));
#pragma unroll
            for (int e = 0; e < (int)sizeof(XT) / 2; ++e) {
                const uint4 x = *reinterpret_cast<const uint4*>(row + (sizeof(XT) == 4 ? ((q + 4 * e) ^ ((g & 1) << 2)) * 16 : q * 16));
                v[h].w[4 * e] = x.x; v[h].w[4 * e + 1] = x.y; v[h].w[4 * e + 2] = x.z; v[h].w[4 * e + 3] = x.w;
            }
        }
    };
#pragma unroll
    for (int k = 0; k < STAGES - 1; ++k)
        fetch();

    if (tr.id >= 0) {
        float acc[NT][4] = {}, part[NT][4] = {};
        Raw<XT, 8> x[2];
        constexpr int BATCH = NT > 4 && !NATIVE ? 4 : NT;      // (more at a time do not fit the registers)
        Raw<WT, 8> w_next[AHEAD ? NT : 1];
        const WT* w_row = w1 + (int64_t)g * ld1;
        int since = 0;
        if (AHEAD && xs > 0)
#pragma unroll
            for (int n = 0; n < NT; ++n)
                load_group<XT, VEC>(w_row + (int64_t)(n * 8) * ld1, first, q, D1, n * 8 + g < R, w_next[n], a.vec_w1);
        for (int i = 0; i < xs; ++i) {
            const int k0 = first + i * step;
#pragma unroll
            for (int n0 = 0; n0 < NT; n0 += BATCH) {
                Raw<WT, 8> w[BATCH];
#pragma unroll
                for (int n = 0; n < BATCH; ++n)
                    if (AHEAD) {
                        w[n] = w_next[n];
                        load_group<XT, VEC>(w_row + (int64_t)(n * 8) * ld1, k0 + step, q, D1, n * 8 + g < R, w_next[n], a.vec_w1);   // (behind the end nothing is loaded)
                    } else {
                        load_group<XT, VEC>(w_row + (int64_t)((n0 + n) * 8) * ld1, k0, q, D1, (n0 + n) * 8 + g < R, w[n], a.vec_w1);
                    }
                if (n0 == 0)
                    take(x);
                if constexpr (NATIVE) {
#pragma unroll
                    for (int st = 0; st < 2; ++st) {
                        const uint32_t v[4] = {x[0].w[2 * st], x[1].w[2 * st], x[0].w[2 * st + 1], x[1].w[2 * st + 1]};
#pragma unroll
                        for (int n = 0; n < BATCH; ++n)
                            mma_16(part[n0 + n], v, w[n].w[2 * st], w[n].w[2 * st + 1], XT());
                    }
                } else {
                    float f[2][8], fw[BATCH][8];
                    x[0].values(f[0]);
                    x[1].values(f[1]);
#pragma unroll
                    for (int n = 0; n < BATCH; ++n)
                        w[n].values(fw[n]);
#pragma unroll
                    for (int st = 0; st < 4; ++st) {
                        const float v[4] = {f[0][2 * st], f[1][2 * st], f[0][2 * st + 1], f[1][2 * st + 1]};
                        uint32_t vh[4], vl[4];
                        split_four<true>(v, vh, vl);
                        float b[BATCH][2];
#pragma unroll
                        for (int n = 0; n < BATCH; ++n) {
                            b[n][0] = fw[n][2 * st];
                            b[n][1] = fw[n][2 * st + 1];
                        }
                        mma_split<true, WIDE<WT>, BATCH>(part + n0, vh, vl, b);
                    }
                }
            }
            if (++since == 2) {                            // 64 columns
                since = 0;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        acc[n][k] += part[n][k];
                        part[n][k] = 0.f;
                    }
            }
        }
        float* mine = parts + (wk * BM + r0) * RP;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            *reinterpret_cast<float2*>(mine + g * RP + n * 8 + 2 * q) = make_float2(acc[n][0] + part[n][0], acc[n][1] + part[n][1]);
            *reinterpret_cast<float2*>(mine + (8 + g) * RP + n * 8 + 2 * q) = make_float2(acc[n][2] + part[n][2], acc[n][3] + part[n][3]);
        }
        __syncthreads();
        if (C > 1) {                                       // the block's own sum first: one array per block to fetch
            for (int i = threadIdx.x; i < BM * RP; i += THREADS) {
                float v = parts[i];
                for (int k = 1; k < WK; ++k)
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
                for (int k = 0; k < WK; ++k)
                    v += parts[k * BM * RP + i];
            }
            if (!finite(v) && r < tr.rows && j < R) {
                v = 0.f;
                for (int k = 0; k < D1; ++k)
                    v = fmaf(as_float(in[r * a.ld_in + k]), as_float(w1[(int64_t)j * ld1 + k]), v);
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

    if (a.out && here > 0) {
        // BF16: t in two terms of 8 bits, 2^-18 of it left out against the 2^-9 that y is rounded by; otherwise TF32 terms
        constexpr bool BF = std::is_same<XT, __nv_bfloat16>::value;
        constexpr int TPER = RP < 32 ? RP / 4 : 8, BLOCKS = RP / (4 * TPER);  // ranks of a thread side by side, and how often
        constexpr bool HOLD = BF || RP <= 32;                                 // t's operands stay in registers
        constexpr bool AHEAD2 = RP * sizeof(WT) <= 64;
        uint32_t th[HOLD ? BLOCKS : 1][TPER / 2][4], tl[HOLD ? BLOCKS : 1][TPER / 2][4];
        auto fetch_t = [&](int b, uint32_t (&h)[TPER / 2][4], uint32_t (&l)[TPER / 2][4]) {
            float t[2][TPER];
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < TPER; i += 4) {
                    const float4 v = *reinterpret_cast<const float4*>(t_smem + (r0 + k * 8 + g) * PITCH + (b * 4 + q) * TPER + i);
                    t[k][i] = v.x; t[k][i + 1] = v.y; t[k][i + 2] = v.z; t[k][i + 3] = v.w;
                }
            if constexpr (BF) {
#pragma unroll
                for (int st = 0; st < TPER / 4; ++st)
#pragma unroll
                    for (int e = 0; e < 4; ++e)            // rows g, g + 8, then the second pair of ranks
                        split_bf16(t[e & 1][4 * st + 2 * (e >> 1)], t[e & 1][4 * st + 2 * (e >> 1) + 1], h[st][e], l[st][e]);
            } else {
#pragma unroll
                for (int st = 0; st < TPER / 2; ++st) {
                    const float v[4] = {t[0][2 * st], t[1][2 * st], t[0][2 * st + 1], t[1][2 * st + 1]};
                    split_four<true>(v, h[st], l[st]);
                }
            }
        };
        if constexpr (HOLD)
            if (tr.id >= 0)
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b)
                    fetch_t(b, th[b], tl[b]);
        // The MMA's column g of tile e is this output column: the two columns 2 q and 2 q + 1 that a thread gets of each of the four
        // tiles are its columns of the group.
        const int n0 = sizeof(XT) == 4 ? 4 * (g >> 1) + (g & 1) : 8 * (g >> 1) + (g & 1);
        auto tile_column = [](int e) { return sizeof(XT) == 4 ? (e >> 1) * 16 + (e & 1) * 2 : 2 * e; };
        auto load_w2 = [&](int c0, int b, Raw<WT, TPER> (&w)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int n = c0 + n0 + tile_column(e);
                if (VEC || a.vec_w2)
                    load_cols<true>(w2 + (int64_t)n * ld2, (b * 4 + q) * TPER, R, n < D2, w[e]);
                else
                    load_cols<false>(w2 + (int64_t)n * ld2, (b * 4 + q) * TPER, R, n < D2, w[e]);
            }
        };
        Raw<WT, TPER> w_next[AHEAD2 ? BLOCKS : 1][4];
        if (AHEAD2 && tr.id >= 0)
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
                load_w2(first, b, w_next[AHEAD2 ? b : 0]);
        XT* out_row[2] = {(XT*)a.out + (tr.row + r0 + g) * a.ld_out, (XT*)a.out + (tr.row + r0 + 8 + g) * a.ld_out};
        for (int c0 = first; c0 < D2; c0 += step) {
            float y[2][8], acc[4][4] = {};
            if (tr.id >= 0) {
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    Raw<WT, TPER> w[4];
                    if constexpr (AHEAD2) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            w[e] = w_next[b][e];
                        load_w2(c0 + step, b, w_next[b]);
                    } else {
                        load_w2(c0, b, w);
                    }
                    if constexpr (!HOLD)
                        fetch_t(b, th[0], tl[0]);
                    const auto& h = th[HOLD ? b : 0];
                    const auto& l = tl[HOLD ? b : 0];
                    if constexpr (BF) {
#pragma unroll
                        for (int st = 0; st < TPER / 4; ++st)
#pragma unroll
                            for (int k = 0; k < 2; ++k)
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    mma_16(acc[e], k ? h[st] : l[st], w[e].w[2 * st], w[e].w[2 * st + 1], __nv_bfloat16());
                    } else {
                        float f[4][TPER];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            w[e].values(f[e]);
                        // (above 64 ranks the sums of 32 are added in registers: cut off throughout, y was 1.1e-6 off instead of 0.4e-6)
                        float part[RP > 64 ? 4 : 1][4] = {};
#pragma unroll
                        for (int st = 0; st < TPER / 2; ++st) {
                            const float v[4][2] = {{f[0][2 * st], f[0][2 * st + 1]}, {f[1][2 * st], f[1][2 * st + 1]},
                                                   {f[2][2 * st], f[2][2 * st + 1]}, {f[3][2 * st], f[3][2 * st + 1]}};
                            mma_split<true, WIDE<WT>, 4>(RP > 64 ? part : acc, h[st], l[st], v);
                        }
                        if constexpr (RP > 64)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    acc[e][k] += part[e][k];
                    }
                }
                float zero = 0.f;                          // becomes NaN if a sum is not finite
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        zero = fmaf(acc[e][k], 0.f, zero);
                if (zero != 0.f) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int h = i >> 3, r = r0 + h * 8 + g, col = c0 + group_column<XT>(q, i & 7);
                        float& v = acc[(i & 7) >> 1][2 * h + (i & 1)];
                        if (!finite(v) && r < tr.rows && col < D2) {
                            v = 0.f;
                            for (int j = 0; j < R; ++j)
                                v = fmaf(t_smem[r * PITCH + j], as_float(w2[(int64_t)col * ld2 + j]), v);
                        }
                    }
                }
            }
            if (bs > 0) {
                Raw<XT, 8> y0[2];
                take(y0);
                y0[0].values(y[0]);
                y0[1].values(y[1]);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    y[i >> 3][i & 7] = 0.f;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    y[h][i] += acc[i >> 1][2 * h + (i & 1)];
                if (8 * h + g >= here)
                    continue;
                XT* o = out_row[h] + c0;
#pragma unroll
                for (int p = 0; p < 8; p += PER) {
                    const int col = group_column<XT>(q, p);
                    if (VEC || a.out_by == 16) {
                        if (c0 + col < D2) {
                            alignas(16) XT v[PER];
#pragma unroll
                            for (int i = 0; i < PER; ++i)
                                v[i] = from_float<XT>(y[h][p + i]);
                            *reinterpret_cast<uint4*>(o + col) = *reinterpret_cast<const uint4*>(v);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < PER; ++i)
                            if (c0 + col + i < D2)
                                o[col + i] = from_float<XT>(y[h][p + i]);
                    }
                }
            }
        }
    }
    __syncwarp();
    if (C > 1 && tr.id >= 0)
        cluster_wait();                                    // nobody still reads this block's sums
}

// Adapters transposed for the backward pass, 32 x 32 at a time: [G][R][K] to [G][K][ldr] and [G][N][R] to [G][R][ldn], rows of which start
// at multiples of 16 bytes, zeros behind their ends; and the tickets of the gradients' blocks set to zero.
template <typename T>
__global__ void __launch_bounds__(THREADS) transpose_adapters_kernel(const T* a, T* at, const T* b, T* bt, int R, int K, int N, int ldr, int ldn,
                                                                     int tiles_a, int tiles, uint32_t* tickets, int n_tickets)
{
    __shared__ T piece[32][33];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0 && (int)blockIdx.x < n_tickets)
        tickets[blockIdx.x] = 0;                           // (there are more blocks than tickets: 32 columns each instead of 64)
    const int g = blockIdx.x / tiles, t = blockIdx.x % tiles;
    const bool is_b = t >= tiles_a;
    const int rows = is_b ? N : R, cols = is_b ? R : K, ld = is_b ? ldn : ldr, across = (cols + 31) / 32, i = is_b ? t - tiles_a : t;
    const T* src = (is_b ? b : a) + (int64_t)g * rows * cols;
    T* dst = (is_b ? bt : at) + (int64_t)g * cols * ld;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, r0 = i / across * 32, c0 = i % across * 32;
#pragma unroll
    for (int k = y; k < 32; k += 8)
        piece[k][x] = r0 + k < rows && c0 + x < cols ? src[(int64_t)(r0 + k) * cols + c0 + x] : T(0);
    __syncthreads();
#pragma unroll
    for (int k = y; k < 32; k += 8)
        if (c0 + k < cols && r0 + x < ld)
            dst[(int64_t)(c0 + k) * ld + r0 + x] = piece[x][k];
}

// ---- gradients of the adapters -----------------------------------------------------------------------------------
// out(col, j) = sum over an adapter's rows of wide[i][col] * thin[i][j]: columns of x with t (dA) and of dy with u (dB).  A
// block takes 64 columns; its warps, and the blocks with the same columns, share the rows in runs.  Sums are added up in a fixed
// order: those of the warps in shared memory, those of the blocks by the one that is the last of them to end (a kernel of its own
// behind this one: 2 us more, 8192 x 640 -> 640).
// Element i of a tile's 64 RP, in the order of the output's contiguous side.
__device__ __forceinline__ void tile_element(int i, int RP, bool is_b, int& col, int& j)
{
    col = is_b ? i / RP : i % 64;
    j = is_b ? i % RP : i / 64;
}

// Every warp has a ring of its own in shared memory: runs of 16 (32) rows of 64 columns and of its JT ranks, fetched asynchronously
// STAGES - 1 runs ahead; no warp waits for another before the end.  (Loads into registers, 8192 x 1280 columns: 40 us; so, 14.)  The pitches keep a quarter warp's
// vectors, and a warp's single words, in different banks.
template <typename XT, int JT>
struct GradRing {
    static constexpr int RUN = sizeof(XT) == 2 && JT == 16 ? 32 : 16;
    static constexpr int WIDE_PITCH = 64 * (int)sizeof(XT) + 16, THIN_PITCH = (JT + 4) * 4;      // bytes
    static constexpr int STAGE = RUN * (WIDE_PITCH + THIN_PITCH);
    static constexpr int STAGES = sizeof(XT) == 2 && JT == 32 ? 3 : 2;                            // two blocks on an SM
};

// JT: ranks of a warp; RP / JT warps share a run of rows.  (Two blocks on an SM leave 128 registers: FP32 rows spill 116 to 140 bytes, FP16 20
// to 44, BF16 4 to 16.)
template <typename XT, int RP, int JT>
__global__ void __launch_bounds__(THREADS, 2) adapter_grad_kernel(const GradArgs a)
{
    using Ring = GradRing<XT, JT>;
    constexpr int NT = JT / 8, WN = RP / JT, WK = WARPS / WN, RUN = Ring::RUN, STAGES = Ring::STAGES;
    constexpr int MB = 4 / NT < 1 ? 1 : 4 / NT;            // four independent MMAs one after the other
    constexpr int CHAIN = NT >= 4 ? 1 : 2;
    extern __shared__ float4 smem4[];
    constexpr int PITCH = RP + 2;                          // (columns of a tile in different banks, for the writes and for the reads)
    float* parts = reinterpret_cast<float*>(smem4);        // at the end: [WK][64][PITCH]
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const GradShare share = share_of(a);
    if (share.z < 0)
        return;
    const int tile = blockIdx.x, id = share.id, splits = share.splits;
    const bool is_b = tile >= a.tiles_k;
    const int64_t D = is_b ? a.N : a.K, ld = is_b ? a.ld_dy : a.ldx, c0 = (int64_t)(is_b ? tile - a.tiles_k : tile) * 64;
    const XT* wide = (const XT*)(is_b ? a.dy : a.x);
    const float* thin = is_b ? a.u : a.t;
    const int R = a.R, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int wn = warp % WN, wk = warp / WN, workers = WK * splits, worker = share.z * WK + wk, j0 = wn * JT;
    uint8_t* ring = reinterpret_cast<uint8_t*>(smem4) + warp * (STAGES * Ring::STAGE);

    // the runs of this warp, in order: every workers-th of all runs of the adapter's segments
    int chunk = -32, my_begin = 0, my_end = 0;             // 32 segments at a time, one to a lane
    uint32_t left = 0;
    int runs = 0;                                          // runs of the segments in front, modulo the workers
    int at = 0, n_runs = 0, begin = 0, end = 0;
    auto next_run = [&](int& row, int& rows) {
        while (at >= n_runs) {
            runs = (runs + n_runs) % workers;
            n_runs = 0;
            while (left == 0) {
                chunk += 32;
                if (chunk >= a.S)
                    return false;
                const int sg = chunk + lane;
                bool mine = false;
                if (sg < a.S) {
                    my_begin = min(max(a.offsets[sg], 0), (int)a.M);
                    my_end = min(max(a.offsets[sg + 1], 0), (int)a.M);
                    mine = a.ids[sg] == id && my_end > my_begin;
                }
                left = __ballot_sync(0xffffffffu, mine);
            }
            const int from = __ffs(left) - 1;
            left &= left - 1;
            begin = __shfl_sync(0xffffffffu, my_begin, from);
            end = __shfl_sync(0xffffffffu, my_end, from);
            n_runs = (end - begin - 1) / RUN + 1;
            at = worker - runs + (worker < runs ? workers : 0);
        }
        row = begin + at * RUN;
        rows = end - row;
        at += workers;                                     // (runs and workers together stay far below 2^31)
        return true;
    };
    constexpr int PER = 16 / (int)sizeof(XT), ACROSS = 64 / PER, EVERY = 32 / ACROSS;      // vectors of a row, rows at a time
    const int wr = lane / ACROSS, wc = lane % ACROSS * PER;
    const bool wide_in = c0 + wc < D;
    const int by = is_b ? a.dy_by : a.x_by;
    constexpr int T_ACROSS = JT / 4, T_EVERY = 32 / T_ACROSS;
    const int tr = lane / T_ACROSS, tc = lane % T_ACROSS * 4;
    const bool thin_in = j0 + tc < R, thin_vec = R % 4 == 0 && (reinterpret_cast<uintptr_t>(thin) & 15) == 0;
    auto fetch = [&](int slot) {
        int row, rows;
        const bool some = next_run(row, rows);
        if (some) {
            uint8_t* w = ring + slot * Ring::STAGE;
            const XT* src = wide + (int64_t)(row + wr) * ld + c0 + wc;
            uint8_t* dst = w + wr * Ring::WIDE_PITCH + wc * (int)sizeof(XT);
            if (by == 16) {
#pragma unroll
                for (int k = 0; k < RUN; k += EVERY) {
                    const bool there = wide_in && wr + k < rows;
                    copy_async16(smem_u32(dst + k * Ring::WIDE_PITCH), there ? src + k * ld : wide, there);
                }
            } else {
#pragma unroll 1
                for (int k = 0; k < RUN; k += 4 * EVERY)
                    copy_pieces<XT, 4>(dst + k * Ring::WIDE_PITCH, EVERY * Ring::WIDE_PITCH, src + k * ld, EVERY * ld, rows - wr - k, EVERY,
                                       (int)min(D - c0 - wc, (int64_t)PER), by, wide);
            }
            uint8_t* t = w + RUN * Ring::WIDE_PITCH;
            if (thin_vec) {
                const float* from = thin + (int64_t)(row + tr) * R + j0 + tc;
#pragma unroll
                for (int k = 0; k < RUN; k += T_EVERY) {
                    const bool there = thin_in && tr + k < rows;
                    copy_async16(smem_u32(t + (tr + k) * Ring::THIN_PITCH + tc * 4), there ? from + k * R : thin, there);
                }
            } else {
#pragma unroll 4
                for (int i = lane; i < RUN * JT; i += 32) {
                    const int r = i / JT, c = i % JT;
                    const bool there = r < rows && j0 + c < R;
                    copy_async4(smem_u32(t + r * Ring::THIN_PITCH + c * 4), there ? thin + (int64_t)(row + r) * R + j0 + c : thin, there);
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        return some;
    };

    float acc[4][NT][4] = {};
    int ahead = 0, stage = 0, put = 0;                     // runs fetched and not yet used
#pragma unroll
    for (int k = 0; k < STAGES - 1; ++k) {
        ahead += fetch(put) ? 1 : 0;
        put = put + 1 == STAGES ? 0 : put + 1;
    }
    while (ahead > 0) {
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
        __syncwarp();
        ahead += fetch(put) ? 0 : -1;                      // into the slot that was read last, by all lanes in front of this barrier
        put = put + 1 == STAGES ? 0 : put + 1;
        const uint8_t* w = ring + stage * Ring::STAGE;
        const float* t = reinterpret_cast<const float*>(w + RUN * Ring::WIDE_PITCH) + g;
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        // MMA k: rows 2 q and 2 q + 1 (and 8 behind them); the sums of a run start from zero and are added in registers
        if constexpr (std::is_same<XT, __nv_bfloat16>::value) {
            // BF16 as it is, with t or u in three terms of 8 bits
#pragma unroll
            for (int st = 0; st < RUN / 16; ++st) {
            uint32_t p[3][NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float x = t[(16 * st + 2 * q + 8 * h) * (JT + 4) + 8 * n], y = t[(16 * st + 2 * q + 1 + 8 * h) * (JT + 4) + 8 * n];
#pragma unroll
                    for (int e = 0; e < 3; ++e) {
                        const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
                        const float2 f = __bfloat1622float2(v);
                        p[e][n][h] = *reinterpret_cast<const uint32_t*>(&v);
                        x -= f.x;
                        y -= f.y;
                    }
                }
            uint4 v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                v[k] = *reinterpret_cast<const uint4*>(w + (16 * st + 2 * q + (k & 1) + 8 * (k >> 1)) * Ring::WIDE_PITCH + g * 16);
            const uint32_t* rows[4] = {&v[0].x, &v[1].x, &v[2].x, &v[3].x};
#pragma unroll
            for (int m0 = 0; m0 < 4; m0 += MB) {
                float part[MB][NT][4];
                uint32_t f[MB][4];
#pragma unroll
                for (int i = 0; i < MB; ++i) {             // MMA rows g and g + 8 are columns 8 g + 2 m and 8 g + 2 m + 1
                    const int m = m0 + i;
                    f[i][0] = __byte_perm(rows[0][m], rows[1][m], 0x5410);
                    f[i][1] = __byte_perm(rows[0][m], rows[1][m], 0x7632);
                    f[i][2] = __byte_perm(rows[2][m], rows[3][m], 0x5410);
                    f[i][3] = __byte_perm(rows[2][m], rows[3][m], 0x7632);
                }
#pragma unroll
                for (int e = 2; e >= 0; --e)
#pragma unroll
                    for (int i = 0; i < MB; ++i)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
                            if (e == 2)
                                mma_16_from_zero(part[i][n], f[i], p[e][n][0], p[e][n][1]);
                            else
                                mma_16(part[i][n], f[i], p[e][n][0], p[e][n][1], __nv_bfloat16());
#pragma unroll
                for (int i = 0; i < MB; ++i)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            acc[m0 + i][n][k] += part[i][n][k];
            }
            }
        } else {
#pragma unroll
            for (int s0 = 0; s0 < RUN / 8; s0 += CHAIN) {  // a sum of 8 or 16 rows starts from zero, and is added in registers
                uint32_t ph[CHAIN][NT][2], pl[CHAIN][NT][2];
                float v[CHAIN][2][8];                          // [rows 2 q, 2 q + 1][both columns of the MMA's four row tiles]
#pragma unroll
                for (int st = 0; st < CHAIN; ++st)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int row = 8 * (s0 + st) + 2 * q + h;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const float x = t[row * (JT + 4) + 8 * n];
                            ph[st][n][h] = high(x);
                            pl[st][n][h] = low(x, ph[st][n][h]);
                        }
                        const uint8_t* r = w + row * Ring::WIDE_PITCH;
                        if constexpr (sizeof(XT) == 4) {   // columns 4 g + m and 32 + 4 g + m
                            const float4 x = *reinterpret_cast<const float4*>(r + g * 16), y = *reinterpret_cast<const float4*>(r + 128 + g * 16);
                            v[st][h][0] = x.x; v[st][h][2] = x.y; v[st][h][4] = x.z; v[st][h][6] = x.w;
                            v[st][h][1] = y.x; v[st][h][3] = y.y; v[st][h][5] = y.z; v[st][h][7] = y.w;
                        } else {                           // columns 8 g + 2 m and 8 g + 2 m + 1
                            Raw<XT, 8> x;
                            const uint4 y = *reinterpret_cast<const uint4*>(r + g * 16);
                            x.w[0] = y.x; x.w[1] = y.y; x.w[2] = y.z; x.w[3] = y.w;
                            x.values(v[st][h]);
                        }
                    }
#pragma unroll
                for (int m0 = 0; m0 < 4; m0 += MB) {
                    float part[MB][NT][4];
#pragma unroll
                    for (int st = 0; st < CHAIN; ++st) {
                        uint32_t wh[MB][4], wl[MB][4];
#pragma unroll
                        for (int i = 0; i < MB; ++i) {
                            const int m = m0 + i;
                            const float f[4] = {v[st][0][2 * m], v[st][0][2 * m + 1], v[st][1][2 * m], v[st][1][2 * m + 1]};
                            split_four<WIDE<XT>>(f, wh[i], wl[i]);
                        }
#pragma unroll
                        for (int e = 0; e < 3; ++e)
#pragma unroll
                            for (int i = 0; i < MB; ++i)
#pragma unroll
                                for (int n = 0; n < NT; ++n)
                                    if (e == 0 && st == 0)
                                        mma_tf32_from_zero(part[i][n], wh[i], pl[st][n][0], pl[st][n][1]);
                                    else if (e == 0)
                                        mma_tf32(part[i][n], wh[i], pl[st][n][0], pl[st][n][1]);
                                    else if (e == 2)
                                        mma_tf32(part[i][n], wh[i], ph[st][n][0], ph[st][n][1]);
                                    else if (WIDE<XT>)
                                        mma_tf32(part[i][n], wl[i], ph[st][n][0], ph[st][n][1]);
                    }
#pragma unroll
                    for (int i = 0; i < MB; ++i)
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                acc[m0 + i][n][k] += part[i][n][k];
                }
            }
        }
    }
    __syncthreads();                                       // the rings are free
    // parts[wk][column][rank]
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int col = sizeof(XT) == 4 ? h * 32 + g * 4 + m : g * 8 + 2 * m + h;
                *reinterpret_cast<float2*>(parts + (wk * 64 + col) * PITCH + j0 + n * 8 + 2 * q) = make_float2(acc[m][n][2 * h], acc[m][n][2 * h + 1]);
            }
    __syncthreads();
    float* sums = a.sums + (((int64_t)share.z * a.G + id) * a.tiles + tile) * 64 * RP;
    for (int i = threadIdx.x; i < 64 * RP; i += THREADS) {
        int col, j;
        tile_element(i, RP, is_b, col, j);
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < WK; ++k)
            v += parts[(k * 64 + col) * PITCH + j];
        if (splits > 1)
            sums[i] = v;
        else if (c0 + col < D && j < R)
            store_gradient<XT>(a, id, is_b, c0 + col, j, v);
    }
    if (splits == 1)
        return;
    __shared__ int last;
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t ended;
        asm volatile("atom.acq_rel.gpu.global.add.u32 %0, [%1], 1;" : "=r"(ended) : "l"(a.tickets + (int64_t)id * a.tiles + tile) : "memory");
        last = ended == (uint32_t)splits - 1;
    }
    __syncthreads();
    if (!last)
        return;
    sums = a.sums + ((int64_t)id * a.tiles + tile) * 64 * RP;
    const int64_t next = (int64_t)a.G * a.tiles * 64 * RP;
#pragma unroll 1
    for (int i = threadIdx.x; i < 64 * RP; i += 4 * THREADS) {
        float v[4] = {};
        for (int z = 0; z < splits; z += 4) {              // (sixteen loads at a time, the last ones too)
            float w[4][4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    w[e][k] = z + e < splits ? sums[(z + e) * next + i + k * THREADS] : 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    v[k] += w[e][k];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            int col, j;
            tile_element(i + k * THREADS, RP, is_b, col, j);
            if (c0 + col < D && j < R)
                store_gradient<XT>(a, id, is_b, c0 + col, j, v[k]);
        }
    }
}

// ---- launches ----------------------------------------------------------------------------------------------------
template <typename Args>
cudaError_t launch_cluster(void (*kernel)(const Args), std::atomic<uint64_t>& known, int most, dim3 grid, int cluster, size_t smem,
                           cudaStream_t st, const Args& args)
{
    // shared memory beyond 48 KB is asked for once per kernel and device: `most`, what any call of this kernel needs
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess)
        return e;
    if (most > 48 * 1024 && (dev >= 64 || !(known.load(std::memory_order_relaxed) >> dev & 1))) {
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
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

// rows at multiples of 16 bytes, a whole number of vectors long
bool vectors(const void* p, int64_t ld, int64_t width, int bytes)
{
    return (uintptr_t)p % 16 == 0 && ld * bytes % 16 == 0 && width * bytes % 16 == 0;
}

int type_bytes(int t) { return t == FPQ_FP32 ? 4 : 2; }

// bytes at a time that rows allow: 16, 4 (words), or 2 where rows of 16-bit values start between words
int bytes_at_a_time(const void* p, int64_t ld, int64_t width, int bytes)
{
    return vectors(p, ld, width, bytes) ? 16 : (uintptr_t)p % 4 == 0 && ld * bytes % 4 == 0 ? 4 : 2;
}

template <typename XT, typename WT, int RP, bool VEC>
cudaError_t launch_rows_as(RowsArgs a, cudaStream_t st)
{
    constexpr int PITCH = RP == 16 ? 16 : RP + 16;
    const int64_t longest = std::max(a.D1, a.out ? a.D2 : 0), groups = (longest + 31) / 32;
    a.wr = 1;
    while (a.wr < 8 && a.M / (16 * a.wr) + a.S > 2 * 148 && a.M >= 24 * a.wr * (int64_t)a.S)
        a.wr *= 2;
    const int BM = 16 * a.wr;
    const size_t smem = (size_t)WARPS * RowsRing<XT, RP>::STAGES * RowsRing<XT, RP>::SLOT + (size_t)(WARPS * 16 * RP + BM * PITCH) * 4;
    const int64_t tiles = a.M / BM + a.S;
    // clusters until there are two blocks for every SM, while every block has a group of columns for most of its warps
    int c = 1;
    const int64_t busy = (a.M + BM - 1) / BM + std::min<int64_t>(a.S, a.M) - 1;
    while (c < 8 && busy * c * 2 <= 2 * 148 && groups > (int64_t)c * (WARPS / a.wr))
        c *= 2;
    static std::atomic<uint64_t> known{0};
    constexpr int MOST = WARPS * RowsRing<XT, RP>::STAGES * RowsRing<XT, RP>::SLOT + (WARPS * 16 * RP + 16 * WARPS * PITCH) * 4;
    return launch_cluster<RowsArgs>(adapter_rows_kernel<XT, WT, RP, VEC>, known, MOST, dim3((unsigned)(tiles * c)), c, smem, st, a);
}

// VEC: everything is read and written by vectors; otherwise each operand as its rows allow.  (Weight rows longer than needed hold zeros
// behind their ends.)
template <typename XT, typename WT>
cudaError_t launch_rows_type(RowsArgs a, cudaStream_t st)
{
    constexpr int XB = sizeof(XT);
    a.in_by = bytes_at_a_time(a.in, a.ld_in, a.D1, XB);
    a.base_by = a.base ? bytes_at_a_time(a.base, a.ld_base, a.D2, XB) : 16;
    a.out_by = a.out ? bytes_at_a_time(a.out, a.ld_out, a.D2, XB) : 16;
    a.vec_w2 = (uintptr_t)a.w2 % 16 == 0 && a.ld_w2 % (a.R <= 16 ? 4 : 8) == 0 && (a.R % (a.R <= 16 ? 4 : 8) == 0 || a.ld_w2 > a.R);
    a.vec_w1 = vectors(a.w1, a.ld_w1, a.ld_w1, sizeof(WT));
    const bool vec = a.vec_w1 && (!a.out || a.vec_w2) && a.in_by == 16 && a.base_by == 16 && a.out_by == 16;
#define FPQ_ROWS(RP) (vec ? launch_rows_as<XT, WT, RP, true>(a, st) : launch_rows_as<XT, WT, RP, false>(a, st))
    return a.R <= 16 ? FPQ_ROWS(16) : a.R <= 32 ? FPQ_ROWS(32) : a.R <= 64 ? FPQ_ROWS(64) : FPQ_ROWS(128);
#undef FPQ_ROWS
}

cudaError_t launch_rows(const RowsArgs& a, int x_type, int w_type, cudaStream_t st)
{
    bool tiles = adapter_tiles_preferred(a, x_type, w_type);
    if (tiles)
        return launch_adapter_tiles(a, x_type, w_type, st) == FPQ_OK ? cudaSuccess : cudaErrorUnknown;
    if (x_type == FPQ_BF16)
        return launch_rows_type<__nv_bfloat16, __nv_bfloat16>(a, st);
    if (x_type == FPQ_FP16)
        return launch_rows_type<__half, __half>(a, st);
    return w_type == FPQ_FP32   ? launch_rows_type<float, float>(a, st)
           : w_type == FPQ_BF16 ? launch_rows_type<float, __nv_bfloat16>(a, st)
                                : launch_rows_type<float, __half>(a, st);
}

int padded_rank(int R) { return R <= 16 ? 16 : R <= 32 ? 32 : R <= 64 ? 64 : 128; }

int column_tiles(int64_t n) { return (int)((n + 63) / 64); }

// How often the rows are split: two blocks for every SM, and 64 rows at least for a block's eight warps.  Of several adapters each gets
// its share of that (splits_of); the sums have room for four times as many blocks.
int grad_splits(int64_t M, int64_t N, int64_t K, int G)
{
    const int64_t tiles = column_tiles(K) + column_tiles(N), rounded_up = std::min(G - 1, 8) / 2;
    const int64_t most = std::min(M / 64, std::min(2 * 148 / tiles - rounded_up, 8 * 148 / (tiles * G)));
    return (int)std::max<int64_t>(most, 1);
}

template <typename XT, int RP, int JT>
cudaError_t launch_grad_as(const GradArgs& a, cudaStream_t st)
{
    using Ring = GradRing<XT, JT>;
    const size_t smem = std::max<size_t>((size_t)(WARPS / (RP / JT)) * 64 * (RP + 2) * 4, (size_t)WARPS * Ring::STAGES * Ring::STAGE);
    static std::atomic<uint64_t> known{0};
    return launch_cluster<GradArgs>(adapter_grad_kernel<XT, RP, JT>, known, (int)smem, grad_grid(a), 1, smem, st, a);
}

template <typename XT>
cudaError_t launch_grad(const GradArgs& a, cudaStream_t st)
{
    return a.R <= 16   ? launch_grad_as<XT, 16, 16>(a, st)
           : a.R <= 32 ? launch_grad_as<XT, 32, 32>(a, st)
           : a.R <= 64 ? launch_grad_as<XT, 64, 32>(a, st)
                       : launch_grad_as<XT, 128, 32>(a, st);
}

// rows of the transposed adapters, in elements: [G][K][ldr] and [G][R][ldn]
int padded_ranks(int R, int bytes) { return (int)round_up(R, bytes == 4 && R <= 16 ? 4 : 8); }
int padded_columns(int64_t N, int bytes) { return (int)round_up(N, 16 / bytes); }

template <typename T>
cudaError_t launch_transpose_as(const AdapterProblem& p, T* at, T* bt, uint32_t* tickets, int n_tickets, cudaStream_t st)
{
    const int64_t r = (p.R + 31) / 32, tiles_a = r * ((p.K + 31) / 32), tiles = tiles_a + r * ((p.N + 31) / 32);
    return launch_overlapped(transpose_adapters_kernel<T>, dim3((unsigned)(tiles * p.G)), THREADS, 0, st, (const T*)p.a, at, (const T*)p.b, bt,
                             p.R, (int)p.K, (int)p.N, padded_ranks(p.R, sizeof(T)), padded_columns(p.N, sizeof(T)), (int)tiles_a, (int)tiles, tickets, n_tickets);
}

size_t pad16(size_t n) { return (n + 15) / 16 * 16; }

// what the rows' pass of a backward call looks like; its weights are the transposed and padded ones
RowsArgs backward_rows(const AdapterProblem& p, const void* dy, int64_t ld_dy, const void* base, int64_t ld_base, void* dx, int64_t ld_dx, const void* at,
                       const void* bt)
{
    const int wb = type_bytes(p.w_type);
    RowsArgs a = {};
    a.in = dy; a.w1 = bt; a.w2 = at; a.scale = p.scale; a.offsets = p.offsets; a.ids = p.ids;
    a.base = base; a.out = dx; a.kept_scaled = 1;
    a.ld_w1 = padded_columns(p.N, wb); a.ld_w2 = padded_ranks(p.R, wb);
    a.M = p.M; a.D1 = p.N; a.D2 = p.K; a.ld_in = ld_dy; a.ld_base = ld_base; a.ld_out = ld_dx;
    a.G = p.G; a.R = p.R; a.S = p.S;
    return a;
}

const void* const ALIGNED = reinterpret_cast<const void*>((uintptr_t)256);     // never followed: only its alignment is looked at

}  // namespace

cudaError_t launch_adapter_forward(const AdapterProblem& p, const void* x, int64_t ldx, const void* base, int64_t ld_base, void* y,
                                   int64_t ldy, float* u, cudaStream_t st)
{
    RowsArgs a = {};
    a.in = x; a.w1 = p.a; a.w2 = p.b; a.scale = p.scale; a.offsets = p.offsets; a.ids = p.ids;
    a.base = base; a.out = y; a.kept = u;
    a.ld_w1 = p.K; a.ld_w2 = p.R;
    a.M = p.M; a.D1 = p.K; a.D2 = p.N; a.ld_in = ldx; a.ld_base = ld_base; a.ld_out = ldy;
    a.G = p.G; a.R = p.R; a.S = p.S;
    return launch_rows(a, p.x_type, p.w_type, st);
}

bool adapter_forward_by_tiles(const AdapterProblem& p, bool base)
{
    RowsArgs a = {};
    a.in = a.w1 = a.w2 = ALIGNED;
    a.out = (void*)ALIGNED;
    a.base = base ? ALIGNED : nullptr;
    a.ld_w1 = p.K; a.ld_w2 = p.R;
    a.M = p.M; a.D1 = a.ld_in = p.K; a.D2 = a.ld_out = a.ld_base = p.N; a.G = p.G; a.R = p.R; a.S = p.S;
    return p.M > 0 && p.S > 0 && adapter_tiles_preferred(a, p.x_type, p.w_type);
}

bool adapter_backward_by_tiles(const AdapterProblem& p, bool dx, bool base)
{
    const RowsArgs a = backward_rows(p, ALIGNED, p.N, dx && base ? ALIGNED : nullptr, p.K, dx ? (void*)ALIGNED : nullptr, p.K, ALIGNED, ALIGNED);
    return p.M > 0 && p.S > 0 && adapter_tiles_preferred(a, p.x_type, p.w_type);
}

// workspace: t [M][R] FP32, A and B transposed, the tickets and the sums of the blocks that share an adapter's rows
size_t adapter_backward_bytes(int64_t M, int64_t N, int64_t K, int G, int R, int w_type)
{
    const size_t wb = type_bytes(w_type), g = (size_t)G * wb;
    const size_t splits = grad_splits(M, N, K, G), tiles = (size_t)G * (column_tiles(K) + column_tiles(N));
    size_t blocks = splits == 1 ? 0 : splits * tiles * 64;
    if (w_type == FPQ_BF16)                                // (of rows in BF16, or in FP32)
        blocks = std::max(blocks, adapter_grad_tile_columns(M, N, K, G, R));
    const size_t sums = blocks == 0 ? 0 : pad16(tiles * 4) + blocks * padded_rank(R) * 4;
    return pad16((size_t)M * R * 4) + pad16(g * K * padded_ranks(R, (int)wb)) + pad16(g * R * padded_columns(N, (int)wb)) + sums;
}

cudaError_t launch_adapter_backward(const AdapterProblem& p, const void* dy, int64_t ld_dy, const void* x, int64_t ldx, const float* u,
                                    const void* base, int64_t ld_base, void* dx, int64_t ld_dx, float* da, float* db, void* workspace,
                                    cudaStream_t st)
{
    float* t = (float*)workspace;
    const size_t wb = type_bytes(p.w_type);
    const int xb = type_bytes(p.x_type);
    uint8_t* at = (uint8_t*)workspace + pad16((size_t)p.M * p.R * 4);
    uint8_t* bt = at + pad16((size_t)p.G * p.K * padded_ranks(p.R, (int)wb) * wb);
    uint32_t* tickets = (uint32_t*)(bt + pad16((size_t)p.G * p.R * padded_columns(p.N, (int)wb) * wb));
    GradArgs b = {};
    b.x = x; b.dy = dy; b.t = t; b.u = u; b.offsets = p.offsets; b.ids = p.ids; b.da = da; b.db = db;
    b.M = p.M; b.N = p.N; b.K = p.K; b.ldx = ldx; b.ld_dy = ld_dy; b.G = p.G; b.R = p.R; b.S = p.M > 0 ? p.S : 0;
    b.scale = b.S > 0 ? p.scale : nullptr;                 // (without rows the callers have not looked at the scales)
    b.x_by = bytes_at_a_time(x, ldx, p.K, xb);
    b.dy_by = bytes_at_a_time(dy, ld_dy, p.N, xb);
    b.tiles_k = column_tiles(p.K);
    b.tiles = b.tiles_k + column_tiles(p.N);
    b.tickets = tickets;
    const bool by_tiles = b.S > 0 && p.x_type == FPQ_BF16 && adapter_grad_tiles_preferred(b);
    b.splits = b.S == 0 ? 1 : by_tiles ? adapter_grad_tile_splits(p.M, p.N, p.K, p.G, p.R) : grad_splits(p.M, p.N, p.K, p.G);
    const int n_tickets = b.splits > 1 ? p.G * b.tiles : 0;    // (below 2^27)
    b.sums = (float*)((uint8_t*)tickets + pad16((size_t)n_tickets * 4));
    if (p.M > 0 && p.S > 0) {
        cudaError_t e = wb == 4 ? launch_transpose_as(p, (uint32_t*)at, (uint32_t*)bt, tickets, n_tickets, st)
                                : launch_transpose_as(p, (uint16_t*)at, (uint16_t*)bt, tickets, n_tickets, st);
        if (e != cudaSuccess)
            return e;
        RowsArgs a = backward_rows(p, dy, ld_dy, base, ld_base, dx, ld_dx, at, bt);
        a.kept = t;
        e = launch_rows(a, p.x_type, p.w_type, st);
        if (e != cudaSuccess)
            return e;
    }
    if (by_tiles)
        return launch_adapter_grad_tiles(b, st);
    return p.x_type == FPQ_FP32 ? launch_grad<float>(b, st) : p.x_type == FPQ_BF16 ? launch_grad<__nv_bfloat16>(b, st) : launch_grad<__half>(b, st);
}

}  // namespace fpq
