// The adapters' pass from rows to t and back for requests of many rows, on the 5th-generation tensor cores.
//
// A block (or a cluster of two, sharing the reduction and the output columns) takes 128 rows of one request:
//   1. t = x W1^T: both come by TMA in stages of 128 bytes of every row, and an MMA of 128 x rank accumulates in tensor memory.  FP32:
//      the tensor core reads the tiles as loaded as their TF32 heads, the other warps write what that leaves off beside them, and
//      three products make one (two for 16-bit weights, which the warps write as FP32).  16-bit rows are multiplied as they are.
//   2. The warps add the accumulators of a few stages each up in registers (the tensor core cuts its sums off), and write s t
//      as an MMA operand of two terms: TF32 heads and tails, or two BF16.
//   3. y = base + t W2^T in chunks of 64 columns, by groups of four warps in turn: W2's chunk comes by TMA, the MMA goes to tensor
//      memory, and every warp adds its 32 rows to base, which came by TMA, in place in shared memory, from where TMA stores
//      them (the rows of a request's last tile, which are fewer, are stored by the warp).
// Bound by memory: 18944 x 64 -> 2560, BF16, rank 64, one block for every SM: 44 us, 4.4 TB/s; the pass by warps (fpq_adapter.cu), which
// spends some 300 instructions on 16 x 32 values, 95 us.  A wave of blocks has some 7 us of its own (finding the tile, the first copies,
// the step from t to y).  32768 x 320 -> 2560, two blocks on an SM: 76 to 80 us against 159.
#include <math.h>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "fpq_adapter.cuh"
#include "fpq_adapter_layout.h"

namespace fpq {

namespace {

template <typename XT, typename WT, int RP, bool TWO>
using TileLayout = TileSizes<(int)sizeof(XT), (int)sizeof(WT), std::is_same<XT, __nv_bfloat16>::value, RP, TWO>;

struct TileArgs {
    RowsArgs a;
    int* status;
    uint32_t idesc1, idesc2;
};

__device__ __forceinline__ void tma_store_2d(const void* tmap, uint32_t src, int c0, int c1)
{
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];"
                 ::"l"(tmap), "r"(src), "r"(c0), "r"(c1)
                 : "memory");
}

// D (+)= A B; acc == 0 overwrites D
template <bool F16>
__device__ __forceinline__ void mma_tile(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t acc)
{
    if (F16)
        asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
                     "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}"
                     ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(SMEM_DESC_HI_K_SW128), "r"(idesc), "r"(acc)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
                     "tcgen05.mma.cta_group::1.kind::tf32 [%0], da, db, %4, p;\n\t}"
                     ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(SMEM_DESC_HI_K_SW128), "r"(idesc), "r"(acc)
                     : "memory");
}

// What an FP32 number loses when the tensor core reads it as TF32 (the low 13 mantissa bits are ignored): exact, and half a step of its own
// TF32 more, so that the core's cutting off rounds it.  (Heads and tails that are all cut off make a product 1.4e-7 smaller on average.
// Of a number that is not finite the head alone makes the sum not finite.)
__device__ __forceinline__ float tail(float x)
{
    return __uint_as_float(__float_as_uint(x - __uint_as_float(__float_as_uint(x) & 0xffffe000u)) + 0x1000u);
}

// N 16-byte pieces of FP32 numbers and, at the same places, what TF32 leaves off of them
template <int N, int THREADS_>
__device__ __forceinline__ void tails(const uint8_t* from, uint8_t* to, int tid)
{
#pragma unroll
    for (int i = 0; i < (N + THREADS_ - 1) / THREADS_; ++i) {
        const int e = tid + i * THREADS_;
        if (N % THREADS_ == 0 || e < N) {
            const float4 v = reinterpret_cast<const float4*>(from)[e];
            reinterpret_cast<float4*>(to)[e] = make_float4(tail(v.x), tail(v.y), tail(v.z), tail(v.w));
        }
    }
}

// ROWS rows of ACROSS x 4 16-bit numbers, side by side, as an operand of FP32 numbers (blocks of ROWS x 128 bytes)
template <int ROWS, int ACROSS, int THREADS_, typename WT>
__device__ __forceinline__ void widen(const uint8_t* from, uint8_t* to, int tid)
{
#pragma unroll
    for (int i = 0; i < (ROWS * ACROSS + THREADS_ - 1) / THREADS_; ++i) {
        const int e = tid + i * THREADS_, r = e / ACROSS, c = e % ACROSS;
        if (ROWS * ACROSS % THREADS_ == 0 || e < ROWS * ACROSS) {
            const uint2 w = reinterpret_cast<const uint2*>(from)[e];
            float v[4];
            unpack(w.x, v, WT());
            unpack(w.y, v + 2, WT());
            *reinterpret_cast<float4*>(to + c / 8 * (ROWS * 128) + swizzled(r, c % 8)) = make_float4(v[0], v[1], v[2], v[3]);
        }
    }
}
template <typename XT, typename WT, int RP, bool TWO>
__global__ void __launch_bounds__(TileLayout<XT, WT, RP, TWO>::THREADS, TWO ? 2 : 1) adapter_tile_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w1,
                                                                       const __grid_constant__ CUtensorMap tm_w2, const __grid_constant__ CUtensorMap tm_base,
                                                                       const __grid_constant__ CUtensorMap tm_out, const TileArgs g)
{
    using T = TileLayout<XT, WT, RP, TWO>;
    constexpr bool NATIVE = !T::FP32, F16_2 = T::BF;
    constexpr int STAGES = T::STAGES, CHUNK = T::CHUNK, SLOTS = T::SLOTS, GROUPS = T::GROUPS, WORK_WARPS = T::WORK_WARPS, SHARE = RP / GROUPS, SETS = T::W2_SETS;
    const RowsArgs& a = g.a;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base_addr = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base_addr - smem_u32(smem_raw));
    const uint32_t bars = base_addr + (uint32_t)T::barriers_at((int)(base_addr - smem_u32(smem_raw)));
    const uint32_t full = bars + T::FULL, empty = bars + T::EMPTY, ready = bars + T::READY, t_full = bars + T::T_FULL, t_free = bars + T::T_FREE,
                   t_ready = bars + T::T_READY, t_done = bars + T::T_DONE, w_full = bars + T::W_FULL, w_empty = bars + T::W_EMPTY, w_ready = bars + T::W_READY,
                   y_full = bars + T::Y_FULL, slot_full = bars + T::SLOT_FULL;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem_raw + (bars + T::TMEM_WORD - smem_u32(smem_raw)));
    if (threadIdx.x == 0) {
        tma_prefetch_desc(&tm_x);
        tma_prefetch_desc(&tm_w1);
        tma_prefetch_desc(&tm_w2);
        tma_prefetch_desc(&tm_base);
        tma_prefetch_desc(&tm_out);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t rank = cluster_rank(), C;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
    const TileRows tr = find_tile(TILE_M, blockIdx.x / C, a.offsets, a.ids, a.S, a.G, a.M);
    if (tr.rows <= 0)
        return;                                            // (every block of the cluster leaves)
    const bool active = tr.id >= 0;
    const int D1 = (int)a.D1, D2 = (int)a.D2, R = a.R;
    const int all_stages = (D1 + T::KE - 1) / T::KE, all_chunks = a.out ? (D2 + NCOLS - 1) / NCOLS : 0;
    const int s_lo = (int)((int64_t)all_stages * rank / C), n_stages = active ? (int)((int64_t)all_stages * (rank + 1) / C) - s_lo : 0;
    const int c_lo = (int)((int64_t)all_chunks * rank / C), n_chunks = (int)((int64_t)all_chunks * (rank + 1) / C) - c_lo;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
            if (T::FP32)
                mbar_init(ready + 8 * s, WORK_WARPS);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(t_full + 8 * b, 1);
            mbar_init(t_free + 8 * b, WORK_WARPS);
        }
        for (int b = 0; b < SETS; ++b) {
            mbar_init(w_full + 8 * b, 1);
            mbar_init(w_empty + 8 * b, 1);
        }
        for (int b = 0; b < GROUPS; ++b) {
            mbar_init(w_ready + 8 * b, 4);
            mbar_init(y_full + 8 * b, 1);
        }
        mbar_init(t_ready, WORK_WARPS);
        mbar_init(t_done, 1);
        for (int s = 0; s < WORK_WARPS * SLOTS; ++s)
            mbar_init(slot_full + 8 * s, 1);
        fence_barrier_init();
    }
    if (warp == 1) {
        tmem_alloc(smem_u32((const void*)tmem_slot), T::TMEM);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // (behind the allocation: a block of the next kernel that moves in could otherwise hold the tensor memory that this one waits for)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t tmem = *tmem_slot;
    bool dead = false;

    if (warp == 0) {
        // ---------------- x, W1 and W2 by TMA ----------------
        const bool copier = elect_one();
        if (copier && active) {
            uint32_t s = 0, ph = 0;
            int k = 0;
            for (; k < n_stages; ++k) {
                if (!mbar_wait(empty + 8 * s, ph ^ 1)) { dead = true; break; }
                mbar_expect_tx(full + 8 * s, X_BYTES + T::W_RAW);
                tma_load_2d(base_addr + s * T::STAGE, &tm_x, full + 8 * s, (s_lo + k) * T::KE, (int)tr.row);
                // (rows behind the adapter's last rank are the next one's: the columns of t that they give are set to zero)
                tma_load_2d(base_addr + s * T::STAGE + T::X_PART, &tm_w1, full + 8 * s, (s_lo + k) * T::KE, tr.id * R);
                if (++s == STAGES) { s = 0; ph ^= 1; }
            }
            if (dead)                                      // the copies in flight end before the block does
                for (int i = max(k - STAGES, 0); i < k; ++i)
                    mbar_wait(full + 8 * (i % STAGES), (i / STAGES) & 1);
        }
        __syncwarp();
        if (active && C > 1) {
            cluster_sync_all();
            cluster_sync_all();
        }
        if (copier && active && n_chunks > 0 && !dead) {
            // W2's sets lie where the stages were: they are free when the last MMA on these has ended.  (A barrier of its own, with one
            // phase: of t_full this thread has not seen the phases in between, and a parity alone does not tell them apart.)
            int j = 0;
            if (n_stages > 0 && !mbar_wait(t_done, 0))
                dead = true;
            for (; j < n_chunks && !dead; ++j) {
                const uint32_t set = j % SETS, at = base_addr + T::W2_BASE + set * T::W2_SET;
                if (!mbar_wait(w_empty + 8 * set, ((j / SETS) & 1) ^ 1)) { dead = true; break; }
                mbar_expect_tx(w_full + 8 * set, T::W2_RAW);
                // (rows behind the adapter's last column are the next one's: they give columns that y does not have)
                const int n = tr.id * D2 + (c_lo + j) * NCOLS;
                tma_load_2d(at, &tm_w2, w_full + 8 * set, 0, n);
                if (T::W2_RAW > NCOLS * 128)
                    tma_load_2d(at + NCOLS * 128, &tm_w2, w_full + 8 * set, 32, n);
            }
            if (dead)
                for (int i = max(j - SETS, 0); i < j; ++i)
                    mbar_wait(w_full + 8 * (i % SETS), (i / SETS) & 1);
        }
        if (dead)
            flag_status(g.status, FPQ_ERR_TIMEOUT);
        __syncwarp();
    } else if (warp == 1) {
        // ---------------- MMAs ----------------
        const bool issuer = elect_one();
        if (issuer && active) {
            uint32_t s = 0, ph = 0;
            for (int k = 0; k < n_stages; ++k) {
                const int chunk = k / CHUNK;
                const uint32_t buf = chunk & 1;
                if (k % CHUNK == 0) {
                    // a fresh accumulator: the warps must have added up what it held two chunks ago
                    if (chunk >= 2 && !mbar_wait(t_free + 8 * buf, ((chunk >> 1) - 1) & 1)) { dead = true; break; }
                    tc_fence_after();
                }
                if (!mbar_wait(full + 8 * s, ph) || (T::FP32 && !mbar_wait(ready + 8 * s, ph))) { dead = true; break; }
                tc_fence_after();
                const uint32_t st = base_addr + s * T::STAGE, d = tmem + buf * RP, wt = st + T::X_PART;
                // FP32 weights: as loaded, and their tails behind; 16-bit ones of FP32 rows: what they are in FP32 behind
                const uint32_t x = smem_desc_lo(st), xl = smem_desc_lo(st + X_BYTES),
                               w = smem_desc_lo(T::FP32 && !T::WIDE_W ? wt + T::W_RAW : wt), wl = smem_desc_lo(wt + T::W_RAW);
                // (32 bytes of every row at a time.  What the heads leave off comes first: each MMA cuts the running sum off, and those on the small
                // sum of the tails cost nothing.)
                uint32_t acc = k % CHUNK != 0;
                if (T::FP32)
#pragma unroll
                    for (uint32_t kk = 0; kk < 4; ++kk) {
                        mma_tile<false>(d, xl + 2 * kk, w + 2 * kk, g.idesc1, acc);
                        if (T::WIDE_W)
                            mma_tile<false>(d, x + 2 * kk, wl + 2 * kk, g.idesc1, 1);
                        acc = 1;
                    }
#pragma unroll
                for (uint32_t kk = 0; kk < 4; ++kk) {
                    mma_tile<NATIVE>(d, x + 2 * kk, w + 2 * kk, g.idesc1, acc);
                    acc = 1;
                }
                mma_commit(empty + 8 * s);                 // the stage is free once these MMAs have read it
                if (++s == STAGES) { s = 0; ph ^= 1; }
                if ((k + 1) % CHUNK == 0 || k + 1 == n_stages)
                    mma_commit(t_full + 8 * buf);
                if (k + 1 == n_stages)
                    mma_commit(t_done);
            }
        }
        __syncwarp();
        if (active && C > 1) {
            cluster_sync_all();
            cluster_sync_all();
        }
        if (issuer && active && !dead && n_chunks > 0) {
            if (!mbar_wait(t_ready, 0))
                dead = true;
            const uint32_t th = smem_desc_lo(base_addr), tl = smem_desc_lo(base_addr + T::T_BYTES);
            for (int j = 0; j < n_chunks && !dead; ++j) {
                const uint32_t set = j % SETS, y = j % GROUPS;
                if (!mbar_wait(w_full + 8 * set, (j / SETS) & 1) || !mbar_wait(w_ready + 8 * y, (j / GROUPS) & 1)) { dead = true; break; }
                tc_fence_after();
                const uint32_t raw = base_addr + T::W2_BASE + set * T::W2_SET, w = T::BF || T::WIDE_W ? raw : raw + T::W2_RAW, d = tmem + y * NCOLS;
#pragma unroll
                for (uint32_t kk = 0; kk < T::T_ROW / 32; ++kk) {      // (the tails first here too)
                    const uint32_t b = kk / 4, o = 2 * (kk % 4), at = b * (TILE_M * 128 / 16) + o;
                    mma_tile<F16_2>(d, tl + at, smem_desc_lo(w + b * (NCOLS * 128)) + o, g.idesc2, kk != 0);
                    if (T::WIDE_W && !T::BF)
                        mma_tile<F16_2>(d, th + at, smem_desc_lo(raw + T::W2_RAW + b * (NCOLS * 128)) + o, g.idesc2, 1);
                }
#pragma unroll
                for (uint32_t kk = 0; kk < T::T_ROW / 32; ++kk) {
                    const uint32_t b = kk / 4, o = 2 * (kk % 4);
                    mma_tile<F16_2>(d, th + b * (TILE_M * 128 / 16) + o, smem_desc_lo(w + b * (NCOLS * 128)) + o, g.idesc2, 1);
                }
                mma_commit(w_empty + 8 * set);
                mma_commit(y_full + 8 * y);
            }
        }
        if (dead)
            flag_status(g.status, FPQ_ERR_TIMEOUT);
        __syncwarp();
    } else {
        // ---------------- sixteen warps ----------------
        const int w = warp - 2, tid = threadIdx.x - 64, quarter = warp & 3, group = w >> 2, row = quarter * 32 + lane;
        const int rows_here = tr.rows - quarter * 32;      // of this warp's 32
        const WT* w1 = (const WT*)a.w1 + (int64_t)max(tr.id, 0) * R * a.ld_w1;
        const WT* w2 = (const WT*)a.w2 + (int64_t)max(tr.id, 0) * D2 * a.ld_w2;
        uint8_t* slots = smem + T::SLOT_BASE + w * SLOTS * SLOT_BYTES;
        const uint32_t slots_addr = base_addr + T::SLOT_BASE + w * SLOTS * SLOT_BYTES, my_full = slot_full + 8 * SLOTS * w;

        // base and y: this warp's 32 rows in pieces of 128 bytes; of its group's chunks, every second
        constexpr int PER_CHUNK = T::FP32 ? 2 : 1, COLS = NCOLS / PER_CHUNK;
        const int my_chunks = rows_here > 0 && n_chunks > group ? (n_chunks - group - 1) / GROUPS + 1 : 0, pieces = my_chunks * PER_CHUNK;
        const bool based = a.base != nullptr;
        auto piece_col = [&](int i) { return (c_lo + group + GROUPS * (i / PER_CHUNK)) * NCOLS + (i % PER_CHUNK) * COLS; };
        auto fetch_base = [&](int i) {                     // lane 0
            if (based && i < pieces) {
                const uint32_t bar = my_full + 8 * (i % SLOTS);
                mbar_expect_tx(bar, SLOT_BYTES);
                tma_load_2d(slots_addr + (i % SLOTS) * SLOT_BYTES, &tm_base, bar, piece_col(i), (int)tr.row + quarter * 32);
            }
        };
        constexpr int FETCH = SLOTS == 1 ? 1 : SLOTS - 1;  // with several slots the one behind a store stays free for it
        if (lane == 0)
            for (int i = 0; i < FETCH; ++i)
                fetch_base(i);
        int fetched = min(FETCH, pieces);                  // (with a base)

        if (active) {
            float sum[SHARE];
#pragma unroll
            for (int i = 0; i < SHARE; ++i)
                sum[i] = 0.f;
            const float scale = a.scale ? a.scale[tr.id] : 1.f;
            int drained = 0;
            auto drain = [&](int c) {
                const uint32_t buf = c & 1;
                if (!mbar_wait(t_full + 8 * buf, (c >> 1) & 1)) { dead = true; return; }
                tc_fence_after();
                uint32_t r[SHARE];
                tmem_load<SHARE>(tmem + buf * RP + group * SHARE + ((uint32_t)(quarter * 32) << 16), r);
                tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < SHARE; ++i)
                    sum[i] += __uint_as_float(r[i]);
                tc_fence_before();
                __syncwarp();
                if (lane == 0)
                    mbar_arrive(t_free + 8 * buf);
            };
            uint32_t s = 0, ph = 0;
            if constexpr (T::FP32)
                for (int k = 0; k < n_stages && !dead; ++k) {
                    if (!mbar_wait(full + 8 * s, ph)) { dead = true; break; }
                    uint8_t *st = smem + s * T::STAGE, *wt = st + T::X_PART;
                    tails<X_BYTES / 16, 32 * WORK_WARPS>(st, st + X_BYTES, tid);
                    if constexpr (T::WIDE_W)
                        tails<RP * 8, 32 * WORK_WARPS>(wt, wt + T::W_RAW, tid);
                    else
                        widen<RP, 8, 32 * WORK_WARPS, WT>(wt, wt + T::W_RAW, tid);
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0)
                        mbar_arrive(ready + 8 * s);
                    if (++s == STAGES) { s = 0; ph ^= 1; }
                    // a stage later the previous chunk's MMAs are done
                    if (k % CHUNK == 0 && k / CHUNK > drained)
                        drain(drained++);
                }
            while (!dead && drained < (n_stages + CHUNK - 1) / CHUNK)
                drain(drained++);

            // t: every rank's sums through the cluster, then kept in FP32 and written as the second MMA's operand
            float* kept = reinterpret_cast<float*>(smem + T::KEPT_BASE);      // [128][RP]
            float* mine = kept + row * RP + group * SHARE;
            if (C > 1) {
#pragma unroll
                for (int i = 0; i < SHARE; i += 4)
                    *reinterpret_cast<float4*>(mine + i) = make_float4(sum[i], sum[i + 1], sum[i + 2], sum[i + 3]);
                __syncwarp();
                cluster_sync_all();
#pragma unroll
                for (int i = 0; i < SHARE; ++i)
                    sum[i] = 0.f;
                for (uint32_t c = 0; c < C; ++c) {
                    const uint32_t from = peer_smem_addr(smem_u32(mine), c);
#pragma unroll
                    for (int i = 0; i < SHARE; i += 4) {
                        const float4 v = ld_cluster_smem4(from + 4 * i);
                        sum[i] += v.x; sum[i + 1] += v.y; sum[i + 2] += v.z; sum[i + 3] += v.w;
                    }
                }
                __syncwarp();
                cluster_sync_all();                        // (nobody reads these sums any more)
            }
            float zero[4] = {};                            // become NaN if a sum is not finite
#pragma unroll
            for (int i = 0; i < SHARE; ++i)
                zero[i % 4] = fmaf(sum[i], 0.f, zero[i % 4]);
            if ((zero[0] + zero[1]) + (zero[2] + zero[3]) != 0.f && row < tr.rows) {
                // (kept out of the way of what runs for every tile: an instruction cache holds it all)
#pragma unroll
                for (int i = 0; i < SHARE; ++i)
                    mine[i] = sum[i];
                const XT* x = (const XT*)a.in + (tr.row + row) * a.ld_in;
#pragma unroll 1
                for (int j = group * SHARE; j < min(group * SHARE + SHARE, R); ++j) {
                    float v = mine[j - group * SHARE];
                    if (!finite(v)) {
                        v = 0.f;
#pragma unroll 1
                        for (int k = 0; k < D1; ++k)
                            v = fmaf(as_float(x[k]), as_float(w1[j * a.ld_w1 + k]), v);
                        mine[j - group * SHARE] = v;
                    }
                }
#pragma unroll
                for (int i = 0; i < SHARE; ++i)
                    sum[i] = mine[i];
            }
#pragma unroll
            for (int i = 0; i < SHARE; ++i)
                if (group * SHARE + i >= R || row >= tr.rows)
                    sum[i] = 0.f;
            float st[SHARE];
#pragma unroll
            for (int i = 0; i < SHARE; ++i)
                st[i] = sum[i] * scale;
#pragma unroll
            for (int i = 0; i < SHARE; i += 4)
                *reinterpret_cast<float4*>(mine + i) = make_float4(st[i], st[i + 1], st[i + 2], st[i + 3]);
            if (T::BF) {
#pragma unroll
                for (int i = 0; i < SHARE; i += 4) {
                    uint32_t h[2], l[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        split_bf16(st[i + 2 * e], st[i + 2 * e + 1], h[e], l[e]);
                    const int j = group * SHARE + i, at = swizzled(row, j / 8) + j % 8 * 2;
                    *reinterpret_cast<uint2*>(smem + at) = make_uint2(h[0], h[1]);
                    *reinterpret_cast<uint2*>(smem + T::T_BYTES + at) = make_uint2(l[0], l[1]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < SHARE; i += 4) {
                    const int j = group * SHARE + i, at = j / 32 * (TILE_M * 128) + swizzled(row, j % 32 / 4);
                    *reinterpret_cast<float4*>(smem + at) = make_float4(st[i], st[i + 1], st[i + 2], st[i + 3]);
                    *reinterpret_cast<float4*>(smem + T::T_BYTES + at) = make_float4(tail(st[i]), tail(st[i + 1]), tail(st[i + 2]), tail(st[i + 3]));
                }
            }
            fence_proxy_async();
            asm volatile("bar.sync 1, %0;" ::"n"(32 * WORK_WARPS) : "memory");                    // all of t is there, for the odd sums too
            if (lane == 0)
                mbar_arrive(t_ready);
            if (a.kept && rank == 0 && row < tr.rows) {    // (while the MMAs begin)
                float* k = a.kept + (tr.row + row) * R + group * SHARE;
                if (R % 4 == 0 && (reinterpret_cast<uintptr_t>(a.kept) & 15) == 0) {
#pragma unroll
                    for (int i = 0; i < SHARE; i += 4)
                        if (group * SHARE + i < R)
                            *reinterpret_cast<float4*>(k + i) = a.kept_scaled ? make_float4(st[i], st[i + 1], st[i + 2], st[i + 3])
                                                                              : make_float4(sum[i], sum[i + 1], sum[i + 2], sum[i + 3]);
                } else {
#pragma unroll
                    for (int i = 0; i < SHARE; ++i)
                        if (group * SHARE + i < R)
                            k[i] = a.kept_scaled ? st[i] : sum[i];
                }
            }
        } else if (a.kept && rank == 0) {
            for (int i = tid; i < tr.rows * R; i += 32 * WORK_WARPS)
                a.kept[tr.row * R + i] = 0.f;
        }

        // y: this group's chunks, while the MMAs of the other groups' run
        const int gid = tid & 127;
        auto prepare = [&](int j) {                        // W2's chunk j as an operand; the accumulator that it gets has been read
            const int set = j % SETS;
            if constexpr (!T::BF) {
                if (!mbar_wait(w_full + 8 * set, (j / SETS) & 1)) { dead = true; return; }
                uint8_t* raw = smem + T::W2_BASE + set * T::W2_SET;
                if constexpr (T::WIDE_W)
                    tails<T::W2_BYTES / 16, 128>(raw, raw + T::W2_RAW, gid);
                else
                    widen<NCOLS, RP / 4, 128, WT>(raw, raw + T::W2_RAW, gid);
                fence_proxy_async();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0)
                mbar_arrive(w_ready + 8 * (j % GROUPS));
        };
        XT* out = (XT*)a.out + (tr.row + quarter * 32) * a.ld_out;
        int piece = 0;
        if (active && n_chunks > group && !dead)
            prepare(group);
        for (int j = group; j < n_chunks; j += GROUPS) {
            const uint32_t tmem_y = tmem + j % GROUPS * NCOLS;
            if (active && !dead) {
                if (!mbar_wait(y_full + 8 * (j % GROUPS), (j / GROUPS) & 1))
                    dead = true;
                tc_fence_after();
            }
#pragma unroll
            for (int part = 0; part < PER_CHUNK; ++part, ++piece) {
                if (rows_here <= 0 || dead)
                    break;
                const int col = piece_col(piece), slot = piece % SLOTS;
                uint8_t* sl = slots + slot * SLOT_BYTES;
                if (based) {
                    if (!mbar_wait(my_full + 8 * slot, (piece / SLOTS) & 1)) { dead = true; break; }
                }
                float zero[4] = {};                        // become NaN if a sum is not finite
                constexpr int PER = 16 / (int)sizeof(XT);
#pragma unroll
                for (int i = 0; i < COLS; i += 32) {
                    uint32_t acc[32];
                    if (active) {
                        tmem_load<32>(tmem_y + part * COLS + i + ((uint32_t)(quarter * 32) << 16), acc);
                        tmem_ld_wait();
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            acc[e] = 0;
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        zero[e % 4] = fmaf(__uint_as_float(acc[e]), 0.f, zero[e % 4]);
#pragma unroll
                    for (int c = 0; c < 32 / PER; ++c) {
                        uint4* p = reinterpret_cast<uint4*>(sl + swizzled(lane, i / PER + c));
                        alignas(16) XT v[PER];
                        if (based)
                            *reinterpret_cast<uint4*>(v) = *p;
#pragma unroll
                        for (int e = 0; e < PER; ++e)
                            v[e] = from_float<XT>((based ? as_float(v[e]) : 0.f) + __uint_as_float(acc[c * PER + e]));
                        *p = *reinterpret_cast<const uint4*>(v);
                    }
                }
                if ((zero[0] + zero[1]) + (zero[2] + zero[3]) != 0.f && row < tr.rows) {
                    // what is not finite again by multiply-adds
                    const float* t = reinterpret_cast<const float*>(smem + T::KEPT_BASE) + row * RP;
                    const XT* b = based ? (const XT*)a.base + (tr.row + row) * a.ld_base + col : nullptr;
#pragma unroll 1
                    for (int i = 0; i < min(COLS, D2 - col); ++i) {
                        XT& y = reinterpret_cast<XT*>(sl + swizzled(lane, i / PER))[i % PER];
                        if (finite(as_float(y)))
                            continue;
                        float v = 0.f;
#pragma unroll 1
                        for (int k = 0; k < R; ++k)
                            v = fmaf(t[k], as_float(w2[(col + i) * a.ld_w2 + k]), v);
                        y = from_float<XT>((b ? as_float(b[i]) : 0.f) + v);
                    }
                }
                if (rows_here >= 32) {
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0)
                        tma_store_2d(&tm_out, slots_addr + slot * SLOT_BYTES, col, (int)tr.row + quarter * 32);
                } else {
                    __syncwarp();
#pragma unroll 1
                    for (int e = lane; e < rows_here * 8; e += 32) {
                        const int r = e >> 3, c = e & 7;
                        if (col + c * PER < D2)
                            *reinterpret_cast<uint4*>(out + r * a.ld_out + col + c * PER) = *reinterpret_cast<const uint4*>(sl + swizzled(r, c));
                    }
                    fence_proxy_async();
                    __syncwarp();
                }
                if (lane == 0) {
                    // the slot in front of this one is free once its store has read it: the next piece of base goes there
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(SLOTS == 1 ? 0 : 1) : "memory");
                    fetch_base(piece + FETCH);
                }
                fetched = min(piece + FETCH + 1, pieces);
                __syncwarp();
            }
            if (active && j + GROUPS < n_chunks && !dead)
                prepare(j + GROUPS);
        }
        if (dead) {
            flag_status(g.status, FPQ_ERR_TIMEOUT);
            if (based)                                     // the copies in flight end before the block does
                for (int i = piece; i < fetched; ++i)
                    mbar_wait(my_full + 8 * (i % SLOTS), (i / SLOTS) & 1);
        }
        if (lane == 0)
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, T::TMEM);
    }
}

int64_t tiles_of(const RowsArgs& a) { return (a.M + TILE_M - 1) / TILE_M + a.S - 1; }

// Up to a tile for every SM one block on each, two sharing a tile's columns where the tiles are at most half as many; more tiles: two blocks on
// each SM, one of which loads while the other stores (65536 rows, 640 -> 2560, BF16, rank 64: 156 us against 167; 8192 rows: 42 against 33).
int cluster_of(const RowsArgs& a) { return tiles_of(a) <= 74 ? 2 : 1; }
bool two_on_an_sm(const RowsArgs& a, int x_type) { return tiles_of(a) > 148 && (a.R <= 32 || x_type == FPQ_BF16); }

template <typename XT, typename WT, int RP, bool TWO>
fpq_status launch_as(const RowsArgs& a, int x_type, int w_type, cudaStream_t st)
{
    using T = TileLayout<XT, WT, RP, TWO>;
    static_assert(T::SMEM <= 232448, "shared memory");
    static_assert(2 * RP <= T::TMEM && T::GROUPS * NCOLS <= T::TMEM, "tensor memory");
    static_assert(!TWO || 2 * (T::SMEM + 1024) <= 233472, "two blocks on an SM");
    EncodeTiledFn enc = tensor_map_encoder();
    TileArgs g;
    g.a = a;
    g.status = status_word();
    int dev = 0;
    if (!enc || !g.status || cudaGetDevice(&dev) != cudaSuccess)
        return FPQ_ERR_CUDA;
    static std::atomic<uint64_t> known{0};
    if (dev >= 64 || !(known.load(std::memory_order_relaxed) >> dev & 1)) {
        if (cudaFuncSetAttribute(adapter_tile_kernel<XT, WT, RP, TWO>, cudaFuncAttributeMaxDynamicSharedMemorySize, T::SMEM) != cudaSuccess)
            return FPQ_ERR_CUDA;
        if (dev < 64)
            known.fetch_or((uint64_t)1 << dev);
    }
    CUtensorMap tx, t1, t2, tb, ty;
    const void* out = a.out ? a.out : a.in;                // (without an output the maps of W2, base and output are not used)
    const int64_t width = a.out ? a.D2 : a.D1, ld = a.out ? a.ld_out : a.ld_in;
    const int xe = 128 / (int)sizeof(XT);
    const bool raw1 = T::FP32 && !T::WIDE_W, raw2 = !T::BF && !T::WIDE_W;
    if (!encode_rows(enc, &tx, a.in, a.M, a.D1, a.ld_in, x_type, TILE_M, xe, true) || !encode_rows(enc, &ty, out, a.M, width, ld, x_type, 32, xe, true) ||
        !encode_rows(enc, &tb, a.out && a.base ? a.base : out, a.M, width, a.out && a.base ? a.ld_base : ld, x_type, 32, xe, true) ||
        !encode_rows(enc, &t1, a.w1, (int64_t)a.G * a.R, a.D1, a.ld_w1, w_type, RP, raw1 ? 32 : xe, !raw1))
        return FPQ_ERR_CUDA;
    if (!a.out)
        t2 = t1;
    else if (!encode_rows(enc, &t2, a.w2, (int64_t)a.G * a.D2, a.R, a.ld_w2, w_type, NCOLS, raw2 ? RP : 128 / (int)sizeof(WT), !raw2))
        return FPQ_ERR_CUDA;
    // FP32 accumulators; operands BF16 (1), FP16 (0) or TF32 (2), K-major; M = 128, N = the rank, or 64 columns
    const uint32_t f1 = x_type == FPQ_FP32 ? 2 : x_type == FPQ_BF16 ? 1 : 0, f2 = T::BF ? 1 : 2;
    g.idesc1 = (1u << 4) | (f1 << 7) | (f1 << 10) | ((uint32_t)(RP >> 3) << 17) | ((uint32_t)(TILE_M >> 4) << 24);
    g.idesc2 = (1u << 4) | (f2 << 7) | (f2 << 10) | ((uint32_t)(NCOLS >> 3) << 17) | ((uint32_t)(TILE_M >> 4) << 24);
    const int c = cluster_of(a);
    const int64_t tiles = a.M / TILE_M + a.S;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * c));
    cfg.blockDim = dim3(T::THREADS);
    cfg.dynamicSmemBytes = T::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = c;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, adapter_tile_kernel<XT, WT, RP, TWO>, tx, t1, t2, tb, ty, g) == cudaSuccess ? FPQ_OK : FPQ_ERR_CUDA;
}

template <typename XT, typename WT, int RP>
fpq_status launch_rank(const RowsArgs& a, int x_type, int w_type, cudaStream_t st)
{
    if constexpr (RP <= 32 || std::is_same<XT, __nv_bfloat16>::value)
        if (two_on_an_sm(a, x_type))
            return launch_as<XT, WT, RP, true>(a, x_type, w_type, st);
    return launch_as<XT, WT, RP, false>(a, x_type, w_type, st);
}

template <typename XT, typename WT>
fpq_status launch_type(const RowsArgs& a, int x_type, int w_type, cudaStream_t st)
{
    if (a.R <= 16) {
        if constexpr (sizeof(XT) == 4)
            return FPQ_ERR_UNSUPPORTED;                    // (adapter_tiles_preferred)
        else
            return launch_rank<XT, WT, 16>(a, x_type, w_type, st);
    }
    return a.R <= 32 ? launch_rank<XT, WT, 32>(a, x_type, w_type, st) : launch_rank<XT, WT, 64>(a, x_type, w_type, st);
}

}  // namespace

bool encode_rows(EncodeTiledFn enc, CUtensorMap* tm, const void* base, int64_t rows, int64_t cols, int64_t ld, int type, int box_rows, int box_cols,
                 bool swizzle)
{
    const int bytes = type == FPQ_FP32 ? 4 : 2;
    const CUtensorMapDataType t = type == FPQ_FP32   ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                  : type == FPQ_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                     : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * bytes};
    cuuint32_t box[2] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return enc(tm, t, 2, (void*)base, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool adapter_tiles_preferred(const RowsArgs& a, int x_type, int w_type)
{
    const int bytes = x_type == FPQ_FP32 ? 4 : 2;
    if (a.R > 64 || !mapped(a.in, a.ld_in, bytes) || a.D1 * bytes % 16 || (a.out && (!mapped(a.out, a.ld_out, bytes) || a.D2 * bytes % 16)) ||
        (a.out && a.base && !mapped(a.base, a.ld_base, bytes)))
        return false;
    const int wb = w_type == FPQ_FP32 ? 4 : 2;
    if (!mapped(a.w1, a.ld_w1, wb) || (a.out && !mapped(a.w2, a.ld_w2, wb)) || (int64_t)a.G * std::max<int64_t>(a.R, a.out ? a.D2 : 0) >= ((int64_t)1 << 31))
        return false;
    // Estimates of both passes in us, fitted to 120 shapes of 8192 to 65536 rows (16 % and 19 % rms; the choice costs 1.3 % over the better
    // one, the pass by warps alone 46 %).  This one: a wave of blocks has its own latency and 31 bytes per ns and block (19 with two on
    // an SM); the pass by warps: so many values a us by type and rank.  (8192 x 640 -> 2560, FP32, rank 16: 46 here, 39 by warps;
    // rank 64: 58 and 98; 65536 rows, BF16, rank 64: 156 and 335.)  FP32 rows of rank 16 gained nothing, requests shorter than two
    // tiles and clusters of more than two blocks were slower in every case.
    const int64_t tiles = tiles_of(a);
    if (tiles <= 37 || a.M < 256 * (int64_t)a.S || (bytes == 4 && a.R <= 16))
        return false;
    const bool two = two_on_an_sm(a, x_type);
    const int c = cluster_of(a), kind = (a.R <= 16 ? 0 : a.R <= 32 ? 1 : 2) + (bytes == 4 ? 0 : 3);
    const double values = (double)a.M * ((double)a.D1 + (a.out ? (double)a.D2 * (a.base ? 2 : 1) : 0)), moved = values * bytes;
    const double blocks = (double)tiles * c, waves = ceil(blocks / (two ? 296 : 148));
    const double here = 6.5 * waves + (c > 1 ? 2.8 : 0) + std::max(moved / 5.3e6, moved / blocks * waves / (two ? 19.3e3 : 31e3));
    static const double rate[6] = {0, 0.71e6, 0.37e6, 1.81e6, 1.39e6, 0.81e6};
    return here < 4.7 + std::max(values / rate[kind], moved / 5.3e6);
}

fpq_status launch_adapter_tiles(const RowsArgs& a, int x_type, int w_type, cudaStream_t st)
{
    if (x_type == FPQ_BF16)
        return launch_type<__nv_bfloat16, __nv_bfloat16>(a, x_type, w_type, st);
    if (x_type == FPQ_FP16)
        return launch_type<__half, __half>(a, x_type, w_type, st);
    return w_type == FPQ_FP32   ? launch_type<float, float>(a, x_type, w_type, st)
           : w_type == FPQ_BF16 ? launch_type<float, __nv_bfloat16>(a, x_type, w_type, st)
                                : launch_type<float, __half>(a, x_type, w_type, st);
}

}  // namespace fpq
