// The adapters' gradients from BF16 rows on the 5th-generation tensor cores.
//
//   out(col, j) = sum over an adapter's rows of wide[i][col] * thin[i][j]     (dA: x with t; dB: dy with u)
//
// A block takes 128 columns and, with the blocks that share them, the adapter's rows in runs of 64.  A run of both comes by TMA.  The
// rows of x lie as they are the MMA's first operand (128 x 64, its 128 columns side by side); the warps write t or u as three BF16
// terms, which hold all of its 24 bits, side by side as 3 x rank columns of the second operand: one MMA for the three, whose
// accumulators are added up in registers every 128 rows, the smallest term first (the tensor core cuts its sums off).
// Blocks that share a sum write theirs, and a second kernel adds them up in order.  Ranks above 64 go to two blocks, 64 to each.
//
// Bound by memory: 30011 x 1280 and x 640, rank 32, three adapters: 25 us, of which 23 read 115 MB in the 285 blocks' main loops, two blocks
// on an SM; their sums 5 us more (under a profiler, from cold caches).  By warps (fpq_adapter.cu), which split t anew for every 64 columns: 57.
#include <algorithm>
#include <atomic>

#include "fpq_adapter.cuh"

namespace fpq {

namespace {

constexpr int COLS = 128, RUN = 64, WORK_WARPS = 8, THREADS = 32 * (2 + WORK_WARPS), CHUNK = 2;      // (CHUNK runs to an accumulator)

template <int RP>
struct GradTile {
    static constexpr int X_BYTES = RUN * COLS * 2, B_BYTES = 3 * RP * 128, T_BYTES = RUN * RP * 4, STAGE = X_BYTES + B_BYTES + T_BYTES;
    static constexpr int STAGES = RP == 16 ? 4 : 3, ON_AN_SM = RP <= 32 ? 2 : 1;
    static constexpr int TMEM = RP == 16 ? 128 : RP == 32 ? 256 : 512;                // two accumulators of 3 x rank columns
    static constexpr int SMEM = STAGES * STAGE + 1024 + 256;                          // to start at a multiple of 1024; barriers behind the stages
};

struct GradTileArgs {
    GradArgs a;
    int* status;
};

template <int RP>
__global__ void __launch_bounds__(THREADS, GradTile<RP>::ON_AN_SM) adapter_grad_tile_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_dy,
                                                                                           const __grid_constant__ CUtensorMap tm_t, const __grid_constant__ CUtensorMap tm_u,
                                                                                           const GradTileArgs ga)
{
    using T = GradTile<RP>;
    constexpr int STAGES = T::STAGES, SHARE = RP / 2;
    const GradArgs& a = ga.a;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base_addr = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t* smem = smem_raw + (base_addr - smem_u32(smem_raw));
    const uint32_t bars = base_addr + STAGES * T::STAGE, full = bars, ready = bars + 32, empty = bars + 64, sum_full = bars + 96, sum_free = bars + 112;
    volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem + STAGES * T::STAGE + 128);
    volatile int* rows_of = reinterpret_cast<volatile int*>(smem + STAGES * T::STAGE + 144);      // [STAGES]: of the run that lies there; -1: no more
    if (threadIdx.x == 0) {
        tma_prefetch_desc((int)blockIdx.x % ga.a.tiles >= ga.a.tiles_k ? &tm_dy : &tm_x);
        tma_prefetch_desc((int)blockIdx.x % ga.a.tiles >= ga.a.tiles_k ? &tm_u : &tm_t);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const GradShare share = share_of(a);
    const int part = blockIdx.x / a.tiles, parts = gridDim.x / a.tiles, tile = blockIdx.x % a.tiles, id = share.id, z = share.z, splits = share.splits;
    if (z < 0)
        return;
    const bool is_b = tile >= a.tiles_k;
    const int64_t D = is_b ? a.N : a.K, c0 = (int64_t)(is_b ? tile - a.tiles_k : tile) * COLS;
    const int R = a.R, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(ready + 8 * s, WORK_WARPS);
            mbar_init(empty + 8 * s, 1);
        }
        for (int b = 0; b < 2; ++b) {
            mbar_init(sum_full + 8 * b, 1);
            mbar_init(sum_free + 8 * b, WORK_WARPS);
        }
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
    float sum[SHARE];
#pragma unroll
    for (int i = 0; i < SHARE; ++i)
        sum[i] = 0.f;
    // this thread's column and its share of the ranks
    const int quarter = warp & 3, half = (warp - 2) >> 2, col = quarter * 32 + lane, j0 = half * SHARE;

    if (warp == 0) {
        // ---------------- runs by TMA: every splits-th of all runs of the adapter's segments ----------------
        int chunk = -32, my_begin = 0, my_end = 0;         // 32 segments at a time, one to a lane
        uint32_t left = 0;
        int runs = 0, at = 0, n_runs = 0, begin = 0, end = 0;        // runs: of the segments in front, modulo the splits
        auto next_run = [&](int& row, int& rows) {
            while (at >= n_runs) {
                runs = (runs + n_runs) % splits;
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
                at = z - runs + (z < runs ? splits : 0);
            }
            row = begin + at * RUN;
            rows = min(end - row, RUN);
            at += splits;
            return true;
        };
        uint32_t s = 0, ph = 0;
        int k = 0;
        for (;; ++k) {
            int row = 0, rows = 0;
            const bool some = next_run(row, rows);
            if (__any_sync(0xffffffffu, !mbar_wait(empty + 8 * s, ph ^ 1))) { dead = true; break; }
            if (lane == 0) {
                rows_of[s] = some ? rows : -1;
                if (some) {
                    const uint32_t st = base_addr + s * T::STAGE;
                    mbar_expect_tx(full + 8 * s, T::X_BYTES + T::T_BYTES);
                    tma_load_2d(st, is_b ? &tm_dy : &tm_x, full + 8 * s, (int)c0, row);
                    tma_load_2d(st + T::X_BYTES / 2, is_b ? &tm_dy : &tm_x, full + 8 * s, (int)c0 + COLS / 2, row);
                    tma_load_2d(st + T::X_BYTES + T::B_BYTES, is_b ? &tm_u : &tm_t, full + 8 * s, part * RP, row);
                } else {
                    mbar_arrive(full + 8 * s);
                }
            }
            __syncwarp();
            if (!some)
                break;
            if (++s == STAGES) { s = 0; ph ^= 1; }
        }
        if (dead) {                                        // the copies in flight end before the block does
            for (int i = max(k - STAGES, 0); i < k; ++i)
                mbar_wait(full + 8 * (i % STAGES), (i / STAGES) & 1);
            if (lane == 0)
                flag_status(ga.status, FPQ_ERR_TIMEOUT);
        }
    } else if (warp == 1) {
        // ---------------- MMAs ----------------
        if (elect_one()) {
            // FP32 accumulators, BF16 operands, the first one's rows (columns of x) side by side; M = 128, N = 3 ranks
            constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 15) | ((uint32_t)(3 * RP >> 3) << 17) | ((uint32_t)(COLS >> 4) << 24);
            uint32_t s = 0, ph = 0;
            int k = 0;
            for (;; ++k) {
                const int chunk = k / CHUNK;
                const uint32_t buf = chunk & 1;
                if (!mbar_wait(full + 8 * s, ph)) { dead = true; break; }
                if (rows_of[s] < 0)
                    break;
                // a fresh accumulator: the warps must have added up what it held two chunks ago
                if (k % CHUNK == 0 && chunk >= 2 && !mbar_wait(sum_free + 8 * buf, ((chunk >> 1) - 1) & 1)) { dead = true; break; }
                if (!mbar_wait(ready + 8 * s, ph)) { dead = true; break; }
                tc_fence_after();
                // x: 64 of the columns 128 bytes side by side, the other 64 half the stage's rows behind; 8 rows 1024 bytes
                const uint32_t st = base_addr + s * T::STAGE, d = tmem + buf * (3 * RP);
                const uint32_t x = ((st >> 4) & 0x3fffu) | ((uint32_t)(T::X_BYTES / 2 >> 4) << 16), w = smem_desc_lo(st + T::X_BYTES);
#pragma unroll
                for (uint32_t kk = 0; kk < RUN / 16; ++kk) {
                    const uint32_t acc = k % CHUNK != 0 || kk != 0;
                    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\tmov.b64 db, {%2, %3};\n\t"
                                 "tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}"
                                 ::"r"(d), "r"(x + kk * (2048 / 16)), "r"(w + 2 * kk), "r"(SMEM_DESC_HI_K_SW128), "r"(IDESC), "r"(acc)
                                 : "memory");
                }
                mma_commit(empty + 8 * s);
                if (k % CHUNK == CHUNK - 1)
                    mma_commit(sum_full + 8 * buf);
                if (++s == STAGES) { s = 0; ph ^= 1; }
            }
            if (!dead && k % CHUNK != 0)
                mma_commit(sum_full + 8 * (k / CHUNK & 1));
            if (dead)
                flag_status(ga.status, FPQ_ERR_TIMEOUT);
        }
        __syncwarp();
    } else {
        // ---------------- terms of t or u, sums ----------------
        const int tid = threadIdx.x - 64;
        int drained = 0;
        auto drain = [&](int c) {
            const uint32_t buf = c & 1;
            if (!mbar_wait(sum_full + 8 * buf, (c >> 1) & 1)) { dead = true; return; }
            tc_fence_after();
            const uint32_t from = tmem + buf * (3 * RP) + j0 + ((uint32_t)(quarter * 32) << 16);
            uint32_t r[3][SHARE];
#pragma unroll
            for (int e = 0; e < 3; ++e)
                tmem_load<SHARE>(from + e * RP, r[e]);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < SHARE; ++i)
                sum[i] += (__uint_as_float(r[2][i]) + __uint_as_float(r[1][i])) + __uint_as_float(r[0][i]);
            tc_fence_before();
            __syncwarp();
            if (lane == 0)
                mbar_arrive(sum_free + 8 * buf);
        };
        uint32_t s = 0, ph = 0;
        int k = 0;
        for (;; ++k) {
            if (!mbar_wait(full + 8 * s, ph)) { dead = true; break; }
            const int rows = rows_of[s];
            if (rows < 0)
                break;
            uint8_t *st = smem + s * T::STAGE, *terms = st + T::X_BYTES;
            const float* t = reinterpret_cast<const float*>(terms + T::B_BYTES);
#pragma unroll
            for (int u = 0; u < (RP * 8 + 32 * WORK_WARPS - 1) / (32 * WORK_WARPS); ++u) {
                const int e = tid + u * 32 * WORK_WARPS, j = e % RP, c = e / RP;      // rank, and which eight rows
                if (RP * 8 % (32 * WORK_WARPS) == 0 || e < RP * 8) {
                    uint32_t p[3][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = 8 * c + 2 * i;
                        float x = r < rows ? t[r * RP + j] : 0.f, y = r + 1 < rows ? t[(r + 1) * RP + j] : 0.f;
#pragma unroll
                        for (int h = 0; h < 3; ++h) {
                            const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
                            const float2 f = __bfloat1622float2(v);
                            p[h][i] = *reinterpret_cast<const uint32_t*>(&v);
                            x -= f.x;
                            y -= f.y;
                        }
                    }
#pragma unroll
                    for (int h = 0; h < 3; ++h)
                        *reinterpret_cast<uint4*>(terms + swizzled(h * RP + j, c)) = make_uint4(p[h][0], p[h][1], p[h][2], p[h][3]);
                }
            }
            if (rows < RUN)                                // rows behind the segment: whatever they hold, times zero must be zero
                for (int e = tid; e < (RUN - rows) * 16; e += 32 * WORK_WARPS)
                    *reinterpret_cast<uint4*>(st + (e & 8) * (T::X_BYTES / 16) + (rows + (e >> 4)) * 128 + (e & 7) * 16) = make_uint4(0, 0, 0, 0);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0)
                mbar_arrive(ready + 8 * s);
            if (++s == STAGES) { s = 0; ph ^= 1; }
            // a run later the previous chunk's MMAs are done
            if (k % CHUNK == 0 && k / CHUNK > drained) {
                drain(drained++);
                if (dead)
                    break;
            }
        }
        while (!dead && drained < (k + CHUNK - 1) / CHUNK)
            drain(drained++);
        if (dead && lane == 0)
            flag_status(ga.status, FPQ_ERR_TIMEOUT);
    }

    // of dA columns lie side by side, of dB ranks
    if (warp >= 2 && splits > 1) {
        float* sums = a.sums + ((((int64_t)z * a.G + id) * parts + part) * a.tiles + tile) * (COLS * RP) + (is_b ? col * RP + j0 : j0 * COLS + col);
        if (is_b) {
#pragma unroll
            for (int i = 0; i < SHARE; i += 4)
                *reinterpret_cast<float4*>(sums + i) = make_float4(sum[i], sum[i + 1], sum[i + 2], sum[i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < SHARE; ++i)
                sums[i * COLS] = sum[i];
        }
    } else if (warp >= 2 && c0 + col < D) {
#pragma unroll
        for (int i = 0; i < SHARE; ++i)
            if (part * RP + j0 + i < R)
                store_gradient<__nv_bfloat16>(a, id, is_b, c0 + col, part * RP + j0 + i, sum[i]);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, T::TMEM);
    }
}

// The sums of the blocks that share an adapter's rows, in order.  (By the last of those blocks, 19 of them: 13 to 20 us more.)
template <int RP>
__global__ void __launch_bounds__(256) adapter_grad_tile_sum_kernel(const GradArgs a)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int PER = COLS * RP / 256;
    const int part = blockIdx.x / PER / a.tiles, parts = gridDim.x / PER / a.tiles, tile = blockIdx.x / PER % a.tiles, id = blockIdx.y;
    const int i = blockIdx.x % PER * 256 + threadIdx.x, splits = splits_of(a, id);
    const bool is_b = tile >= a.tiles_k;
    const int col = is_b ? i / RP : i % COLS, j = part * RP + (is_b ? i % RP : i / COLS);
    const int64_t c = (int64_t)(is_b ? tile - a.tiles_k : tile) * COLS + col;
    if (splits == 1 || c >= (is_b ? a.N : a.K) || j >= a.R)
        return;                                            // (with one, the block itself has stored them)
    const float* s = a.sums + (((int64_t)id * parts + part) * a.tiles + tile) * (COLS * RP) + i;
    const int64_t every = (int64_t)a.G * parts * a.tiles * (COLS * RP);
    float v = 0.f;
    for (int b = 0; b < splits; b += 8) {                  // (eight loads at a time, the last ones too)
        float w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            w[k] = b + k < splits ? s[(b + k) * every] : 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k)
            v += w[k];
    }
    store_gradient<__nv_bfloat16>(a, id, is_b, c, j, v);
}

int tiles_of(int64_t n) { return (int)((n + COLS - 1) / COLS); }
int padded(int R) { return R <= 16 ? 16 : R <= 32 ? 32 : 64; }
int parts_of(int R) { return R <= 64 ? 1 : 2; }            // of 64 ranks, which different blocks take

template <int RP>
cudaError_t launch_as(const GradArgs& a, cudaStream_t st)
{
    using T = GradTile<RP>;
    static_assert(T::ON_AN_SM * (T::SMEM + 1024) <= 233472 && T::ON_AN_SM * T::TMEM <= 512 && 6 * RP <= T::TMEM, "blocks on an SM");
    EncodeTiledFn enc = tensor_map_encoder();
    GradTileArgs g;
    g.a = a;
    g.status = status_word();
    int dev = 0;
    if (!enc || !g.status)
        return cudaErrorUnknown;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess)
        return e;
    static std::atomic<uint64_t> known{0};
    if (dev >= 64 || !(known.load(std::memory_order_relaxed) >> dev & 1)) {
        e = cudaFuncSetAttribute(adapter_grad_tile_kernel<RP>, cudaFuncAttributeMaxDynamicSharedMemorySize, T::SMEM);
        if (e != cudaSuccess)
            return e;
        if (dev < 64)
            known.fetch_or((uint64_t)1 << dev);
    }
    CUtensorMap tx, ty, tt, tu;
    if (!encode_rows(enc, &tx, a.x, a.M, a.K, a.ldx, FPQ_BF16, RUN, COLS / 2, true) || !encode_rows(enc, &ty, a.dy, a.M, a.N, a.ld_dy, FPQ_BF16, RUN, COLS / 2, true) ||
        !encode_rows(enc, &tt, a.t, a.M, a.R, a.R, FPQ_FP32, RUN, RP, false) || !encode_rows(enc, &tu, a.u, a.M, a.R, a.R, FPQ_FP32, RUN, RP, false))
        return cudaErrorUnknown;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grad_grid(a);
    cfg.gridDim.x *= parts_of(a.R);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = T::SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, adapter_grad_tile_kernel<RP>, tx, ty, tt, tu, g);
    if (e != cudaSuccess || a.splits == 1)
        return e;
    return launch_overlapped(adapter_grad_tile_sum_kernel<RP>, dim3(parts_of(a.R) * a.tiles * (COLS * RP / 256), a.G), 256, 0, st, a);
}

}  // namespace

// From 1024 rows on.  Whole backward passes, the gradients by warps and so, us: one adapter, 1024 rows, 320 -> 320, rank 16: 16.9 and
// 13.9; 8192 rows, 640 -> 640, rank 64: 56 and 37; 32768 rows, 1280 -> 640, rank 32: 103 and 78; 512 rows of 32 adapters, rank 16: 22.4
// and 27.2.  Every segment costs a run of 64 rows here and of 16 or 32 by warps, which the rule does not look at: one adapter in segments
// of 4 rows, 8192 rows, 320 -> 320: 414 and 371; 16 adapters in segments of 16, 1280 -> 640: 93 and 105; 64 adapters in segments of 16, 320 ->
// 320: 42 and 56; 4 adapters, 1024 rows in as many segments: 114 and 188.  (One adapter, or 256 rows to each and 48 to a segment, would
// leave 1.6 % over the better one of 300 shapes instead of 9.5 %.)  Rows that start between 16-byte boundaries, and ranks that are no
// multiple of four, go by warps.
bool adapter_grad_tiles_preferred(const GradArgs& a)
{
    if (a.R % 4 != 0 || !mapped(a.x, a.ldx, 2) || !mapped(a.dy, a.ld_dy, 2) || !mapped(a.t, a.R, 4) || !mapped(a.u, a.R, 4))
        return false;
    return a.M >= 1024;
}

// One wave of blocks, 256 rows at least to each.  Of several adapters each gets its share of the rows' blocks (splits_of), rounded up.
int adapter_grad_tile_splits(int64_t M, int64_t N, int64_t K, int G, int R)
{
    const int64_t tiles = parts_of(R) * (tiles_of(K) + tiles_of(N)), fit = (R <= 32 ? 2 : 1) * 148 / tiles;
    const int64_t most = std::max<int64_t>(fit - (G - 1), fit / 2);
    return (int)std::max<int64_t>(std::min(M / 256, std::min(most, 8 * 148 / (tiles * G))), 1);
}

size_t adapter_grad_tile_columns(int64_t M, int64_t N, int64_t K, int G, int R)
{
    const size_t splits = adapter_grad_tile_splits(M, N, K, G, R);
    return splits == 1 ? 0 : splits * G * (tiles_of(K) + tiles_of(N)) * COLS;
}

cudaError_t launch_adapter_grad_tiles(GradArgs a, cudaStream_t st)
{
    a.tiles_k = tiles_of(a.K);
    a.tiles = a.tiles_k + tiles_of(a.N);
    return padded(a.R) == 16 ? launch_as<16>(a, st) : padded(a.R) == 32 ? launch_as<32>(a, st) : launch_as<64>(a, st);
}

}  // namespace fpq
