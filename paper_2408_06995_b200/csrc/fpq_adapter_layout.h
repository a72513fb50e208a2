// Shared memory of the adapters' tile kernel (fpq_adapter_tile.cu), as numbers alone: the kernel takes its addresses from here, and
// a host program can look at them.
#pragma once

#ifdef __CUDACC__
#define FPQ_HOST_DEVICE __host__ __device__
#else
#define FPQ_HOST_DEVICE
#endif

namespace fpq {

constexpr int TILE_M = 128, NCOLS = 64;
constexpr int X_BYTES = TILE_M * 128, SLOT_BYTES = 32 * 128;

// XB, WB: bytes of a value of x and of the weights.  BF_: BF16 rows.  TWO: two blocks on an SM, of eight working warps each; otherwise
// one of sixteen (of eight, where t takes 64 KB)
template <int XB, int WB, bool BF_, int RP, bool TWO>
struct TileSizes {
    static constexpr bool FP32 = XB == 4;
    static constexpr bool WIDE_W = WB == 4;
    static constexpr bool BF = BF_;                                                 // t in two BF16 terms, otherwise TF32 terms
    static constexpr int GROUPS = TWO || (RP == 64 && !BF) ? 2 : 4, WORK_WARPS = 4 * GROUPS, THREADS = 32 * (2 + WORK_WARPS);
    static constexpr int KE = 128 / XB;                                             // columns of a stage
    // W1's part of a stage: the operand as it lies in memory; FP32 rows: with its tails, or 16-bit weights and what they are in FP32
    static constexpr int W_BYTES = RP * 128, W_RAW = FP32 && !WIDE_W ? RP * 64 : W_BYTES, W_MORE = FP32 ? W_BYTES : 0;
    static constexpr int X_PART = X_BYTES * (FP32 ? 2 : 1), STAGE = X_PART + W_RAW + W_MORE;
    static constexpr int STAGES = FP32 ? (TWO ? 2 : 3) : TWO ? 3 : 4;
    static constexpr int CHUNK = FP32 ? 2 : 4;                                      // stages whose products the tensor core adds up
    static constexpr int T_ROW = RP * (BF ? 2 : 4), KB = (T_ROW + 127) / 128;       // bytes of a row of t, and blocks of 128
    static constexpr int T_BYTES = KB * TILE_M * 128;                               // one term
    // the same of W2, 64 columns
    static constexpr int W2_BYTES = KB * NCOLS * 128, W2_RAW = BF || WIDE_W ? W2_BYTES : NCOLS * RP * 2, W2_MORE = BF ? 0 : W2_BYTES;
    static constexpr int W2_SET = (W2_RAW + W2_MORE + 1023) / 1024 * 1024, W2_SETS = GROUPS;       // (a group's own)
    static constexpr int T_KEPT = TILE_M * RP * 4;                                  // t in FP32, for the cluster and for odd sums
    static constexpr int W2_BASE = 2 * T_BYTES, KEPT_BASE = W2_BASE + W2_SETS * W2_SET, PHASE2 = KEPT_BASE + T_KEPT;
    static constexpr int WORK = STAGES * STAGE > PHASE2 ? STAGES * STAGE : PHASE2;
    static constexpr int SLOTS = TWO || (FP32 && GROUPS == 4) ? 1 : 2;                 // of each warp: 32 rows x 128 bytes of base and y
    static constexpr int SLOT_BASE = WORK, END = SLOT_BASE + WORK_WARPS * SLOTS * SLOT_BYTES;
    static constexpr int TMEM = 64 * GROUPS;                                        // 2 x rank columns of t, later 64 of y for each group

    // The barriers, 8 bytes each, and behind the last of them the word that gets the address of the tensor memory
    static constexpr int FULL = 0, EMPTY = FULL + 8 * STAGES, READY = EMPTY + 8 * STAGES;         // (READY: FP32 rows only)
    static constexpr int T_FULL = READY + (FP32 ? 8 * STAGES : 0), T_FREE = T_FULL + 16, T_READY = T_FREE + 16, T_DONE = T_READY + 8;
    static constexpr int W_FULL = T_DONE + 8, W_EMPTY = W_FULL + 8 * W2_SETS, W_READY = W_EMPTY + 8 * W2_SETS, Y_FULL = W_READY + 8 * GROUPS;
    static constexpr int SLOT_FULL = Y_FULL + 8 * GROUPS, TMEM_WORD = SLOT_FULL + 8 * WORK_WARPS * SLOTS;       // SLOT_FULL: [warp][SLOTS]
    static constexpr int BARRIERS = (TMEM_WORD + 4 + 15) / 16 * 16;

    // The stages start at the next multiple of 1024 behind the dynamic shared memory's own start (a multiple of 16); the barriers lie
    // in front of them where they fit, else behind the end
    static constexpr int SMEM = END + 1024;
    FPQ_HOST_DEVICE static constexpr int barriers_at(int gap) { return gap >= BARRIERS ? -BARRIERS : END; }       // from the stages' start
    static_assert(BARRIERS - 16 + BARRIERS <= 1024, "the barriers behind the end, behind the widest gap that does not hold them");
};

}  // namespace fpq
