// What the tcgen05 kernels (ffn_rows.cuh, ffn_q4.cuh, layer_tc.cuh) have in common: the group table's
// entry, unit arithmetic and the set of tensor maps of the split-K kernels.
#pragma once

#include "common.cuh"
#include "ffn_stream.cuh"
#include "ptx.cuh"

namespace s2moe {

constexpr int kTcKT = 4;                       // k-tiles (of 64) per unit of the split-K kernels
constexpr int kTcWTile = 128 * 128;            // bytes of one bf16 weight k-tile in shared memory
constexpr int kTcQ4KG = 4;                     // int4: k-tiles per ring stage (a whole unit)
static_assert(kTcQ4KG == kTcKT, "an int4 stage is a whole unit");
constexpr int kTcQ4Packed = 128 * 32;          // bytes of one packed weight k-tile (128 rows x 64 nibbles)
constexpr int kTcQ4Scales = 128 * 16;          // 8 binary16 scales per row: the 256 columns of the unit
constexpr int kTcQ4ACol = 256;                 // int4: TMEM columns 256.. hold the A operand (32 per k-tile), 0..255 the accumulators
#ifndef S2MOE_MAX_STAGES
#define S2MOE_MAX_STAGES 10
#endif
constexpr int kTcMaxStages = S2MOE_MAX_STAGES;
constexpr int kTcMaxSmem = 232448 - 9216;      // dynamic shared memory; the rest is static (unit table, barriers)
constexpr unsigned kTcSpinLimit = 1u << 22;
// Share of the experts in wave 0 of the split-K kernels (by units of the first projection).  The second
// projection of wave 0 is what hides the hand-over of wave 1, the first projection of wave 1 what hides
// that of wave 0.
#ifndef S2MOE_SPLIT_NUM
#define S2MOE_SPLIT_NUM 7
#define S2MOE_SPLIT_DEN 16
#endif
constexpr int kTcSplitNum = S2MOE_SPLIT_NUM, kTcSplitDen = S2MOE_SPLIT_DEN;
constexpr int kTcReady = 512;                  // ws.sync[kTcReady - 8 + w], [kTcReady - 4 + w]: the two counters of wave w

// one active group in shared memory: 32 bytes, so that an entry is two aligned 16-byte reads
// (wider entries were measured: 48 bytes cost 0.7 us per layer)
struct TcGroup {
    unsigned long long mask;   // tokens of the batch bucketed to this group
    int group, T, off, f;      // group id (offloaded experts: device slot), tokens, first slot, inner dim
    int p1, p2;                // first phase-1 / phase-2 unit of the group
};
static_assert(sizeof(TcGroup) == 32, "layout");

// units of a group: phase 1 = 2 matrices x row blocks x k-pieces, phase 2 = row blocks x k-pieces
__host__ __device__ __forceinline__ int tc_kpieces(int K) { return ((K + 63) / 64 + kTcKT - 1) / kTcKT; }
__host__ __device__ __forceinline__ int tc_units1(int f_g, int d) { return 2 * ((f_g + 127) / 128) * tc_kpieces(d); }
__host__ __device__ __forceinline__ int tc_units2(int f_g, int d) { return ((d + 127) / 128) * tc_kpieces(f_g); }

// Barrier among the four epilogue warps on an mbarrier (count 4), so that the wait is bounded.
__device__ __forceinline__ bool tc_bar(uint64_t *bar, uint32_t &phase, int lane)
{
    __syncwarp();
    if (lane == 0) mbar_arrive(bar);
    const bool ok = mbar_wait(bar, phase);
    phase ^= 1u;
    return ok;
}

// counter += 1 with release semantics at GPU scope (one instruction instead of fence + atomic)
__device__ __forceinline__ void tc_red_release(int32_t *counter)
{
    asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(counter) : "memory");
}

// next slot of the ring; the parity flips on wrap-around
__device__ __forceinline__ void tc_ring_next(int &s, uint32_t &parity, int S)
{
    if (++s == S) { s = 0; parity ^= 1u; }
}

// tensor maps: 0 gate, 1 up, 2 down, 3 sh_gate, 4 sh_up, 5 sh_down, 6 hidden, 7 activations of the
// routed slots, 8 of the shared slots: 3-D {k, slot, hi|lo}, so that one copy of box {64, 16, 2}
// lands the hi tile and, right behind it, the lo tile of 16 slots
// block-int4 weights: 0..5 are the packed matrices (bytes, boxes of four k-tiles), 9..14 their scales
// (binary16), 6 is the (column-permuted) hidden states as {k in tile, row, k-tile} with a box of all rows x kg
// k-tiles, 7 and 8 the activations as {k in tile, slot, k-tile, hi|lo} with a box {64, 8, kg, 2}:
// one copy per stage (per 8 slots) instead of one per k-tile
struct TcMaps {
    CUtensorMap m[15];
};

}  // namespace s2moe
