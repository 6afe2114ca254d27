// Attention over packed sequences: the work list that the host plans and the
// arguments that the kernels take.
#pragma once

#include "attn_common.h"

namespace gt {

constexpr int kMaxBuckets = 64;   // learned bias: rows of the table
constexpr int kTableStride = 65;  // a head's table in LDS; entries from n_buckets on are -inf

// One tile of one sequence.  Forward and dQ: rows tile .. of the sequence's
// lq * g query rows of one kv head (row r is query r / g, head r % g of the
// group), walking the keys s0 .. s1 - 1.  dK/dV: the keys tile .., walking the
// rows s0 .. s1 - 1.
struct PackedItem {
    int32_t q0, lq, k0, lk;  // the sequence's first query and key, and their numbers
    int32_t tile, s0, s1;
    int32_t slot;            // partial result's slot, -1: the tile's only item
    int64_t pair;            // first byte of the sequence's bucket ids
};

// What gt_packed_plan.layout holds: where the lists lie in `items` and how long
// they are.
enum PackedLayout {
    kRowsSmall = 0,   // 32-row tiles of sequences with at most 32 rows: one wavefront each
    kRowsLarge = 1,   // 128-row tiles: four wavefronts each
    kKeysSmall = 2,   // the same for the keys
    kKeysLarge = 3,
    kPackedLists = 4
};

constexpr int kRowTile = 128;

struct PackedArgs {
    const PackedItem* items;
    int n_items;
    int H, Hkv, gs, causal;  // gs: log2 of the query heads per kv head
    const void *Q, *K, *V, *O, *dO;
    int64_t ldq, ldk, ldv;   // elements between consecutive nodes
    float scale;
    const float* table;      // [B, H]
    const uint8_t* ids;
    int B;
    void *out0, *out1, *out2;  // O; dQ; dK, dV
    float* LSE;
    float *Dv, *Lg;          // row statistics [nq, H]: D, and log2 of the weights' sum under the given LSE
    float* hist;             // [blocks, g, B] partial gradients of the table
};

inline int ilog2(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

// Launchers, one set per element type (packed_fwd_*.hip, packed_bwd_*.hip).
template <typename T>
gt_status packed_fwd(const gt_packed_plan* p, int d, PackedArgs a, hipStream_t s);
template <typename T>
gt_status packed_bwd(const gt_packed_plan* p, int d, PackedArgs a, float* dtable, hipStream_t s);

// The blocks that a list's kernel runs, and the list.
inline int64_t packed_items(const gt_packed_plan* p, int list) { return p->layout[2 * list + 1]; }
inline const PackedItem* packed_list(const gt_packed_plan* p, int list) {
    return reinterpret_cast<const PackedItem*>(static_cast<const char*>(p->items) + p->layout[2 * list]);
}

}  // namespace gt
