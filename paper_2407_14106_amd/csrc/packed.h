// Attention over packed sequences: the work list that the host plans and the
// arguments that the kernels take.
#pragma once

#include "attn_common.h"

namespace gt {

constexpr int kMaxBuckets = 64;   // learned bias: rows of the table
constexpr int kTableStride = 65;  // a head's table in LDS; entries from n_buckets on are -inf

// One tile of one sequence.  The row lists (forward and dQ): rows tile .. of the
// sequence's lq * g query rows of one kv head (row r is query r / g, head r % g
// of the group), walking the keys s0 .. s1 - 1.  The key lists (dK, dV): the keys
// tile .., walking the rows s0 .. s1 - 1.  A tile whose walk is split has an item
// for each part; part p leaves its result for the tile's u-th 32 rows (or keys) in
// slot + u.  The merge lists: 32 rows (or keys) from tile on, whose s0 parts lie in
// the slots slot, slot + s1, ...
struct PackedItem {
    int32_t q0, lq, k0, lk;  // the sequence's first query and key, and their numbers
    int32_t tile, s0, s1;
    int32_t slot;            // partial result's first slot, -1: the tile's only item
    int64_t pair;            // first byte of the sequence's bucket ids
};

// The lists in plan->items; layout[2 l] is list l's first byte and
// layout[2 l + 1] its length.
enum PackedList {
    kPairs,     // at most 32 rows and 32 keys: one wavefront does all of it
    kRowsFew,   // tiles of 32 rows (sequences of no more): wavefronts share the walk
    kRows64,    // tiles of 64, 128 and 256 rows: wavefronts of 32 or 64 rows walk together
    kRows128,
    kRows256,
    kKeysFew,   // the same for the keys
    kKeys64,
    kKeys128,
    kKeys256,
    kRowMerges,
    kKeyMerges,
    kPackedLists
};
constexpr int kRowSlotsAt = 28, kKeySlotsAt = 29;      // layout: numbers of slots
constexpr int kRowSharedAt = 26, kKeySharedAt = 27;    // layout: whether two sets share a walk

// Whether two sets of wavefronts share the walks of tiles of 128.
template <typename T>
bool packed_shared(const gt_packed_plan* p, int at) {
    return p->layout[at] >= (sizeof(T) == 4 ? 1 : 2);
}

struct PackedArgs {
    const PackedItem* items;
    int n_items;
    int H, Hkv, gs, causal;  // gs: log2 of the query heads per kv head
    const void *Q, *K, *V, *O, *dO;
    uint32_t ldq, ldk, ldv;  // elements between consecutive nodes, below 2^23
    float scale;
    const float* table;      // [B, H]
    const uint8_t* ids;
    int B;                   // 0: no bias
    void *out0, *out1, *out2;  // O or dQ; dK, dV
    float* LSE;
    float *Dv, *Lg;          // row statistics [nq, H]: D, and log2 of the weights' sum under the given LSE
    float* slots;            // partial results
    float* hist;             // [blocks, g, B] partial gradients of the table
};

// Adds a value to a lane's own column of a [bucket][lane] sum in LDS: no two lanes
// meet, so a load and a store do what an atomic would (ds_add_f32 goes lane by lane,
// 193 cycles a wavefront's addition; a load and a store 12), in the program's order.
// (Four at a time, a value whose bucket one before it had taking that sum: one wait
// for four, but the comparisons cost more: 61 -> 74 us in the row pass.)
__device__ __forceinline__ void hist_add(float* col, uint32_t id, float v) { col[id * kWave] += v; }

inline int ilog2(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

inline int64_t packed_items(const gt_packed_plan* p, int list) { return p->layout[2 * list + 1]; }
inline const PackedItem* packed_list(const gt_packed_plan* p, int list) {
    return reinterpret_cast<const PackedItem*>(static_cast<const char*>(p->items) + p->layout[2 * list]);
}

// Wavefronts of a workgroup: of the pair kernels (a pair each) and for tiles of 32
// (shares of one walk).  They follow from the LDS that a wavefront's stages take
// (row bytes x 32 rows x 4 buffers).
constexpr int pair_waves(int row_bytes) { return row_bytes <= 128 ? 4 : row_bytes <= 256 ? 2 : 1; }
constexpr int few_waves(int row_bytes) { return row_bytes <= 64 ? 8 : row_bytes <= 256 ? 4 : 2; }
// With the table's gradient each of them needs its columns in LDS besides.
constexpr int few_waves_hist(int row_bytes) { return row_bytes <= 128 ? 4 : row_bytes <= 256 ? 2 : 1; }
// Wavefronts per SIMD that the stages (STAGE rows x 4 buffers x sets) leave room
// for, at most 2: what a kernel's registers are held to.
constexpr int waves_per_simd(int stage_bytes, int waves) {
    const int w = (160 << 10) / stage_bytes * waves / 4;
    return w < 1 ? 1 : w > 2 ? 2 : w;
}

// Floats of one slot (32 rows or keys): forward m, l and O;
// statistics; dQ; dK and dV.
constexpr int64_t kFewRows = 32;
inline int64_t fwd_slot_floats(int d) { return kFewRows * (d + 2); }
inline int64_t row_slot_floats(int d) { return kFewRows * d; }
inline int64_t key_slot_floats(int d) { return kFewRows * 2 * d; }

// Workgroups of the pair backward with a bias: each wavefront stays and goes through
// its sequences, so a partial table is left for a wavefront, not for a sequence.
constexpr int64_t kPairBlocks = 1024;
inline int64_t pair_blocks(const gt_packed_plan* p, int row_bytes) {
    // whole sets of heads on each XCD: a wavefront's pairs are all of one head, and an XCD works on the neighbouring
    // heads of a run of sequences, whose rows share cache lines
    const int64_t units = packed_items(p, kPairs) * p->Hkv, set = int64_t(kXcds) * p->Hkv, w = pair_waves(row_bytes);
    const int64_t want = cdiv(units, w * set) * set, most = cdiv(kPairBlocks, set) * set;
    return want < most ? want : most;
}

// Launchers, one set per element type (packed_fwd_*.hip, packed_bwd_*.hip).
template <typename T>
gt_status packed_fwd(const gt_packed_plan* p, int d, PackedArgs a, hipStream_t s);
template <typename T>
gt_status packed_bwd(const gt_packed_plan* p, int d, PackedArgs a, float* dtable, hipStream_t s);

// Merges of split walks (packed_merge.hip).
gt_status packed_merge_fwd(const gt_packed_plan* p, int d, gt_dtype dt, PackedArgs a, hipStream_t s);
gt_status packed_merge_stat(const gt_packed_plan* p, PackedArgs a, hipStream_t s);
gt_status packed_merge_rows(const gt_packed_plan* p, int d, gt_dtype dt, PackedArgs a, hipStream_t s);
gt_status packed_merge_keys(const gt_packed_plan* p, int d, gt_dtype dt, PackedArgs a, hipStream_t s);
// dtable[b, h] = the sum of the blocks' partial tables.
struct TableParts {
    int64_t at[6], n[6];  // per launch: n partial tables [g][B] from `at` on, the i-th of kv head i % Hkv
    int count;
};
gt_status packed_table_sum(const TableParts& t, PackedArgs a, float* dtable, hipStream_t s);

}  // namespace gt
