// The work list of packed-sequence attention, planned on the host: the tiles of
// every sequence, the longest first, in lists by the kernel that runs them.
#include <algorithm>
#include <cstring>
#include <utility>

#include "packed.h"

using namespace gt;

namespace {

constexpr int64_t kPlanMark = 0x67745061636b6564;  // set by init, checked by every call
constexpr int kMarkAt = 31;

struct Seqs {
    int64_t n;
    const int64_t *q, *k;
    int gs, Hkv;
    bool causal;
    bool fold;  // small sequences in the lists of tiles of 128
};

// How the tiles of one side (rows or keys) are cut; from the whole batch, so that
// init and fill agree.
struct Cut {
    bool large;         // tiles of 256 where a sequence has as many
    int shared;         // two sets of wavefronts share the walk of a tile of 128: 2 always, 1 in fp32
    int64_t chunk;      // longest walk of one item
    int64_t few_chunk;  // the same for tiles of 32
};
struct Cuts {
    Cut rows, keys;
};

// A CU works on two workgroups of four wavefronts at a time: where walks are longer
// than a workgroup's share of all of them by more than a merge costs, they are cut to
// two thirds of it (to the share: four causal prompts' backward 307 us, two thirds
// 274, half 277, a third 286; whole walks of up to two shares, 8,192 x 32 / 8 heads of
// 128 causal: its key passes 1500 and 1001 us, cut 973 and 655).
constexpr int64_t kCus = 256;
// Walks are not split into shorter parts than this: parts cost a second launch
// and a merge.
constexpr int64_t kMinChunk = 1024;
constexpr int64_t kLongWalk = 2048;

// A launch has fewer than 2^32 threads (with the grids' padding); the most that a kernel of a list takes for an item
// and kv head.
constexpr int64_t kMostThreads = (int64_t(1) << 32) - (int64_t(1) << 22);
int64_t list_threads(int list) { return list == kPairs ? kWave : list >= kRowMerges ? 32 * kWave : 8 * kWave; }

int64_t row_walk(const Seqs& s, int64_t lk, int64_t off, int64_t last) {  // keys that rows up to `last` attend to
    return s.causal ? std::max<int64_t>(0, std::min(lk, off + (last >> s.gs) + 1)) : lk;
}
int64_t first_row(const Seqs& s, int64_t rows, int64_t off, int64_t key) {  // first row that attends to `key`
    return s.causal ? std::min(rows, std::max<int64_t>(0, key - off) << s.gs) : 0;
}

// Sequences of every size in one small batch: each list is a launch, which costs more than the lanes that small
// sequences leave idle in tiles of 128, up to about four of those a CU (60 sequences of 10 to 100, 8 heads of 64, step
// 50 -> 31 us, 100 of them 51 -> 33; 200 of 20 to 60, nearly eight a CU, 42 -> 49).  Not where the wavefronts of few
// rows share a longer walk.
constexpr int64_t kFoldWalk = 256;
bool folds(const Seqs& s) {
    int64_t tiles = 0;
    bool rows_over = false, keys_over = false;
    for (int64_t i = 0; i < s.n; ++i) {
        const int64_t rows = (s.q[i + 1] - s.q[i]) << s.gs, lk = s.k[i + 1] - s.k[i];
        tiles += (std::max(rows, lk) + 127) / 128;
        rows_over |= rows > 32;
        keys_over |= lk > 32;
    }
    return rows_over && keys_over && tiles * s.Hkv <= 4 * kCus;
}
bool is_pair(const Seqs& s, int64_t rows, int64_t lk) { return !s.fold && rows <= 32 && lk <= 32; }
// Rows (or keys) for the list of tiles of 32, and how long their walk can be.
bool is_few(const Seqs& s, int64_t own, int64_t walk) { return own <= 32 && !(s.fold && walk <= kFoldWalk); }

// Walks of the tiles of one size.
struct Load {
    int64_t n = 0, total = 0, most = 0;
    void add(int64_t walk) {
        ++n;
        total += walk;
        most = std::max(most, walk);
    }
};
Cut cut_side(const Load& few, const Load& t128, const Load& t256, int64_t Hkv) {
    Cut c;
    auto share = [&](const Load& l, int64_t blocks) { return (l.total * Hkv + blocks - 1) / blocks; };
    // Large tiles read the partners less often, but take all of a CU and its other work cannot hide their start: for
    // long walks, where none is more than half its share (8,192 x 16 x 64: 913 against 990 us backward; 128 sequences
    // of 512: 427 against 415 for half the work).
    c.large = t256.n * Hkv >= 2 * kCus && t256.most <= share(t256, 2 * kCus) && t256.total >= kLongWalk * t256.n;
    // Two sets on one walk wait for each other (four prompts' dQ 94 -> 116 us), so only where there are fewer workgroups
    // than CUs and walks too short to be split over all of them (2,000 x 8 heads of 64, backward 76 -> 69 us), or in
    // fp32, whose products take so long that the wait is small, for up to four workgroups a CU (48 graphs 212 -> 199).
    c.shared = t128.n * Hkv < kCus && t128.total * Hkv < 2 * kCus * kMinChunk ? 2 : t128.n * Hkv < 4 * kCus;
    auto chunk = [&](int64_t x) { return std::max(kMinChunk, (x + 255) & ~int64_t(255)); };
    const int64_t slack = t128.n * Hkv < 2 * kCus ? 0 : 2 * kMinChunk;  // what a merge costs; idle CUs cost more
    c.chunk = t128.most <= share(t128, 2 * kCus) + slack ? std::max<int64_t>(t128.most, 1) : chunk(share(t128, 3 * kCus));
    c.few_chunk = chunk(share(few, 2 * kCus));
    return c;
}

// Calls f(tile, walk) for the tiles of `size`.
template <typename F>
void row_tiles(const Seqs& s, int64_t rows, int64_t lk, int64_t off, int64_t size, F f) {
    for (int64_t t = 0; t < rows; t += size) f(t, row_walk(s, lk, off, std::min(rows, t + size) - 1));
}
template <typename F>
void key_tiles(const Seqs& s, int64_t rows, int64_t lk, int64_t off, int64_t size, F f) {
    for (int64_t t = 0; t < lk; t += size) f(t, rows - first_row(s, rows, off, t));
}

Cuts cut(const Seqs& s) {
    Load few[2], t128[2], t256[2];
    for (int64_t i = 0; i < s.n; ++i) {
        const int64_t lq = s.q[i + 1] - s.q[i], lk = s.k[i + 1] - s.k[i], rows = lq << s.gs, off = lk - lq;
        if (is_pair(s, rows, lk)) continue;
        if (rows > 0 && is_few(s, rows, lk)) few[0].add(row_walk(s, lk, off, rows - 1));
        else row_tiles(s, rows, lk, off, 128, [&](int64_t, int64_t w) { t128[0].add(w); });
        if (rows >= 256) row_tiles(s, rows, lk, off, 256, [&](int64_t, int64_t w) { t256[0].add(w); });
        if (lk > 0 && is_few(s, lk, rows)) few[1].add(rows - first_row(s, rows, off, 0));
        else key_tiles(s, rows, lk, off, 128, [&](int64_t, int64_t w) { t128[1].add(w); });
        if (lk >= 256) key_tiles(s, rows, lk, off, 256, [&](int64_t, int64_t w) { t256[1].add(w); });
    }
    return {cut_side(few[0], t128[0], t256[0], s.Hkv), cut_side(few[1], t128[1], t256[1], s.Hkv)};
}

// Calls f(list, item) for every item of the work list, sequence by sequence.
// Returns the numbers of slots (row lists, key lists).
template <typename F>
std::pair<int64_t, int64_t> each_item(const Seqs& s, const Cuts& c, F f) {
    constexpr int64_t kTile[] = {32, 64, 128, 256};
    int64_t pair = 0, row_slots = 0, key_slots = 0;
    for (int64_t i = 0; i < s.n; ++i) {
        PackedItem it = {};
        it.q0 = int32_t(s.q[i]);
        it.k0 = int32_t(s.k[i]);
        it.lq = int32_t(s.q[i + 1] - s.q[i]);
        it.lk = int32_t(s.k[i + 1] - s.k[i]);
        it.pair = pair;
        pair += int64_t(it.lq) * ((int64_t(it.lk) + 15) / 16 * 16);
        const int64_t rows = int64_t(it.lq) << s.gs, lk = it.lk, off = lk - it.lq;
        it.slot = -1;
        if (is_pair(s, rows, lk)) {
            if (rows > 0 || lk > 0) f(kPairs, it);
            continue;
        }
        // one tile's walk, in parts of at most `chunk`
        auto walk = [&](int list, int merges, int64_t& slots, int64_t tile, int64_t units, int64_t s0, int64_t s1,
                        int64_t chunk) {
            it.tile = int32_t(tile);
            const int64_t parts = std::max<int64_t>(1, (s1 - s0 + chunk - 1) / chunk);
            it.slot = -1;
            if (parts > 1) {
                PackedItem m = it;
                m.s0 = int32_t(parts);
                m.s1 = int32_t(units);
                for (int64_t u = 0; u < units; ++u) {
                    m.tile = int32_t(tile + 32 * u);
                    m.slot = int32_t(slots + u);
                    f(merges, m);
                }
                it.slot = int32_t(slots);
                slots += parts * units;
            }
            // parts of equal length, whole blocks of 32 each
            const int64_t each = ((s1 - s0 + parts - 1) / parts + 31) & ~int64_t(31);
            for (int64_t p = 0; p < parts; ++p) {
                it.s0 = int32_t(std::min(s1, s0 + p * each));
                it.s1 = int32_t(parts > 1 ? std::min(s1, s0 + (p + 1) * each) : s1);
                f(list, it);
                if (parts > 1) it.slot += int32_t(units);
            }
        };
        const int row_list = is_few(s, rows, lk)               ? kRowsFew
                             : rows <= 64 && !s.fold           ? kRows64
                             : c.rows.large && rows >= 256     ? kRows256
                                                               : kRows128;
        const int64_t row_tile = kTile[row_list - kRowsFew];
        row_tiles(s, rows, lk, off, row_tile, [&](int64_t t, int64_t w) {
            walk(row_list, kRowMerges, row_slots, t, (std::min(rows - t, row_tile) + 31) / 32, 0, w,
                 row_list == kRowsFew ? c.rows.few_chunk : c.rows.chunk);
        });
        const int key_list = is_few(s, lk, rows)               ? kKeysFew
                             : lk <= 64 && !s.fold             ? kKeys64
                             : c.keys.large && lk >= 256       ? kKeys256
                                                               : kKeys128;
        const int64_t key_tile = kTile[key_list - kKeysFew];
        key_tiles(s, rows, lk, off, key_tile, [&](int64_t t, int64_t w) {
            walk(key_list, kKeyMerges, key_slots, t, (std::min(lk - t, key_tile) + 31) / 32, rows - w, rows,
                 key_list == kKeysFew ? c.keys.few_chunk : c.keys.chunk);
        });
    }
    return {row_slots, key_slots};
}

gt_status check_seqs(const char* who, const Seqs& s, int64_t* pair_bytes) {
    const std::string w(who);
    if (s.q[0] != 0 || s.k[0] != 0) return fail(GT_ERR_OUT_OF_RANGE, w + ": q_ptr and k_ptr start at 0");
    for (int64_t i = 0; i < s.n; ++i)
        if (s.q[i + 1] < s.q[i] || s.k[i + 1] < s.k[i])
            return fail(GT_ERR_UNSORTED, w + ": q_ptr and k_ptr must not decrease");
    if (s.q[s.n] >= (int64_t(1) << 31) || s.k[s.n] >= (int64_t(1) << 31))
        return fail(GT_ERR_INVALID_ARG, w + ": more than 2^31 - 1 rows");
    int64_t pair = 0;
    for (int64_t i = 0; i < s.n; ++i) {
        const int64_t lq = s.q[i + 1] - s.q[i], lk = s.k[i + 1] - s.k[i];
        // row numbers of one kv head, with a tile's slack, are 32-bit in the kernels
        if ((lq << s.gs) > (int64_t(1) << 31) - 4096 || lk > (int64_t(1) << 31) - 4096)
            return fail(GT_ERR_UNSUPPORTED, w + ": a sequence of this many rows");
        pair += lq * ((lk + 15) / 16 * 16);
    }
    *pair_bytes = pair;
    return GT_OK;
}

std::pair<int64_t, int64_t> plan_lists(const Seqs& s, const Cuts& c, int64_t (&count)[kPackedLists]) {
    for (auto& x : count) x = 0;
    return each_item(s, c, [&](int list, const PackedItem&) { ++count[list]; });
}

}  // namespace

namespace gt {
bool packed_plan_ok(const gt_packed_plan* p) { return p && p->layout[kMarkAt] == kPlanMark; }
}  // namespace gt

extern "C" gt_status gt_packed_plan_init(int64_t n_seq, const int64_t* q_ptr, const int64_t* k_ptr, int32_t H,
                                         int32_t Hkv, int32_t causal, gt_packed_plan* plan) {
    const char* who = "gt_packed_plan_init";
    if (!plan) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null plan");
    std::memset(plan, 0, sizeof *plan);
    if (n_seq < 0 || n_seq >= (int64_t(1) << 31) || !q_ptr || !k_ptr)
        return fail(GT_ERR_INVALID_ARG, std::string(who) + ": bad n_seq or null pointer");
    if (H < 1 || Hkv < 1 || H > 256 || H % Hkv != 0)
        return fail(GT_ERR_UNSUPPORTED, std::string(who) + ": H must be a multiple of Hkv, at most 256");
    const int g = H / Hkv;
    if (g > 16 || (g & (g - 1))) return fail(GT_ERR_UNSUPPORTED, std::string(who) + ": H / Hkv must be 1, 2, 4, 8 or 16");
    Seqs s = {n_seq, q_ptr, k_ptr, ilog2(g), Hkv, causal != 0, false};
    int64_t pair = 0;
    gt_status st = check_seqs(who, s, &pair);
    if (st != GT_OK) return st;
    int64_t count[kPackedLists];
    s.fold = folds(s);
    const Cuts c = cut(s);
    const auto slots = plan_lists(s, c, count);
    if (slots.first * Hkv >= (int64_t(1) << 26) || slots.second * Hkv >= (int64_t(1) << 26))
        return fail(GT_ERR_UNSUPPORTED, std::string(who) + ": more than 2^26 partial results");
    int64_t at = 0;
    for (int l = 0; l < kPackedLists; ++l) {
        if (count[l] * Hkv > kMostThreads / list_threads(l))
            return fail(GT_ERR_UNSUPPORTED, std::string(who) + ": more tiles than one launch takes");
        plan->layout[2 * l] = at;
        plan->layout[2 * l + 1] = count[l];
        at += count[l] * int64_t(sizeof(PackedItem));
    }
    plan->n_seq = n_seq;
    plan->nq = q_ptr[n_seq];
    plan->nk = k_ptr[n_seq];
    plan->pair_bytes = pair;
    plan->item_bytes = at;
    plan->H = H;
    plan->Hkv = Hkv;
    plan->causal = causal != 0;
    plan->layout[kRowSharedAt] = c.rows.shared;
    plan->layout[kKeySharedAt] = c.keys.shared;
    plan->layout[kRowSlotsAt] = slots.first;
    plan->layout[kKeySlotsAt] = slots.second;
    plan->layout[kMarkAt] = kPlanMark;
    return GT_OK;
}

extern "C" gt_status gt_packed_plan_fill(int64_t n_seq, const int64_t* q_ptr, const int64_t* k_ptr,
                                         const gt_packed_plan* plan, void* host_items, size_t bytes) {
    const char* who = "gt_packed_plan_fill";
    if (!packed_plan_ok(plan) || !q_ptr || !k_ptr)
        return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null pointer, or a plan that init did not make");
    if (n_seq != plan->n_seq) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": n_seq differs from init's");
    if (bytes < size_t(plan->item_bytes)) return fail(GT_ERR_WORKSPACE, std::string(who) + ": item buffer too small");
    if (plan->item_bytes > 0 && !host_items) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    Seqs s = {n_seq, q_ptr, k_ptr, ilog2(plan->H / plan->Hkv), plan->Hkv, plan->causal != 0, false};
    int64_t pair = 0;
    gt_status st = check_seqs(who, s, &pair);
    if (st != GT_OK) return st;
    int64_t count[kPackedLists];
    s.fold = folds(s);
    const Cuts c = cut(s);
    const auto slots = plan_lists(s, c, count);
    // the slots too: the workspace has as many as init counted
    bool same = pair == plan->pair_bytes && q_ptr[n_seq] == plan->nq && k_ptr[n_seq] == plan->nk &&
                slots.first == plan->layout[kRowSlotsAt] && slots.second == plan->layout[kKeySlotsAt] &&
                c.rows.shared == plan->layout[kRowSharedAt] && c.keys.shared == plan->layout[kKeySharedAt];
    for (int l = 0; l < kPackedLists; ++l) same = same && count[l] == plan->layout[2 * l + 1];
    if (!same) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": the sequences differ from init's");
    PackedItem* list[kPackedLists];
    for (int l = 0; l < kPackedLists; ++l)
        list[l] = reinterpret_cast<PackedItem*>(static_cast<char*>(host_items) + plan->layout[2 * l]);
    int64_t fill[kPackedLists] = {};
    each_item(s, c, [&](int l, const PackedItem& it) { list[l][fill[l]++] = it; });
    // the longest walks first, so that no long one starts when the chip runs empty (pairs are all alike)
    for (int l = kPairs + 1; l < kRowMerges; ++l)
        std::sort(list[l], list[l] + count[l], [](const PackedItem& a, const PackedItem& b) {
            const int32_t ca = a.s1 - a.s0, cb = b.s1 - b.s0;
            return ca != cb ? ca > cb : a.q0 != b.q0 ? a.q0 < b.q0 : a.k0 != b.k0 ? a.k0 < b.k0
                                                                   : a.tile != b.tile ? a.tile < b.tile
                                                                                      : a.s0 < b.s0;
        });
    return GT_OK;
}
