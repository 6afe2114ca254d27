// The work list of packed-sequence attention, planned on the host: the tiles of
// every sequence, the longest first, in lists by the kernel that runs them.
#include <algorithm>
#include <cstring>

#include "packed.h"

using namespace gt;

namespace {

constexpr int64_t kPlanMark = 0x67745061636b6564;  // set by init, checked by every call
constexpr int kMarkAt = 31;

struct Seqs {
    int64_t n;
    const int64_t *q, *k;
    int gs;
    bool causal;
};

// Calls f(list, item) for every item of the work list, sequence by sequence.
template <typename F>
void each_item(const Seqs& s, F f) {
    int64_t pair = 0;
    for (int64_t i = 0; i < s.n; ++i) {
        PackedItem it = {};
        it.q0 = int32_t(s.q[i]);
        it.k0 = int32_t(s.k[i]);
        it.lq = int32_t(s.q[i + 1] - s.q[i]);
        it.lk = int32_t(s.k[i + 1] - s.k[i]);
        it.slot = -1;
        it.pair = pair;
        pair += int64_t(it.lq) * ((int64_t(it.lk) + 15) / 16 * 16);
        const int64_t rows = int64_t(it.lq) << s.gs, off = int64_t(it.lk) - it.lq;
        const bool small_rows = rows <= 32, small_keys = it.lk <= 32;
        for (int64_t t = 0; t < rows; t += small_rows ? 32 : kRowTile) {
            const int64_t last = std::min(rows, t + (small_rows ? 32 : kRowTile)) - 1;
            it.tile = int32_t(t);
            it.s0 = 0;
            it.s1 = int32_t(s.causal ? std::max<int64_t>(0, std::min<int64_t>(it.lk, off + (last >> s.gs) + 1)) : it.lk);
            f(small_rows ? kRowsSmall : kRowsLarge, it);
        }
        for (int64_t t = 0; t < it.lk; t += small_keys ? 32 : kRowTile) {
            it.tile = int32_t(t);
            it.s0 = int32_t(s.causal ? std::min(rows, std::max<int64_t>(0, t - off) << s.gs) : 0);
            it.s1 = int32_t(rows);
            f(small_keys ? kKeysSmall : kKeysLarge, it);
        }
    }
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
        if ((lq << s.gs) > (int64_t(1) << 31) - 4 * kRowTile || lk > (int64_t(1) << 31) - 4 * kRowTile)
            return fail(GT_ERR_UNSUPPORTED, w + ": a sequence of this many rows");
        pair += lq * ((lk + 15) / 16 * 16);
    }
    *pair_bytes = pair;
    return GT_OK;
}

gt_status plan_lists(const Seqs& s, int64_t (&count)[kPackedLists]) {
    for (auto& c : count) c = 0;
    each_item(s, [&](int list, const PackedItem&) { ++count[list]; });
    return GT_OK;
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
    const Seqs s = {n_seq, q_ptr, k_ptr, ilog2(g), causal != 0};
    int64_t pair = 0;
    gt_status st = check_seqs(who, s, &pair);
    if (st != GT_OK) return st;
    int64_t count[kPackedLists];
    if ((st = plan_lists(s, count)) != GT_OK) return st;
    int64_t at = 0;
    for (int l = 0; l < kPackedLists; ++l) {
        if (count[l] * Hkv > (int64_t(1) << 31) - 64)  // one block for each item and kv head
            return fail(GT_ERR_UNSUPPORTED, std::string(who) + ": more than 2^31 tiles");
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
    const Seqs s = {n_seq, q_ptr, k_ptr, ilog2(plan->H / plan->Hkv), plan->causal != 0};
    int64_t pair = 0;
    gt_status st = check_seqs(who, s, &pair);
    if (st != GT_OK) return st;
    int64_t count[kPackedLists];
    if ((st = plan_lists(s, count)) != GT_OK) return st;
    bool same = pair == plan->pair_bytes && q_ptr[n_seq] == plan->nq && k_ptr[n_seq] == plan->nk;
    for (int l = 0; l < kPackedLists; ++l) same = same && count[l] == plan->layout[2 * l + 1];
    if (!same) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": the sequences differ from init's");
    PackedItem* list[kPackedLists];
    for (int l = 0; l < kPackedLists; ++l)
        list[l] = reinterpret_cast<PackedItem*>(static_cast<char*>(host_items) + plan->layout[2 * l]);
    int64_t fill[kPackedLists] = {};
    each_item(s, [&](int l, const PackedItem& it) { list[l][fill[l]++] = it; });
    // the longest walks first, so that no long one starts when the chip runs empty
    for (int l = 0; l < kPackedLists; ++l)
        std::sort(list[l], list[l] + count[l], [](const PackedItem& a, const PackedItem& b) {
            const int32_t ca = a.s1 - a.s0, cb = b.s1 - b.s0;
            return ca != cb ? ca > cb : a.q0 != b.q0 ? a.q0 < b.q0 : a.k0 != b.k0 ? a.k0 < b.k0 : a.tile < b.tile;
        });
    return GT_OK;
}
