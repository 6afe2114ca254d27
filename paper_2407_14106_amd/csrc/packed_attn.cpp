// Entry points of packed-sequence attention: argument checks and workspaces.
#include "packed.h"

using namespace gt;

namespace gt {
bool packed_plan_ok(const gt_packed_plan* p);

extern template gt_status packed_fwd<uint16_t>(const gt_packed_plan*, int, PackedArgs, hipStream_t);
extern template gt_status packed_fwd<float>(const gt_packed_plan*, int, PackedArgs, hipStream_t);
extern template gt_status packed_bwd<uint16_t>(const gt_packed_plan*, int, PackedArgs, float*, hipStream_t);
extern template gt_status packed_bwd<float>(const gt_packed_plan*, int, PackedArgs, float*, hipStream_t);
}  // namespace gt

namespace {

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

gt_status check(const char* who, const gt_packed_plan* p, int32_t d, gt_dtype dt, const void* Q, int64_t ldq,
                const void* K, int64_t ldk, const void* V, int64_t ldv) {
    const std::string w(who);
    if (!packed_plan_ok(p)) return fail(GT_ERR_INVALID_ARG, w + ": null plan, or one that gt_packed_plan_init did not make");
    if (p->item_bytes > 0 && !p->items) return fail(GT_ERR_INVALID_ARG, w + ": plan->items is null");
    if (off16(p->items)) return fail(GT_ERR_UNSUPPORTED, w + ": plan->items must start at a multiple of 16 bytes");
    if ((dt != GT_BF16 && dt != GT_F32) || (d != 32 && d != 64 && d != 128))
        return fail(GT_ERR_UNSUPPORTED, w + ": unsupported (dtype, d)");
    if ((p->nq > 0 && !Q) || (p->nk > 0 && (!K || !V))) return fail(GT_ERR_INVALID_ARG, w + ": null pointer");
    const int64_t piece = dt == GT_BF16 ? 8 : 4;
    if (ldq < int64_t(p->H) * d || ldk < int64_t(p->Hkv) * d || ldv < int64_t(p->Hkv) * d ||
        ldq >= (int64_t(1) << 23) || ldk >= (int64_t(1) << 23) || ldv >= (int64_t(1) << 23))
        return fail(GT_ERR_INVALID_ARG, w + ": a node stride below the node's features, or 2^23 or more");
    if (off16(Q) || off16(K) || off16(V) || ldq % piece || ldk % piece || ldv % piece)
        return fail(GT_ERR_UNSUPPORTED, w + ": features must lie at multiples of 16 bytes");
    return GT_OK;
}

gt_status check_bias(const char* who, const gt_packed_plan* p, const float* table, int32_t B, const uint8_t* ids) {
    const std::string w(who);
    if (B < 1 || B > GT_MAX_BUCKETS) return fail(GT_ERR_UNSUPPORTED, w + ": 1 to 64 buckets");
    if (!table || (p->pair_bytes > 0 && !ids)) return fail(GT_ERR_INVALID_ARG, w + ": null pointer");
    if (off16(ids)) return fail(GT_ERR_UNSUPPORTED, w + ": buckets must start at a multiple of 16 bytes");
    return GT_OK;
}

PackedArgs args(const gt_packed_plan* p, const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V,
                int64_t ldv, float scale) {
    PackedArgs a = {};
    a.H = p->H;
    a.Hkv = p->Hkv;
    a.gs = ilog2(p->H / p->Hkv);
    a.causal = p->causal;
    a.Q = Q, a.K = K, a.V = V;
    a.ldq = uint32_t(ldq), a.ldk = uint32_t(ldk), a.ldv = uint32_t(ldv);
    a.scale = scale;
    return a;
}

gt_status run_fwd(const gt_packed_plan* p, int32_t d, gt_dtype dt, PackedArgs a, hipStream_t s) {
    return dt == GT_BF16 ? packed_fwd<uint16_t>(p, d, a, s) : packed_fwd<float>(p, d, a, s);
}

// The largest slot of each pass times the slots there are.
int64_t row_slots(const gt_packed_plan* p) { return p->layout[kRowSlotsAt] * p->Hkv; }
int64_t key_slots(const gt_packed_plan* p) { return p->layout[kKeySlotsAt] * p->Hkv; }

struct BwdWs {
    float *Dv, *Lg = nullptr, *slots, *hist = nullptr;
    BwdWs(Ws& w, const gt_packed_plan* p, int32_t d, gt_dtype dt, int32_t B) {
        Dv = w.take<float>(size_t(p->nq) * p->H);
        const int64_t a = row_slots(p) * row_slot_floats(d), b = key_slots(p) * key_slot_floats(d);
        slots = w.take<float>(size_t(a > b ? a : b));
        if (B == 0) return;
        Lg = w.take<float>(size_t(p->nq) * p->H);
        const int row = d * (dt == GT_BF16 ? 2 : 4);
        int64_t blocks = packed_items(p, kPairs) > 0 ? pair_blocks(p, row) * pair_waves(row) : 0;
        for (int l = kRowsFew; l <= kRows256; ++l) blocks += packed_items(p, l) * p->Hkv * (l == kRows256 ? 2 : 1);
        hist = w.take<float>(size_t(blocks) * (p->H / p->Hkv) * B);
    }
};

size_t bwd_ws(const gt_packed_plan* p, int32_t d, gt_dtype dt, int32_t B) {
    if (!packed_plan_ok(p) || d < 1 || d > 128) return 0;
    Ws w(nullptr);
    BwdWs b(w, p, d, dt, B);
    return w.size();
}

size_t fwd_ws(const gt_packed_plan* p, int32_t d) {
    if (!packed_plan_ok(p) || d < 1 || d > 128) return 0;
    Ws w(nullptr);
    w.take<float>(size_t(row_slots(p) * fwd_slot_floats(d)));
    return w.size();
}

gt_status take_fwd_ws(const char* who, const gt_packed_plan* p, int32_t d, PackedArgs& a, void* ws, size_t ws_bytes) {
    const size_t need = fwd_ws(p, d);
    if (ws_bytes < need) return fail(GT_ERR_WORKSPACE, std::string(who) + ": workspace too small");
    if (need > 0 && !ws) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    a.slots = static_cast<float*>(ws);
    return GT_OK;
}

gt_status run_bwd(const char* who, const gt_packed_plan* p, int32_t d, gt_dtype dt, PackedArgs a, const void* O,
                  const void* dO, const float* LSE, void* dQ, void* dK, void* dV, float* dtable, void* ws,
                  size_t ws_bytes, hipStream_t s) {
    const std::string w(who);
    if ((p->nq > 0 && (!dO || !LSE || !dQ || (a.B == 0 && !O))) || (p->nk > 0 && (!dK || !dV)))
        return fail(GT_ERR_INVALID_ARG, w + ": null pointer");
    if (off16(O) || off16(dO) || off16(dQ) || off16(dK) || off16(dV))
        return fail(GT_ERR_UNSUPPORTED, w + ": features must lie at multiples of 16 bytes");
    const size_t need = bwd_ws(p, d, dt, a.B);
    if (ws_bytes < need) return fail(GT_ERR_WORKSPACE, w + ": workspace too small");
    if (need > 0 && !ws) return fail(GT_ERR_INVALID_ARG, w + ": null pointer");
    Ws wk(ws);
    const BwdWs b(wk, p, d, dt, a.B);
    a.O = O, a.dO = dO;
    a.LSE = const_cast<float*>(LSE);
    a.out0 = dQ, a.out1 = dK, a.out2 = dV;
    a.Dv = b.Dv, a.Lg = b.Lg, a.slots = b.slots, a.hist = b.hist;
    return dt == GT_BF16 ? packed_bwd<uint16_t>(p, d, a, dtable, s) : packed_bwd<float>(p, d, a, dtable, s);
}

}  // namespace

extern "C" size_t gt_packed_attn_fwd_workspace_size(const gt_packed_plan* p, int32_t d, gt_dtype) {
    return fwd_ws(p, d);
}

extern "C" gt_status gt_packed_attn_fwd(const gt_packed_plan* p, int32_t d, gt_dtype dt, const void* Q, int64_t ldq,
                                        const void* K, int64_t ldk, const void* V, int64_t ldv, float scale, void* O,
                                        float* LSE, void* ws, size_t ws_bytes, hipStream_t s) {
    const char* who = "gt_packed_attn_fwd";
    gt_status st = check(who, p, d, dt, Q, ldq, K, ldk, V, ldv);
    if (st != GT_OK) return st;
    if (p->nq > 0 && (!O || !LSE)) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    if (off16(O)) return fail(GT_ERR_UNSUPPORTED, std::string(who) + ": features must lie at multiples of 16 bytes");
    PackedArgs a = args(p, Q, ldq, K, ldk, V, ldv, scale);
    a.out0 = O;
    a.LSE = LSE;
    if ((st = take_fwd_ws(who, p, d, a, ws, ws_bytes)) != GT_OK) return st;
    return run_fwd(p, d, dt, a, s);
}

extern "C" size_t gt_packed_attn_fwd_bias_workspace_size(const gt_packed_plan* p, int32_t d, gt_dtype, int32_t) {
    return fwd_ws(p, d);
}

extern "C" gt_status gt_packed_attn_fwd_bias(const gt_packed_plan* p, int32_t d, gt_dtype dt, const void* Q,
                                             int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                                             const float* table, int32_t B, const uint8_t* ids, float scale, void* O,
                                             float* LSE, void* ws, size_t ws_bytes, hipStream_t s) {
    const char* who = "gt_packed_attn_fwd_bias";
    gt_status st = check(who, p, d, dt, Q, ldq, K, ldk, V, ldv);
    if (st == GT_OK) st = check_bias(who, p, table, B, ids);
    if (st != GT_OK) return st;
    if (p->nq > 0 && (!O || !LSE)) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    if (off16(O)) return fail(GT_ERR_UNSUPPORTED, std::string(who) + ": features must lie at multiples of 16 bytes");
    PackedArgs a = args(p, Q, ldq, K, ldk, V, ldv, scale);
    a.out0 = O;
    a.LSE = LSE;
    a.table = table, a.B = B, a.ids = ids;
    if ((st = take_fwd_ws(who, p, d, a, ws, ws_bytes)) != GT_OK) return st;
    return run_fwd(p, d, dt, a, s);
}

extern "C" size_t gt_packed_attn_bwd_workspace_size(const gt_packed_plan* p, int32_t d, gt_dtype dt) {
    return bwd_ws(p, d, dt, 0);
}

extern "C" gt_status gt_packed_attn_bwd(const gt_packed_plan* p, int32_t d, gt_dtype dt, const void* Q, int64_t ldq,
                                        const void* K, int64_t ldk, const void* V, int64_t ldv, const void* O,
                                        const void* dO, const float* LSE, float scale, void* dQ, void* dK, void* dV,
                                        void* ws, size_t ws_bytes, hipStream_t s) {
    const char* who = "gt_packed_attn_bwd";
    const gt_status st = check(who, p, d, dt, Q, ldq, K, ldk, V, ldv);
    if (st != GT_OK) return st;
    return run_bwd(who, p, d, dt, args(p, Q, ldq, K, ldk, V, ldv, scale), O, dO, LSE, dQ, dK, dV, nullptr, ws,
                   ws_bytes, s);
}

extern "C" size_t gt_packed_attn_bwd_bias_workspace_size(const gt_packed_plan* p, int32_t d, gt_dtype dt, int32_t B) {
    return B < 1 || B > GT_MAX_BUCKETS ? 0 : bwd_ws(p, d, dt, B);
}

extern "C" gt_status gt_packed_attn_bwd_bias(const gt_packed_plan* p, int32_t d, gt_dtype dt, const void* Q,
                                             int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                                             const float* table, int32_t B, const uint8_t* ids, const void* dO,
                                             const float* LSE, float scale, void* dQ, void* dK, void* dV, float* dtable,
                                             void* ws, size_t ws_bytes, hipStream_t s) {
    const char* who = "gt_packed_attn_bwd_bias";
    gt_status st = check(who, p, d, dt, Q, ldq, K, ldk, V, ldv);
    if (st == GT_OK) st = check_bias(who, p, table, B, ids);
    if (st != GT_OK) return st;
    if (!dtable) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    PackedArgs a = args(p, Q, ldq, K, ldk, V, ldv, scale);
    a.table = table, a.B = B, a.ids = ids;
    return run_bwd(who, p, d, dt, a, nullptr, dO, LSE, dQ, dK, dV, dtable, ws, ws_bytes, s);
}
