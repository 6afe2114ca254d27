// Packed-sequence attention, forward: for every row of a tile an online softmax
// over its keys, one pass over K and V.
#pragma once

#include "packed_kernels.h"

namespace gt {
namespace {

// The running reference m of a row is checked after the fact: a block's weights
// are summed anyway, and only where a lane's sum of 16 exceeds 2^8 (or is not a
// number) are the scores formed again, the true maximum taken and the
// accumulators rescaled.  m starts at the lowest finite value, so a row that
// attends to nothing keeps weights of zero.  Without a bias m and the scores are
// in the exp2 domain; with one they stay in the natural domain (a bias of the
// type's lowest value times log2 e would overflow to -inf).
template <typename T, int D, int NB, int WAVES, bool BIAS>
__global__ __launch_bounds__(WAVES * kWave) void k_packed_fwd(PackedArgs a) {
    using B = Blk<T, D>;
    __shared__ __attribute__((aligned(16))) T sK0[B::kElems], sK1[B::kElems], sV0[B::kElems], sV1[B::kElems];
    extern __shared__ float s_tab[];
    PackedItem it;
    int hk;
    int64_t block;
    if (!packed_place<WAVES == 1>(a, it, hk, block)) return;
    const int lane = lane_id(), wave = uniform(int(threadIdx.x) / kWave);
    const int gs = a.gs, gm = (1 << gs) - 1, R = it.lq << gs, off = it.lk - it.lq;
    const int row0 = it.tile + wave * 32 * NB;
    if constexpr (BIAS) load_table(s_tab, a, hk);
    auto limit = [&](int q) {  // how many of the item's keys query q attends to
        const int l = a.causal ? off + q + 1 : it.s1;
        return l < it.s1 ? l : it.s1;
    };
    const T* K = static_cast<const T*>(a.K) + int64_t(it.k0) * a.ldk + hk * D;
    const T* V = static_cast<const T*>(a.V) + int64_t(it.k0) * a.ldv + hk * D;
    auto fetch = [&](int kbase, T* toK, T* toV) {
        const int rows = it.s1 - kbase;
        auto key = [&](int r) { return int64_t(kbase + r < it.lk ? kbase + r : it.lk - 1); };
        B::template fetch<WAVES>(toK, rows, wave, lane, [&](int r) { return K + key(r) * a.ldk; });
        B::template fetch<WAVES>(toV, rows, wave, lane, [&](int r) { return V + key(r) * a.ldv; });
    };
    if (it.s0 < it.s1) fetch(it.s0, sK0, sV0);
    typename B::Row qf[NB];
    int lim[NB], q_of[NB], hg[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int r = row0 + 32 * b + (lane & 31), rc = r < R ? r : R - 1;
        q_of[b] = rc >> gs;
        hg[b] = rc & gm;
        lim[b] = limit(q_of[b]);
        qf[b].load(static_cast<const T*>(a.Q) + int64_t(it.q0 + q_of[b]) * a.ldq + ((hk << gs) + hg[b]) * D, lane);
    }
    const int first = row0 < R ? row0 : R - 1, last = row0 + 32 * NB - 1 < R ? row0 + 32 * NB - 1 : R - 1;
    const int lo = uniform(limit(first >> gs)), hi = uniform(row0 < R ? limit(last >> gs) : 0);
    f32x16_t acc[NB][D / 32];
    float m[NB], l[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int db = 0; db < D / 32; ++db) acc[b][db] = splat16(0.f);
        m[b] = kLowest;
        l[b] = 0.f;
    }
    const float sl2 = a.scale * kLog2e;
    const int64_t wide = (int64_t(it.lk) + 15) & ~int64_t(15);
    stage_done<WAVES>();
    auto stage = [&](int kbase, const T* cK, const T* cV, T* nK, T* nV) {
        if (kbase + B::kStage < it.s1) fetch(kbase + B::kStage, nK, nV);
#pragma unroll
        for (int kb = 0; kb < B::kStage / 32; ++kb) {
            const int key0 = kbase + 32 * kb;
            if (key0 >= hi) break;  // uniform
            const bool masked = key0 + 32 > lo;
            uint32_t id4[NB][4];
            if constexpr (BIAS) {
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int k = key0 + 8 * j + 4 * (lane >> 5);
                        id4[b][j] = k < wide ? *reinterpret_cast<const uint32_t*>(a.ids + it.pair + q_of[b] * wide + k)
                                             : ~0u;
                    }
            }
            f32x16_t s[NB];
            auto scores = [&] {
#pragma unroll
                for (int b = 0; b < NB; ++b) s[b] = splat16(0.f);
                B::template rows<NB>(cK, 32 * kb, qf, s, lane);
                if constexpr (BIAS)
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const uint32_t id = (id4[b][i >> 2] >> (8 * (i & 3))) & 255u;
                            s[b][i] = fmaf(s[b][i], a.scale,
                                           s_tab[hg[b] * kTableStride + (id < kMaxBuckets ? id : kMaxBuckets)]);
                        }
            };
            float ls[NB];
            auto weights = [&] {  // s becomes the weights, ls this lane's sums of them
#pragma unroll
                for (int b = 0; b < NB; ++b) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[b][i] = BIAS ? (s[b][i] - m[b]) * kLog2e : fmaf(s[b][i], sl2, -m[b]);
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (key0 + crow(i, lane) >= lim[b]) s[b][i] = -kInf;
                    }
                    float x[2] = {0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        s[b][i] = ex2(s[b][i]);
                        x[i & 1] += s[b][i];
                    }
                    ls[b] = x[0] + x[1];
                }
            };
            scores();
            typename B::Cols vt;
            vt.load(cV, 32 * kb, lane);
            if (key0 + 32 > it.s1) vt.drop(it.s1 - key0, lane);
            __builtin_amdgcn_sched_barrier(0);
            weights();
            bool high = false;
#pragma unroll
            for (int b = 0; b < NB; ++b) high |= !(ls[b] <= 256.f);
            if (__builtin_expect(__builtin_amdgcn_ballot_w64(high) != 0, 0)) {
                scores();
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    float mx = -kInf;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        mx = fmaxf(mx, key0 + crow(i, lane) >= lim[b] ? -kInf : BIAS ? s[b][i] : s[b][i] * sl2);
                    const float mn = fmaxf(m[b], pair_max(mx));
                    const float alpha = ex2(BIAS ? (m[b] - mn) * kLog2e : m[b] - mn);
                    l[b] *= alpha;
#pragma unroll
                    for (int db = 0; db < D / 32; ++db)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[b][db][i] *= alpha;
                    m[b] = mn;
                }
                weights();
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) l[b] += ls[b];
            B::template apply<NB>(vt, s, acc);
        }
        stage_done<WAVES>();
    };
    for (int kbase = it.s0; kbase < it.s1; kbase += 2 * B::kStage) {
        stage(kbase, sK0, sV0, sK1, sV1);
        if (kbase + B::kStage < it.s1) stage(kbase + B::kStage, sK1, sV1, sK0, sV0);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const float lt = pair_sum(l[b]);
        if (row0 + 32 * b + (lane & 31) >= R) continue;
        const int64_t at = int64_t(it.q0 + q_of[b]) * a.H + (hk << gs) + hg[b];
        if (lane < 32)
            a.LSE[at] = lt == 0.f ? -kInf : BIAS ? fmaf(__log2f(lt), kLn2, m[b]) : (m[b] + __log2f(lt)) * kLn2;
        B::store(static_cast<T*>(a.out0) + at * D, acc[b], lt == 0.f ? 0.f : 1.f / lt, lane);
    }
}

template <typename T, int D, bool BIAS>
gt_status packed_fwd_d(const gt_packed_plan* p, PackedArgs a, hipStream_t s) {
    const size_t lds = BIAS ? size_t(kTableStride << a.gs) * sizeof(float) : 0;
    a.items = packed_list(p, kRowsSmall);
    if ((a.n_items = int(packed_items(p, kRowsSmall))) > 0)
        k_packed_fwd<T, D, 1, 1, BIAS><<<packed_grid(a.n_items, a.Hkv), kWave, lds, s>>>(a);
    GT_LAUNCH_CHECK("packed_fwd");
    a.items = packed_list(p, kRowsLarge);
    if ((a.n_items = int(packed_items(p, kRowsLarge))) > 0)
        k_packed_fwd<T, D, 1, 4, BIAS><<<packed_grid(a.n_items, a.Hkv), 4 * kWave, lds, s>>>(a);
    GT_LAUNCH_CHECK("packed_fwd");
    return GT_OK;
}

}  // namespace

template <typename T>
gt_status packed_fwd(const gt_packed_plan* p, int d, PackedArgs a, hipStream_t s) {
    const bool bias = a.B > 0;
    switch (d) {
        case 32: return bias ? packed_fwd_d<T, 32, true>(p, a, s) : packed_fwd_d<T, 32, false>(p, a, s);
        case 64: return bias ? packed_fwd_d<T, 64, true>(p, a, s) : packed_fwd_d<T, 64, false>(p, a, s);
        case 128: return bias ? packed_fwd_d<T, 128, true>(p, a, s) : packed_fwd_d<T, 128, false>(p, a, s);
    }
    return fail(GT_ERR_UNSUPPORTED, "packed attention: d must be 32, 64 or 128");
}

}  // namespace gt
