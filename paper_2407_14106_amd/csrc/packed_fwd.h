// Packed-sequence attention, forward: for every row of a tile an online softmax
// over its keys, one pass over K and V.
#pragma once

#include "packed_kernels.h"

namespace gt {
namespace {

// Pairs: a sequence of at most 32 rows and 32 keys is one block, done by one
// wavefront with nothing shared.  Bound by reading and writing the features and by
// the block's chain of waits, which more wavefronts hide: 4,000 molecules of 23 to 26
// nodes, 8 heads of 32, with a bias, 46 us (133 MB).
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(pair_waves(D * int(sizeof(T))) * kWave) void k_pair_fwd(PackedArgs a) {
    using B = Blk<T, D>;
    constexpr int W = pair_waves(D * int(sizeof(T)));
    __shared__ __attribute__((aligned(16))) T sK[W][B::kElems], sV[W][B::kElems];
    extern __shared__ float s_tabs[];
    const int lane = lane_id(), wave = uniform(int(threadIdx.x) / kWave);
    const uint32_t unit = uint32_t(xcd_block(blockIdx.x, gridDim.x)) * W + wave;
    if (unit >= uint32_t(a.n_items) * uint32_t(a.Hkv)) return;
    const PackedItem it = a.items[unit / uint32_t(a.Hkv)];
    const int hk = int(unit % uint32_t(a.Hkv));
    const int gs = a.gs, gm = (1 << gs) - 1, R = it.lq << gs, off = it.lk - it.lq;
    if (R == 0) return;  // keys without queries are listed for the backward
    if (it.lk > 0) {
        B::template fetch<1>(sK[wave], static_cast<const T*>(a.K) + int64_t(it.k0) * a.ldk + hk * D, it.lk, 0, lane,
                             [&](int r) { return uint32_t(r) * a.ldk; });
        B::template fetch<1>(sV[wave], static_cast<const T*>(a.V) + int64_t(it.k0) * a.ldv + hk * D, it.lk, 0, lane,
                             [&](int r) { return uint32_t(r) * a.ldv; });
    }
    const int r = lane & 31, rc = r < R ? r : R - 1, q = rc >> gs, h = (hk << gs) + (rc & gm);
    typename B::Row qf[1];
    qf[0].load(static_cast<const T*>(a.Q) + int64_t(it.q0 + q) * a.ldq + h * D, lane);
    const int lim = a.causal && off + q + 1 < it.lk ? off + q + 1 : it.lk;
    uint4 ids;
    float* tab = s_tabs + wave * (kTableStride << gs);
    if constexpr (BIAS) {
        if (it.lk > 0) ids = load_ids(a.ids + it.pair + q * ids_width(it.lk), 0, it.lk, lane);
        load_table<kWave>(tab, a, hk, lane);
    }
    f32x16_t s[1] = {splat16(0.f)}, acc[1][D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[0][db] = splat16(0.f);
    wave_done();
    float m = kLowest, l = 0.f;
    if (it.lk > 0) {
        const typename B::At at(lane, 0);
        B::template rows<1>(sK[wave], at, qf, s);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if constexpr (BIAS) {
                s[0][i] = fmaf(s[0][i], a.scale, tab[(rc & gm) * kTableStride + id_of(ids, i, a.B)]);
            } else {
                s[0][i] *= a.scale;
            }
            if (i >= lim - part(0, lane)) s[0][i] = -kInf;
            m = fmaxf(m, s[0][i]);
        }
        m = pair_max(m);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[0][i] = ex2((s[0][i] - m) * kLog2e);
            l += s[0][i];
        }
        l = pair_sum(l);
        typename B::Cols vt;
        vt.load(sV[wave], at);
        B::template apply<1>(vt, s, acc);
    }
    if (r < R) {
        const int64_t out = int64_t(it.q0 + q) * a.H + h;
        if (lane < 32) a.LSE[out] = l == 0.f ? -kInf : fmaf(__log2f(l), kLn2, m);
        B::store(static_cast<T*>(a.out0) + out * D, acc[0], l == 0.f ? 0.f : 1.f / l, lane);
    }
}

// Tiles of 32 NB W rows.  KS sets of W wavefronts take turns at the stages of the
// walk; a set's wavefronts share a stage.  The running reference m of a row is
// checked after the fact: a block's weights are summed anyway, and only where a
// lane's sum of 16 exceeds 2^8 (or is not a number) are the scores formed again,
// the true maximum taken and the accumulators rescaled.  m starts at the lowest
// finite value, so a row that attends to nothing keeps weights of zero.  Without
// a bias m and the scores are in the exp2 domain; with one they stay in the
// natural domain (a bias of the type's lowest value times log2 e would overflow
// to -inf).
// Bound by the matrix cores, then the exponentials: 8,192 x 16 heads bf16 at 950
// (64 wide) and 1,025 TFLOP/s (128), four causal prompts of up to 6,000 (16 / 4
// heads of 128) 206 us, 920 TFLOP/s.  Few rows are bound by reading K and V: 16
// tokens over up to 65,536 keys 293 us, 4.85 TB/s.  With a bias by waiting (38% of
// the wavefronts' time, at two a SIMD) and its vector work (30%): 16 graphs of up to
// 1,000, 8 heads of 64, 36 us.
template <typename T, int D, int STAGE, int NB, int W, int KS, bool BIAS>
__global__ __launch_bounds__(W * KS * kWave) __attribute__((amdgpu_waves_per_eu(
    waves_per_simd(KS * 4 * STAGE * D * int(sizeof(T)), W* KS)))) void k_packed_fwd(PackedArgs a) {
    using B = Blk<T, D, STAGE>;
    // one variable per buffer: the compiler then knows that a stage's reads do not touch the buffer being filled, and
    // does not wait for its loads
    __shared__ __attribute__((aligned(16))) T sK0[KS * B::kElems], sK1[KS * B::kElems];
    __shared__ __attribute__((aligned(16))) T sV0[KS * B::kElems], sV1[KS * B::kElems];
    extern __shared__ float s_tab[];
    PackedItem it;
    int hk, sub;
    uint32_t block;
    if (!packed_place<W == 1>(a, it, hk, sub, block)) return;
    const int lane = lane_id(), wave = uniform(int(threadIdx.x) / kWave);
    const int set = KS == 1 ? 0 : wave / W, row_wave = wave - set * W;
    const int gs = a.gs, gm = (1 << gs) - 1, R = it.lq << gs, off = it.lk - it.lq;
    const int row0 = it.tile + row_wave * 32 * NB;
    if constexpr (BIAS) load_table<W * KS * kWave>(s_tab, a, hk, int(threadIdx.x));
    auto limit = [&](int q) {  // how many of the item's keys query q attends to
        const int l = a.causal ? off + q + 1 : it.s1;
        return l < it.s1 ? l : it.s1;
    };
    const T* K = static_cast<const T*>(a.K) + int64_t(it.k0) * a.ldk + hk * D;
    const T* V = static_cast<const T*>(a.V) + int64_t(it.k0) * a.ldv + hk * D;
    auto fetch = [&](int kbase, T* toK, T* toV) {
        if (kbase >= it.s1) return;
        B::template fetch<W>(toK + set * B::kElems, K + int64_t(kbase) * a.ldk, it.s1 - kbase, row_wave, lane,
                             [&](int r) { return __umul24(r, a.ldk); });
        B::template fetch<W>(toV + set * B::kElems, V + int64_t(kbase) * a.ldv, it.s1 - kbase, row_wave, lane,
                             [&](int r) { return __umul24(r, a.ldv); });
    };
    fetch(it.s0 + set * STAGE, sK0, sV0);
    typename B::Row qf[NB];
    int lim[NB], q_of[NB], hg[NB];
    const uint8_t* id_row[NB];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        const int r = row0 + 32 * b + (lane & 31), rc = r < R ? r : R - 1;
        q_of[b] = rc >> gs;
        hg[b] = rc & gm;
        lim[b] = limit(q_of[b]);
        if constexpr (BIAS) id_row[b] = a.ids + it.pair + q_of[b] * ids_width(it.lk);
        qf[b].load(static_cast<const T*>(a.Q) + int64_t(it.q0 + q_of[b]) * a.ldq + ((hk << gs) + hg[b]) * D, lane);
    }
    const int last = row0 + 32 * NB - 1 < R ? row0 + 32 * NB - 1 : R - 1;
    const int hi = uniform(row0 < R ? limit(last >> gs) : 0);
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
    stage_done<(W > 1) || BIAS>();
    const typename B::At lds(lane, set * B::kElems * int(sizeof(T)));
    // one block of 32 keys; masked: some row does not attend to all of them
    auto block32 = [&](auto masked, int key0, const T* bK, const T* bV, const uint4(&ids)[NB]) {
        int left[NB];  // how many of the lane's 16 keys its row attends to
#pragma unroll
        for (int b = 0; b < NB; ++b) left[b] = lim[b] - key0 - part(0, lane);
        f32x16_t s[NB];
        auto scores = [&] {
#pragma unroll
            for (int b = 0; b < NB; ++b) s[b] = splat16(0.f);
            B::template rows<NB>(bK, lds, qf, s);
            if constexpr (BIAS)
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[b][i] = fmaf(s[b][i], a.scale, s_tab[hg[b] * kTableStride + id_of(ids[b], i, a.B)]);
        };
        float ls[NB];
        auto weights = [&] {  // s becomes the weights, ls this lane's sums of them
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                float x[2] = {0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    float t = BIAS ? (s[b][i] - m[b]) * kLog2e : fmaf(s[b][i], sl2, -m[b]);
                    if constexpr (masked.value) t = i >= left[b] ? -kInf : t;
                    s[b][i] = ex2(t);
                    x[i & 1] += s[b][i];
                }
                ls[b] = x[0] + x[1];
            }
        };
        scores();
        typename B::Cols vt;
        vt.load(bV, lds);
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
                for (int i = 0; i < 16; ++i) {
                    const float t = BIAS ? s[b][i] : s[b][i] * sl2;
                    mx = fmaxf(mx, masked.value && i >= left[b] ? -kInf : t);
                }
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
    };
    uint4 ids[STAGE / 32][NB];  // the buckets of a stage, loaded a stage ahead
    auto next_ids = [&](int kbase) {
        if constexpr (BIAS)
#pragma unroll
            for (int kb = 0; kb < STAGE / 32; ++kb)
#pragma unroll
                for (int b = 0; b < NB; ++b) ids[kb][b] = load_ids(id_row[b], kbase + 32 * kb, it.lk, lane);
    };
    if (it.s0 < it.s1) next_ids(it.s0 + set * STAGE);
    auto stage = [&](auto masked, int kbase, const T* cK, const T* cV, T* nK, T* nV) {
        fetch(kbase + KS * STAGE, nK, nV);
        uint4 now[STAGE / 32][NB];
        if constexpr (BIAS)
#pragma unroll
            for (int kb = 0; kb < STAGE / 32; ++kb)
#pragma unroll
                for (int b = 0; b < NB; ++b) now[kb][b] = ids[kb][b];
        next_ids(kbase + KS * STAGE);
        if constexpr (masked.value) {
#pragma unroll
            for (int kb = 0; kb < STAGE / 32; ++kb)
                if (kbase + 32 * kb < hi)  // uniform
                    block32(masked, kbase + 32 * kb, cK + 32 * kb * D, cV + 32 * kb * D, now[kb]);
        } else {
#pragma unroll
            for (int kb = 0; kb < STAGE / 32; ++kb) {
                __builtin_amdgcn_sched_barrier(0);  // two blocks' operands at once do not fit the registers
                block32(masked, kbase + 32 * kb, cK + 32 * kb * D, cV + 32 * kb * D, now[kb]);
            }
        }
        stage_done<(W > 1)>();
    };
    // every set goes through the same number of stages, the last ones of some behind the walk's end; the stages
    // that every row of the tile attends to whole come first, an even number of them
    constexpr int kRound = KS * STAGE;
    const int first_row = it.tile < R ? it.tile : R - 1, lo = uniform(limit(first_row >> gs));
    int kbase = it.s0;
    for (int n = lo > it.s0 ? (lo - it.s0) / (2 * kRound) : 0; n > 0; --n, kbase += 2 * kRound) {
        stage(Flag<false>{}, kbase + set * STAGE, sK0, sV0, sK1, sV1);
        stage(Flag<false>{}, kbase + kRound + set * STAGE, sK1, sV1, sK0, sV0);
    }
    for (; kbase < it.s1; kbase += 2 * kRound) {
        stage(Flag<true>{}, kbase + set * STAGE, sK0, sV0, sK1, sV1);
        if (kbase + kRound < it.s1) stage(Flag<true>{}, kbase + kRound + set * STAGE, sK1, sV1, sK0, sV0);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) l[b] = pair_sum(l[b]);
    if constexpr (KS > 1) {  // the sets' states: scaled to a common reference, then added by the first set
        __shared__ float s_ml[2 * NB][KS][W * kWave];
        __shared__ float s_acc[KS - 1][8][W * kWave];
        const int at = row_wave * kWave + lane;
#pragma unroll
        for (int b = 0; b < NB; ++b) s_ml[b][set][at] = m[b], s_ml[NB + b][set][at] = l[b];
        __syncthreads();
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            float mn = kLowest, lt = 0.f;
#pragma unroll
            for (int p = 0; p < KS; ++p) mn = fmaxf(mn, s_ml[b][p][at]);
#pragma unroll
            for (int p = 0; p < KS; ++p) {
                const float x = s_ml[b][p][at] - mn;
                lt = fmaf(s_ml[NB + b][p][at], ex2(BIAS ? x * kLog2e : x), lt);
            }
            const float w = ex2(BIAS ? (m[b] - mn) * kLog2e : m[b] - mn);
            m[b] = mn;
            l[b] = lt;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (set > 0)
#pragma unroll
                        for (int i = 0; i < 8; ++i) s_acc[set - 1][i][at] = acc[b][db][8 * half + i] * w;
                    __syncthreads();
                    if (set == 0)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float t = acc[b][db][8 * half + i] * w;
#pragma unroll
                            for (int p = 0; p < KS - 1; ++p) t += s_acc[p][i][at];
                            acc[b][db][8 * half + i] = t;
                        }
                    __syncthreads();
                }
        }
        if (set > 0) return;
    }
    if (it.slot >= 0) {  // a part of a split walk
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if (row0 + 32 * b >= R) break;  // uniform
            float* o = a.slots + (int64_t(it.slot + row_wave * NB + b) * a.Hkv + hk) * (kFewRows * (D + 2));
            const int r = lane & 31;
            if (lane < 32) o[r] = m[b], o[kFewRows + r] = l[b];
            Blk<float, D>::store(o + 2 * kFewRows + r * D, acc[b], 1.f, lane);
        }
        return;
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        if (row0 + 32 * b + (lane & 31) >= R) continue;
        const int64_t at = int64_t(it.q0 + q_of[b]) * a.H + (hk << gs) + hg[b];
        if (lane < 32)
            a.LSE[at] = l[b] == 0.f ? -kInf : BIAS ? fmaf(__log2f(l[b]), kLn2, m[b]) : (m[b] + __log2f(l[b])) * kLn2;
        B::store(static_cast<T*>(a.out0) + at * D, acc[b], l[b] == 0.f ? 0.f : 1.f / l[b], lane);
    }
}

template <typename T, int D, bool BIAS>
gt_status packed_fwd_d(const gt_packed_plan* p, PackedArgs a, hipStream_t s) {
    constexpr int kRow = D * int(sizeof(T)), kStage = sizeof(T) == 2 ? 64 : 32;
    const size_t lds = BIAS ? size_t(kTableStride << a.gs) * sizeof(float) : 0;
    auto list = [&](int l) {
        a.items = packed_list(p, l);
        a.n_items = int(packed_items(p, l));
        return a.n_items > 0;
    };
    if (list(kPairs)) {
        constexpr int W = pair_waves(kRow);
        k_pair_fwd<T, D, BIAS><<<xcd_grid(cdiv(int64_t(a.n_items) * a.Hkv, W)), W * kWave, W * lds, s>>>(a);
        GT_LAUNCH_CHECK("packed_fwd pairs");
    }
#define GT_FWD(LIST, STAGE, NB, W, KS)                                                                            \
    if (list(LIST)) {                                                                                             \
        k_packed_fwd<T, D, STAGE, NB, W, KS, BIAS><<<packed_grid(a.n_items, a.Hkv), W * KS * kWave, lds, s>>>(a); \
        GT_LAUNCH_CHECK("packed_fwd");                                                                            \
    }
    GT_FWD(kRowsFew, 32, 1, 1, few_waves(kRow))
    GT_FWD(kRows64, kStage, 1, 2, 1)
    if (packed_shared<T>(p, kRowSharedAt)) {
        GT_FWD(kRows128, (kRow <= 128 ? kStage : 32), 1, 4, (kRow <= 256 ? 2 : 1))
    } else {
        GT_FWD(kRows128, kStage, 1, 4, 1)
    }
    if constexpr (kRow <= 128 && !BIAS) {  // two blocks of rows and their buckets do not fit the registers
        GT_FWD(kRows256, kStage, 2, 4, 1)
    } else {
        GT_FWD(kRows256, kStage, 1, 8, 1)
    }
#undef GT_FWD
    return list(kRowMerges) ? packed_merge_fwd(p, D, sizeof(T) == 2 ? GT_BF16 : GT_F32, a, s) : GT_OK;
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
