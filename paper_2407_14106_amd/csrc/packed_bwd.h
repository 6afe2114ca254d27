// Packed-sequence attention, backward, from the forward's LSE: the row pass (dQ,
// and with a learned bias the table's gradient) and the key pass (dK, dV); no
// atomics on results, so they are the same run to run.
#pragma once

#include "packed_kernels.h"

namespace gt {
namespace {

enum RowPass { kStat, kGrad };

// kGrad: dQ_i = scale sum_j dS_ij K_j with dS_ij = P_ij (dP_ij - D_i); the dP
// products start from -D_i, so their sum is dP - D with no subtraction.  Without
// a bias D_i = <dO_i, O_i> (written here for the key pass).
// kStat (before it, with a bias): D_i = sum_j P_ij dP_ij from the scores, since a
// bf16 O is off by 2^-9, which moves the table's gradient (fp32) by as much,
// and the weights' sum under the given LSE: an fp32 LSE beside a large bias
// holds log(sum) only roughly, so P is normalised again by it.
// The table's gradient: every lane adds the dS of its row to a column of its own
// in LDS ([bucket][lane]: no two lanes meet, and the order of additions is the
// program's), summed over the lanes at the end.
template <typename T, int D, int WAVES, bool BIAS, RowPass PASS>
__global__ __launch_bounds__(WAVES * kWave) void k_packed_rows(PackedArgs a) {
    using B = Blk<T, D>;
    __shared__ __attribute__((aligned(16))) T sK0[B::kElems], sK1[B::kElems], sV0[B::kElems], sV1[B::kElems];
    extern __shared__ float s_dyn[];
    PackedItem it;
    int hk;
    int64_t block;
    if (!packed_place<WAVES == 1>(a, it, hk, block)) return;
    const int lane = lane_id(), wave = uniform(int(threadIdx.x) / kWave);
    const int gs = a.gs, gm = (1 << gs) - 1, R = it.lq << gs, off = it.lk - it.lq;
    const int row0 = it.tile + wave * 32;
    float* s_tab = s_dyn;
    float* hist = s_dyn + (kTableStride << gs) + wave * (a.B + 1) * kWave;
    if constexpr (BIAS) {
        load_table(s_tab, a, hk);
        if constexpr (PASS == kGrad)
            for (int x = 0; x <= a.B; ++x) hist[x * kWave + lane] = 0.f;
    }
    auto limit = [&](int q) {
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
    const int r = row0 + (lane & 31), rc = r < R ? r : R - 1;
    const int q = rc >> gs, hg = rc & gm;
    const int64_t at = int64_t(it.q0 + q) * a.H + (hk << gs) + hg;
    const int lim = r < R ? limit(q) : 0;  // a row past the end takes no part, in the table's gradient either
    const int lo = uniform(row0 + 32 <= R ? limit(row0 >> gs) : 0);
    const int hi = uniform(row0 < R ? limit((row0 + 31 < R ? row0 + 31 : R - 1) >> gs) : 0);
    typename B::Row qf[1], gf[1];
    qf[0].load(static_cast<const T*>(a.Q) + int64_t(it.q0 + q) * a.ldq + ((hk << gs) + hg) * D, lane);
    gf[0].load(static_cast<const T*>(a.dO) + at * D, lane);
    const float sl2 = a.scale * kLog2e;
    float L = a.LSE[at], lg = 0.f, Dq = 0.f;
    if (L == -kInf) L = 0.f;  // an empty row: every score is masked
    if constexpr (!BIAS) {
        L *= kLog2e;
        typename B::Row of;
        of.load(static_cast<const T*>(a.O) + at * D, lane);
        Dq = pair_sum(gf[0].dot(of));
        if (r < R && lane < 32) a.Dv[at] = Dq;
    } else if constexpr (PASS == kGrad) {
        lg = a.Lg[at];
        Dq = a.Dv[at];
    }
    f32x16_t acc[1][D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[0][db] = splat16(0.f);
    float sum = 0.f, dsum = 0.f;
    const int64_t wide = (int64_t(it.lk) + 15) & ~int64_t(15);
    stage_done<WAVES>();
    auto stage = [&](int kbase, const T* cK, const T* cV, T* nK, T* nV) {
        if (kbase + B::kStage < it.s1) fetch(kbase + B::kStage, nK, nV);
#pragma unroll
        for (int kb = 0; kb < B::kStage / 32; ++kb) {
            const int key0 = kbase + 32 * kb;
            if (key0 >= hi) break;  // uniform
            uint32_t id4[4];
            if constexpr (BIAS) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int k = key0 + 8 * j + 4 * (lane >> 5);
                    id4[j] = k < wide ? *reinterpret_cast<const uint32_t*>(a.ids + it.pair + q * wide + k) : ~0u;
                }
            }
            f32x16_t s[1] = {splat16(0.f)}, dp[1] = {splat16(-Dq)};
            B::template rows<1>(cK, 32 * kb, qf, s, lane);
            B::template rows<1>(cV, 32 * kb, gf, dp, lane);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if constexpr (BIAS) {
                    const uint32_t id = (id4[i >> 2] >> (8 * (i & 3))) & 255u;
                    const float u = fmaf(s[0][i], a.scale,
                                         s_tab[hg * kTableStride + (id < kMaxBuckets ? id : kMaxBuckets)]);
                    s[0][i] = fmaf(u - L, kLog2e, -lg);
                } else {
                    s[0][i] = fmaf(s[0][i], sl2, -L);
                }
            }
            if (key0 + 32 > lo) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (key0 + crow(i, lane) >= lim) s[0][i] = -kInf, dp[0][i] = 0.f;
            }
            if constexpr (PASS == kStat) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float p = ex2(s[0][i]);
                    sum += p;
                    dsum = fmaf(p, dp[0][i], dsum);
                }
            } else {
                typename B::Cols kt;
                kt.load(cK, 32 * kb, lane);
                if (key0 + 32 > it.s1) kt.drop(it.s1 - key0, lane);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[0][i] = ex2(s[0][i]) * dp[0][i];
                    if constexpr (BIAS) {
                        const int id = int((id4[i >> 2] >> (8 * (i & 3))) & 255u);
                        hist[(id < a.B ? id : a.B) * kWave + lane] += s[0][i];
                    }
                }
                B::template apply<1>(kt, s, acc);
            }
        }
        stage_done<WAVES>();
    };
    for (int kbase = it.s0; kbase < it.s1; kbase += 2 * B::kStage) {
        stage(kbase, sK0, sV0, sK1, sV1);
        if (kbase + B::kStage < it.s1) stage(kbase + B::kStage, sK1, sV1, sK0, sV0);
    }
    if constexpr (PASS == kStat) {
        sum = pair_sum(sum);
        dsum = pair_sum(dsum);
        if (r < R && lane < 32) {
            a.Dv[at] = sum == 0.f ? 0.f : dsum / sum;
            a.Lg[at] = sum == 0.f ? 0.f : __log2f(sum);
        }
    } else {
        if (r < R) B::store(static_cast<T*>(a.out0) + at * D, acc[0], a.scale, lane);
        if constexpr (BIAS) {
            __syncthreads();
            // a lane's rows all belong to head lane % g of the group (tiles start at multiples of 32)
            for (int x = int(threadIdx.x); x < (a.B << gs); x += int(blockDim.x)) {
                const int head = x / a.B, b = x % a.B;
                const float* h0 = s_dyn + (kTableStride << gs) + b * kWave;
                float t = 0.f;
                for (int w = 0; w < WAVES; ++w)
                    for (int k = 0; k < kWave >> gs; ++k)
                        t += h0[w * (a.B + 1) * kWave + ((((k + x) & ((kWave >> gs) - 1)) << gs) | head)];
                a.hist[block * (int64_t(a.B) << gs) + x] = t;
            }
        }
    }
}

// dK_j = scale sum_i dS_ij Q_i and dV_j = sum_i P_ij dO_i over the rows of the
// whole group, with the wavefront owning 32 keys and the rows streaming through
// LDS; the dP products start from the rows' -D_i.
template <typename T, int D, int WAVES, bool BIAS>
__global__ __launch_bounds__(WAVES * kWave) void k_packed_keys(PackedArgs a) {
    using B = Blk<T, D>;
    __shared__ __attribute__((aligned(16))) T sQ0[B::kElems], sQ1[B::kElems], sG0[B::kElems], sG1[B::kElems];
    // per row of a stage: LSE (exp2 domain without a bias), -D, log2 of the weights' sum
    __shared__ __attribute__((aligned(16))) float sR0[3][B::kStage], sR1[3][B::kStage];
    extern __shared__ float s_tab[];
    PackedItem it;
    int hk;
    int64_t block;
    if (!packed_place<WAVES == 1>(a, it, hk, block)) return;
    const int lane = lane_id(), wave = uniform(int(threadIdx.x) / kWave);
    const int gs = a.gs, gm = (1 << gs) - 1, off = it.lk - it.lq;
    const int key0 = it.tile + wave * 32;
    if constexpr (BIAS) load_table(s_tab, a, hk);
    float rs[3] = {0.f, 0.f, 0.f};
    auto load_stats = [&](int base) {
        if (wave != 0) return;
        const int r = base + lane;
        rs[0] = BIAS ? 0.f : kInf;  // rows past the end weigh nothing
        rs[1] = 0.f;
        rs[2] = BIAS ? kInf : 0.f;
        if (lane < B::kStage && r < it.s1) {
            const int64_t at = int64_t(it.q0 + (r >> gs)) * a.H + (hk << gs) + (r & gm);
            const float L = a.LSE[at];
            rs[0] = L == -kInf ? 0.f : BIAS ? L : L * kLog2e;
            rs[1] = -a.Dv[at];
            if constexpr (BIAS) rs[2] = a.Lg[at];
        }
    };
    auto store_stats = [&](float(&to)[3][B::kStage]) {
        if (wave == 0 && lane < B::kStage) to[0][lane] = rs[0], to[1][lane] = rs[1], to[2][lane] = rs[2];
    };
    const T* Q = static_cast<const T*>(a.Q) + int64_t(it.q0) * a.ldq + (hk << gs) * D;
    const T* G = static_cast<const T*>(a.dO) + (int64_t(it.q0) * a.H + (hk << gs)) * D;
    auto fetch = [&](int base, T* toQ, T* toG) {
        const int rows = it.s1 - base;
        auto row = [&](int r) { return base + r < it.s1 ? base + r : it.s1 - 1; };
        B::template fetch<WAVES>(toQ, rows, wave, lane,
                                 [&](int r) { return Q + int64_t(row(r) >> gs) * a.ldq + (row(r) & gm) * D; });
        B::template fetch<WAVES>(toG, rows, wave, lane, [&](int r) {
            return G + (int64_t(row(r) >> gs) * a.H + (row(r) & gm)) * D;
        });
    };
    if (it.s0 < it.s1) {
        load_stats(it.s0);
        fetch(it.s0, sQ0, sG0);
    }
    const int j = key0 + (lane & 31), jc = j < it.lk ? j : it.lk - 1;
    auto first_row = [&](int key) { return a.causal && key > off ? (key - off) << gs : 0; };
    const int rmin = first_row(jc);
    const int rlo = uniform(first_row(key0 < it.lk ? key0 : it.lk - 1));
    const int rhi = uniform(first_row(key0 + 31 < it.lk ? key0 + 31 : it.lk - 1));
    typename B::Row kf[1], vf[1];
    kf[0].load(static_cast<const T*>(a.K) + int64_t(it.k0 + jc) * a.ldk + hk * D, lane);
    vf[0].load(static_cast<const T*>(a.V) + int64_t(it.k0 + jc) * a.ldv + hk * D, lane);
    f32x16_t dk[1][D / 32], dv[1][D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) dk[0][db] = dv[0][db] = splat16(0.f);
    const float sl2 = a.scale * kLog2e;
    const int64_t wide = (int64_t(it.lk) + 15) & ~int64_t(15);
    store_stats(sR0);
    stage_done<WAVES>();
    auto stage = [&](int base, const T* cQ, const T* cG, const float(&cR)[3][B::kStage], T* nQ, T* nG,
                     float(&nR)[3][B::kStage]) {
        const bool more = base + B::kStage < it.s1;
        if (more) {
            load_stats(base + B::kStage);
            fetch(base + B::kStage, nQ, nG);
        }
#pragma unroll
        for (int rb = 0; rb < B::kStage / 32; ++rb) {
            const int r0 = base + 32 * rb;
            if (r0 >= it.s1 || key0 >= it.lk) break;  // uniform
            if (r0 + 32 <= rlo) continue;             // before every key of this wavefront
            uint32_t id[16];
            if constexpr (BIAS) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int r = r0 + crow(i, lane);
                    id[i] = r < it.s1 ? a.ids[it.pair + (r >> gs) * wide + jc] : 255u;
                }
            }
            f32x16_t s[1] = {splat16(0.f)}, dp[1];
            float L[16], lg[16];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int r = 32 * rb + 8 * x + 4 * (lane >> 5);
                const float4 l4 = *reinterpret_cast<const float4*>(&cR[0][r]);
                const float4 d4 = *reinterpret_cast<const float4*>(&cR[1][r]);
                L[4 * x] = l4.x, L[4 * x + 1] = l4.y, L[4 * x + 2] = l4.z, L[4 * x + 3] = l4.w;
                dp[0][4 * x] = d4.x, dp[0][4 * x + 1] = d4.y, dp[0][4 * x + 2] = d4.z, dp[0][4 * x + 3] = d4.w;
                if constexpr (BIAS) {
                    const float4 g4 = *reinterpret_cast<const float4*>(&cR[2][r]);
                    lg[4 * x] = g4.x, lg[4 * x + 1] = g4.y, lg[4 * x + 2] = g4.z, lg[4 * x + 3] = g4.w;
                }
            }
            B::template rows<1>(cQ, 32 * rb, kf, s, lane);
            B::template rows<1>(cG, 32 * rb, vf, dp, lane);
            typename B::Cols gt_, qt;
            gt_.load(cG, 32 * rb, lane);
            qt.load(cQ, 32 * rb, lane);
            if (r0 + 32 > it.s1) {
                gt_.drop(it.s1 - r0, lane);
                qt.drop(it.s1 - r0, lane);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if constexpr (BIAS) {
                    const float u = fmaf(s[0][i], a.scale, s_tab[((r0 + crow(i, lane)) & gm) * kTableStride +
                                                                 (id[i] < kMaxBuckets ? id[i] : kMaxBuckets)]);
                    s[0][i] = fmaf(u - L[i], kLog2e, -lg[i]);
                } else {
                    s[0][i] = fmaf(s[0][i], sl2, -L[i]);
                }
            }
            if (r0 < rhi || r0 + 32 > it.s1) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int r = r0 + crow(i, lane);
                    if (r < rmin || r >= it.s1) s[0][i] = -kInf, dp[0][i] = 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[0][i] = ex2(s[0][i]);
                dp[0][i] *= s[0][i];
            }
            B::template apply<1>(gt_, s, dv);
            B::template apply<1>(qt, dp, dk);
        }
        if (more) store_stats(nR);
        stage_done<WAVES>();
    };
    for (int base = it.s0; base < it.s1; base += 2 * B::kStage) {
        stage(base, sQ0, sG0, sR0, sQ1, sG1, sR1);
        if (base + B::kStage < it.s1) stage(base + B::kStage, sQ1, sG1, sR1, sQ0, sG0, sR0);
    }
    if (j < it.lk) {
        const int64_t at = int64_t(it.k0 + j) * a.Hkv + hk;
        B::store(static_cast<T*>(a.out1) + at * D, dk[0], a.scale, lane);
        B::store(static_cast<T*>(a.out2) + at * D, dv[0], 1.f, lane);
    }
}

// dtable[b, h]: the blocks' partial sums, one workgroup per head; thread t of a
// bucket adds the blocks t, t + 64, ... of that head, then the 64 are added.
template <bool SMALL>
__device__ __forceinline__ int64_t hist_block(int64_t i, int hk, int64_t items, int Hkv) {
    return SMALL ? i * Hkv + hk : hk * items + i;
}
__global__ __launch_bounds__(256) void k_packed_table(int64_t n_small, int64_t n_large, int H, int Hkv, int gs, int B,
                                                      const float* __restrict__ hist, float* __restrict__ out) {
    const int h = int(blockIdx.x), b = int(blockIdx.y), hk = h >> gs, hg = h & ((1 << gs) - 1);
    const int64_t per = int64_t(B) << gs;
    float t = 0.f;
    for (int64_t i = threadIdx.x; i < n_small + n_large; i += 256) {
        const int64_t blk = i < n_small ? hist_block<true>(i, hk, n_small, Hkv)
                                        : n_small * Hkv + hist_block<false>(i - n_small, hk, n_large, Hkv);
        t += hist[blk * per + hg * B + b];
    }
    __shared__ float s[4];
    t = wave_sum(t);
    if (lane_id() == 0) s[threadIdx.x / kWave] = t;
    __syncthreads();
    if (threadIdx.x == 0) out[int64_t(b) * H + h] = (s[0] + s[1]) + (s[2] + s[3]);
}

template <typename T, int D, bool BIAS>
gt_status packed_bwd_d(const gt_packed_plan* p, PackedArgs a, float* dtable, hipStream_t s) {
    const size_t tab = BIAS ? size_t(kTableStride << a.gs) * sizeof(float) : 0;
    const size_t col = BIAS ? size_t(a.B + 1) * kWave * sizeof(float) : 0;
    const int64_t n1 = packed_items(p, kRowsSmall), n4 = packed_items(p, kRowsLarge);
    float* hist = a.hist;
    auto rows = [&](auto pass) -> gt_status {
        constexpr RowPass P = decltype(pass)::value;
        a.items = packed_list(p, kRowsSmall);
        a.hist = hist;
        if ((a.n_items = int(n1)) > 0)
            k_packed_rows<T, D, 1, BIAS, P><<<packed_grid(n1, a.Hkv), kWave, tab + (P == kGrad ? col : 0), s>>>(a);
        GT_LAUNCH_CHECK("packed_bwd rows");
        a.items = packed_list(p, kRowsLarge);
        a.hist = BIAS ? hist + n1 * a.Hkv * (int64_t(a.B) << a.gs) : nullptr;
        if ((a.n_items = int(n4)) > 0)
            k_packed_rows<T, D, 4, BIAS, P><<<packed_grid(n4, a.Hkv), 4 * kWave, tab + (P == kGrad ? 4 * col : 0), s>>>(a);
        GT_LAUNCH_CHECK("packed_bwd rows");
        return GT_OK;
    };
    if constexpr (BIAS) {
        const gt_status st = rows(std::integral_constant<RowPass, kStat>{});
        if (st != GT_OK) return st;
    }
    const gt_status st = rows(std::integral_constant<RowPass, kGrad>{});
    if (st != GT_OK) return st;
    a.items = packed_list(p, kKeysSmall);
    if ((a.n_items = int(packed_items(p, kKeysSmall))) > 0)
        k_packed_keys<T, D, 1, BIAS><<<packed_grid(a.n_items, a.Hkv), kWave, tab, s>>>(a);
    GT_LAUNCH_CHECK("packed_bwd keys");
    a.items = packed_list(p, kKeysLarge);
    if ((a.n_items = int(packed_items(p, kKeysLarge))) > 0)
        k_packed_keys<T, D, 4, BIAS><<<packed_grid(a.n_items, a.Hkv), 4 * kWave, tab, s>>>(a);
    GT_LAUNCH_CHECK("packed_bwd keys");
    if constexpr (BIAS) {
        k_packed_table<<<dim3(a.H, a.B), 256, 0, s>>>(n1, n4, a.H, a.Hkv, a.gs, a.B, hist, dtable);
        GT_LAUNCH_CHECK("packed_bwd table");
    }
    return GT_OK;
}

}  // namespace

template <typename T>
gt_status packed_bwd(const gt_packed_plan* p, int d, PackedArgs a, float* dtable, hipStream_t s) {
    const bool bias = a.B > 0;
    switch (d) {
        case 32: return bias ? packed_bwd_d<T, 32, true>(p, a, dtable, s) : packed_bwd_d<T, 32, false>(p, a, dtable, s);
        case 64: return bias ? packed_bwd_d<T, 64, true>(p, a, dtable, s) : packed_bwd_d<T, 64, false>(p, a, dtable, s);
        case 128:
            return bias ? packed_bwd_d<T, 128, true>(p, a, dtable, s) : packed_bwd_d<T, 128, false>(p, a, dtable, s);
    }
    return fail(GT_ERR_UNSUPPORTED, "packed attention: d must be 32, 64 or 128");
}

}  // namespace gt
