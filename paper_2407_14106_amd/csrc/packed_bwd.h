// Packed-sequence attention, backward, from the forward's LSE: the row pass (dQ,
// and with a learned bias the table's gradient) and the key pass (dK, dV); no
// atomics on results, so they are the same run to run.
#pragma once

#include "packed_kernels.h"

namespace gt {
namespace {

// A block's dS to the lane's column of the table's gradient.
__device__ __forceinline__ void add_block(float* col, const uint4& ids, int B, const f32x16_t& ds) {
#pragma unroll
    for (int i = 0; i < 16; ++i) hist_add(col, id_of(ids, i, B), ds[i]);
}

// Pairs: a sequence of at most 32 rows and 32 keys, all of its backward by one
// wavefront from one reading of Q, K, V and dO: the weights P and dS of the one
// block, D from them, dQ; then the two turned round through LDS, dV and dK.
// With a bias a wavefront keeps to one head and goes through its sequences, its
// part of the table's gradient in LDS (56 KB a workgroup at 21 buckets: two a CU, so
// two wavefronts a SIMD, which wait 56% of their time).  4,000 molecules 94 us.
template <typename T, int D, bool BIAS>
__global__ __launch_bounds__(pair_waves(D * int(sizeof(T))) * kWave)
    __attribute__((amdgpu_waves_per_eu(D * int(sizeof(T)) <= 64 ? 3 : D * int(sizeof(T)) <= 128 ? 2 : 1))) void k_pair_bwd(PackedArgs a) {
    using B = Blk<T, D>;
    using S = Blk<T, 32>;
    constexpr int W = pair_waves(D * int(sizeof(T)));
    __shared__ __attribute__((aligned(16))) T s_q[W][B::kElems], s_k[W][B::kElems], s_v[W][B::kElems], s_g[W][B::kElems];
    extern __shared__ float s_dyn[];
    const int lane = lane_id(), wave = uniform(int(threadIdx.x) / kWave);
    T *sQ = s_q[wave], *sK = s_k[wave], *sV = s_v[wave], *sG = s_g[wave];
    const int gs = a.gs, gm = (1 << gs) - 1;
    const uint32_t first = uint32_t(xcd_block(blockIdx.x, gridDim.x)) * W + wave, step = gridDim.x * W, units = uint32_t(a.n_items) * uint32_t(a.Hkv);
    const int hk = int(first % uint32_t(a.Hkv));  // of every unit: step is a multiple of Hkv
    float* tab = s_dyn + wave * (kTableStride << gs);
    float* hist = s_dyn + W * (kTableStride << gs) + wave * (a.B + 1) * kWave;
    if constexpr (BIAS) {
        load_table<kWave>(tab, a, hk, lane);
        for (int b = 0; b <= a.B; ++b) hist[b * kWave + lane] = 0.f;
    }
    const typename B::At at(lane, 0);
    const typename S::At turned_at(lane, 0);
    PackedItem next = a.items[first < units ? first / uint32_t(a.Hkv) : 0];
    for (uint32_t unit = first; unit < units; unit += step) {
        const PackedItem it = next;
        next = a.items[(unit + step < units ? unit + step : unit) / uint32_t(a.Hkv)];
        const int R = it.lq << gs, off = it.lk - it.lq;
        const int64_t row_at = int64_t(it.q0) * a.H + (hk << gs), key_at = int64_t(it.k0) * a.Hkv + hk;
        const bool some = R > 0 && it.lk > 0;
        const int r = lane & 31, q = r >> gs;
        float L = 0.f;
        uint4 ids;
        if (some) {
            B::template fetch<1>(sK, static_cast<const T*>(a.K) + int64_t(it.k0) * a.ldk + hk * D, it.lk, 0, lane,
                                 [&](int x) { return __umul24(x, a.ldk); });
            B::template fetch<1>(sV, static_cast<const T*>(a.V) + int64_t(it.k0) * a.ldv + hk * D, it.lk, 0, lane,
                                 [&](int x) { return __umul24(x, a.ldv); });
            B::template fetch<1>(sQ, static_cast<const T*>(a.Q) + int64_t(it.q0) * a.ldq + (hk << gs) * D, R, 0, lane,
                                 [&](int x) { return __umul24(x >> gs, a.ldq) + uint32_t((x & gm) * D); });
            B::template fetch<1>(sG, static_cast<const T*>(a.dO) + row_at * D, R, 0, lane,
                                 [&](int x) { return uint32_t(((x >> gs) * a.H + (x & gm)) * D); });
            if (r < R) L = a.LSE[row_at + q * a.H + (r & gm)];
            if (L == -kInf) L = 0.f;  // an empty row: every score is masked
            if constexpr (BIAS)
                ids = load_ids(a.ids + it.pair + (r < R ? q : it.lq - 1) * ids_width(it.lk), 0, it.lk, lane);
        }
        wave_done();
        f32x16_t dq[1][D / 32], dk[1][D / 32], dv[1][D / 32];
#pragma unroll
        for (int db = 0; db < D / 32; ++db) dq[0][db] = dk[0][db] = dv[0][db] = splat16(0.f);
        if (some) {
            f32x16_t s[1] = {splat16(0.f)}, dp[1] = {splat16(0.f)};
            typename B::Row own[1];
            own[0].staged(sQ, lane);
            B::template rows<1>(sK, at, own, s);
            own[0].staged(sG, lane);
            B::template rows<1>(sV, at, own, dp);
            const int lim = r >= R ? 0 : a.causal && off + q + 1 < it.lk ? off + q + 1 : it.lk;
            float sum = 0.f, dsum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float u;
                if constexpr (BIAS) u = fmaf(s[0][i], a.scale, tab[(r & gm) * kTableStride + id_of(ids, i, a.B)]);
                else u = s[0][i] * a.scale;
                s[0][i] = ex2((u - L) * kLog2e);
                if (i >= lim - part(0, lane)) s[0][i] = 0.f;
                sum += s[0][i];
                dsum = fmaf(s[0][i], dp[0][i], dsum);
            }
            sum = pair_sum(sum);
            const float inv = sum == 0.f ? 0.f : 1.f / sum, Dr = pair_sum(dsum) * inv;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[0][i] *= inv;
                dp[0][i] = s[0][i] * (dp[0][i] - Dr);
            }
            if constexpr (BIAS) add_block(hist + lane, ids, a.B, dp[0]);
            typename B::Cols x;
            x.load(sK, at);
            B::template apply<1>(x, dp, dq);
            typename B::Weights w[1];
            lds_done();  // K and V are read: their places take P and dS
            lay_block<T>(sK, s[0], lane);
            lay_block<T>(sV, dp[0], lane);
            lds_done();
            // acc += (staged rows) x (block turned round)
            auto turned = [&](const T* block, const T* rows, f32x16_t(&acc)[1][D / 32]) {
                typename S::Cols t;
                t.load(block, turned_at);
#pragma unroll
                for (int i = 0; i < (B::kHalf ? 2 : 16); ++i) w[0].v[i] = t.v[0][i];
                x.load(rows, at);
                B::template apply<1>(x, w, acc);
            };
            turned(sK, sG, dv);
            turned(sV, sQ, dk);
        }
        if (r < R) B::store(static_cast<T*>(a.out0) + (row_at + q * a.H + (r & gm)) * D, dq[0], a.scale, lane);
        if (r < it.lk) {
            B::store(static_cast<T*>(a.out1) + (key_at + r * a.Hkv) * D, dk[0], a.scale, lane);
            B::store(static_cast<T*>(a.out2) + (key_at + r * a.Hkv) * D, dv[0], 1.f, lane);
        }
        lds_done();  // the next sequence's loads may land
    }
    if constexpr (BIAS)
        hist_flush<kWave>(hist, 1, a.B, gs, a.hist + int64_t(first) * (int64_t(a.B) << gs), lane);
}

// The sum of KS sets' accumulators in the first set (false for the others).
template <int KS, int W, int N>
__device__ __forceinline__ bool add_sets(f32x16_t (&acc)[N], int set, int at) {
    if constexpr (KS > 1) {
        __shared__ float s_acc[KS - 1][8][W * kWave];
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (set > 0)
#pragma unroll
                    for (int i = 0; i < 8; ++i) s_acc[set - 1][i][at] = acc[k][8 * half + i];
                __syncthreads();
                if (set == 0)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int p = 0; p < KS - 1; ++p) acc[k][8 * half + i] += s_acc[p][i][at];
                __syncthreads();
            }
    }
    return set == 0;
}

enum RowPass { kStat, kGrad };

// kGrad: dQ_i = scale sum_j dS_ij K_j with dS_ij = P_ij (dP_ij - D_i); the dP
// products start from -D_i, so their sum is dP - D with no subtraction.  Without
// a bias D_i = <dO_i, O_i> (written here for the key pass); a bf16 O is off by 2^-8
// of its size, which shrinks with the number of keys, so rows of the few keys of one
// stage form D_i from their weights (causal sequences of up to 275, dQ's and dK's
// error 0.0026 -> 0.0023 of their size).
// Bound by the matrix cores: four causal prompts of up to 4,096 (16 / 4 heads of 64)
// 89 us, 895 TFLOP/s of its three products; with a bias by waiting (46% of the
// wavefronts' time, at two a SIMD; the LDS instructions, most of them the table's
// gradient's, take 9%): 16 graphs of up to 1,000 51 us, kStat 36.
// kStat (before it, with a bias): D_i = sum_j P_ij dP_ij from the scores, since a
// bf16 O is off by 2^-8, which moves the table's gradient (fp32) by as much,
// and the weights' sum under the given LSE: an fp32 LSE beside a large bias
// holds log(sum) only roughly, so P is normalised again by it.
template <typename T, int D, int STAGE, int W, int KS, int SUB, bool BIAS, RowPass PASS>
__global__ __launch_bounds__(W * KS * kWave) __attribute__((amdgpu_waves_per_eu(
    D * int(sizeof(T)) <= 256 ? waves_per_simd(KS * 4 * STAGE * D * int(sizeof(T)), W* KS) : 1))) void k_packed_rows(PackedArgs a) {
    using B = Blk<T, D, STAGE>;
    __shared__ __attribute__((aligned(16))) T sK0[KS * B::kElems], sK1[KS * B::kElems];
    __shared__ __attribute__((aligned(16))) T sV0[KS * B::kElems], sV1[KS * B::kElems];
    extern __shared__ float s_dyn[];
    PackedItem it;
    int hk, sub;
    uint32_t block;
    if (!packed_place<W == 1, SUB>(a, it, hk, sub, block)) return;
    const int lane = lane_id(), wave = uniform(int(threadIdx.x) / kWave);
    const int set = KS == 1 ? 0 : wave / W, row_wave = wave - set * W;
    const int gs = a.gs, gm = (1 << gs) - 1, R = it.lq << gs, off = it.lk - it.lq;
    const int row0 = it.tile + (sub * W + row_wave) * 32;
    float* s_tab = s_dyn;
    float* hist = s_dyn + (kTableStride << gs) + wave * (a.B + 1) * kWave + lane;
    if constexpr (BIAS) {
        load_table<W * KS * kWave>(s_tab, a, hk, int(threadIdx.x));
        if constexpr (PASS == kGrad)
            for (int x = 0; x <= a.B; ++x) hist[x * kWave] = 0.f;
    }
    auto limit = [&](int q) {
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
    const int r = row0 + (lane & 31), rc = r < R ? r : R - 1;
    const int q = rc >> gs, hg = rc & gm;
    const int64_t at = int64_t(it.q0 + q) * a.H + (hk << gs) + hg;
    const int lim = limit(q);
    const int hi = uniform(row0 < R ? limit((row0 + 31 < R ? row0 + 31 : R - 1) >> gs) : 0);
    const uint8_t* id_row = BIAS ? a.ids + it.pair + q * ids_width(it.lk) : nullptr;
    typename B::Row qf[1], gf[1];
    qf[0].load(static_cast<const T*>(a.Q) + int64_t(it.q0 + q) * a.ldq + ((hk << gs) + hg) * D, lane);
    gf[0].load(static_cast<const T*>(a.dO) + at * D, lane);
    const float sl2 = a.scale * kLog2e;
    float L = a.LSE[at], lg = 0.f, Dq = 0.f;
    if (L == -kInf) L = 0.f;  // an empty row: every score is masked
    if (r >= R) L = kInf;     // a row past the end weighs nothing, in the table's gradient either
    if constexpr (!BIAS) {
        L *= kLog2e;
        typename B::Row of;
        of.load(static_cast<const T*>(a.O) + at * D, lane);
        Dq = pair_sum(gf[0].dot(of));
    } else if constexpr (PASS == kGrad) {
        lg = a.Lg[at];
        Dq = a.Dv[at];
    }
    f32x16_t acc[1][D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) acc[0][db] = splat16(0.f);
    float sum = 0.f, dsum = 0.f;
    stage_done<(W > 1) || BIAS>();
    const typename B::At lds(lane, set * B::kElems * int(sizeof(T)));
    if constexpr (!BIAS) {
        if (it.s0 == 0 && set == 0) {
            if (B::kHalf && hi <= STAGE) {  // uniform; this set's first stage holds all that the rows attend to
                float ps = 0.f, ds = 0.f;
#pragma unroll 1
                for (int key0 = 0; key0 < hi; key0 += 32) {
                    f32x16_t s[1] = {splat16(0.f)}, dp[1] = {splat16(0.f)};
                    B::template rows<1>(sK0 + key0 * D, lds, qf, s);
                    B::template rows<1>(sV0 + key0 * D, lds, gf, dp);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float p = key0 + part(i, lane) < lim ? ex2(fmaf(s[0][i], sl2, -L)) : 0.f;
                        ps += p;
                        ds = fmaf(p, dp[0][i], ds);
                    }
                }
                ps = pair_sum(ps);
                ds = pair_sum(ds);
                if (ps > 0.f) Dq = ds / ps;
            }
            if (r < R && lane < 32) a.Dv[at] = Dq;
        }
    }
    auto block32 = [&](auto masked, int key0, const T* bK, const T* bV, const uint4& ids) {
        const int left = lim - key0 - part(0, lane);  // how many of the lane's 16 keys its row attends to
        f32x16_t s[1] = {splat16(0.f)}, dp[1] = {splat16(-Dq)};
        B::template rows<1>(bK, lds, qf, s);
        B::template rows<1>(bV, lds, gf, dp);
        typename B::Cols kt;
        if constexpr (PASS == kGrad) {
            kt.load(bK, lds);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float t;
            if constexpr (BIAS) {
                t = fmaf(fmaf(s[0][i], a.scale, s_tab[hg * kTableStride + id_of(ids, i, a.B)]) - L, kLog2e, -lg);
            } else {
                t = fmaf(s[0][i], sl2, -L);
            }
            if constexpr (masked.value) t = i >= left ? -kInf : t;
            const float p = ex2(t);
            s[0][i] = p * dp[0][i];
            if constexpr (PASS == kStat) {
                sum += p;
                dsum += s[0][i];
            }
        }
        if constexpr (PASS == kGrad) {
            if constexpr (BIAS) add_block(hist, ids, a.B, s[0]);
            B::template apply<1>(kt, s, acc);
        }
    };
    uint4 ids[STAGE / 32];  // the buckets of a stage, loaded a stage ahead
    auto next_ids = [&](int kbase) {
        if constexpr (BIAS)
#pragma unroll
            for (int kb = 0; kb < STAGE / 32; ++kb) ids[kb] = load_ids(id_row, kbase + 32 * kb, it.lk, lane);
    };
    if (it.s0 < it.s1) next_ids(it.s0 + set * STAGE);
    auto stage = [&](auto masked, int kbase, const T* cK, const T* cV, T* nK, T* nV) {
        fetch(kbase + KS * STAGE, nK, nV);
        uint4 now[STAGE / 32];
        if constexpr (BIAS)
#pragma unroll
            for (int kb = 0; kb < STAGE / 32; ++kb) now[kb] = ids[kb];
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
    // as in the forward
    constexpr int kRound = KS * STAGE;
    const int first_row = it.tile + sub * W * 32 < R ? it.tile + sub * W * 32 : R - 1, lo = uniform(limit(first_row >> gs));
    int kbase = it.s0;
    for (int n = lo > it.s0 ? (lo - it.s0) / (2 * kRound) : 0; n > 0; --n, kbase += 2 * kRound) {
        stage(Flag<false>{}, kbase + set * STAGE, sK0, sV0, sK1, sV1);
        stage(Flag<false>{}, kbase + kRound + set * STAGE, sK1, sV1, sK0, sV0);
    }
    for (; kbase < it.s1; kbase += 2 * kRound) {
        stage(Flag<true>{}, kbase + set * STAGE, sK0, sV0, sK1, sV1);
        if (kbase + kRound < it.s1) stage(Flag<true>{}, kbase + kRound + set * STAGE, sK1, sV1, sK0, sV0);
    }
    if constexpr (PASS == kStat) {
        sum = pair_sum(sum);
        dsum = pair_sum(dsum);
        if constexpr (KS > 1) {
            __shared__ float s_sum[2][KS][W * kWave];
            s_sum[0][set][row_wave * kWave + lane] = sum;
            s_sum[1][set][row_wave * kWave + lane] = dsum;
            __syncthreads();
            if (set > 0) return;
#pragma unroll
            for (int p = 1; p < KS; ++p) {
                sum += s_sum[0][p][row_wave * kWave + lane];
                dsum += s_sum[1][p][row_wave * kWave + lane];
            }
        }
        if (lane >= 32) return;
        if (it.slot >= 0) {  // a part of a split walk
            if (row0 >= R) return;
            float* o = a.slots + (int64_t(it.slot + sub * W + row_wave) * a.Hkv + hk) * (2 * kFewRows);
            o[lane] = sum, o[kFewRows + lane] = dsum;
        } else if (r < R) {
            a.Dv[at] = sum == 0.f ? 0.f : dsum / sum;
            a.Lg[at] = sum == 0.f ? 0.f : __log2f(sum);
        }
    } else {
        if constexpr (BIAS) {
            __syncthreads();
            // a lane's rows all belong to head lane % g of the group: tiles start at multiples of 32
            hist_flush<W * KS * kWave>(s_dyn + (kTableStride << gs), W * KS, a.B, gs,
                                       a.hist + int64_t(block) * (int64_t(a.B) << gs), int(threadIdx.x));
        }
        if (!add_sets<KS, W>(acc[0], set, row_wave * kWave + lane)) return;
        if (it.slot >= 0) {
            if (row0 < R)  // uniform
                Blk<float, D>::store(
                    a.slots + ((int64_t(it.slot + sub * W + row_wave) * a.Hkv + hk) * kFewRows + (lane & 31)) * D, acc[0],
                    1.f, lane);
        } else if (r < R)
            B::store(static_cast<T*>(a.out0) + at * D, acc[0], a.scale, lane);
    }
}

// kBoth: dK and dV of a block from one forming of its weights.  Wide rows' accumulators
// for both leave room for one wavefront a SIMD, which waits for everything it reads
// (D = 128, bf16); there a pass for each (kOnlyV: Q, dO; kOnlyK) forms the scores
// twice, five products for four, with two wavefronts.
enum KeyPass { kBoth, kOnlyV, kOnlyK };

// dK_j = scale sum_i dS_ij Q_i and dV_j = sum_i P_ij dO_i over the rows of the
// whole group, with the wavefront owning 32 keys and the rows streaming through
// LDS; the dP products start from the rows' -D_i.  Bound by the matrix cores and a
// barrier a stage: four causal prompts of up to 4,096 (16 / 4 heads of 64) 133 us,
// 800 TFLOP/s of its four products; with a bias (16 graphs of up to 1,000) 52 us.
template <typename T, int D, int STAGE, int W, int KS, int SUB, bool BIAS, KeyPass PASS>
__global__ __launch_bounds__(W * KS * kWave) __attribute__((amdgpu_waves_per_eu(
    PASS != kBoth || D * int(sizeof(T)) <= 128 ? waves_per_simd(KS * 4 * STAGE * D * int(sizeof(T)), W* KS) : 1))) void k_packed_keys(PackedArgs a) {
    using B = Blk<T, D, STAGE>;
    __shared__ __attribute__((aligned(16))) T sQ0[KS * B::kElems], sQ1[KS * B::kElems];
    __shared__ __attribute__((aligned(16))) T sG0[KS * B::kElems], sG1[KS * B::kElems];
    // per row of a stage: LSE (exp2 domain without a bias), -D, log2 of the weights' sum
    typedef float Stats[KS][3][STAGE];
    __shared__ __attribute__((aligned(16))) Stats sR0, sR1;
    // with a bias, the buckets of a stage's rows and a wavefront's 32 keys: loaded a row a lane, read turned round, a key a lane
    typedef uint8_t Buckets[BIAS ? W * KS : 1][BIAS ? STAGE : 1][32];
    __shared__ __attribute__((aligned(16))) Buckets sI0, sI1;
    extern __shared__ float s_tab[];
    PackedItem it;
    int hk, sub;
    uint32_t block;
    if (!packed_place<W == 1, SUB>(a, it, hk, sub, block)) return;
    const int lane = lane_id(), wave = uniform(int(threadIdx.x) / kWave);
    const int set = KS == 1 ? 0 : wave / W, key_wave = wave - set * W;
    const int gs = a.gs, gm = (1 << gs) - 1, off = it.lk - it.lq;
    const int key0 = it.tile + (sub * W + key_wave) * 32;
    if constexpr (BIAS) load_table<W * KS * kWave>(s_tab, a, hk, int(threadIdx.x));
    float rs[3] = {0.f, 0.f, 0.f};
    auto load_stats = [&](int base) {
        if (key_wave != 0) return;
        const int r = base + lane;
        rs[0] = BIAS ? 0.f : kInf;  // rows past the end weigh nothing
        rs[1] = 0.f;
        rs[2] = BIAS ? kInf : 0.f;
        if (lane < STAGE && r < it.s1) {
            const int64_t at = int64_t(it.q0 + (r >> gs)) * a.H + (hk << gs) + (r & gm);
            const float L = a.LSE[at];
            rs[0] = L == -kInf ? 0.f : BIAS ? L : L * kLog2e;
            rs[1] = -a.Dv[at];
            if constexpr (BIAS) rs[2] = a.Lg[at];
        }
    };
    uint4 ids[STAGE / 32];
    const int64_t wide = ids_width(it.lk);
    auto load_rows = [&](int base) {
        load_stats(base);
        if constexpr (BIAS)
#pragma unroll
            for (int rb = 0; rb < STAGE / 32; ++rb) {
                const int r = base + 32 * rb + (lane & 31), rc = r < it.s1 ? r : it.s1 - 1;
                ids[rb] = load_ids(a.ids + it.pair + (rc >> gs) * wide, key0, it.lk, lane);
            }
    };
    auto store_rows = [&](Stats& to, Buckets& toI) {
        if (key_wave == 0 && lane < STAGE) to[set][0][lane] = rs[0], to[set][1][lane] = rs[1], to[set][2][lane] = rs[2];
        if constexpr (BIAS)
#pragma unroll
            for (int rb = 0; rb < STAGE / 32; ++rb)
                *reinterpret_cast<uint4*>(&toI[wave][32 * rb + (lane & 31)][16 * (lane >> 5)]) = ids[rb];
    };
    const T* Q = static_cast<const T*>(a.Q) + int64_t(it.q0) * a.ldq + (hk << gs) * D;
    const T* G = static_cast<const T*>(a.dO) + (int64_t(it.q0) * a.H + (hk << gs)) * D;
    const uint32_t ldg = uint32_t(a.H) * D;
    auto fetch = [&](int base, T* toQ, T* toG) {  // base is a multiple of the group
        if (base >= it.s1) return;
        B::template fetch<W>(toQ + set * B::kElems, Q + int64_t(base >> gs) * a.ldq, it.s1 - base, key_wave, lane,
                             [&](int r) { return __umul24(r >> gs, a.ldq) + uint32_t((r & gm) * D); });
        B::template fetch<W>(toG + set * B::kElems, G + int64_t(base >> gs) * ldg, it.s1 - base, key_wave, lane,
                             [&](int r) { return __umul24(r >> gs, ldg) + uint32_t((r & gm) * D); });
    };
    if (it.s0 < it.s1) load_rows(it.s0 + set * STAGE);
    fetch(it.s0 + set * STAGE, sQ0, sG0);
    const int j = key0 + (lane & 31), jc = j < it.lk ? j : it.lk - 1;
    auto first_row = [&](int key) { return a.causal && key > off ? (key - off) << gs : 0; };
    const int rmin = first_row(jc);
    const int rlo = uniform(first_row(key0 < it.lk ? key0 : it.lk - 1));
    typename B::Row kf[1], vf[1];
    kf[0].load(static_cast<const T*>(a.K) + int64_t(it.k0 + jc) * a.ldk + hk * D, lane);
    vf[0].load(static_cast<const T*>(a.V) + int64_t(it.k0 + jc) * a.ldv + hk * D, lane);
    f32x16_t dk[1][D / 32], dv[1][D / 32];
#pragma unroll
    for (int db = 0; db < D / 32; ++db) dk[0][db] = dv[0][db] = splat16(0.f);
    const float sl2 = a.scale * kLog2e;
    store_rows(sR0, sI0);
    stage_done<(W > 1) || BIAS>();
    const typename B::At lds(lane, set * B::kElems * int(sizeof(T)));
    auto block32 = [&](auto masked, int r0, const T* bQ, const T* bG, const float(&bR)[3][STAGE], const uint8_t* bI, int rb) {
        const int from = rmin - r0 - part(0, lane);  // of the lane's 16 rows the first that attends to its key
        f32x16_t s[1] = {splat16(0.f)}, dp[1];
        const int rs0 = 32 * rb + part(0, lane);  // the lane's rows in the stage's statistics
        if constexpr (PASS != kOnlyV) {
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float4 d4 = *reinterpret_cast<const float4*>(&bR[1][rs0 + 4 * x]);
                dp[0][4 * x] = d4.x, dp[0][4 * x + 1] = d4.y, dp[0][4 * x + 2] = d4.z, dp[0][4 * x + 3] = d4.w;
            }
        }
        B::template rows<1>(bQ, lds, kf, s);
        if constexpr (PASS != kOnlyV) B::template rows<1>(bG, lds, vf, dp);
        // operands and statistics are read where they are used: held together they do not fit the registers
        __builtin_amdgcn_sched_barrier(0);
        typename B::Cols x;
        x.load(PASS == kOnlyK ? bQ : bG, lds);
        uint4 ids;
        if constexpr (BIAS) ids = turned_ids(bI + 32 * 32 * rb, lane);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float4 l4 = *reinterpret_cast<const float4*>(&bR[0][rs0 + 4 * k]);
            float4 g4;
            if constexpr (BIAS) g4 = *reinterpret_cast<const float4*>(&bR[2][rs0 + 4 * k]);
            const float L[4] = {l4.x, l4.y, l4.z, l4.w}, lg[4] = {g4.x, g4.y, g4.z, g4.w};
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int i = 4 * k + y;
                float t;
                if constexpr (BIAS) {
                    const float bias = s_tab[(part(i, lane) & gm) * kTableStride + id_of(ids, i, a.B)];
                    t = fmaf(fmaf(s[0][i], a.scale, bias) - L[y], kLog2e, -lg[y]);
                } else {
                    t = fmaf(s[0][i], sl2, -L[y]);
                }
                if constexpr (masked.value) t = i < from ? -kInf : t;
                s[0][i] = ex2(t);
                if constexpr (PASS != kOnlyV) dp[0][i] *= s[0][i];
            }
        }
        if constexpr (PASS == kOnlyK) {
            B::template apply<1>(x, dp, dk);
            return;
        }
        B::template apply<1>(x, s, dv);
        if constexpr (PASS == kBoth) {
            __builtin_amdgcn_sched_barrier(0);
            x.load(bQ, lds);
            B::template apply<1>(x, dp, dk);
        }
    };
    auto stage = [&](auto masked, int base, const T* cQ, const T* cG, const Stats& cR, const Buckets& cI, T* nQ, T* nG,
                     Stats& nR, Buckets& nI) {
        load_rows(base + KS * STAGE);
        fetch(base + KS * STAGE, nQ, nG);
        if constexpr (masked.value) {
#pragma unroll 1
            for (int rb = 0; rb < STAGE / 32; ++rb) {
                const int r0 = base + 32 * rb;
                if (r0 < it.s1 && r0 + 32 > rlo && key0 < it.lk)  // uniform
                    block32(masked, r0, cQ + 32 * rb * D, cG + 32 * rb * D, cR[set], &cI[BIAS ? wave : 0][0][0], rb);
            }
        } else if (key0 < it.lk) {  // uniform
#pragma unroll
            for (int rb = 0; rb < STAGE / 32; ++rb) {
                __builtin_amdgcn_sched_barrier(0);
                block32(masked, base + 32 * rb, cQ + 32 * rb * D, cG + 32 * rb * D, cR[set], &cI[BIAS ? wave : 0][0][0], rb);
            }
        }
        store_rows(nR, nI);
        stage_done<(W > 1)>();
    };
    // the stages whose rows attend to every key of the tile lie between the first ones (causal) and the last (ragged);
    // an even number of stages before them and of them
    constexpr int kRound = KS * STAGE;
    const int end_key = it.tile + (sub + 1) * W * 32, last_key = end_key < it.lk ? end_key - 1 : it.lk - 1;
    const int all = uniform(first_row(last_key)) - it.s0;  // rows before the first that attends to every key
    const int before = it.s0 + (all > 0 ? (all + 2 * kRound - 1) / (2 * kRound) * (2 * kRound) : 0);
    const int after = it.s1 > before ? before + (it.s1 - before) / (2 * kRound) * (2 * kRound) : it.s0;
    int base = it.s0;
#pragma unroll 1
    for (int phase = 0; phase < 2; ++phase) {
        const int end = phase == 0 && before < it.s1 ? before : it.s1;
#pragma unroll 1
        for (; base < end; base += 2 * kRound) {
            stage(Flag<true>{}, base + set * STAGE, sQ0, sG0, sR0, sI0, sQ1, sG1, sR1, sI1);
            if (base + kRound < it.s1)
                stage(Flag<true>{}, base + kRound + set * STAGE, sQ1, sG1, sR1, sI1, sQ0, sG0, sR0, sI0);
        }
        if (phase == 0)
            for (; base < after; base += 2 * kRound) {
                stage(Flag<false>{}, base + set * STAGE, sQ0, sG0, sR0, sI0, sQ1, sG1, sR1, sI1);
                stage(Flag<false>{}, base + kRound + set * STAGE, sQ1, sG1, sR1, sI1, sQ0, sG0, sR0, sI0);
            }
    }
    const int thread = key_wave * kWave + lane;
    if constexpr (PASS != kOnlyV) add_sets<KS, W>(dk[0], set, thread);
    if constexpr (PASS != kOnlyK) add_sets<KS, W>(dv[0], set, thread);
    if (set > 0) return;
    if (it.slot >= 0) {
        if (key0 >= it.lk) return;  // uniform
        float* o = a.slots + ((int64_t(it.slot + sub * W + key_wave) * a.Hkv + hk) * (2 * kFewRows) + (lane & 31)) * D;
        if constexpr (PASS != kOnlyV) Blk<float, D>::store(o, dk[0], 1.f, lane);
        if constexpr (PASS != kOnlyK) Blk<float, D>::store(o + kFewRows * D, dv[0], 1.f, lane);
    } else if (j < it.lk) {
        const int64_t at = int64_t(it.k0 + j) * a.Hkv + hk;
        if constexpr (PASS != kOnlyV) B::store(static_cast<T*>(a.out1) + at * D, dk[0], a.scale, lane);
        if constexpr (PASS != kOnlyK) B::store(static_cast<T*>(a.out2) + at * D, dv[0], 1.f, lane);
    }
}

template <typename T, int D, bool BIAS>
gt_status packed_bwd_d(const gt_packed_plan* p, PackedArgs a, float* dtable, hipStream_t s) {
    constexpr int kRow = D * int(sizeof(T)), kStage = sizeof(T) == 2 ? 64 : 32;
    const gt_dtype dt = sizeof(T) == 2 ? GT_BF16 : GT_F32;
    const size_t tab = BIAS ? size_t(kTableStride << a.gs) * sizeof(float) : 0;
    const size_t col = BIAS ? size_t(a.B + 1) * kWave * sizeof(float) : 0;
    const int64_t per = int64_t(a.B) << a.gs;
    float* const hist = a.hist;
    TableParts parts = {};
    auto list = [&](int l) {
        a.items = packed_list(p, l);
        a.n_items = int(packed_items(p, l));
        return a.n_items > 0;
    };
    // where a launch of n blocks (or wavefronts) leaves its partial tables
    auto part = [&](int64_t n) {
        const int k = parts.count++;
        parts.at[k] = k == 0 ? 0 : parts.at[k - 1] + parts.n[k - 1] * per;
        parts.n[k] = n;
        a.hist = BIAS ? hist + parts.at[k] : nullptr;
    };
    if (list(kPairs)) {
        constexpr int W = pair_waves(kRow);
        const int64_t blocks = BIAS ? pair_blocks(p, kRow) : cdiv(int64_t(a.n_items) * a.Hkv, W * kXcds * a.Hkv) * kXcds * a.Hkv;
        part(blocks * W);
        k_pair_bwd<T, D, BIAS><<<unsigned(blocks), W * kWave, W * (tab + col), s>>>(a);
        GT_LAUNCH_CHECK("packed_bwd pairs");
    }
#define GT_ROWS(LIST, STAGE, W, KS, SUB, PASS)                                                                  \
    if (list(LIST)) {                                                                                           \
        if (PASS == kGrad) part(int64_t(a.n_items) * SUB * a.Hkv);                                              \
        k_packed_rows<T, D, STAGE, W, KS, SUB, BIAS, PASS><<<packed_grid(a.n_items, a.Hkv, SUB),                \
                            W * KS * kWave, tab + (PASS == kGrad ? W * KS * col : 0), s>>>(a);                  \
        GT_LAUNCH_CHECK("packed_bwd rows");                                                                     \
    }
    if constexpr (BIAS) {
        GT_ROWS(kRowsFew, 32, 1, few_waves(kRow), 1, kStat)
        GT_ROWS(kRows64, kStage, 2, 1, 1, kStat)
        if (kRow <= 128 && packed_shared<T>(p, kRowSharedAt)) {
            GT_ROWS(kRows128, kStage, 4, (kRow <= 128 ? 2 : 1), 1, kStat)
        } else {
            GT_ROWS(kRows128, kStage, 4, 1, 1, kStat)
        }
        GT_ROWS(kRows256, kStage, 4, 1, 2, kStat)
        if (list(kRowMerges)) {
            const gt_status st = packed_merge_stat(p, a, s);
            if (st != GT_OK) return st;
        }
        // the table's gradient takes 16 KB of LDS a wavefront: smaller workgroups
        GT_ROWS(kRowsFew, 32, 1, few_waves_hist(kRow), 1, kGrad)
        GT_ROWS(kRows64, kStage, 2, 1, 1, kGrad)
        // two sets where their columns fit beside the stages (and the sums' exchange)
        if (kRow <= 128 && packed_shared<T>(p, kRowSharedAt) && 8 * (kStage * kRow + col) + tab + (16 << 10) <= (160 << 10)) {
            GT_ROWS(kRows128, kStage, 4, (kRow <= 128 ? 2 : 1), 1, kGrad)
        } else {
            GT_ROWS(kRows128, kStage, 4, 1, 1, kGrad)
        }
        GT_ROWS(kRows256, kStage, 4, 1, 2, kGrad)
    } else {
        GT_ROWS(kRowsFew, 32, 1, few_waves(kRow), 1, kGrad)
        GT_ROWS(kRows64, kStage, 2, 1, 1, kGrad)
        if (kRow <= 128 && packed_shared<T>(p, kRowSharedAt)) {
            GT_ROWS(kRows128, kStage, 4, (kRow <= 128 ? 2 : 1), 1, kGrad)
        } else {
            GT_ROWS(kRows128, kStage, 4, 1, 1, kGrad)
        }
        if constexpr (kRow <= 128 || sizeof(T) == 2) {
            GT_ROWS(kRows256, kStage, 8, 1, 1, kGrad)
        } else {
            GT_ROWS(kRows256, kStage, 4, 1, 2, kGrad)
        }
    }
#undef GT_ROWS
    if (list(kRowMerges)) {
        const gt_status st = packed_merge_rows(p, D, dt, a, s);
        if (st != GT_OK) return st;
    }
#define GT_KEYS(LIST, STAGE, W, KS, SUB, PASS)                                                                  \
    if (list(LIST)) {                                                                                           \
        k_packed_keys<T, D, STAGE, W, KS, SUB, BIAS, PASS>                                                      \
            <<<packed_grid(a.n_items, a.Hkv, SUB), W * KS * kWave, tab, s>>>(a);                                \
        GT_LAUNCH_CHECK("packed_bwd keys");                                                                     \
    }
    GT_KEYS(kKeysFew, 32, 1, few_waves(kRow), 1, kBoth)
    if constexpr (kRow <= 128) {
        GT_KEYS(kKeys64, kStage, 2, 1, 1, kBoth)
        if (packed_shared<T>(p, kKeySharedAt)) {
            GT_KEYS(kKeys128, kStage, 4, 2, 1, kBoth)
        } else {
            GT_KEYS(kKeys128, kStage, 4, 1, 1, kBoth)
        }
        GT_KEYS(kKeys256, kStage, 8, 1, 1, kBoth)
    } else if constexpr (sizeof(T) == 2) {
        GT_KEYS(kKeys64, kStage, 2, 1, 1, kBoth)
        if (packed_shared<T>(p, kKeySharedAt)) {
            GT_KEYS(kKeys128, 32, 4, 2, 1, kOnlyV)
            GT_KEYS(kKeys128, 32, 4, 2, 1, kOnlyK)
        } else {
            GT_KEYS(kKeys128, kStage, 4, 1, 1, kOnlyV)
            GT_KEYS(kKeys128, kStage, 4, 1, 1, kOnlyK)
        }
        GT_KEYS(kKeys256, kStage, 8, 1, 1, kOnlyV)
        GT_KEYS(kKeys256, kStage, 8, 1, 1, kOnlyK)
    } else {
        GT_KEYS(kKeys64, kStage, 2, 1, 1, kBoth)
        GT_KEYS(kKeys128, kStage, 4, 1, 1, kBoth)
        GT_KEYS(kKeys256, kStage, 4, 1, 2, kBoth)
    }
#undef GT_KEYS
    if (list(kKeyMerges)) {
        const gt_status st = packed_merge_keys(p, D, dt, a, s);
        if (st != GT_OK) return st;
    }
    if constexpr (BIAS) {
        a.hist = hist;
        return packed_table_sum(parts, a, dtable, s);
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
