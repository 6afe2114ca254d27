// Packed-sequence attention: the parts of split walks put together, and the
// table's gradient from the blocks' partial tables.  An item is 32 rows (or keys);
// their parts are added in their order, so results do not depend on which finished
// first.
#include "packed.h"

namespace gt {
namespace {

constexpr int kThreads = 256;
constexpr int kOut = kThreads / kWave;  // rows (or keys) per workgroup, one a wavefront

template <typename T>
__device__ __forceinline__ T from_f32(float v) {
    if constexpr (sizeof(T) == 2) return f32_to_bf16(v);
    else return v;
}

// Which item, kv head and row of the item this wavefront has.
__device__ __forceinline__ void merge_place(const PackedArgs& a, PackedItem& it, int& hk, int& r) {
    const uint32_t per = kFewRows / kOut, b = blockIdx.x;
    hk = int(b / per % uint32_t(a.Hkv));
    it = a.items[b / per / uint32_t(a.Hkv)];
    r = int(b % per) * kOut + uniform(int(threadIdx.x) / kWave);
}
unsigned merge_grid(const PackedArgs& a) { return unsigned(int64_t(a.n_items) * a.Hkv * (kFewRows / kOut)); }

__device__ __forceinline__ int64_t row_at(const PackedArgs& a, const PackedItem& it, int hk, int row) {
    return int64_t(it.q0 + (row >> a.gs)) * a.H + (hk << a.gs) + (row & ((1 << a.gs) - 1));
}

// Calls add(load(p)) for the parts in their order, four loads at a time (one after the
// other: 16 tokens over up to 65,536 keys 17 us, now 8).
template <typename L, typename A>
__device__ __forceinline__ void each_part(int parts, L load, A add) {
    for (int p0 = 0; p0 < parts; p0 += 4) {
        decltype(load(0)) v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = load(p0 + u < parts ? p0 + u : parts - 1);
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (p0 + u < parts) add(v[u]);
    }
}

// O = sum of w_p O_p / sum of w_p l_p, w_p = exp(m_p - max m): a lane a part for the
// weights, then a lane a feature.
template <typename T>
__global__ __launch_bounds__(kThreads) void k_merge_fwd(PackedArgs a, int D) {
    PackedItem it;
    int hk, r;
    merge_place(a, it, hk, r);
    if (it.tile + r >= it.lq << a.gs) return;
    const int lane = lane_id();
    const int64_t slot = kFewRows * (D + 2), step = it.s1 * int64_t(a.Hkv) * slot;
    const float* s = a.slots + (int64_t(it.slot) * a.Hkv + hk) * slot;
    const float to2 = a.B > 0 ? kLog2e : 1.f;  // m is in the exp2 domain without a bias
    float m = -3.402823466e38f, l = 0.f, o[2] = {0.f, 0.f};
    for (int p = lane; p < it.s0; p += kWave) m = fmaxf(m, s[p * step + r]);
    m = wave_max(m);
    for (int p = lane; p < it.s0; p += kWave)
        l = fmaf(ex2((s[p * step + r] - m) * to2), s[p * step + kFewRows + r], l);
    l = wave_sum(l);
    const int c0 = lane < D ? lane : 0, c1 = lane + kWave < D ? lane + kWave : 0;
    each_part(
        it.s0,
        [&](int p) {
            const float* x = s + p * step;
            return make_float3(x[r], x[2 * kFewRows + r * D + c0], x[2 * kFewRows + r * D + c1]);
        },
        [&](const float3& x) {
            const float w = ex2((x.x - m) * to2);
            o[0] = fmaf(w, x.y, o[0]);
            o[1] = fmaf(w, x.z, o[1]);
        });
    const int64_t at = row_at(a, it, hk, it.tile + r);
    if (lane == 0) a.LSE[at] = l == 0.f ? -__builtin_huge_valf() : fmaf(__log2f(l), kLn2, a.B > 0 ? m : m * kLn2);
    const float f = l == 0.f ? 0.f : 1.f / l;
    for (int k = 0; k < 2; ++k)
        if (lane + kWave * k < D) static_cast<T*>(a.out0)[at * D + lane + kWave * k] = from_f32<T>(o[k] * f);
}

// The row statistics from the parts' sums of P and of P dP.
__global__ __launch_bounds__(kThreads) void k_merge_stat(PackedArgs a) {
    const uint32_t x = blockIdx.x * kThreads + threadIdx.x, tile = x / kFewRows;
    if (tile >= uint32_t(a.n_items) * uint32_t(a.Hkv)) return;
    const PackedItem it = a.items[tile / uint32_t(a.Hkv)];
    const int hk = int(tile % uint32_t(a.Hkv)), r = int(x % kFewRows);
    if (it.tile + r >= it.lq << a.gs) return;
    float sum = 0.f, dsum = 0.f;
    for (int p = 0; p < it.s0; ++p) {
        const float* s = a.slots + ((it.slot + int64_t(p) * it.s1) * a.Hkv + hk) * (2 * kFewRows);
        sum += s[r];
        dsum += s[kFewRows + r];
    }
    const int64_t at = row_at(a, it, hk, it.tile + r);
    a.Dv[at] = sum == 0.f ? 0.f : dsum / sum;
    a.Lg[at] = sum == 0.f ? 0.f : __log2f(sum);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_merge_rows(PackedArgs a, int D) {
    PackedItem it;
    int hk, r;
    merge_place(a, it, hk, r);
    if (it.tile + r >= it.lq << a.gs) return;
    const int64_t at = row_at(a, it, hk, it.tile + r);
    for (int c = lane_id(); c < D; c += kWave) {
        float t = 0.f;
        each_part(
            it.s0,
            [&](int p) { return a.slots[(((it.slot + int64_t(p) * it.s1) * a.Hkv + hk) * kFewRows + r) * D + c]; },
            [&](float x) { t += x; });
        static_cast<T*>(a.out0)[at * D + c] = from_f32<T>(t * a.scale);
    }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void k_merge_keys(PackedArgs a, int D) {
    PackedItem it;
    int hk, r;
    merge_place(a, it, hk, r);
    if (it.tile + r >= it.lk) return;
    const int64_t at = int64_t(it.k0 + it.tile + r) * a.Hkv + hk;
    for (int c = lane_id(); c < D; c += kWave) {
        float k = 0.f, v = 0.f;
        each_part(
            it.s0,
            [&](int p) {
                const float* s = a.slots + (((it.slot + int64_t(p) * it.s1) * a.Hkv + hk) * (2 * kFewRows) + r) * D + c;
                return make_float2(s[0], s[kFewRows * D]);
            },
            [&](const float2& x) {
                k += x.x;
                v += x.y;
            });
        static_cast<T*>(a.out1)[at * D + c] = from_f32<T>(k * a.scale);
        static_cast<T*>(a.out2)[at * D + c] = from_f32<T>(v);
    }
}

// One workgroup per head and bucket.
__global__ __launch_bounds__(kThreads) void k_table_sum(TableParts t, int H, int Hkv, int gs, int B,
                                                        const float* __restrict__ hist, float* __restrict__ out) {
    const int h = int(blockIdx.x), b = int(blockIdx.y), hk = h >> gs, hg = h & ((1 << gs) - 1);
    const int64_t per = int64_t(B) << gs;
    float x = 0.f;
    for (int k = 0; k < t.count; ++k) {
        for (int64_t i = threadIdx.x; i < t.n[k] / Hkv; i += kThreads) x += hist[t.at[k] + (i * Hkv + hk) * per + hg * B + b];
    }
    __shared__ float s[kThreads / kWave];
    x = wave_sum(x);
    if (lane_id() == 0) s[threadIdx.x / kWave] = x;
    __syncthreads();
    if (threadIdx.x == 0) out[int64_t(b) * H + h] = (s[0] + s[1]) + (s[2] + s[3]);
}

}  // namespace

#define GT_MERGE(K, NAME)                                                    \
    do {                                                                     \
        if (dt == GT_BF16) K<uint16_t><<<merge_grid(a), kThreads, 0, s>>>(a, d); \
        else K<float><<<merge_grid(a), kThreads, 0, s>>>(a, d);              \
        GT_LAUNCH_CHECK(NAME);                                               \
        return GT_OK;                                                        \
    } while (0)

gt_status packed_merge_fwd(const gt_packed_plan* p, int d, gt_dtype dt, PackedArgs a, hipStream_t s) {
    a.items = packed_list(p, kRowMerges);
    a.n_items = int(packed_items(p, kRowMerges));
    GT_MERGE(k_merge_fwd, "packed_merge_fwd");
}
gt_status packed_merge_rows(const gt_packed_plan* p, int d, gt_dtype dt, PackedArgs a, hipStream_t s) {
    a.items = packed_list(p, kRowMerges);
    a.n_items = int(packed_items(p, kRowMerges));
    GT_MERGE(k_merge_rows, "packed_merge_rows");
}
gt_status packed_merge_keys(const gt_packed_plan* p, int d, gt_dtype dt, PackedArgs a, hipStream_t s) {
    a.items = packed_list(p, kKeyMerges);
    a.n_items = int(packed_items(p, kKeyMerges));
    GT_MERGE(k_merge_keys, "packed_merge_keys");
}
gt_status packed_merge_stat(const gt_packed_plan* p, PackedArgs a, hipStream_t s) {
    a.items = packed_list(p, kRowMerges);
    a.n_items = int(packed_items(p, kRowMerges));
    k_merge_stat<<<unsigned(cdiv(int64_t(a.n_items) * a.Hkv * kFewRows, kThreads)), kThreads, 0, s>>>(a);
    GT_LAUNCH_CHECK("packed_merge_stat");
    return GT_OK;
}
gt_status packed_table_sum(const TableParts& t, PackedArgs a, float* dtable, hipStream_t s) {
    k_table_sum<<<dim3(unsigned(a.H), unsigned(a.B)), kThreads, 0, s>>>(t, a.H, a.Hkv, a.gs, a.B, a.hist, dtable);
    GT_LAUNCH_CHECK("packed_table_sum");
    return GT_OK;
}

}  // namespace gt
