// The learned bias by buckets on the edges of a sparse layer (the structural
// encoding of §2.1 Eq. (3)): its values, and the table's gradient.
#include "packed.h"

using namespace gt;

namespace {

// Rows of float4 at any multiple of 4 bytes (dwordx4 accesses need no more).
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kThreads = 256;

// bias[e, h] = table[bucket[e], h].  Bound by its stores: 4 H bytes an edge
// against one byte read.  A thread writes 16 bytes at a time from the table in
// LDS; workgroups stay (a short one spends its time on loading the table) and
// take turns at runs of UNROLL x 4 KB.  30.7M edges of 8 heads: 187 us, 5.4 TB/s.
constexpr int64_t kFwdBlocks = 2048;

template <int HS, int UNROLL>
__global__ __launch_bounds__(kThreads) void k_bucket_fwd(int64_t nnz, int B, const float* __restrict__ table,
                                                         const uint8_t* __restrict__ bucket,
                                                         float* __restrict__ bias) {
    constexpr int H = 1 << HS, E = H >= 4 ? 1 : 4 / H;  // edges in 16 bytes
    __shared__ float s_tab[(kMaxBuckets + 1) << HS];
    for (int x = int(threadIdx.x); x < (kMaxBuckets + 1) << HS; x += kThreads)
        s_tab[x] = x < (B << HS) ? table[x] : -__builtin_huge_valf();
    __syncthreads();
    const int64_t total = nnz << HS, run = int64_t(kThreads) * 4 * UNROLL, step = run * gridDim.x;
    // a result beyond the 256 MiB of last-level cache goes past it: what reads it next does not find it there, and what
    // runs next does not wait for its write-back (fwd and bwd of 30.7M edges of 8 heads 425 -> 367 us)
    const bool far = total > (int64_t(256) << 20) / 4;
    const int mine = 4 * int(threadIdx.x), head = mine & (H - 1);  // a run is whole edges
    for (int64_t base = run * blockIdx.x; base < total; base += step) {
        const bool whole = base + run <= total;  // uniform
        const uint8_t* q = bucket + ((base + mine) >> HS);
        uint32_t id[UNROLL][E];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int k = 0; k < E; ++k) {
                const int64_t e = ((base + mine + u * (kThreads * 4)) >> HS) + k;
                id[u][k] = whole ? q[((u * (kThreads * 4)) >> HS) + k] : bucket[e < nnz ? e : nnz - 1];
            }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            f32x4u_t v;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const uint32_t b = id[u][E == 1 ? 0 : t / H];
                v[t] = s_tab[(b < uint32_t(B) ? b : uint32_t(kMaxBuckets)) * H + (E == 1 ? head + t : t & (H - 1))];
            }
            const int64_t at = base + mine + u * (kThreads * 4);
            if (whole && far) __builtin_nontemporal_store(v, reinterpret_cast<f32x4u_t*>(bias + at));
            else if (whole) *reinterpret_cast<f32x4u_t*>(bias + at) = v;
            else
                for (int t = 0; t < 4 && at + t < total; ++t) bias[at + t] = v[t];
        }
    }
}

// dtable[b, h] = the sum of dbias[e, h] over the edges of bucket b.  Bound by the
// reads of dbias.  A lane's values all belong to one head (64 is a multiple of
// H); it adds each to a column of its own in LDS ([bucket][lane]), so no two
// lanes meet and the order of additions is the program's.  A workgroup leaves
// one partial table, and k_bucket_sum adds those.  30.7M edges of 8 heads: 170 us,
// 6.0 TB/s.
constexpr int kBurst = 16;  // values a lane loads together
constexpr int64_t kSumBlocks = 1024;

__global__ __launch_bounds__(kThreads) void k_bucket_bwd(int64_t nnz, int hs, int B,
                                                         const uint8_t* __restrict__ bucket,
                                                         const float* __restrict__ dbias, float* __restrict__ part) {
    extern __shared__ float s_col[];  // [4][B + 1][64]
    const int lane = lane_id(), wave = int(threadIdx.x) / kWave;
    float* col = s_col + wave * (B + 1) * kWave;
    for (int b = 0; b <= B; ++b) col[b * kWave + lane] = 0.f;
    const int64_t total = nnz << hs, step = int64_t(kBurst) * kWave;
    const int64_t waves = int64_t(gridDim.x) * (kThreads / kWave);
    for (int64_t base = (int64_t(blockIdx.x) * (kThreads / kWave) + wave) * step; base < total; base += waves * step) {
        float v[kBurst];
        uint32_t id[kBurst];
        if (base + step <= total) {
            // whole bursts at constant distances from one address (a check and an address for every load: 346 us for
            // 30.7M edges of 8 heads, 1.01 GB, against 165)
            const float* p = dbias + base + lane;
            const uint8_t* q = bucket + ((base + lane) >> hs);
#pragma unroll
            for (int u = 0; u < kBurst; ++u) {
                v[u] = p[u * kWave];
                id[u] = q[(u * kWave) >> hs];
            }
        } else {
#pragma unroll
            for (int u = 0; u < kBurst; ++u) {
                const int64_t at = base + u * kWave + lane, safe = at < total ? at : total - 1;
                v[u] = dbias[safe];
                id[u] = at < total ? bucket[safe >> hs] : uint32_t(B);
            }
        }
#pragma unroll
        for (int u = 0; u < kBurst; ++u) hist_add(col + lane, id[u] < uint32_t(B) ? id[u] : uint32_t(B), v[u]);
    }
    __syncthreads();
    const int H = 1 << hs, per = kWave >> hs;
    for (int x = int(threadIdx.x); x < (B << hs); x += kThreads) {
        const int b = x >> hs, h = x & (H - 1);
        float t = 0.f;
        for (int w = 0; w < kThreads / kWave; ++w)
            for (int k = 0; k < per; ++k) t += s_col[(w * (B + 1) + b) * kWave + (((k + x) & (per - 1)) << hs | h)];
        part[int64_t(blockIdx.x) * (B << hs) + x] = t;
    }
}

// out[x] = the sum over the partial tables, 16 entries a workgroup: 64 threads
// for each, every one a 64th of the tables, then those 64.
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void k_bucket_sum(int64_t parts, int n, const float* __restrict__ part,
                                                            float* __restrict__ out) {
    __shared__ float s[kSumThreads];
    const int x = int(blockIdx.x) * 16 + int(threadIdx.x & 15);
    float t = 0.f;
    if (x < n)
#pragma unroll 8
        for (int64_t p = threadIdx.x / 16; p < parts; p += kSumThreads / 16) t += part[p * n + x];
    s[threadIdx.x] = t;
    __syncthreads();
    if (threadIdx.x >= 16 || x >= n) return;
    for (int k = 1; k < kSumThreads / 16; ++k) t += s[16 * k + threadIdx.x];
    out[x] = t;
}

int64_t sum_blocks(int64_t nnz, int32_t H) {
    const int64_t want = cdiv(nnz * H, int64_t(kBurst) * kThreads);
    return want < kSumBlocks ? want : kSumBlocks;
}

gt_status bucket_check(const char* who, int64_t nnz, int32_t H, int32_t B, const void* a, const void* b) {
    const std::string w(who);
    if (nnz < 0 || nnz >= (int64_t(1) << 32)) return fail(GT_ERR_INVALID_ARG, w + ": nnz out of range");
    if (!(H == 1 || H == 2 || H == 4 || H == 8 || H == 16)) return fail(GT_ERR_UNSUPPORTED, w + ": unsupported H");
    if (B < 1 || B > GT_MAX_BUCKETS) return fail(GT_ERR_UNSUPPORTED, w + ": 1 to 64 buckets");
    if (nnz > 0 && (!a || !b)) return fail(GT_ERR_INVALID_ARG, w + ": null pointer");
    return GT_OK;
}

}  // namespace

extern "C" gt_status gt_bucket_bias_fwd(int64_t nnz, int32_t H, int32_t B, const float* table, const uint8_t* bucket,
                                        float* bias, hipStream_t s) {
    const char* who = "gt_bucket_bias_fwd";
    const gt_status st = bucket_check(who, nnz, H, B, bucket, bias);
    if (st != GT_OK) return st;
    if (!table) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    if (nnz == 0) return GT_OK;
    constexpr int U = 4;
    const int64_t runs = cdiv(nnz * H, int64_t(kThreads) * 4 * U);
    const unsigned grid = unsigned(runs < kFwdBlocks ? runs : kFwdBlocks);
    switch (H) {
        case 1: k_bucket_fwd<0, U><<<grid, kThreads, 0, s>>>(nnz, B, table, bucket, bias); break;
        case 2: k_bucket_fwd<1, U><<<grid, kThreads, 0, s>>>(nnz, B, table, bucket, bias); break;
        case 4: k_bucket_fwd<2, U><<<grid, kThreads, 0, s>>>(nnz, B, table, bucket, bias); break;
        case 8: k_bucket_fwd<3, U><<<grid, kThreads, 0, s>>>(nnz, B, table, bucket, bias); break;
        default: k_bucket_fwd<4, U><<<grid, kThreads, 0, s>>>(nnz, B, table, bucket, bias); break;
    }
    GT_LAUNCH_CHECK("bucket_bias_fwd");
    return GT_OK;
}

extern "C" size_t gt_bucket_bias_bwd_workspace_size(int64_t nnz, int32_t H, int32_t B) {
    if (nnz < 0 || H < 1 || H > 16 || B < 1 || B > GT_MAX_BUCKETS) return 0;
    Ws w(nullptr);
    w.take<float>(size_t(sum_blocks(nnz, H)) * B * H);
    return w.size();
}

extern "C" gt_status gt_bucket_bias_bwd(int64_t nnz, int32_t H, int32_t B, const uint8_t* bucket, const float* dbias,
                                        float* dtable, void* ws, size_t ws_bytes, hipStream_t s) {
    const char* who = "gt_bucket_bias_bwd";
    const gt_status st = bucket_check(who, nnz, H, B, bucket, dbias);
    if (st != GT_OK) return st;
    const size_t need = gt_bucket_bias_bwd_workspace_size(nnz, H, B);
    if (!dtable || (need > 0 && !ws)) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    if (ws_bytes < need) return fail(GT_ERR_WORKSPACE, std::string(who) + ": workspace too small");
    const int64_t blocks = sum_blocks(nnz, H);
    Ws w(ws);
    float* part = w.take<float>(size_t(blocks) * B * H);
    if (blocks > 0) {
        k_bucket_bwd<<<unsigned(blocks), kThreads, size_t(4) * (B + 1) * kWave * sizeof(float), s>>>(
            nnz, ilog2(H), B, bucket, dbias, part);
        GT_LAUNCH_CHECK("bucket_bias_bwd");
    }
    k_bucket_sum<<<unsigned(cdiv(B * H, 16)), kSumThreads, 0, s>>>(blocks, B * H, part, dtable);
    GT_LAUNCH_CHECK("bucket_bias_bwd sum");
    return GT_OK;
}
