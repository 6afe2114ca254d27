// Dropout from a counter-based generator, with the residual's addition.
//
// y_i = (add_i +) x_i / (1 - p) where word i of the generator is at or above
// T = round(p 2^32), (add_i +) 0 elsewhere.  The words are those of Philox4x32-10
// (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// SC 2011): four for each 64-bit counter, so any element's word is found from its
// index alone and no mask is kept.  Key and first counter are read on the device.
//
// Bound by memory (x, add in, y out: 5.3 to 5.9 TB/s beyond the caches, bf16 and fp32;
// a million rows of 256 bf16 186 us): the generator's 20 products of a counter are vector
// work beside the loads.  A lane takes 16 bytes of each array, two counters of bf16
// elements or one of fp32.
#include <cmath>

#include "rows.h"

using namespace gt;

namespace {

// The four words of a counter (its high 64 bits are zero).
__device__ __forceinline__ void words(uint64_t counter, uint64_t seed, uint32_t (&w)[4]) {
    uint32_t x0 = uint32_t(counter), x1 = uint32_t(counter >> 32), x2 = 0, x3 = 0;
    uint32_t k0 = uint32_t(seed), k1 = uint32_t(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t a = uint64_t(x0) * 0xD2511F53u, b = uint64_t(x2) * 0xCD9E8D57u;
        x0 = uint32_t(b >> 32) ^ x1 ^ k0;
        x2 = uint32_t(a >> 32) ^ x3 ^ k1;
        x1 = uint32_t(b), x3 = uint32_t(a);
        k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
    }
    w[0] = x0, w[1] = x1, w[2] = x2, w[3] = x3;
}

template <typename T, bool ADD>
__global__ __launch_bounds__(256) void k_dropout(int64_t n, uint32_t limit, float up, const uint64_t* rng, const T* x,
                                                  const T* add, T* y, bool far) {
    constexpr int E = Piece<T>::E;
    const uint64_t seed = rng[0], offset = rng[1];
    const int64_t pieces = cdiv(n, E), step = int64_t(gridDim.x) * blockDim.x;
    for (int64_t c = blockIdx.x * int64_t(blockDim.x) + threadIdx.x; c < pieces; c += step) {
        const int64_t i0 = c * E;
        const bool whole = i0 + E <= n;
        float v[E], r[E];
        if (whole) {
            load_piece(v, x + i0);
            if constexpr (ADD) load_piece(r, add + i0);
        } else {
#pragma unroll
            for (int t = 0; t < E; ++t) {
                v[t] = i0 + t < n ? load_one(x + i0 + t) : 0.f;
                if constexpr (ADD) r[t] = i0 + t < n ? load_one(add + i0 + t) : 0.f;
            }
        }
#pragma unroll
        for (int q = 0; q < E / 4; ++q) {
            uint32_t w[4];
            words(offset + uint64_t(c) * (E / 4) + q, seed, w);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int k = 4 * q + t;
                // chosen, not multiplied by 0: what a dropped element held does not matter
                const float d = w[t] >= limit ? v[k] * up : 0.f;
                v[k] = ADD ? r[k] + d : d;
            }
        }
        if (whole) {
            store_piece(y + i0, v, far);
        } else {
#pragma unroll
            for (int t = 0; t < E; ++t)
                if (i0 + t < n) store_one(y + i0 + t, v[t]);
        }
    }
}

template <typename T>
void run(int64_t n, uint32_t limit, float up, const uint64_t* rng, const void* x, const void* add, void* y, bool far,
         hipStream_t s) {
    const unsigned grid = grid_for(cdiv(n, Piece<T>::E), 256, 1 << 16);
    const T* px = static_cast<const T*>(x);
    const T* pa = static_cast<const T*>(add);
    if (add) k_dropout<T, true><<<grid, 256, 0, s>>>(n, limit, up, rng, px, pa, static_cast<T*>(y), far);
    else k_dropout<T, false><<<grid, 256, 0, s>>>(n, limit, up, rng, px, pa, static_cast<T*>(y), far);
}

}  // namespace

extern "C" gt_status gt_dropout(int64_t n, gt_dtype dt, double p, const uint64_t* rng, const void* x, const void* add,
                                void* y, hipStream_t s) {
    if (dt != GT_BF16 && dt != GT_F32) return fail(GT_ERR_UNSUPPORTED, "gt_dropout: unsupported dtype");
    if (n < 0 || n >= (int64_t(1) << 48)) return fail(GT_ERR_INVALID_ARG, "gt_dropout: n out of range");
    if (!(p >= 0.0 && p < 1.0)) return fail(GT_ERR_INVALID_ARG, "gt_dropout: p must be in [0, 1)");
    // the share of words below the limit; a p that rounds to all of them is not dropout
    const double limit = std::nearbyint(p * 4294967296.0);
    if (limit >= 4294967296.0) return fail(GT_ERR_INVALID_ARG, "gt_dropout: p must be in [0, 1)");
    if (n == 0) return GT_OK;
    if (!rng || !x || !y) return fail(GT_ERR_INVALID_ARG, "gt_dropout: null pointer");
    if (reinterpret_cast<uintptr_t>(rng) & 7) return fail(GT_ERR_UNSUPPORTED, "gt_dropout: rng must start at a multiple of 8 bytes");
    const bool far = n * (dt == GT_BF16 ? 2 : 4) > kFarBytes;
    const float up = float(1.0 / (1.0 - p));
    if (dt == GT_BF16) run<uint16_t>(n, uint32_t(limit), up, rng, x, add, y, far, s);
    else run<float>(n, uint32_t(limit), up, rng, x, add, y, far, s);
    GT_LAUNCH_CHECK("dropout");
    return GT_OK;
}
