// Matrix-core building blocks of the packed-sequence attention kernels, for
// bf16 and fp32 features, and what the forward and backward kernels share.
//
// Every product is formed in 32 x 32 blocks with the owned rows as columns, so a
// lane holds one owned row and 16 of its partners (accumulator element i is
// partner crow(i, lane)).  Row statistics then need one exchange between the
// half-waves, and the weights become the next product's B operand straight from
// the accumulators.  bf16 blocks are v_mfma_f32_32x32x16_bf16; fp32 blocks
// v_mfma_f32_32x32x2_f32, whose operands are single fp32 values, so nothing is
// rounded.
#pragma once

#include "packed.h"

namespace gt {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr float kInf = __builtin_huge_valf();
constexpr float kLowest = -3.402823466e38f;  // a running maximum's start: -inf minus it is -inf, no NaN

__device__ __forceinline__ int crow(int i, int lane) { return 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3); }

__device__ __forceinline__ f32x16_t splat16(float x) {
    f32x16_t z;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] = x;
    return z;
}

__device__ __forceinline__ float pair_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// 16 bytes from global memory straight into LDS: lane i's land at `lds` + 16 i.
__device__ __forceinline__ void load_to_lds(void* lds, const void* src) {
    __builtin_amdgcn_global_load_lds(
        reinterpret_cast<const __attribute__((address_space(1))) uint32_t*>(reinterpret_cast<uintptr_t>(src)),
        reinterpret_cast<__attribute__((address_space(3))) uint32_t*>(reinterpret_cast<uintptr_t>(lds)), 16, 0, 0);
}

// The stage fetched last is in LDS for every wavefront of the workgroup, and
// every wavefront is done reading the one before.
template <int WAVES>
__device__ __forceinline__ void stage_done() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    if constexpr (WAVES > 1) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
}

// Operands of the block products.  A stage of partner rows lies row-major in
// LDS, each row's 16-byte pieces permuted by the row number, which spreads the
// same piece of neighbouring rows over the LDS banks.
template <typename T, int D>
struct Blk {
    static constexpr bool kHalf = sizeof(T) == 2;
    static constexpr int kStage = kHalf ? 64 : 32;         // partner rows per stage
    static constexpr int kElems = kStage * D;              // one staged operand
    static constexpr int kPiece = 16 / int(sizeof(T));     // features per 16-byte piece
    static constexpr int kPieces = D / kPiece;             // pieces per row
    static constexpr int kLoads = kElems * int(sizeof(T)) / 1024;  // 1 KiB wavefront loads per operand
    static constexpr int kSteps = D / (2 * kPiece);        // pieces a lane holds of one row

    // the pieces' permutation in row r; rows of 256 bytes and more span all banks
    __device__ __forceinline__ static int turn(int r) {
        return kPieces >= 16 ? r & 15 : kPieces == 8 ? (kHalf ? r & 7 : (r >> 1) & 7) : (r >> 1) & 3;
    }

    // One owned row as a B operand: pieces 2 c + lane / 32.
    struct Row {
        uint4 v[kSteps];
        __device__ __forceinline__ void load(const T* p, int lane) {
#pragma unroll
            for (int c = 0; c < kSteps; ++c)
                v[c] = *reinterpret_cast<const uint4*>(p + kPiece * (2 * c + (lane >> 5)));
        }
        __device__ __forceinline__ float dot(const Row& o) const {
            float s = 0.f;
#pragma unroll
            for (int c = 0; c < kSteps; ++c) {
                const uint32_t a[4] = {v[c].x, v[c].y, v[c].z, v[c].w}, b[4] = {o.v[c].x, o.v[c].y, o.v[c].z, o.v[c].w};
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    if constexpr (kHalf) {
                        s = fmaf(bf16lo(a[t]), bf16lo(b[t]), s);
                        s = fmaf(bf16hi(a[t]), bf16hi(b[t]), s);
                    } else {
                        s = fmaf(__uint_as_float(a[t]), __uint_as_float(b[t]), s);
                    }
                }
            }
            return s;
        }
    };

    // This wavefront's share of a stage: `rows` partner rows (of kStage) are
    // wanted; row(r) is the address of row r's features.
    template <int WAVES, typename F>
    __device__ __forceinline__ static void fetch(T* s, int rows, int wave, int lane, F row) {
#pragma unroll
        for (int q0 = 0; q0 < kLoads; q0 += WAVES) {
            const int q = q0 + wave;
            if (q >= kLoads || q * 64 / kPieces >= rows) break;  // uniform
            const int at = q * 64 + lane, r = at / kPieces, c = (at % kPieces) ^ turn(r);
            load_to_lds(s + q * (1024 / int(sizeof(T))), row(r) + kPiece * c);
        }
    }

    // c += (staged rows r0 .. r0 + 31) x (owned rows), over the features.
    __device__ __forceinline__ static f32x16_t mul_piece(uint4 a, uint4 b, f32x16_t c) {
        if constexpr (kHalf) {
            return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a),
                                                           __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
        } else {
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
            return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
        }
    }
    __device__ __forceinline__ static uint4 piece(const T* s, int r, int c, int lane) {
        return *reinterpret_cast<const uint4*>(s + r * D + kPiece * ((2 * c + (lane >> 5)) ^ turn(r)));
    }
    template <int NB>
    __device__ __forceinline__ static void rows(const T* s, int r0, const Row (&o)[NB], f32x16_t (&c)[NB], int lane) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const uint4 a = piece(s, r0 + (lane & 31), k, lane);
#pragma unroll
            for (int b = 0; b < NB; ++b) c[b] = mul_piece(a, o[b].v[k], c[b]);
        }
    }

    // The staged rows r0 .. r0 + 31 turned round (features x partners), in the
    // partner order of an accumulator used as B operand.
    struct Cols {
        // bf16: partners 16 half + 4 (lane / 32) + {0..3, 8..11}; fp32: partner crow(i, lane)
        typename std::conditional<kHalf, bf16x8_t, float>::type v[D / 32][kHalf ? 2 : 16];

        __device__ __forceinline__ void load(const T* s, int r0, int lane) {
            if constexpr (kHalf) {
                typedef short s16x4_t __attribute__((ext_vector_type(4)));
                typedef short s16x8_t __attribute__((ext_vector_type(8)));
                const int k = 4 * (lane >> 5) + ((lane & 15) >> 2);
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int c = 4 * db + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
                        const T* x = s + (r0 + 16 * half + k) * D + 8 * (c ^ turn(k)) + 4 * (lane & 1);
                        const T* y = s + (r0 + 16 * half + k + 8) * D + 8 * (c ^ turn(k + 8)) + 4 * (lane & 1);
                        const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            reinterpret_cast<__attribute__((address_space(3))) s16x4_t*>(reinterpret_cast<uintptr_t>(x)));
                        const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            reinterpret_cast<__attribute__((address_space(3))) s16x4_t*>(reinterpret_cast<uintptr_t>(y)));
                        v[db][half] =
                            __builtin_bit_cast(bf16x8_t, s16x8_t{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
                    }
            } else {
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int r = r0 + crow(i, lane), f = 32 * db + (lane & 31);
                        v[db][i] = s[r * D + 4 * ((f >> 2) ^ turn(r)) + (f & 3)];
                    }
            }
        }
        // Zero the partners from the `left`-th on: rows behind the end hold
        // whatever lies there, and a zero weight times an infinity would be NaN.
        __device__ __forceinline__ void drop(int left, int lane) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (crow(i, lane) >= left)
#pragma unroll
                    for (int db = 0; db < D / 32; ++db) {
                        if constexpr (kHalf) v[db][i / 8][i % 8] = (__bf16)0.f;
                        else v[db][i] = 0.f;
                    }
        }
    };
    // acc (features x owned rows) += Cols x w, w an accumulator block (partners x
    // owned rows); bf16 rounds w to bf16 (half a step, 2^-9 of a weight: the
    // size of the features' own rounding).
    template <int NB>
    __device__ __forceinline__ static void apply(const Cols& a, const f32x16_t (&w)[NB], f32x16_t (&acc)[NB][D / 32]) {
        if constexpr (kHalf) {
            bf16x8_t p[NB][2];
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) p[b][i / 8][i % 8] = (__bf16)w[b][i];
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        acc[b][db] =
                            __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v[db][half], p[b][half], acc[b][db], 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int b = 0; b < NB; ++b)
                        acc[b][db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[db][i], w[b][i], acc[b][db], 0, 0, 0);
        }
    }
    // One owned row of acc times f, as T.
    __device__ __forceinline__ static void store(T* o, const f32x16_t (&a)[D / 32], float f, int lane) {
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                T* to = o + 32 * db + 8 * j + 4 * (lane >> 5);
                const float x = a[db][4 * j] * f, y = a[db][4 * j + 1] * f, z = a[db][4 * j + 2] * f,
                            w = a[db][4 * j + 3] * f;
                if constexpr (kHalf) *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(x, y), pack_bf16x2(z, w));
                else *reinterpret_cast<float4*>(to) = make_float4(x, y, z, w);
            }
    }
};

// A block's place: which item and which kv head; false for the grid's padding.
// Small items lie head by head, so the heads of one sequence, whose features
// share cache lines, run together; large ones item by item within a head, so an
// XCD works on few heads' keys at a time.
template <bool SMALL>
__device__ __forceinline__ bool packed_place(const PackedArgs& a, PackedItem& it, int& hk, int64_t& block) {
    const int64_t b = xcd_block(blockIdx.x, gridDim.x);
    if (b >= int64_t(a.n_items) * a.Hkv) return false;
    block = b;
    const int64_t i = SMALL ? b / a.Hkv : b % a.n_items;
    hk = int(SMALL ? b % a.Hkv : b / a.n_items);
    it = a.items[i];
    return true;
}
inline unsigned packed_grid(int64_t items, int Hkv) { return xcd_grid(items * Hkv); }

// The learned bias's table of one kv head's group in LDS: [g][kTableStride],
// -inf from the B-th bucket on.
__device__ __forceinline__ void load_table(float* s, const PackedArgs& a, int hk) {
    for (int x = int(threadIdx.x); x < (kTableStride << a.gs); x += int(blockDim.x)) {
        const int hg = x / kTableStride, b = x % kTableStride;
        s[x] = b < a.B ? a.table[int64_t(b) * a.H + (hk << a.gs) + hg] : -kInf;
    }
}

}  // namespace gt
