// Matrix-core building blocks of the packed-sequence attention kernels, for
// bf16 and fp32 features, and what the forward and backward kernels share.
//
// Every product is formed in 32 x 32 blocks with the owned rows as columns, so a
// lane holds one owned row and 16 of its partners.  Partner rows are staged in an
// order that makes those 16 consecutive: accumulator element i of a lane is
// partner part(i, lane) of the block.  Row statistics then need one exchange between the
// half-waves, and the weights become the next product's B operand straight from
// the accumulators.  bf16 blocks are v_mfma_f32_32x32x16_bf16; fp32 blocks
// v_mfma_f32_32x32x2_f32, whose operands are single fp32 values, so nothing is
// rounded.
#pragma once

#include "lanes.h"
#include "packed.h"

namespace gt {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr float kInf = __builtin_huge_valf();
constexpr float kLowest = -3.402823466e38f;  // a running maximum's start: -inf minus it is -inf, no NaN

__device__ __forceinline__ int part(int i, int lane) { return 16 * (lane >> 5) + i; }
// The partner (of a block of 32) that lies in LDS row r of the block, and back:
// the matrix cores give lane half h the LDS rows 8 a + 4 h + b, a, b < 4.
__device__ __forceinline__ int row_partner(int r) { return 16 * ((r >> 2) & 1) + 4 * (r >> 3) + (r & 3); }
__device__ __forceinline__ int partner_row(int p) { return 8 * ((p >> 2) & 3) + 4 * (p >> 4) + (p & 3); }

// A compile-time flag passed as a value (generic lambdas take it as auto).
template <bool B>
struct Flag {
    static constexpr bool value = B;
};

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

// The wavefront's own loads into LDS have landed and its reads of LDS are done.
__device__ __forceinline__ void wave_done() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}
// The wavefront's accesses to LDS are done (its stores to memory need not be).
__device__ __forceinline__ void lds_done() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
}
// The first for a workgroup (or, where no wavefront shares a stage, for each).
template <bool SHARED>
__device__ __forceinline__ void stage_done() {
    wave_done();
    if constexpr (SHARED) __syncthreads();
}

// Operands of the block products.  A stage of partner rows lies row-major in
// LDS, each row's 16-byte pieces permuted by the row number, which spreads the
// same piece of neighbouring rows over the LDS banks.
template <typename T, int D, int STAGE = 32>
struct Blk {
    static constexpr bool kHalf = sizeof(T) == 2;
    static constexpr int kStage = STAGE;                   // partner rows per stage
    static constexpr int kElems = kStage * D;              // one staged operand
    static constexpr int kPiece = 16 / int(sizeof(T));     // features per 16-byte piece
    static constexpr int kPieces = D / kPiece;             // pieces per row
    static constexpr int kLoads = kElems * int(sizeof(T)) / 1024;  // 1 KiB wavefront loads per operand
    static constexpr int kSteps = D / (2 * kPiece);        // pieces a lane holds of one row

    // the pieces' permutation in row r; rows of 256 bytes and more span all banks
    __device__ __forceinline__ static int turn(int r) {
        return kPieces >= 16 ? r & 15 : kPieces == 8 ? (kHalf ? r & 7 : (r >> 1) & 7) : (r >> 1) & 3;
    }

    // A lane's byte offsets into a staged block, of the row operand's pieces and of
    // the turned operand; set: offset of the wavefront's stage.  What varies with
    // the block, the stage's buffer and the element is added as a constant, so the
    // reads of a whole walk share these few registers.
    static constexpr int kTurned = kHalf ? D / 32 : D == 32 ? 4 : 8;
    struct At {
        uint32_t row[kSteps], col[kTurned];
        __device__ __forceinline__ At(int lane, int set) {
            const int r = lane & 31, half = lane >> 5;
#pragma unroll
            for (int c = 0; c < kSteps; ++c) row[c] = set + int(sizeof(T)) * (r * D + kPiece * ((2 * c + half) ^ turn(r)));
            if constexpr (kHalf) {
                const int k = 4 * half + ((lane & 15) >> 2), c = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
#pragma unroll
                for (int x = 0; x < kTurned; ++x)
                    col[x] = set + 2 * (k * D + 8 * ((c ^ turn(k)) ^ (4 * x)) + 4 * (lane & 1));
            } else {
#pragma unroll
                for (int x = 0; x < kTurned; ++x)
                    col[x] = set + 4 * (4 * half * D + 4 * (((r >> 2) ^ turn(4 * half)) ^ turned_bits(x)) + (r & 3));
            }
#pragma unroll
            for (int c = 0; c < kSteps; ++c) asm("" : "+v"(row[c]));
#pragma unroll
            for (int x = 0; x < kTurned; ++x) asm("" : "+v"(col[x]));
        }
        __device__ __forceinline__ static constexpr int turned_bits(int x) {
            return D == 32 ? (x & 1) | (x >> 1) << 2 : (x & 3) | (x >> 2) << 3;
        }
    };

    // One owned row as a B operand: pieces 2 c + lane / 32.
    struct Row {
        uint4 v[kSteps];
        __device__ __forceinline__ void load(const T* p, int lane) {
#pragma unroll
            for (int c = 0; c < kSteps; ++c)
                v[c] = *reinterpret_cast<const uint4*>(p + kPiece * (2 * c + (lane >> 5)));
        }
        // the lane's row of a staged block
        __device__ __forceinline__ void staged(const T* s, int lane) {
            const int r = partner_row(lane & 31);
#pragma unroll
            for (int c = 0; c < kSteps; ++c)
                v[c] = *reinterpret_cast<const uint4*>(s + r * D + kPiece * ((2 * c + (lane >> 5)) ^ turn(r)));
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

    // This wavefront's share of a stage: the `left` (at least 1) partner rows from
    // `base` on, up to a stage; off(r) is row r's offset in elements, below 2^30.
    // Rows behind the last one repeat it where their block of 32 is begun, so a
    // block never holds values that are not the sequence's own: weights of zero
    // need nothing else.
    template <int WAVES, typename F>
    __device__ __forceinline__ static void fetch(T* s, const T* base, int left, int wave, int lane, F off) {
        constexpr int kRowsPerLoad = 64 / kPieces;
#pragma unroll
        for (int q0 = 0; q0 < kLoads; q0 += WAVES) {
            const int q = q0 + wave;
            if (q >= kLoads || ((q * kRowsPerLoad) & ~31) >= left) break;  // uniform
            const int at = q * kRowsPerLoad + lane / kPieces, c = (lane % kPieces) ^ turn(at);
            const int p = (at & ~31) + row_partner(at & 31);
            const uint32_t o = off(p < left ? p : left - 1) + uint32_t(kPiece * c);
            load_to_lds(s + q * (1024 / int(sizeof(T))), reinterpret_cast<const char*>(base) + o * uint32_t(sizeof(T)));
        }
    }

    // c += (the 32 staged rows at s) x (owned rows), over the features.
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
    template <int NB>
    __device__ __forceinline__ static void rows(const T* s, const At& at, const Row (&o)[NB], f32x16_t (&c)[NB]) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const uint4 a = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(s) + at.row[k]);
#pragma unroll
            for (int b = 0; b < NB; ++b) c[b] = mul_piece(a, o[b].v[k], c[b]);
        }
    }

    // The 32 staged rows at s turned round (features x partners), in the
    // partner order of an accumulator used as B operand.
    struct Cols {
        // element 8 half + t (bf16) or i (fp32) of a lane: partner part(.., lane)
        typename std::conditional<kHalf, bf16x8_t, float>::type v[D / 32][kHalf ? 2 : 16];

        __device__ __forceinline__ void load(const T* s, const At& at) {
            const char* p = reinterpret_cast<const char*>(s);
            if constexpr (kHalf) {
                typedef short s16x4_t __attribute__((ext_vector_type(4)));
                typedef short s16x8_t __attribute__((ext_vector_type(8)));
                typedef __attribute__((address_space(3))) s16x4_t* lds_t;
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        // eight rows on, rows of 256 bytes are turned by another 8 pieces
                        const char* x = p + 2 * 16 * half * D + at.col[db];
                        const char* y = p + 2 * (16 * half + 8) * D + at.col[kPieces >= 16 ? db ^ 2 : db];
                        const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            reinterpret_cast<lds_t>(reinterpret_cast<uintptr_t>(x)));
                        const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            reinterpret_cast<lds_t>(reinterpret_cast<uintptr_t>(y)));
                        v[db][half] =
                            __builtin_bit_cast(bf16x8_t, s16x8_t{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
                    }
            } else {
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int x = D == 32 ? ((i >> 1) & 1) + 2 * ((i >> 2) & 1) : (i & 3) + 4 * (((i >> 2) ^ db) & 1);
                        v[db][i] = *reinterpret_cast<const float*>(p + 4 * (8 * (i >> 2) + (i & 3)) * D +
                                                                   256 * (db >> 1) + at.col[x]);
                    }
            }
        }
    };
    // Weights (partners x owned rows) as the B operand of a product with Cols:
    // bf16 rounds them to bf16 (half a step, 2^-8 of a weight at most: the size of
    // the features' own rounding), fp32 takes them as they are.
    struct Weights {
        typename std::conditional<kHalf, bf16x8_t, float>::type v[kHalf ? 2 : 16];
        __device__ __forceinline__ void set(const f32x16_t& w) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if constexpr (kHalf) v[i / 8][i % 8] = (__bf16)w[i];
                else v[i] = w[i];
            }
        }
    };
    // acc (features x owned rows) += Cols x weights.
    template <int NB>
    __device__ __forceinline__ static void apply(const Cols& a, const Weights (&w)[NB], f32x16_t (&acc)[NB][D / 32]) {
#pragma unroll
        for (int k = 0; k < (kHalf ? 2 : 16); ++k)
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    if constexpr (kHalf)
                        acc[b][db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v[db][k], w[b].v[k], acc[b][db], 0, 0, 0);
                    else
                        acc[b][db] = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[db][k], w[b].v[k], acc[b][db], 0, 0, 0);
                }
    }
    template <int NB>
    __device__ __forceinline__ static void apply(const Cols& a, const f32x16_t (&w)[NB], f32x16_t (&acc)[NB][D / 32]) {
        Weights p[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) p[b].set(w[b]);
        apply<NB>(a, p, acc);
    }
    // One owned row of acc times f, as T.  A lane holds every other 4 features of its
    // row; bf16 lanes exchange with the other half-wave first, so that each writes 16
    // bytes (8-byte writes are twice the requests).
    __device__ __forceinline__ static void store(T* o, const f32x16_t (&a)[D / 32], float f, int lane) {
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
            if constexpr (kHalf) {
#pragma unroll
                for (int j = 0; j < 4; j += 2) {
                    uint32_t x[2][2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint32_t u = pack_bf16x2(a[db][4 * j + 2 * k] * f, a[db][4 * j + 2 * k + 1] * f);
                        const uint32_t v = pack_bf16x2(a[db][4 * j + 4 + 2 * k] * f, a[db][4 * j + 5 + 2 * k] * f);
                        const auto r = __builtin_amdgcn_permlane32_swap(u, v, false, false);
                        x[0][k] = r[0], x[1][k] = r[1];
                    }
                    *reinterpret_cast<uint4*>(o + 32 * db + 8 * (j + (lane >> 5))) =
                        make_uint4(x[0][0], x[0][1], x[1][0], x[1][1]);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<float4*>(o + 32 * db + 8 * j + 4 * (lane >> 5)) =
                        make_float4(a[db][4 * j] * f, a[db][4 * j + 1] * f, a[db][4 * j + 2] * f, a[db][4 * j + 3] * f);
            }
        }
    }
};

// A block of 32 x 32 values (owned row = lane, partners part(i, lane)) laid down
// so that Cols of a Blk<T, 32> reads it turned round: partner = lane, the owned
// rows as its 16 elements.
template <typename T>
__device__ __forceinline__ void lay_block(T* s, const f32x16_t& w, int lane) {
    using B = Blk<T, 32>;
    const int r = partner_row(lane & 31);
#pragma unroll
    for (int c = 0; c < 16 / B::kPiece; ++c) {
        const int p = (16 / B::kPiece) * (lane >> 5) + c;  // piece of the row
        uint4 x;
        if constexpr (B::kHalf)
            x = make_uint4(pack_bf16x2(w[8 * c], w[8 * c + 1]), pack_bf16x2(w[8 * c + 2], w[8 * c + 3]),
                           pack_bf16x2(w[8 * c + 4], w[8 * c + 5]), pack_bf16x2(w[8 * c + 6], w[8 * c + 7]));
        else
            x = make_uint4(__float_as_uint(w[4 * c]), __float_as_uint(w[4 * c + 1]), __float_as_uint(w[4 * c + 2]),
                           __float_as_uint(w[4 * c + 3]));
        *reinterpret_cast<uint4*>(s + r * 32 + B::kPiece * (p ^ B::turn(r))) = x;
    }
}

// A workgroup's place: which item and which kv head; false for the grid's padding.
// Workgroups go to the 8 XCDs in turn and items lie with the longest walk first, so
// the XCDs' shares are alike only where each takes every 8th item.  Few rows: an
// item's heads, whose features share cache lines, follow each other on one XCD.
// Tiles of many rows: the heads take turns, so an XCD works on every 8th head only
// (a head's keys stay in its L2).  (An eighth of the list for each XCD gave some the
// long walks: four causal prompts of 128-wide heads 343 us forward against 222.)
// An item's tile may be shared by SUB workgroups (sub: which one).
template <bool BY_HEAD, int SUB = 1>
__device__ __forceinline__ bool packed_place(const PackedArgs& a, PackedItem& it, int& hk, int& sub, uint32_t& block) {
    const uint32_t b = blockIdx.x, n = uint32_t(a.n_items) * SUB, heads = uint32_t(a.Hkv);
    const uint32_t p = BY_HEAD ? b / kXcds : b;
    const uint32_t i = BY_HEAD ? p / heads * kXcds + b % kXcds : p / heads;
    if (i >= n) return false;
    hk = int(p % heads);
    block = i * heads + uint32_t(hk);
    sub = int(i % SUB);
    it = a.items[i / SUB];
    return true;
}
inline unsigned packed_grid(int64_t items, int Hkv, int sub = 1) {
    return unsigned(cdiv(items * sub, kXcds) * kXcds * Hkv);
}

// The learned bias's table of one kv head's group in LDS: [g][kTableStride],
// -inf from the B-th bucket on.
template <int THREADS>
__device__ __forceinline__ void load_table(float* s, const PackedArgs& a, int hk, int thread) {
    for (int x = thread; x < (kTableStride << a.gs); x += THREADS) {
        const int hg = x / kTableStride, b = x % kTableStride;
        s[x] = b < a.B ? a.table[int64_t(b) * a.H + (hk << a.gs) + hg] : -kInf;
    }
}

// The buckets of a lane's row and 16 partners of a block: 16 bytes, at a multiple
// of 16 (rows of buckets are padded to that).  Behind the row's end, where every
// pair is masked, the row's first ones are read again (lk is at least 1).
__device__ __forceinline__ uint4 load_ids(const uint8_t* row, int key0, int lk, int lane) {
    const int k = key0 + 16 * (lane >> 5);
    return *reinterpret_cast<const uint4*>(row + (k < lk ? k : 0));
}
// Bucket i of the 16, B for any that the table does not hold.
__device__ __forceinline__ uint32_t id_of(const uint4& ids, int i, uint32_t B) {
    const uint32_t w = i < 4 ? ids.x : i < 8 ? ids.y : i < 12 ? ids.z : ids.w;
    const uint32_t b = (w >> (8 * (i & 3))) & 255u;
    return b < B ? b : B;
}
// The buckets of a lane's key (lane & 31) and rows part(0 .., lane), from 32 rows of
// 32 keys in LDS: 16 lanes read 8 rows of 16 keys and each takes a column.
__device__ __forceinline__ uint4 turned_ids(const uint8_t* s, int lane) {
    typedef int i32x2_t __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) i32x2_t* lds_t;
    const uint8_t* p = s + (16 * (lane >> 5) + ((lane & 15) >> 1)) * 32 + 16 * ((lane >> 4) & 1) + 8 * (lane & 1);
    const i32x2_t a = __builtin_amdgcn_ds_read_tr8_b64_v2i32(reinterpret_cast<lds_t>(reinterpret_cast<uintptr_t>(p)));
    const i32x2_t b =
        __builtin_amdgcn_ds_read_tr8_b64_v2i32(reinterpret_cast<lds_t>(reinterpret_cast<uintptr_t>(p + 8 * 32)));
    return make_uint4(uint32_t(a[0]), uint32_t(a[1]), uint32_t(b[0]), uint32_t(b[1]));
}
__device__ __forceinline__ int64_t ids_width(int lk) { return (int64_t(lk) + 15) & ~int64_t(15); }

// out[head of the group][bucket] = the sums over the lanes (whose row's head is
// lane % g) of `waves` such columns, each B + 1 buckets; a wavefront a bucket.
template <int THREADS>
__device__ __forceinline__ void hist_flush(const float* s, int waves, int B, int gs, float* out, int thread) {
    // four buckets side by side: the exchanges wait for each other only inside one
    constexpr int kSide = 4;
    const int lane = thread % kWave;
    for (int b0 = thread / kWave * kSide; b0 < B; b0 += THREADS / kWave * kSide) {
        float t[kSide];
#pragma unroll
        for (int k = 0; k < kSide; ++k) {
            const int b = b0 + k < B ? b0 + k : B;
            t[k] = 0.f;
            for (int w = 0; w < waves; ++w) t[k] += s[(w * (B + 1) + b) * kWave + lane];
        }
#pragma unroll
        for (int k = 0; k < kSide; ++k) t[k] = pair_sum(t[k]);
#pragma unroll
        for (int o = 16; o > 0; o /= 2)
            if (o >> gs)  // uniform
#pragma unroll
                for (int k = 0; k < kSide; ++k) t[k] += __int_as_float(xor_lane_pow2(__float_as_int(t[k]), o));
#pragma unroll
        for (int k = 0; k < kSide; ++k)
            if (lane >> gs == 0 && b0 + k < B) out[lane * B + b0 + k] = t[k];
    }
}

}  // namespace gt
