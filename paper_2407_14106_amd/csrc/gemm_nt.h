// Matrix products whose operands both lie along the summed dimension, on the matrix
// cores: C[n][m] = sum_k A[m][k] B[n][k], bf16 or fp32, accumulated in fp32.
//
// A workgroup forms a BM x BN block of C.  A step takes 128 bytes of every row of A
// and B into one of two LDS buffers, straight from memory, while the other is
// multiplied.  A row's eight 16-byte pieces are permuted by the row number, so that
// the same piece of neighbouring rows lies in different banks.  Products are 32 x 32
// blocks (bf16 v_mfma_f32_32x32x16_bf16, fp32 v_mfma_f32_32x32x2_f32: the order of
// the summed elements is the same for both operands, so a lane's 16-byte piece is an
// operand as it lies).  Accumulator element i of a lane is
// C[lane % 32][8 (i / 4) + 4 (lane / 32) + i % 4] of its block: four consecutive m.
#pragma once

#include "attn_common.h"

namespace gt {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kStepBytes = 128;  // of every row, a step

__device__ __forceinline__ void mma_piece(uint16_t, const uint4& a, const uint4& b, f32x16_t& c) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0,
                                                0, 0);
}
__device__ __forceinline__ void mma_piece(float, const uint4& a, const uint4& b, f32x16_t& c) {
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
}

__device__ __forceinline__ void copy_to_lds(char* lds, const char* src) {
    __builtin_amdgcn_global_load_lds(
        reinterpret_cast<const __attribute__((address_space(1))) uint32_t*>(reinterpret_cast<uintptr_t>(src)),
        reinterpret_cast<__attribute__((address_space(3))) uint32_t*>(reinterpret_cast<uintptr_t>(lds)), 16, 0, 0);
}

// What orders the compiler's memory accesses around a barrier that waits for no more
// than is needed.
template <int LOADS>
__device__ __forceinline__ void wait_loads() {  // all but the last LOADS loads of the wavefront have landed
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LOADS) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// WM x WN wavefronts, each TM x TN blocks of 32 x 32.
template <typename T, int WM, int WN, int TM, int TN>
struct GemmNT {
    static constexpr int kThreads = WM * WN * kWave;
    static constexpr int BM = WM * TM * 32, BN = WN * TN * 32;
    static constexpr int kStage = (BM + BN) * kStepBytes;
    static constexpr int kLoads = kStage / 1024 / (WM * WN);  // 1 KiB loads of a wavefront, a step
    static_assert(kStage % (1024 * WM * WN) == 0, "whole loads a wavefront");

    f32x16_t acc[TM][TN];

    struct Frag {
        uint4 a[TM], b[TN];
    };

    // lds0, lds1: two arrays of kStage bytes (two objects: the compiler makes a read of
    // one wait for loads into the same object).  Rows m0.. of A and n0.. of B (rows at
    // or above M and N repeat the last one; B's rows through the list, if there is
    // one), steps [s0, s1) of kStepBytes.
    //
    // A step's four quarters (two pieces of each row) are read a quarter ahead of their
    // products, the next step's first quarter too: the one barrier of a step stands
    // before its last products, whose operands are in registers, and behind it the
    // buffer just read takes the loads of the step after the next.
    __device__ __forceinline__ void run(char* lds0, char* lds1, const char* A, int64_t lda, int64_t m0, int64_t M,
                                        const char* B, int64_t ldb, int64_t n0, int64_t N, const int32_t* rows,
                                        int64_t s0, int64_t s1) {
        const int tid = threadIdx.x, wave = uniform(tid / kWave), lane = tid % kWave;
        const int wm = wave % WM, wn = wave / WM;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        if (s0 >= s1) return;
        const char* src[kLoads];
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            const int r = (wave * kLoads + l) * 8 + lane / 8;  // row of the stage: BM of A, then BN of B
            const int piece = (lane % 8) ^ turn(r);
            if (r < BM) {
                const int64_t m = m0 + r < M ? m0 + r : M - 1;
                src[l] = A + m * lda + piece * 16 + s0 * kStepBytes;
            } else {
                int64_t n = n0 + (r - BM) < N ? n0 + (r - BM) : N - 1;
                if (rows) n = rows[n];
                src[l] = B + n * ldb + piece * 16 + s0 * kStepBytes;
            }
        }
        const auto fetch = [&](char* lds) {
#pragma unroll
            for (int l = 0; l < kLoads; ++l) {
                copy_to_lds(lds + (wave * kLoads + l) * 1024, src[l]);
                src[l] += kStepBytes;
            }
        };
        uint32_t at_a[4], at_b[4];  // a lane's places in a stage, by quarter
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int r = lane & 31, p = ((2 * c + (lane >> 5)) ^ turn(r)) * 16 + r * kStepBytes;
            at_a[c] = wm * TM * 32 * kStepBytes + p;
            at_b[c] = (BM + wn * TN * 32) * kStepBytes + p;
        }
        const auto read = [&](Frag& f, const char* lds, int c) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
                f.a[i] = *reinterpret_cast<const uint4*>(lds + at_a[c] + i * 32 * kStepBytes);
#pragma unroll
            for (int j = 0; j < TN; ++j)
                f.b[j] = *reinterpret_cast<const uint4*>(lds + at_b[c] + j * 32 * kStepBytes);
        };
        const auto mul = [&](const Frag& f) {
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) mma_piece(T(), f.a[i], f.b[j], acc[i][j]);
        };
        Frag f0, f1;
        const auto step = [&](char* cur, const char* nxt, bool more) {
            read(f1, cur, 1);
            mul(f0);
            mix();
            read(f0, cur, 2);
            mul(f1);
            mix();
            read(f1, cur, 3);
            mul(f0);
            mix();
            wait_loads<0>();
            if (more) fetch(cur);
            read(f0, nxt, 0);  // behind the last step what lies there, multiplied by nothing
            mul(f1);
            mix();
        };
        int64_t left = s1 - s0;
        fetch(left & 1 ? lds1 : lds0);
        if (left & 1) {  // one step by itself, the others go in pairs
            if (left > 1) {
                fetch(lds0);
                wait_loads<kLoads>();
            } else {
                wait_loads<0>();
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                read(f0, lds1, c);
                mul(f0);
            }
            wait_loads<kLoads>();  // lds1 has been read
            --left;
        }
        if (left) {
            fetch(lds1);
            wait_loads<kLoads>();
            read(f0, lds0, 0);
        }
        for (; left; left -= 2) {
            step(lds0, lds1, left > 2);
            step(lds1, lds0, left > 2);
        }
    }

private:
    // the pieces' permutation in row r: rows are half a pass over the banks
    __device__ __forceinline__ static int turn(int r) { return (r >> 1) & 7; }

    // reads between the products
    __device__ __forceinline__ static void mix() {
        constexpr int reads = TM + TN, products = TM * TN * (sizeof(T) == 2 ? 1 : 4);
#pragma unroll
        for (int k = 0; k < reads; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, products / reads, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, products - products / reads * reads, 0);
        __builtin_amdgcn_sched_barrier(0);
    }
};

}  // namespace gt
