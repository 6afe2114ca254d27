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
//
// The products alone, stored as they are, 2,048 x 8,192 x 16,384 in bf16, blocks of 256 x
// 256 by eight wavefronts: 1,320 TFLOP/s (a library's 1,300 to 1,390), the matrix cores
// busy 72% of the time at 1.85 GHz; with no loads from memory 1,680.  Reading a quarter
// step ahead took it to 1,200, rows that are no multiple of 32 KB apart to 1,320.  Power
// bounds the clock: logits of 8,192 x 2,048 over 128,000 classes run at 1.65 GHz, and with
// zeros as data at 2.24 in 23% less time, the matrix cores busy 60% of the time in both.
// Tried and not kept, at 1,290 to 1,320: four stages of half the depth (1,250), the loads
// spread over the step's quarters (1,260) or between the products (1,210 to 1,300), four
// wavefronts with 128 x 128 each (1,160), staging through registers (275); at 1,200, a
// wave priority around the products (1,180); workgroups that stay and begin the next
// block's loads before they store (no faster: 80 registers spill).
#pragma once

#include "attn_common.h"

namespace gt {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kStepBytes = 128;  // of every row, a step

// One matrix instruction of a 16-byte piece of each operand: bf16 takes the pieces
// whole, fp32 an element e of each.
__device__ __forceinline__ void mma_part(uint16_t, const uint4& a, const uint4& b, f32x16_t& c, int) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0,
                                                0, 0);
}
__device__ __forceinline__ void mma_part(float, const uint4& a, const uint4& b, f32x16_t& c, int e) {
    const uint32_t x = e == 0 ? a.x : e == 1 ? a.y : e == 2 ? a.z : a.w;
    const uint32_t y = e == 0 ? b.x : e == 1 ? b.y : e == 2 ? b.z : b.w;
    c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(x), __uint_as_float(y), c, 0, 0, 0);
}

__device__ __forceinline__ void copy_to_lds(char* lds, const char* src) {
    __builtin_amdgcn_global_load_lds(
        reinterpret_cast<const __attribute__((address_space(1))) uint32_t*>(reinterpret_cast<uintptr_t>(src)),
        reinterpret_cast<__attribute__((address_space(3))) uint32_t*>(reinterpret_cast<uintptr_t>(lds)), 16, 0, 0);
}

// Loads before it are issued before loads behind it; no instruction.
__device__ __forceinline__ void issue_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A barrier that waits for no more than is needed (and what orders the compiler's
// memory accesses around it): all but the last LOADS loads of the wavefront have landed
// and its reads of LDS are done.  That a stage has landed when LOADS are on their way
// needs as many loads behind its own: issue_order() between one stage's and the next's.
template <int LOADS>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LOADS) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
// The same for accesses to LDS alone.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
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
    static constexpr int kParts = sizeof(T) == 2 ? 1 : 4;     // matrix instructions of a piece
    static_assert(kStage % (1024 * WM * WN) == 0, "whole loads a wavefront");

    struct Frag {
        uint4 a[TM], b[TN];
    };
    f32x16_t acc[TM][TN];
    const char* src[kLoads];  // where a lane's loads of the next step come from
    int64_t left;             // steps of the block

    // The steps [s0, s1) of kStepBytes of the rows m0.. of A and n0.. of B (B's through the
    // list, if there is one); rows at or above M and N repeat the last one.  A stage holds
    // BM rows of A, then BN of B; eight rows, a load of a wavefront, are of one of the two.
    __device__ __forceinline__ void source(int wave, int lane, const char* A, int64_t lda, int64_t m0, int64_t M,
                                           const char* B, int64_t ldb, int64_t n0, int64_t N, const int32_t* list,
                                           int64_t s0, int64_t s1) {
        left = s0 < s1 ? s1 - s0 : 0;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            const int at = (wave * kLoads + l) * 8, r = at + lane / 8, piece = (lane % 8) ^ turn(r);
            const bool b = at >= BM;
            const int64_t limit = b ? N : M, c = (b ? n0 - BM : m0) + r;
            int64_t row = c < limit ? c : limit - 1;
            if (list && b) row = list[row];
            src[l] = (b ? B : A) + row * (b ? ldb : lda) + piece * 16 + s0 * kStepBytes;
        }
    }

    __device__ __forceinline__ void fetch(char* lds, int wave) {
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            copy_to_lds(lds + (wave * kLoads + l) * 1024, src[l]);
            src[l] += kStepBytes;
        }
    }

    // The loads of the first two steps; nothing reads or writes the stages before run().
    // lds0, lds1: two arrays of kStage bytes (two objects: the compiler makes a read of
    // one wait for loads into the same object).
    __device__ __forceinline__ void start(char* lds0, char* lds1, int wave) {
        if (left & 1) {
            fetch(lds1, wave);
            issue_order();
            if (left > 1) fetch(lds0, wave);
        } else if (left) {
            fetch(lds0, wave);
            issue_order();
            fetch(lds1, wave);
        }
    }

    // The products.  A step's four quarters (two pieces of each row) are read a quarter
    // ahead of their products, the next step's first quarter too: the one barrier of a
    // step stands before its last products, whose operands are in registers, and behind
    // it the buffer just read takes the loads of the step after the next.
    __device__ __forceinline__ void run(char* lds0, char* lds1, int wave, int lane) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
        if (left == 0) return;
        const int wm = wave % WM, wn = wave / WM;
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
            for (int e = 0; e < kParts; ++e)
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j) mma_part(T(), f.a[i], f.b[j], acc[i][j], e);
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
            if (more) fetch(cur, wave);
            read(f0, nxt, 0);  // behind the last step what lies there, multiplied by nothing
            mul(f1);
            mix();
        };
        if (left > 1) wait_loads<kLoads>();
        else wait_loads<0>();
        if (left & 1) {  // one step by itself, the others go in pairs
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                read(f0, lds1, c);
                mul(f0);
            }
            lds_barrier();  // lds1 has been read
            if (--left) {
                fetch(lds1, wave);
                wait_loads<kLoads>();
            }
        }
        if (left) read(f0, lds0, 0);
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
        constexpr int reads = TM + TN, products = TM * TN * kParts;
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
