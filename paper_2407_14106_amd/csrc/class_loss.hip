// Softmax cross entropy over many classes, straight from the features and the class
// weights, and its gradients; the logits are never kept.
//
//   s_iv = <X_i, W_v>,  lse_i = log sum_v exp s_iv,  loss_i = lse_i - s_i,y(i),
//   dL_iv = dloss_i (exp(s_iv - lse_i) - [v = y(i)]),  dX = dL W,  dW = dL^T X.
//
// Rows without a label take no part: where there are more rows than a block takes, the
// labelled ones are listed first (on the device, in order), and every product runs over
// the list.
//
// Forward: the product s with the classes as its rows, so that a lane holds one
// token and a block's classes: the block leaves (max, sum of exp) for each of its
// tokens, and one small kernel joins the blocks of a token.
// Backward: the classes go by in pieces, and where there are many rows these too.  A
// piece's s is formed again, dL is rounded to the features' type and written both ways
// round, and two products give its part of dW and of dX, which are summed in fp32 over
// the pieces.  W and X are laid out the other way round for these, so that one product
// serves for all.
// Where a product has few blocks its sum is split over the grid and the parts are
// added in order.  No atomics on a sum: results are the same run to run.
//
// Bound by the matrix cores from some thousand tokens and classes on: 6,963 labelled of
// 8,192 tokens x 2,048 over 128,000 classes in bf16 3.3 ms forward (1,115 TFLOP/s; without
// the exponentials and sums 9% less time), 10.4 backward (eight pieces of 16,384 classes:
// dL 466 us, dX 447, dW 374: 980, 1,020 and 1,220 TFLOP/s), where a library's products of
// such sizes reach 1,150 to 1,170 (logits, dL) and 1,360 to 1,460 (dX, dW); in fp32, 2,048
// x 512 over 32,000, 0.52 and 1.6 ms (127 TFLOP/s).  By the class weights for a few tokens
// (16 x 2,048 over 128,000: 4.2 TB/s), by memory and the chain of small kernels for few
// classes (200,000 nodes x 256, three in ten labelled, 172 classes: 160 us, where the
// features, dL, its turn and the results are 0.3 GB).
#include "gemm_nt.h"
#include "lanes.h"
#include "rows.h"

using namespace gt;

namespace {

constexpr int kListThreads = 1024, kListRounds = 8, kListRows = kListThreads * kListRounds;
constexpr int64_t kPieceBytes = int64_t(256) << 20;  // of a piece's dL, one way round: the last-level cache
constexpr int64_t kMinPiece = 1024;                  // classes of a piece
constexpr int64_t kPartBytes = int64_t(1) << 30;     // of dL, one way round, where a piece has that few classes or all:
                                                     // more rows go by in parts (parts of 256 MB: 400,000 x 64 over
                                                     // 1,000 11% slower, a million rows 14%; of 512 MB 7 and 7; 2% of 1 GB)
constexpr int kSplitBlocks = 256;                    // blocks that fill the chip
constexpr int64_t kCutBlocks = int64_t(1) << 20;     // of a product whose blocks' shape is chosen
constexpr int64_t kFewBlocks = 8;                    // of classes, that one lane joins
constexpr double kParts = 2.4e5;                     // of the tokens' statistics, joined in a microsecond
constexpr double kSlotBytes = 2e6;                   // of a split sum's parts, joined in a microsecond
constexpr int64_t kLaunchBlocks = int64_t(1) << 22;  // of a launch (its threads are counted in 32 bits)
constexpr int64_t kGatherClasses = 2048;             // above, X's listed rows are laid out once: every block of
                                                     // classes would read them through the list (3% of its time)
constexpr int64_t kListed = 256;                     // up to so many rows none is left out: they are one block
constexpr int64_t kOff = 64;                         // elements behind a row of a turned or dL array: rows whose
                                                     // stride is a large power of two meet in few channels
constexpr int64_t kOffBytes = 4096;                  // of such a row of dL along few classes, which has none (its stride
                                                     // with or without: 0.99 to 1.01 times as fast)
constexpr int kSplitSteps = 8;                       // of a split sum, at least

constexpr float kNegInf = -__builtin_huge_valf();

// ------------------------------------------------------------ labelled rows

// One workgroup's labels: bit r of the result is set where row
// b kListRows + r kListThreads + tid has one.
__device__ __forceinline__ uint32_t labelled(const void* labels, bool wide, int64_t n, int64_t V) {
    uint32_t m = 0;
#pragma unroll
    for (int r = 0; r < kListRounds; ++r) {
        const int64_t i = int64_t(blockIdx.x) * kListRows + r * kListThreads + threadIdx.x;
        if (i < n && load_id(labels, wide, i, V) >= 0) m |= 1u << r;
    }
    return m;
}

__global__ __launch_bounds__(kListThreads) void k_list_count(int64_t n, int64_t V, bool wide, const void* labels,
                                                              int32_t* cnt, uint32_t* top) {
    __shared__ int s_n[kListThreads / kWave];
    if (top && blockIdx.x == 0 && threadIdx.x == 0) *top = 0;
    const int c = wave_sum(__popc(labelled(labels, wide, n, V)));
    if (lane_id() == 0) s_n[threadIdx.x / kWave] = c;
    __syncthreads();
    if (threadIdx.x == 0) {
        int t = 0;
        for (int w = 0; w < kListThreads / kWave; ++w) t += s_n[w];
        cnt[blockIdx.x] = t;
    }
}

// Bits of |x|, which compare as |x| does.
__device__ __forceinline__ uint32_t size_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The list; for the forward, what a row without a label has in its results; for the
// backward, the largest |dloss| of a listed row (top, as bits).
__global__ __launch_bounds__(kListThreads) void k_list_place(int64_t n, int64_t V, bool wide, const void* labels,
                                                              const int32_t* cnt, int32_t* list, int32_t* count,
                                                              float* loss, float* lse, const float* dloss,
                                                              uint32_t* top) {
    constexpr int W = kListThreads / kWave;
    __shared__ int s_n[kListRounds * W], s_before[W];
    __shared__ uint32_t s_top[W];
    const int wave = threadIdx.x / kWave, lane = lane_id();
    const uint32_t m = labelled(labels, wide, n, V);
    int rank[kListRounds];
#pragma unroll
    for (int r = 0; r < kListRounds; ++r) {
        const uint64_t b = ballot((m >> r) & 1u);
        rank[r] = __popcll(b & lanemask_lt());
        if (lane == 0) s_n[r * W + wave] = __popcll(b);
    }
    int before = 0;
    for (int64_t b = threadIdx.x; b < int64_t(blockIdx.x); b += kListThreads) before += cnt[b];
    before = wave_sum(before);
    uint32_t most = 0;
    if (top) {
#pragma unroll
        for (int r = 0; r < kListRounds; ++r)
            if ((m >> r) & 1u) {
                const uint32_t b = size_bits(dloss[int64_t(blockIdx.x) * kListRows + r * kListThreads + threadIdx.x]);
                most = most > b ? most : b;
            }
        most = wave_max(most);
    }
    if (lane == 0) s_before[wave] = before, s_top[wave] = most;
    __syncthreads();
    if (threadIdx.x == 0) {
        int t = 0;
        for (int w = 0; w < W; ++w) {
            t += s_before[w];
            most = most > s_top[w] ? most : s_top[w];
        }
        if (top) {
            if (gridDim.x == 1) *top = most;
            else atomicMax(top, most);
        }
        for (int k = 0; k < kListRounds * W; ++k) {
            const int c = s_n[k];
            s_n[k] = t;
            t += c;
        }
        if (blockIdx.x == gridDim.x - 1) *count = t;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kListRounds; ++r) {
        const int64_t i = int64_t(blockIdx.x) * kListRows + r * kListThreads + threadIdx.x;
        if ((m >> r) & 1u) {
            list[s_n[r * W + wave] + rank[r]] = int32_t(i);
        } else if (i < n && loss) {
            loss[i] = 0.f;
            lse[i] = 0.f;
        }
    }
}

// Rows without a label have no gradient (140,000 rows of 256 bf16 14 us): a wavefront looks at `span` labels (64, or fewer
// where rows are few), then groups of its lanes clear the rows without one, a 16-byte piece a lane (the last one ending with
// the row).
template <typename T>
__global__ __launch_bounds__(256) void k_zero_rows(int64_t n, int D, int64_t V, bool wide, const void* labels, T* dx,
                                                    int shift, int span, bool far) {
    constexpr int E = Piece<T>::E;
    const float zero[E] = {};
    const int lane = lane_id(), lanes = 1 << shift, groups = kWave >> shift, x = lane & (lanes - 1);
    const int pieces = int(cdiv(D, E));
    for (int64_t i0 = (int64_t(blockIdx.x) * 4 + threadIdx.x / kWave) * span; i0 < n;
         i0 += int64_t(gridDim.x) * 4 * span) {
        const uint64_t none = ballot(lane < span && i0 + lane < n && load_id(labels, wide, i0 + lane, V) < 0);
        for (int r = lane >> shift; r < span; r += groups) {
            if (!((none >> r) & 1u)) continue;
            T* row = dx + (i0 + r) * D;
            if (D < E) {
                for (int c = x; c < D; c += lanes) row[c] = T(0);
            } else {
                for (int p = x; p < pieces; p += lanes) store_piece(row + (p * E + E <= D ? p * E : D - E), zero, far);
            }
        }
    }
}
template <typename T>
__global__ __launch_bounds__(256) void k_zero(int64_t n, T* p) {
    for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) p[i] = T(0);
}

// ------------------------------------------------------------------ layouts

// dst[r][0 .. ldd) = src[r][0 .. C), zeros behind; rows through the list, if there is
// one, count of them.  whole: both are whole 16-byte pieces.
template <typename T>
__global__ __launch_bounds__(256) void k_pad(int64_t R, const int32_t* list, const int32_t* count, int C, const T* src,
                                              int64_t lds, T* dst, int ldd, bool whole) {
    constexpr int E = Piece<T>::E;
    if (count) R = *count;
    for (int64_t r = int64_t(blockIdx.x) * 4 + threadIdx.x / kWave; r < R; r += int64_t(gridDim.x) * 4) {
        const T* from = src + (list ? int64_t(list[r]) : r) * lds;
        if (whole)
            for (int c = lane_id() * E; c < ldd; c += kWave * E)
                *reinterpret_cast<uint4*>(dst + r * ldd + c) = *reinterpret_cast<const uint4*>(from + c);
        else
            for (int c = lane_id(); c < ldd; c += kWave) dst[r * ldd + c] = c < C ? from[c] : T(0);
    }
}

// dst[c][r] = src[r][c] for the rows r < R, zeros for R <= r < R rounded up to 64.
// Rows through a list, or all of them, those without a label as zeros.  Source rows
// are whole 16-byte pieces (zeros behind column C).
struct Turn {
    int64_t R;
    const int32_t *count, *list;
    const void* labels;  // or null
    bool wide;
    int64_t V;
    const void* src;
    int64_t lds;
    void* dst;
    int64_t ldd;
};
struct Turns {
    Turn t[2];
    // of a call without a list, by the way: the largest |dloss| of a row with a label
    const float* dloss;
    uint32_t* top;
};
template <typename T>
__global__ __launch_bounds__(256) void k_turn(Turns both, int C) {
    constexpr int E = 16 / int(sizeof(T)), P = 64 / E;  // pieces of 64 elements
    __shared__ T s[64][64 + 4 / sizeof(T)];
    const Turn& a = both.t[blockIdx.z];
    if (both.top && a.labels && blockIdx.x == 0 && blockIdx.y == 0) {
        __shared__ uint32_t s_top[4];
        const int i = threadIdx.x;  // there are no more rows than threads
        uint32_t most = i < a.R && load_id(a.labels, a.wide, i, a.V) >= 0 ? size_bits(both.dloss[i]) : 0u;
        most = wave_max(most);
        if (lane_id() == 0) s_top[i / kWave] = most;
        __syncthreads();
        if (i == 0) {
            for (int w = 1; w < 4; ++w) most = most > s_top[w] ? most : s_top[w];
            *both.top = most;
        }
    }
    const int64_t R = a.count ? int64_t(*a.count) : a.R, r0 = int64_t(blockIdx.x) * 64;
    if (r0 >= R) return;
    const int c0 = blockIdx.y * 64;
#pragma unroll
    for (int k = 0; k < 64 * P / 256; ++k) {
        const int y = (k * 256 + int(threadIdx.x)) / P, c = int(threadIdx.x) % P * E;
        const int64_t r = r0 + y;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (r < R && c0 + c < C) {
            const int64_t row = a.list ? int64_t(a.list[r]) : r;
            if (!a.labels || load_id(a.labels, a.wide, row, a.V) >= 0)
                v = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.src) + row * a.lds + c0 + c);
        }
        uint32_t* o = reinterpret_cast<uint32_t*>(&s[y][c]);
        o[0] = v.x, o[1] = v.y, o[2] = v.z, o[3] = v.w;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 64 * P / 256; ++k) {
        const int c = (k * 256 + int(threadIdx.x)) / P, y = int(threadIdx.x) % P * E;
        if (c0 + c >= C) continue;
        union {
            T e[E];
            uint4 v;
        } x;
#pragma unroll
        for (int e = 0; e < E; ++e) x.e[e] = s[y + e][c];
        *reinterpret_cast<uint4*>(static_cast<T*>(a.dst) + int64_t(c0 + c) * a.ldd + r0 + y) = x.v;
    }
}

// ----------------------------------------------------------------- products

// kStats: the forward's statistics; kGrad: dL, both ways round; kStore: dX or dW.
enum What { kStats, kGrad, kStore };

struct LossArgs {
    const char *A, *B;      // rows of A: classes or features; rows of B: tokens or classes
    int64_t lda, ldb;       // bytes
    int64_t M, N;
    const int32_t* n_count;  // rows of the list (on the device; N at most of them count), or null
    int64_t steps;           // of the sum
    const int32_t* k_count;  // the same of the sum's elements (steps at most), or null
    int64_t first;           // of the list's rows, those before this part
    int splits;
    // kStats, kGrad: B's rows are tokens, listed if there is a list
    int64_t v0, V;  // class of A's first row; classes
    const int32_t* list;
    bool gather;  // B's rows too go through the list (they do not lie in its order already)
    const void* labels;
    bool wide;
    float *part, *hit;  // kStats: part[block][token] of two floats; with one block of classes, null and
    float *loss, *lse;  // the results themselves
    int64_t part_ld;
    const float *lse_in, *dloss;  // kGrad; kStore: dloss, the rows' factors, or null
    const uint32_t* top;          // kGrad: what dlt is relative to; kStore: a factor, or null
    void *dl, *dlt;               // kGrad: dL without dloss [token][dl_ld], and with it [class][dlt_ld], or null
    int64_t dl_ld, dlt_ld;
    // kStore: out[split][row][M], or the result itself
    float* slots;
    int64_t slot_rows;
    bool add;
    void* out;
    const int32_t* out_rows;
};

// The size that dL^T is relative to: the largest |dloss|.  In a mean all rows' dloss are
// the same number, and dloss (p - 1) of the many labels with a small p would all be off
// by the rounding of that one number (0.3% of dW at 1 / 6963); relative to it they are
// -1.  dX takes its row's dloss at the end, in fp32.
__device__ __forceinline__ float whole_size(const uint32_t* top) {
    const float u = __uint_as_float(*top);
    return u > 0.f ? u : 1.f;
}

// What a row of a stored result is multiplied by.
__device__ __forceinline__ float factor_of(const float* dloss, const void* labels, bool wide, int64_t V,
                                           const uint32_t* top, int64_t row) {
    float f = top ? whole_size(top) : 1.f;
    if (dloss) f = row >= 0 && (!labels || load_id(labels, wide, row, V) >= 0) ? f * dloss[row] : 0.f;
    return f;
}

// exp(x - top)
__device__ __forceinline__ float exp_below(float x, float top) { return ex2((x - top) * kLog2e); }

// A token's results from its largest logit, the sum of exp below it and its label's logit.
// The largest and the label's are subtracted first: a label whose logit is the largest has
// a loss of log sum, 0 or more, whatever the logits' size (lse - hit would be off by half
// a step of lse, either way, where the loss is next to 0).  Differences before the factor
// log2 e cost an instruction a logit more than one fma: 0.3% of the forward at 2,048
// features, 3% at 64.
struct Result {
    float lse, loss;
    __device__ __forceinline__ Result(float top, float sum, float hit) {
        const float more = log2f(sum) * kLn2;
        lse = top + more;
        loss = (top - hit) + more;
    }
};

// The block of C, or of a part of a split sum, that a workgroup forms.  Each XCD takes
// a contiguous share of the blocks, those that are formed together close to each other
// in both directions.
struct Block {
    uint32_t m, n, split;
    // false: none
    __device__ __forceinline__ bool at(int64_t mt_, int64_t nt_, int splits) {
        const uint32_t mt = uint32_t(mt_), nt = uint32_t(nt_), each = mt * nt, total = each * uint32_t(splits);
        const uint32_t per = (total + kXcds - 1) / kXcds, i = blockIdx.x / kXcds;
        uint32_t t = blockIdx.x % kXcds * per + i;
        if (i >= per || t >= total) return false;
        split = t / each;
        t -= split * each;
        constexpr uint32_t G = 4;
        const uint32_t g = t / (G * mt), w = nt - g * G < G ? nt - g * G : G, r = t - g * G * mt;
        m = r / w;
        n = g * G + r % w;
        return true;
    }
};

// A lane's four values (consecutive columns of its row) of each lane of a quad, turned:
// lane k of the quad gets column k of the quad's rows, as two packed words.
__device__ __forceinline__ uint2 turn_quad(uint32_t lo, uint32_t hi, int lane) {
    const uint32_t lo1 = uint32_t(xor_lane<1>(int(lo))), hi1 = uint32_t(xor_lane<1>(int(hi)));
    // columns 0 and 2 of a pair of rows in its even lane, 1 and 3 in its odd one
    const bool odd = lane & 1;
    const uint32_t sel = odd ? 0x07060302u : 0x05040100u;
    const uint32_t x = __builtin_amdgcn_perm(odd ? lo : lo1, odd ? lo1 : lo, sel);
    const uint32_t y = __builtin_amdgcn_perm(odd ? hi : hi1, odd ? hi1 : hi, sel);
    const uint32_t got = uint32_t(xor_lane<2>(int(lane & 2 ? x : y)));
    return lane & 2 ? make_uint2(got, y) : make_uint2(x, got);
}

// 32 rows of C of one wavefront (its blocks j), through LDS, so that stores to memory
// are whole runs of a row.  put(i, q, v): the lane's four values of block i, columns
// 8 q + 4 (lane / 32) + 0..3; out(row of the 32, first column, 16 bytes' values).
template <typename O, int TM>
struct Rows32 {
    static constexpr int E = 16 / int(sizeof(O));
    static constexpr int kBlocks = sizeof(O) == 2 && TM > 1 ? 2 : 1;  // at a time: rows of at most 128 bytes
    static constexpr int kRow = kBlocks * 32 * int(sizeof(O)), kPieces = kRow / 16;
    static constexpr int kRounds = TM / kBlocks;

    // a row's pieces are permuted by its number, as in a stage
    __device__ __forceinline__ static char* place(char* lds, int row, int piece) {
        return lds + row * kRow + (piece ^ ((kPieces == 8 ? row >> 1 : row >> 2) & (kPieces - 1))) * 16;
    }
    template <typename Get, typename Out>
    __device__ __forceinline__ static void run(char* lds, int lane, const Get& get, const Out& out) {
        const int row = lane & 31, half = lane >> 5;
#pragma unroll
        for (int r = 0; r < kRounds; ++r) {
#pragma unroll
            for (int i = 0; i < kBlocks; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
                    get(r * kBlocks + i, q, v);
                    if constexpr (sizeof(O) == 2)
                        *reinterpret_cast<uint2*>(place(lds, row, 4 * i + q) + 8 * half) =
                            make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
                    else
                        *reinterpret_cast<float4*>(place(lds, row, 8 * i + 2 * q + half)) =
                            make_float4(v[0], v[1], v[2], v[3]);
                }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_wave_barrier();
            constexpr int rows = kWave / kPieces;
#pragma unroll
            for (int k = 0; k < 32; k += rows) {
                const int at = k + lane / kPieces, p = lane % kPieces;
                const uint4 x = *reinterpret_cast<const uint4*>(place(lds, at, p));
                out(at, r * kBlocks * 32 + p * E, x);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_wave_barrier();
        }
    }
};
constexpr int kRowsBytes = 4096;  // of LDS for a wavefront's rows

// 16 bytes of a row of which `room` elements are left, at any alignment
template <typename O>
__device__ __forceinline__ void store_room(O* p, const uint4& x, int64_t room) {
    typedef typename Piece<O>::type piece_t;
    constexpr int E = Piece<O>::E;
    if (room >= E) {
        const piece_t v = {x.x, x.y, x.z, x.w};
        *reinterpret_cast<piece_t*>(p) = v;
    } else {
        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < room) {
                if constexpr (sizeof(O) == 2) p[e] = O(w[e / 2] >> 16 * (e % 2));
                else p[e] = __uint_as_float(w[e]);
            }
    }
}

// Of the list's rows those from `first` on, `most` at most.
__device__ __forceinline__ int64_t left_of(const int32_t* count, int64_t first, int64_t most) {
    const int64_t n = int64_t(*count) - first;
    return n < 0 ? 0 : n < most ? n : most;
}

// The largest blocks hold 212 (bf16 logits) to 230 registers and none lies in scratch; the
// logits' keep 236 scalars in vector lanes (dL 60, dX and dW 14 at most): the masks of the
// labels' search and of the last block's classes, beside the exponentials.
template <typename T, int WHAT, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(WM * WN * 64) void k_product(LossArgs a) {
    using G = GemmNT<T, WM, WN, TM, TN>;
    // two objects: the compiler makes a read of one wait for loads into the same object
    __shared__ __attribute__((aligned(1024))) char s_0[G::kStage], s_1[G::kStage];
    static_assert(WM * WN * kRowsBytes <= G::kStage, "the wavefronts' rows fit");
    char* const s_out = s_0;
    const int64_t N = !a.n_count ? a.N : WHAT == kStats ? int64_t(*a.n_count) : left_of(a.n_count, a.first, a.N);
    constexpr int64_t kStep = kStepBytes / int64_t(sizeof(T));  // elements
    const int64_t steps =
        WHAT == kStore && a.k_count ? cdiv(left_of(a.k_count, a.first, a.steps * kStep), kStep) : a.steps;
    const int64_t each = cdiv(steps, a.splits);
    const int lane = lane_id(), wave = uniform(threadIdx.x / kWave), wm = wave % WM, wn = wave / WM;
    Block blk;
    if (!blk.at(cdiv(a.M, G::BM), cdiv(N, G::BN), a.splits)) return;
    const int64_t bm = blk.m, split = blk.split, m0 = bm * G::BM, n0 = int64_t(blk.n) * G::BN, s0 = split * each;
    const int64_t mw = m0 + wm * TM * 32, nw = n0 + wn * TN * 32;  // of the wavefront
    const int mh = 4 * (lane >> 5);  // the lane's classes: mw + mh + 32 i + 8 (e / 4) + e % 4
    const bool last = m0 + G::BM > a.M;
    G g;
    g.source(wave, lane, a.A, a.lda, m0, a.M, a.B, a.ldb, n0, N, a.gather ? a.list : nullptr, s0,
             s0 + each < steps ? s0 + each : steps);
    g.start(s_0, s_1, wave);
    // What the lane's tokens bring along, read beside the first steps' loads: the label's place
    // behind the wavefront's first class (-1 if it is not among its classes), whether
    // there is one at all, and the backward's statistics.
    int place[TN];
    bool labelled[TN];
    float lse[TN], up[TN];
    if constexpr (WHAT != kStore) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t t = nw + 32 * j + (lane & 31);
            const int64_t row = t < N ? (a.list ? int64_t(a.list[t]) : t) : -1;
            const int64_t id = row >= 0 ? load_id(a.labels, a.wide, row, a.V) : -1, at = id - a.v0 - mw;
            labelled[j] = id >= 0;
            place[j] = id >= 0 && at >= 0 && at < TM * 32 ? int(at) : -1;
            if constexpr (WHAT == kGrad) {
                lse[j] = id >= 0 ? a.lse_in[row] : 0.f;
                up[j] = id >= 0 && a.dlt ? a.dloss[row] / whole_size(a.top) : 0.f;
            }
        }
    }
    g.run(s_0, s_1, wave, lane);
    lds_barrier();  // the stages have been read
    if constexpr (WHAT == kStats) {
        // the largest product and the sum of exp of what lies below it; exponents go to base 2 as differences, so that
        // the largest term is 1 exactly
        float2* s_part = reinterpret_cast<float2*>(s_out);                // [WM][BN]
        float* s_hit = reinterpret_cast<float*>(s_out + WM * G::BN * 8);  // [BN], of one block of classes
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int c = wn * TN * 32 + 32 * j + (lane & 31);
            if (ballot(place[j] >= 0)) {  // few wavefronts hold any
                float hit = 0.f;
                bool mine = false;
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (place[j] == mh + 32 * i + 8 * (e / 4) + e % 4) hit = g.acc[i][j][e], mine = true;
                if (mine) (a.loss ? s_hit + c : a.hit + n0 + c)[0] = hit;
            }
            float top = kNegInf;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    if (last && mw + mh + 32 * i + 8 * (e / 4) + e % 4 >= a.M) g.acc[i][j][e] = kNegInf;
                    top = fmaxf(top, g.acc[i][j][e]);
                }
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            const float ref = top == kNegInf ? 0.f : top;
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum[e % 4] += exp_below(g.acc[i][j][e], ref);
            float all = (sum[0] + sum[1]) + (sum[2] + sum[3]);
            all += __shfl_xor(all, 32, kWave);
            if (lane < 32) s_part[wm * G::BN + c] = make_float2(top, all);
        }
        lds_barrier();
        for (int c = threadIdx.x; c < G::BN; c += G::kThreads) {
            const int64_t t = n0 + c;
            if (t >= N) break;
            float top = kNegInf, sum = 0.f;
#pragma unroll
            for (int w = 0; w < WM; ++w) top = fmaxf(top, s_part[w * G::BN + c].x);
            const float ref = top == kNegInf ? 0.f : top;
#pragma unroll
            for (int w = 0; w < WM; ++w) {
                const float2 p = s_part[w * G::BN + c];
                sum += p.y * exp_below(p.x, ref);
            }
            if (a.loss) {
                const int64_t row = a.list ? int64_t(a.list[t]) : t;
                const bool has = load_id(a.labels, a.wide, row, a.V) >= 0;
                const Result r(ref, sum, has ? s_hit[c] : 0.f);
                a.lse[row] = has ? r.lse : 0.f;
                a.loss[row] = has ? r.loss : 0.f;
            } else {
                reinterpret_cast<float2*>(a.part)[bm * a.part_ld + t] = make_float2(top, sum);
            }
        }
    } else {
        char* const lds = s_out + wave * kRowsBytes;
        if constexpr (WHAT == kGrad) {
            using R = Rows32<T, TM>;
            T* dl = static_cast<T*>(a.dl);
            T* dlt = static_cast<T*>(a.dlt);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int64_t t0 = nw + 32 * j;
                const bool label = ballot(place[j] >= 0);  // few wavefronts hold any
                const auto value = [&](int i, int q, float(&v)[4]) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = exp_below(g.acc[i][j][4 * q + e], lse[j]);
                        v[e] = labelled[j] ? p : 0.f;
                    }
                    if (label) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (place[j] == mh + 32 * i + 8 * q + e) v[e] -= 1.f;
                    }
                    if (last) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (mw + mh + 32 * i + 8 * q + e >= a.M) v[e] = 0.f;
                    }
                    if (dlt) {
                        T* o = dlt + (mw + mh + 32 * i + 8 * q) * a.dlt_ld + t0;
                        if constexpr (sizeof(T) == 2) {
                            const uint2 x = turn_quad(pack_bf16x2(v[0] * up[j], v[1] * up[j]),
                                                      pack_bf16x2(v[2] * up[j], v[3] * up[j]), lane);
                            *reinterpret_cast<uint2*>(o + (lane & 3) * a.dlt_ld + (lane & 28)) = x;
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[e * a.dlt_ld + (lane & 31)] = v[e] * up[j];
                        }
                    }
                };
                R::run(lds, lane, value, [&](int at, int m, const uint4& x) {
                    if (dl) *reinterpret_cast<uint4*>(dl + (t0 + at) * a.dl_ld + mw + m) = x;
                });
            }
        } else {
            const auto rows = [&](auto o, int j, float factor, const auto& out) {
                Rows32<decltype(o), TM>::run(
                    lds, lane,
                    [&](int i, int q, float(&v)[4]) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = g.acc[i][j][4 * q + e] * factor;
                    },
                    out);
            };
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                const int64_t t0 = nw + 32 * j;
                if (a.slots) {
                    float* o = a.slots + split * a.slot_rows * a.M;
                    rows(float(), j, 1.f, [&](int at, int m, uint4 x) {
                        const int64_t n = t0 + at, room = a.M - mw - m;
                        if (n >= N || room <= 0) return;
                        float* p = o + n * a.M + mw + m;
                        if (a.add) {
                            float v[4] = {__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z),
                                          __uint_as_float(x.w)};
                            if (room >= 4) {
                                float w[4];
                                load_piece(w, p);
#pragma unroll
                                for (int e = 0; e < 4; ++e) v[e] += w[e];
                            } else {
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (e < room) v[e] += p[e];
                            }
                            x = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                                           __float_as_uint(v[3]));
                        }
                        store_room(p, x, room);
                    });
                } else {
                    const int64_t n = t0 + (lane & 31);
                    const float factor = factor_of(a.dloss, a.labels, a.wide, a.V, a.top,
                                                   n < N ? (a.out_rows ? int64_t(a.out_rows[n]) : n) : -1);
                    rows(T(), j, factor, [&](int at, int m, const uint4& x) {
                        const int64_t n = t0 + at, room = a.M - mw - m;
                        if (n >= N || room <= 0) return;
                        const int64_t r = a.out_rows ? int64_t(a.out_rows[n]) : n;
                        store_room(static_cast<T*>(a.out) + r * a.M + mw + m, x, room);
                    });
                }
            }
        }
    }
}

// A token's statistics, taken on by U more parts.
template <int U>
__device__ __forceinline__ void join(float& top, float& sum, const float2 (&p)[U]) {
    float m = top;
#pragma unroll
    for (int k = 0; k < U; ++k) m = fmaxf(m, p[k].x);
    const float ref = m == kNegInf ? 0.f : m;
    sum *= exp_below(top, ref);
#pragma unroll
    for (int k = 0; k < U; ++k) sum += p[k].y * exp_below(p[k].x, ref);
    top = m;
}
struct Joined {
    const float* hit;
    const void* labels;
    bool wide;
    int64_t V;
    const int32_t* list;
    float *loss, *lse;
    __device__ __forceinline__ void put(int64_t t, float top, float sum) const {
        const int64_t i = list ? int64_t(list[t]) : t;
        const bool has = load_id(labels, wide, i, V) >= 0;
        const Result r(top == kNegInf ? 0.f : top, sum, has ? hit[t] : 0.f);
        lse[i] = has ? r.lse : 0.f;
        loss[i] = has ? r.loss : 0.f;
    }
};

// The parts of a token's statistics, joined.  Of a few blocks of classes: a lane a token
// (60,000 tokens of three blocks 5 us, by 64 lanes each 24).
__global__ __launch_bounds__(256) void k_loss_few(int blocks, const float2* part, int64_t ld, const int32_t* count,
                                                  int64_t n, Joined j) {
    if (count) n = *count;
    for (int64_t t = int64_t(blockIdx.x) * 256 + threadIdx.x; t < n; t += int64_t(gridDim.x) * 256) {
        float top = kNegInf, sum = 0.f;
        for (int b = 0; b < blocks; ++b) {
            const float2 p[1] = {part[b * ld + t]};
            join(top, sum, p);
        }
        j.put(t, top, sum);
    }
}

// Of more: 64 lanes take a token's blocks in turn, four at a time.
__global__ __launch_bounds__(1024) void k_loss(int64_t blocks, const float2* part, int64_t ld, const int32_t* count,
                                                int64_t n, Joined j) {
    constexpr int P = 16, G = 1024 / P;  // tokens of a workgroup
    __shared__ float2 s[G][P + 1];
    const int x = threadIdx.x % P, y = threadIdx.x / P;
    if (count) n = *count;
    for (int64_t t0 = int64_t(blockIdx.x) * P; t0 < n; t0 += int64_t(gridDim.x) * P) {
        float top = kNegInf, sum = 0.f;
        if (t0 + x < n)
            for (int64_t b = y; b < blocks; b += 4 * G) {
                float2 p[4];
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    p[k] = b + k * G < blocks ? part[(b + k * G) * ld + t0 + x] : make_float2(kNegInf, 0.f);
                join(top, sum, p);
            }
        s[y][x] = make_float2(top, sum);
        __syncthreads();
        if (y < P) {  // turned: a wavefront's 16 lanes of a token take its 64 sums
            top = kNegInf;
            float2 p[G / P];
#pragma unroll
            for (int k = 0; k < G / P; ++k) p[k] = s[x + P * k][y], top = fmaxf(top, p[k].x);
#pragma unroll
            for (int o = 1; o < P; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
            const float ref = top == kNegInf ? 0.f : top;
            sum = 0.f;
#pragma unroll
            for (int k = 0; k < G / P; ++k) sum += p[k].y * exp_below(p[k].x, ref);
#pragma unroll
            for (int o = 1; o < P; o <<= 1) sum += __shfl_xor(sum, o, kWave);
            if (x == 0 && t0 + y < n) j.put(t0 + y, top, sum);
        }
        __syncthreads();
    }
}

// out[row][c] = the sum of the slots, four columns a lane where rows are whole such;
// the slots go by over L lanes.
struct Factors {
    const float* dloss;
    const void* labels;
    bool wide;
    int64_t V;
    const uint32_t* top;
    __device__ __forceinline__ float of(int64_t row) const { return factor_of(dloss, labels, wide, V, top, row); }
};
template <typename T, int L>
__global__ __launch_bounds__(256) void k_sum_slots(int splits, int64_t slot_rows, int64_t R, const int32_t* count,
                                                    int64_t C, const float* slots, const int32_t* rows, T* out,
                                                    Factors f) {
    constexpr int P = 256 / L;
    __shared__ float4 s[L][P];
    if (count) R = *count;
    const int64_t total = R * C, each = slot_rows * C;
    const int x = threadIdx.x % P, y = threadIdx.x / P;
    for (int64_t i0 = int64_t(blockIdx.x) * P * 4; i0 < total; i0 += int64_t(gridDim.x) * P * 4) {
        const int64_t i = i0 + 4 * x, room = total - i;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (room >= 4) {
#pragma unroll 4
            for (int k = y; k < splits; k += L) {
                float w[4];
                load_piece(w, slots + k * each + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += w[e];
            }
        } else if (room > 0) {
            for (int k = y; k < splits; k += L)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < room) v[e] += slots[k * each + i + e];
        }
        if constexpr (L > 1) {
            s[y][x] = make_float4(v[0], v[1], v[2], v[3]);
            __syncthreads();
            if (y == 0) {
#pragma unroll
                for (int k = 1; k < L; ++k) {
                    const float4 w = s[k][x];
                    v[0] += w.x, v[1] += w.y, v[2] += w.z, v[3] += w.w;
                }
            }
            __syncthreads();
        }
        if (y) continue;
        const int64_t r = i / C;
        if (room >= 4 && (i + 3) / C == r) {
            const float by = f.of(rows ? int64_t(rows[r]) : r);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] *= by;
            T* o = rows ? out + int64_t(rows[r]) * C + (i - r * C) : out + i;
            if constexpr (sizeof(T) == 2) {
                typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
                const u2 p = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                *reinterpret_cast<u2*>(o) = p;
            } else {
                store_piece(o, v, false);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < room) {
                    const int64_t re = (i + e) / C;
                    const int64_t row = rows ? int64_t(rows[re]) : re;
                    store_one(out + row * C + (i + e - re * C), v[e] * f.of(row));
                }
        }
    }
}

// How a product is cut: rows of A and of B a block, and parts of the sum.
struct Cut {
    int m, n, splits;
};

template <typename T, int WHAT>
gt_status product(const LossArgs& a, const Cut& cut, hipStream_t s) {
#define GT_CALL(WM, WN, TM, TN)                                                                       \
    do {                                                                                              \
        using G = GemmNT<T, WM, WN, TM, TN>;                                                          \
        const unsigned blocks = xcd_grid(cdiv(a.M, G::BM) * cdiv(a.N, G::BN) * a.splits);             \
        k_product<T, WHAT, WM, WN, TM, TN><<<blocks, G::kThreads, 0, s>>>(a);                         \
    } while (0)
    if (cut.m == 64) {
        if (cut.n == 64) GT_CALL(2, 2, 1, 1);
        else GT_CALL(2, 4, 1, 2);
    } else if (cut.m == 128) {
        GT_CALL(2, 2, 2, 2);
    } else {
        if (cut.n == 64) GT_CALL(4, 1, 2, 2);
        else GT_CALL(2, 4, 4, 2);
    }
#undef GT_CALL
    GT_LAUNCH_CHECK("class_loss product");
    return GT_OK;
}

// A block shape's microseconds: what a block takes beside its steps, a step of a block
// that has its CU to itself and of one that shares it with as many as fit, in bf16 and
// fp32.  Logits are measured at 200 to 8,192 rows, classes and features.  The sums over
// classes and tokens, whose operands come from beyond L2, have a table of their own,
// fitted to every shape's times at 48 sizes (100 to 300,000 rows, 30 to 150,000 classes,
// 50 to 4,000 features; half of them held back from a first fit).  What the two choose
// takes 1.03 times (fp32 1.02) the time of the best shape at these sizes, for logits and
// for the sums; 256 x 256 wherever both sides pass 64, 1.35 (1.85) and 1.33 (1.65).
struct Times {
    float fixed, lone[2], full[2];
};
struct Side {
    int m, n, fit;
    Times logits, sum;
};
constexpr Side kSides[] = {
    {256, 256, 1, {10.6f, {1.09f, 7.17f}, {1.62f, 7.34f}}, {7.0f, {1.6f, 7.3f}, {1.6f, 7.3f}}},
    {128, 128, 2, {6.7f, {0.43f, 1.86f}, {0.44f, 1.88f}}, {5.5f, {0.78f, 1.9f}, {0.54f, 1.9f}}},
    {256, 64, 2, {6.3f, {0.48f, 1.93f}, {0.52f, 1.94f}}, {5.1f, {0.89f, 2.0f}, {0.57f, 1.9f}}},
    {64, 256, 2, {4.8f, {0.43f, 1.79f}, {0.57f, 1.89f}}, {4.9f, {0.81f, 2.0f}, {0.61f, 1.9f}}},
    {64, 64, 5, {4.2f, {0.21f, 0.48f}, {0.17f, 0.52f}}, {3.6f, {0.52f, 0.63f}, {0.21f, 0.53f}}},
};

// The shape of the least time by that table, and for the sums the parts: as many as fill
// the chip once, or as many as its CUs hold.  A product of few large blocks would leave
// CUs idle: fp32 logits of 3,447 x 214 classes x 924, 14 blocks of 256 x 256, 218 us, in
// blocks of 64 x 64 19; 1,118 x 1,596 x 960 227 and 37; but 8,192 x 8,192 x 1,024 970 and
// 1,119, in bf16 147 and 226.  Logits of up to 64 tokens are bound by the class weights'
// loads, of which small blocks have more on the way (16 x 1,024 over 128,000 classes in
// bf16 68 us, 256 x 64 77); one block of up to 256 classes needs no join (2 x 896 over 213
// in bf16 13 us, four and a join 17).
Cut cut_of(What what, int64_t M, int64_t N, int64_t steps, int size) {
    const bool split = what == kStore;
    Cut best = {M <= 64 ? 64 : 256, N <= 64 ? 64 : 256, 1};
    if (!split && N <= 64 && M > 256) return {64, 64, 1};
    const int f = size == 2 ? 0 : 1;
    double least = 1e30;
    for (const Side& c : kSides) {
        const int64_t blocks = cdiv(M, c.m) * cdiv(N, c.n);
        if (blocks > kCutBlocks) continue;
        const Times& t = split ? c.sum : c.logits;
        for (int full = 0; full <= (split && c.fit > 1 ? 1 : 0); ++full) {
            int64_t s = split ? kSplitBlocks * (full ? c.fit : 1) / blocks : 1;
            if (s > steps / kSplitSteps) s = steps / kSplitSteps;
            if (s < 1) s = 1;
            const double k = double(cdiv(blocks * s, kSplitBlocks)), n = double(cdiv(steps, s));
            const double lone = double(cdiv(int64_t(k), c.fit)) * (t.fixed + n * t.lone[f]);
            const double shared = k * (t.fixed / c.fit + n * t.full[f]);
            double time = lone > shared ? lone : shared;
            if (what == kStats && M > c.m) time += 7 + double(cdiv(M, c.m)) * double(N) / kParts;  // the join
            if (s > 1) time += 2 + double(s) * double(M) * double(N) * 4 / kSlotBytes;  // the parts' sum
            if (time < least) least = time, best = {c.m, c.n, int(s)};
        }
    }
    return best;
}

// ----------------------------------------------------------------- workspace

struct Shape {
    int64_t n, V, ldx, ldw;
    int D, size;
    bool whole_x, copy_x, copy_w;
    int64_t row;   // bytes of a padded row
    int64_t mp;    // tokens, whole blocks
    int64_t ldt;   // row stride of X laid out along the tokens
    int64_t piece, ldp;  // classes a piece, row stride of the arrays along them
    int64_t held;        // classes of a piece in whole blocks
    int64_t rows, ldr;   // tokens a piece (whole blocks), row stride of dL along them
    Cut logits, grad, dx, dw;
    bool slots_x, slots_w;
};

Shape shape_of(int64_t n, int64_t V, int32_t D, gt_dtype dt, int64_t ldx, int64_t ldw) {
    Shape h = {};
    h.n = n, h.V = V, h.D = D, h.ldx = ldx, h.ldw = ldw;
    h.size = dt == GT_BF16 ? 2 : 4;
    h.row = cdiv(int64_t(D) * h.size, kStepBytes) * kStepBytes;
    const bool whole = h.row == int64_t(D) * h.size;
    h.whole_x = whole && ldx * h.size % 16 == 0;
    h.copy_w = !whole || ldw * h.size % 16 != 0;
    h.copy_x = !h.whole_x || (n > kListed && V > kGatherClasses);
    h.mp = cdiv(n, 256) * 256;
    h.ldt = h.mp + kOff;
    int64_t piece = kPieceBytes / (h.mp * h.size) / 256 * 256;
    if (piece < kMinPiece) piece = kMinPiece;
    h.piece = piece < V ? piece : V;
    // rows of a piece: all that fit, or equal parts
    const int64_t most = kPartBytes / (cdiv(h.piece, 64) * 64 * h.size);
    h.rows = h.mp <= most ? h.mp : cdiv(cdiv(n, cdiv(n, most)), 256) * 256;
    h.ldr = h.rows + kOff;
    const int64_t rows = h.rows < n ? h.rows : n;
    h.logits = cut_of(kStats, V, n, h.row / kStepBytes, h.size);
    h.grad = cut_of(kGrad, h.piece, rows, h.row / kStepBytes, h.size);
    h.dx = cut_of(kStore, D, rows, cdiv(h.piece * h.size, kStepBytes), h.size);
    h.dw = cut_of(kStore, D, h.piece, h.rows * h.size / kStepBytes, h.size);
    h.held = cdiv(h.piece, h.grad.m) * h.grad.m;
    h.ldp = h.held + (h.held * h.size < kOffBytes ? 0 : kOff);
    h.slots_x = h.dx.splits > 1 || h.piece < V;
    h.slots_w = h.dw.splits > 1 || h.rows < n;
    return h;
}

struct List {
    int32_t *list, *count, *cnt;
    uint32_t* top;  // the largest |dloss|
};
List list_ws(Ws& w, int64_t n) {
    List l;
    l.list = w.take<int32_t>(size_t(n));
    l.count = w.take<int32_t>(1);
    l.cnt = w.take<int32_t>(size_t(cdiv(n, kListRows)));
    l.top = w.take<uint32_t>(1);
    return l;
}

struct FwdWs {
    List l;
    char *x, *w;
    float *part, *hit;
};
FwdWs fwd_ws(Ws& w, const Shape& h) {
    FwdWs f;
    f.l = list_ws(w, h.n);
    f.x = h.copy_x ? w.take<char>(size_t(h.n * h.row)) : nullptr;
    f.w = h.copy_w ? w.take<char>(size_t(h.V * h.row)) : nullptr;
    f.part = w.take<float>(size_t(2 * h.mp * cdiv(h.V, h.logits.m)));
    f.hit = w.take<float>(size_t(h.n));
    return f;
}

struct BwdWs {
    List l;
    char *x, *w, *xt, *wt, *dl, *dlt;
    float *slots_x, *slots_w;
};
BwdWs bwd_ws(Ws& w, const Shape& h) {
    BwdWs b;
    b.l = list_ws(w, h.n);
    b.x = h.copy_x ? w.take<char>(size_t(h.n * h.row)) : nullptr;
    b.w = h.copy_w ? w.take<char>(size_t(h.V * h.row)) : nullptr;
    b.xt = w.take<char>(size_t(h.D) * size_t(h.ldt * h.size));
    b.wt = w.take<char>(size_t(h.D) * size_t(h.ldp * h.size));
    b.dl = w.take<char>(size_t(h.rows) * size_t(h.ldp * h.size));
    b.dlt = w.take<char>(size_t(h.held) * size_t(h.ldr * h.size));
    b.slots_x = h.slots_x ? w.take<float>(size_t(h.dx.splits) * size_t(h.n) * h.D) : nullptr;
    b.slots_w = h.slots_w ? w.take<float>(size_t(h.dw.splits) * size_t(h.piece) * h.D) : nullptr;
    return b;
}

gt_status make_list(const Shape& h, bool wide, const void* labels, List& l, float* loss, float* lse, const float* dloss,
                    hipStream_t s) {
    if (h.n <= kListed) {
        l.list = l.count = nullptr;
        return GT_OK;
    }
    const unsigned blocks = unsigned(cdiv(h.n, kListRows));
    if (blocks > 1) {
        k_list_count<<<blocks, kListThreads, 0, s>>>(h.n, h.V, wide, labels, l.cnt, dloss ? l.top : nullptr);
        GT_LAUNCH_CHECK("class_loss count");
    }
    k_list_place<<<blocks, kListThreads, 0, s>>>(h.n, h.V, wide, labels, l.cnt, l.list, l.count, loss, lse, dloss,
                                                   dloss ? l.top : nullptr);
    GT_LAUNCH_CHECK("class_loss list");
    return GT_OK;
}

// X and W as the products take them; a copy of X has the listed rows alone, in order
template <typename T>
gt_status make_rows(const Shape& h, const List& l, const void*& X, int64_t& ldx, char* x, const void*& W, int64_t& ldw,
                    char* w, hipStream_t s) {
    const int ldd = int(h.row / h.size);
    if (h.copy_x) {
        k_pad<T><<<grid_for(h.n, 4, 1 << 16), 256, 0, s>>>(h.n, l.list, l.count, h.D, static_cast<const T*>(X), ldx,
                                                           reinterpret_cast<T*>(x), ldd, h.whole_x);
        GT_LAUNCH_CHECK("class_loss rows");
        X = x, ldx = ldd;
    }
    if (h.copy_w) {
        k_pad<T><<<grid_for(h.V, 4, 1 << 16), 256, 0, s>>>(h.V, nullptr, nullptr, h.D, static_cast<const T*>(W), ldw,
                                                           reinterpret_cast<T*>(w), ldd, false);
        GT_LAUNCH_CHECK("class_loss rows");
        W = w, ldw = ldd;
    }
    return GT_OK;
}

template <typename T>
gt_status run_fwd(const Shape& h, const void* X, const void* W, bool wide, const void* labels, float* loss, float* lse,
                  FwdWs f, hipStream_t s) {
    gt_status st = make_list(h, wide, labels, f.l, loss, lse, nullptr, s);
    if (st != GT_OK) return st;
    int64_t ldx = h.ldx, ldw = h.ldw;
    st = make_rows<T>(h, f.l, X, ldx, f.x, W, ldw, f.w, s);
    if (st != GT_OK) return st;
    const int64_t side = h.logits.m, blocks = cdiv(h.V, side);
    LossArgs a = {};
    a.lda = ldw * h.size;
    a.B = static_cast<const char*>(X), a.ldb = ldx * h.size, a.N = h.n;
    a.n_count = f.l.count, a.list = f.l.list, a.gather = !h.copy_x;
    a.steps = h.row / kStepBytes, a.splits = 1;
    a.V = h.V, a.labels = labels, a.wide = wide;
    if (blocks == 1) a.loss = loss, a.lse = lse;
    else a.part_ld = h.mp, a.hit = f.hit;
    // as many classes as a launch takes
    const int64_t piece = side * (kLaunchBlocks / cdiv(h.n, h.logits.n));
    for (int64_t v0 = 0; v0 < h.V; v0 += piece) {
        a.A = static_cast<const char*>(W) + v0 * a.lda;
        a.M = h.V - v0 < piece ? h.V - v0 : piece;
        a.v0 = v0;
        a.part = f.part + 2 * (v0 / side) * h.mp;
        st = product<T, kStats>(a, h.logits, s);
        if (st != GT_OK) return st;
    }
    if (blocks == 1) return GT_OK;
    const Joined j = {f.hit, labels, wide, h.V, f.l.list, loss, lse};
    const float2* part = reinterpret_cast<float2*>(f.part);
    if (blocks <= kFewBlocks)
        k_loss_few<<<grid_for(h.n, 256, 1 << 16), 256, 0, s>>>(int(blocks), part, h.mp, f.l.count, h.n, j);
    else
        k_loss<<<grid_for(h.n, 16, 1 << 16), 1024, 0, s>>>(blocks, part, h.mp, f.l.count, h.n, j);
    GT_LAUNCH_CHECK("class_loss join");
    return GT_OK;
}

template <typename T>
gt_status sum_slots(int splits, int64_t slot_rows, int64_t R, const int32_t* count, int64_t C, const float* slots,
                    const int32_t* rows, T* out, const LossArgs& a, hipStream_t s) {
    const Factors f = {a.dloss, a.labels, a.wide, a.V, a.top};
    if (splits > 4)
        k_sum_slots<T, 8><<<grid_for(R * C, 128, 1 << 16), 256, 0, s>>>(splits, slot_rows, R, count, C, slots, rows,
                                                                        out, f);
    else
        k_sum_slots<T, 1><<<grid_for(R * C, 1024, 1 << 16), 256, 0, s>>>(splits, slot_rows, R, count, C, slots, rows,
                                                                        out, f);
    GT_LAUNCH_CHECK("class_loss sum");
    return GT_OK;
}

template <typename T>
gt_status run_bwd(const Shape& h, const void* X, const void* W, bool wide, const void* labels, const float* lse,
                  const float* dloss, void* dX, void* dW, BwdWs b, hipStream_t s) {
    if (h.n == 0) {
        k_zero<T><<<grid_for(h.V * h.D, 256, 1 << 16), 256, 0, s>>>(h.V * h.D, static_cast<T*>(dW));
        GT_LAUNCH_CHECK("class_loss zero");
        return GT_OK;
    }
    gt_status st = make_list(h, wide, labels, b.l, nullptr, nullptr, dW ? dloss : nullptr, s);
    if (st != GT_OK) return st;
    int64_t ldx = h.ldx, ldw = h.ldw;
    st = make_rows<T>(h, b.l, X, ldx, b.x, W, ldw, b.w, s);
    if (st != GT_OK) return st;
    if (dX && b.l.list) {
        int shift = 0;
        while (shift < 6 && (Piece<T>::E << shift) < h.D) ++shift;
        const int span = h.n >= 65536 ? 64 : 8;
        k_zero_rows<T><<<grid_for(h.n, 4 * span, 1 << 16), 256, 0, s>>>(
            h.n, h.D, h.V, wide, labels, static_cast<T*>(dX), shift, span, h.n * h.D * h.size > kFarBytes);
        GT_LAUNCH_CHECK("class_loss zero rows");
    }
    LossArgs last_x = {};
    for (int64_t v0 = 0; v0 < h.V; v0 += h.piece) {
        const int64_t vn = h.V - v0 < h.piece ? h.V - v0 : h.piece;
        const char* w = static_cast<const char*>(W) + v0 * ldw * h.size;
        Turns turns = {};
        int jobs = 0;
        int64_t most = 0;
        if (dX) {
            turns.t[jobs++] = {vn, nullptr, nullptr, nullptr, false, 0, w, ldw, b.wt, h.ldp};
            most = vn;
        }
        if (dW && v0 == 0) {
            if (!b.l.list) turns.dloss = dloss, turns.top = b.l.top;
            turns.t[jobs++] = {h.n, b.l.count, h.copy_x ? nullptr : b.l.list, b.l.list ? nullptr : labels,
                               wide, h.V, X, ldx, b.xt, h.ldt};
            most = most > h.n ? most : h.n;
        }
        if (jobs) {
            k_turn<T><<<dim3(unsigned(cdiv(most, 64)), unsigned(cdiv(h.D, 64)), unsigned(jobs)), 256, 0, s>>>(
                turns, h.D);
            GT_LAUNCH_CHECK("class_loss turn");
        }
        LossArgs last_w = {};
        T* out = dW ? static_cast<T*>(dW) + v0 * h.D : nullptr;
        for (int64_t r0 = 0; r0 < h.n; r0 += h.rows) {
            const int64_t rn = h.n - r0 < h.rows ? h.n - r0 : h.rows;
            const int32_t* list = b.l.list ? b.l.list + r0 : nullptr;
            LossArgs a = {};
            a.A = w, a.lda = ldw * h.size, a.M = vn;
            a.B = static_cast<const char*>(X) + (h.copy_x ? r0 * ldx * h.size : 0), a.ldb = ldx * h.size, a.N = rn;
            a.n_count = b.l.count, a.first = r0, a.list = list, a.gather = !h.copy_x;
            a.steps = h.row / kStepBytes, a.splits = 1;
            a.v0 = v0, a.V = h.V, a.labels = labels, a.wide = wide, a.lse_in = lse, a.dloss = dloss;
            a.dl = dX ? b.dl : nullptr, a.dl_ld = h.ldp;
            a.dlt = dW ? b.dlt : nullptr, a.dlt_ld = h.ldr, a.top = b.l.top;
            st = product<T, kGrad>(a, h.grad, s);
            if (st != GT_OK) return st;
            if (dX) {
                LossArgs x = {};
                x.A = b.wt, x.lda = h.ldp * h.size, x.M = h.D;
                x.B = b.dl, x.ldb = h.ldp * h.size, x.N = rn, x.n_count = b.l.count, x.first = r0;
                x.steps = cdiv(vn * h.size, kStepBytes), x.splits = h.dx.splits;
                x.slots = b.slots_x ? b.slots_x + r0 * h.D : nullptr, x.slot_rows = h.n, x.add = v0 > 0;
                x.out = dX, x.out_rows = list;
                x.dloss = dloss, x.labels = list ? nullptr : labels, x.wide = wide, x.V = h.V;
                last_x = x;
                st = product<T, kStore>(x, h.dx, s);
                if (st != GT_OK) return st;
            }
            if (dW) {
                LossArgs x = {};
                x.A = b.xt + r0 * h.size, x.lda = h.ldt * h.size, x.M = h.D;
                x.B = b.dlt, x.ldb = h.ldr * h.size, x.N = vn;
                x.steps = cdiv(rn * h.size, kStepBytes), x.k_count = b.l.count, x.first = r0, x.splits = h.dw.splits;
                x.slots = b.slots_w, x.slot_rows = h.piece, x.add = r0 > 0;
                x.out = out, x.top = b.l.top;
                last_w = x;
                st = product<T, kStore>(x, h.dw, s);
                if (st != GT_OK) return st;
            }
        }
        if (dW && b.slots_w) {
            st = sum_slots<T>(h.dw.splits, h.piece, vn, nullptr, h.D, b.slots_w, nullptr, out, last_w, s);
            if (st != GT_OK) return st;
        }
    }
    if (dX && b.slots_x)
        return sum_slots<T>(h.dx.splits, h.n, h.n, b.l.count, h.D, b.slots_x, b.l.list, static_cast<T*>(dX), last_x, s);
    return GT_OK;
}

bool loss_sizes(int64_t n, int64_t V, int32_t D, gt_dtype dt, int64_t ldx, int64_t ldw) {
    const int64_t most = int64_t(1) << 31;
    return (dt == GT_BF16 || dt == GT_F32) && n >= 0 && n < most / 8 && V >= 1 && V < most && D >= 1 &&
           D <= GT_MAX_WIDTH && ldx >= D && ldw >= D && ldx < most && ldw < most;
}
gt_status loss_check(const char* who, int64_t n, int64_t V, int32_t D, gt_dtype dt, gt_itype it, const void* X,
                     int64_t ldx, const void* W, int64_t ldw, const void* labels) {
    const std::string w(who);
    if ((dt != GT_BF16 && dt != GT_F32) || (it != GT_I32 && it != GT_I64))
        return fail(GT_ERR_UNSUPPORTED, w + ": unsupported dtype");
    if (!loss_sizes(n, V, D, dt, ldx, ldw)) return fail(GT_ERR_INVALID_ARG, w + ": n, V, D or a stride out of range");
    if (n > 0 && (!X || !W || !labels)) return fail(GT_ERR_INVALID_ARG, w + ": null pointer");
    if ((reinterpret_cast<uintptr_t>(X) | reinterpret_cast<uintptr_t>(W)) & 15)
        return fail(GT_ERR_UNSUPPORTED, w + ": X and W must start at multiples of 16 bytes");
    return GT_OK;
}

}  // namespace

extern "C" size_t gt_class_loss_fwd_workspace_size(int64_t n, int64_t V, int32_t D, gt_dtype dt, int64_t ldx,
                                                   int64_t ldw) {
    if (!loss_sizes(n, V, D, dt, ldx, ldw)) return 0;
    if (n == 0) return 256;
    Ws w(nullptr);
    fwd_ws(w, shape_of(n, V, D, dt, ldx, ldw));
    return w.size();
}

extern "C" gt_status gt_class_loss_fwd(int64_t n, int64_t V, int32_t D, gt_dtype dt, gt_itype it, const void* X,
                                       int64_t ldx, const void* W, int64_t ldw, const void* labels, float* loss,
                                       float* lse, void* ws, size_t ws_bytes, hipStream_t s) {
    const gt_status st = loss_check("gt_class_loss_fwd", n, V, D, dt, it, X, ldx, W, ldw, labels);
    if (st != GT_OK) return st;
    if (n == 0) return GT_OK;
    if (!loss || !lse || !ws) return fail(GT_ERR_INVALID_ARG, "gt_class_loss_fwd: null pointer");
    if (ws_bytes < gt_class_loss_fwd_workspace_size(n, V, D, dt, ldx, ldw))
        return fail(GT_ERR_WORKSPACE, "gt_class_loss_fwd: workspace too small");
    const Shape h = shape_of(n, V, D, dt, ldx, ldw);
    Ws w(ws);
    const FwdWs f = fwd_ws(w, h);
    if (dt == GT_BF16) return run_fwd<uint16_t>(h, X, W, it == GT_I64, labels, loss, lse, f, s);
    return run_fwd<float>(h, X, W, it == GT_I64, labels, loss, lse, f, s);
}

extern "C" size_t gt_class_loss_bwd_workspace_size(int64_t n, int64_t V, int32_t D, gt_dtype dt, int64_t ldx,
                                                   int64_t ldw) {
    if (!loss_sizes(n, V, D, dt, ldx, ldw)) return 0;
    if (n == 0) return 256;
    Ws w(nullptr);
    bwd_ws(w, shape_of(n, V, D, dt, ldx, ldw));
    return w.size();
}

extern "C" gt_status gt_class_loss_bwd(int64_t n, int64_t V, int32_t D, gt_dtype dt, gt_itype it, const void* X,
                                       int64_t ldx, const void* W, int64_t ldw, const void* labels, const float* lse,
                                       const float* dloss, void* dX, void* dW, void* ws, size_t ws_bytes,
                                       hipStream_t s) {
    const gt_status st = loss_check("gt_class_loss_bwd", n, V, D, dt, it, X, ldx, W, ldw, labels);
    if (st != GT_OK) return st;
    if (n > 0 && (!lse || !dloss)) return fail(GT_ERR_INVALID_ARG, "gt_class_loss_bwd: null pointer");
    if (!dX && !dW) return GT_OK;
    if (n == 0 && !dW) return GT_OK;
    if (!ws) return fail(GT_ERR_INVALID_ARG, "gt_class_loss_bwd: null pointer");
    if (ws_bytes < gt_class_loss_bwd_workspace_size(n, V, D, dt, ldx, ldw))
        return fail(GT_ERR_WORKSPACE, "gt_class_loss_bwd: workspace too small");
    Shape h = {};
    BwdWs b = {};
    if (n > 0) {
        h = shape_of(n, V, D, dt, ldx, ldw);
        Ws w(ws);
        b = bwd_ws(w, h);
    } else {
        h.V = V, h.D = D;
    }
    if (dt == GT_BF16) return run_bwd<uint16_t>(h, X, W, it == GT_I64, labels, lse, dloss, dX, dW, b, s);
    return run_bwd<float>(h, X, W, it == GT_I64, labels, lse, dloss, dX, dW, b, s);
}
