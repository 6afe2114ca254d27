// Softmax cross entropy over many classes, straight from the features and the class
// weights, and its gradients; the logits are never kept.
//
//   s_iv = <X_i, W_v>,  lse_i = log sum_v exp s_iv,  loss_i = lse_i - s_i,y(i),
//   dL_iv = dloss_i (exp(s_iv - lse_i) - [v = y(i)]),  dX = dL W,  dW = dL^T X.
//
// Rows without a label take no part: the labelled rows are listed first (on the
// device, in order), and every product runs over the list.
//
// Forward: the product s with the classes as its rows, so that a lane holds one
// token and a block's classes: the block leaves (max, sum of exp) for each of its
// tokens, and one small kernel joins the blocks of a token.
// Backward: the classes go by in pieces.  A piece's s is formed again, dL is rounded
// to the features' type and written both ways round, and two products give the
// piece's dW and its part of dX, which is summed in fp32 over the pieces.  W and X
// are laid out the other way round for these, so that one product serves for all.
// Where a product has few blocks its sum is split over the grid and the parts are
// added in order.  No atomics: results are the same run to run.
#include "gemm_nt.h"
#include "rows.h"

using namespace gt;

namespace {

constexpr int kListThreads = 1024, kListRounds = 8, kListRows = kListThreads * kListRounds;
constexpr int64_t kPieceBytes = int64_t(256) << 20;  // of dL, one way round: the last-level cache
constexpr int64_t kMinPiece = 1024;                  // classes
constexpr int kSplitBlocks = 256;                    // blocks that fill the chip
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
                                                              int32_t* cnt) {
    __shared__ int s_n[kListThreads / kWave];
    const int c = wave_sum(__popc(labelled(labels, wide, n, V)));
    if (lane_id() == 0) s_n[threadIdx.x / kWave] = c;
    __syncthreads();
    if (threadIdx.x == 0) {
        int t = 0;
        for (int w = 0; w < kListThreads / kWave; ++w) t += s_n[w];
        cnt[blockIdx.x] = t;
    }
}

// The list, and what a row without a label has in the forward's results.
__global__ __launch_bounds__(kListThreads) void k_list_place(int64_t n, int64_t V, bool wide, const void* labels,
                                                              const int32_t* cnt, int32_t* list, int32_t* count,
                                                              float* loss, float* lse) {
    constexpr int W = kListThreads / kWave;
    __shared__ int s_n[kListRounds * W], s_before[W];
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
    if (lane == 0) s_before[wave] = before;
    __syncthreads();
    if (threadIdx.x == 0) {
        int t = 0;
        for (int w = 0; w < W; ++w) t += s_before[w];
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

// Rows without a label have no gradient.
template <typename T>
__global__ __launch_bounds__(256) void k_zero_rows(int64_t n, int D, int64_t V, bool wide, const void* labels, T* dx) {
    for (int64_t i = int64_t(blockIdx.x) * 4 + threadIdx.x / kWave; i < n; i += int64_t(gridDim.x) * 4) {
        if (load_id(labels, wide, i, V) >= 0) continue;
        for (int c = lane_id(); c < D; c += kWave) dx[i * D + c] = T(0);
    }
}
template <typename T>
__global__ __launch_bounds__(256) void k_zero(int64_t n, T* p) {
    for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < n; i += int64_t(gridDim.x) * 256) p[i] = T(0);
}

// ------------------------------------------------------------------ layouts

// dst[r][0 .. ldd) = src[r][0 .. C), zeros behind
template <typename T>
__global__ __launch_bounds__(256) void k_pad(int64_t R, int C, const T* src, int64_t lds, T* dst, int ldd) {
    for (int64_t r = int64_t(blockIdx.x) * 4 + threadIdx.x / kWave; r < R; r += int64_t(gridDim.x) * 4)
        for (int c = lane_id(); c < ldd; c += kWave) dst[r * ldd + c] = c < C ? src[r * lds + c] : T(0);
}

// dst[c][r] = src[r][c], for r < R; zeros for R <= r < R rounded up to 64
template <typename T>
__global__ __launch_bounds__(256) void k_turn(int64_t R, const int32_t* count, const int32_t* list, int C,
                                               const T* src, int64_t lds, T* dst, int64_t ldd) {
    __shared__ T s[64][65 + (sizeof(T) == 2)];
    if (count) R = *count;
    const int64_t r0 = int64_t(blockIdx.x) * 64;
    if (r0 >= R) return;
    const int c0 = blockIdx.y * 64, x = threadIdx.x % 64, y = threadIdx.x / 64;
#pragma unroll
    for (int k = 0; k < 64; k += 4) {
        const int64_t r = r0 + k + y;
        T v = T(0);
        if (r < R && c0 + x < C) v = src[(list ? int64_t(list[r]) : r) * lds + c0 + x];
        s[k + y][x] = v;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 64; k += 4)
        if (c0 + k + y < C) dst[int64_t(c0 + k + y) * ldd + r0 + x] = s[x][k + y];
}

// ----------------------------------------------------------------- products

enum What { kStats, kGrad, kStore };

struct LossArgs {
    const char *A, *B;      // rows of A: classes or features; rows of B: tokens or classes
    int64_t lda, ldb;       // bytes
    int64_t M, N;
    const int32_t* n_count;  // N on the device, or null
    const int32_t* rows;     // B's rows through the list, or null
    int64_t steps;           // of the sum
    const int32_t* k_count;  // the sum's length in elements on the device, or null
    int splits;
    // kStats, kGrad
    int64_t v0, V;  // class of A's first row; classes
    const int32_t* list;
    const void* labels;
    bool wide;
    float *part, *hit;  // kStats: part[block][token] of two floats
    int64_t part_ld;
    const float *lse, *dloss;  // kGrad
    void *dl, *dlt;            // [token][dl_ld], [class][dlt_ld] or null
    int64_t dl_ld, dlt_ld;
    // kStore: out[split][row][M], or the result itself
    float* slots;
    int64_t slot_rows;
    bool add;
    void* out;
    const int32_t* out_rows;
};

// The block of C that a workgroup forms: consecutive blocks of an XCD are close to
// each other in both directions.  False: none.
__device__ __forceinline__ bool block_of(int64_t mt, int64_t nt, int64_t& m, int64_t& n) {
    const int64_t total = mt * nt, per = cdiv(total, kXcds), i = int64_t(blockIdx.x) / kXcds;
    const int64_t t = int64_t(blockIdx.x) % kXcds * per + i;
    if (i >= per || t >= total) return false;
    constexpr int64_t G = 4;
    const int64_t g = t / (G * mt), w = nt - g * G < G ? nt - g * G : G, at = t - g * G * mt;
    m = at / w;
    n = g * G + at % w;
    return true;
}

template <typename T>
__device__ __forceinline__ void store4(T* p, float a, float b, float c, float d, int64_t room) {
    if (room >= 4) {
        if constexpr (sizeof(T) == 2) {
            typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
            const u2 x = {pack_bf16x2(a, b), pack_bf16x2(c, d)};
            *reinterpret_cast<u2*>(p) = x;
        } else {
            typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
            const f4 x = {a, b, c, d};
            *reinterpret_cast<f4*>(p) = x;
        }
    } else {
        if (room > 0) store_one(p, a);
        if (room > 1) store_one(p + 1, b);
        if (room > 2) store_one(p + 2, c);
    }
}

template <typename T, int WHAT, int WM, int WN, int TM, int TN>
__global__ __launch_bounds__(WM * WN * 64) void k_product(LossArgs a) {
    using G = GemmNT<T, WM, WN, TM, TN>;
    __shared__ __attribute__((aligned(1024))) char s_buf[G::kStage], s_buf2[G::kStage];
    const int64_t N = a.n_count ? *a.n_count : a.N;
    int64_t bm, bn;
    if (!block_of(cdiv(a.M, G::BM), cdiv(N, G::BN), bm, bn)) return;
    const int64_t m0 = bm * G::BM, n0 = bn * G::BN;
    int64_t steps = a.steps;
    if (a.k_count) steps = cdiv(int64_t(*a.k_count) * int64_t(sizeof(T)), kStepBytes);
    const int64_t each = cdiv(steps, a.splits), s0 = int64_t(blockIdx.y) * each;
    G g;
    g.run(s_buf, s_buf2, a.A, a.lda, m0, a.M, a.B, a.ldb, n0, N, a.rows, s0, s0 + each < steps ? s0 + each : steps);

    const int lane = lane_id(), wave = threadIdx.x / kWave, wm = wave % WM, wn = wave / WM;
    const int64_t mw = m0 + wm * TM * 32 + 4 * (lane >> 5);       // + 32 i + 8 (e / 4) + e % 4
    const int64_t nw = n0 + wn * TN * 32 + (lane & 31);           // + 32 j
    if constexpr (WHAT == kStats) {
        __syncthreads();
        float2* s_part = reinterpret_cast<float2*>(s_buf);  // [WM][BN]
        const bool last = m0 + G::BM > a.M;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t t = nw + 32 * j;
            float top = kNegInf;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    if (last && mw + 32 * i + 8 * (e / 4) + e % 4 >= a.M) g.acc[i][j][e] = kNegInf;
                    top = fmaxf(top, g.acc[i][j][e]);
                }
            top = fmaxf(top, __shfl_xor(top, 32, kWave));
            const float ref = top == kNegInf ? 0.f : top;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) sum += ex2((g.acc[i][j][e] - ref) * kLog2e);
            sum += __shfl_xor(sum, 32, kWave);
            if (lane < 32) s_part[wm * G::BN + wn * TN * 32 + 32 * j + lane] = make_float2(top, sum);
            if (t < N) {
                const int64_t y = load_id(a.labels, a.wide, a.list[t], a.V) - mw;  // the label's place among the lane's classes
#pragma unroll
                for (int i = 0; i < TM; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (y == 32 * i + 8 * (e / 4) + e % 4) a.hit[t] = g.acc[i][j][e];
            }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < G::BN; c += G::kThreads) {
            if (n0 + c >= N) break;
            float top = kNegInf, sum = 0.f;
#pragma unroll
            for (int w = 0; w < WM; ++w) top = fmaxf(top, s_part[w * G::BN + c].x);
            const float ref = top == kNegInf ? 0.f : top;
#pragma unroll
            for (int w = 0; w < WM; ++w) {
                const float2 p = s_part[w * G::BN + c];
                sum += p.y * ex2((p.x - ref) * kLog2e);
            }
            reinterpret_cast<float2*>(a.part)[bm * a.part_ld + n0 + c] = make_float2(top, sum);
        }
    } else if constexpr (WHAT == kGrad) {
        T* dl = static_cast<T*>(a.dl);
        T* dlt = static_cast<T*>(a.dlt);
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t t = nw + 32 * j;
            const bool in = t < N;
            const int64_t row = in ? a.list[t] : 0;
            const float lse = in ? a.lse[row] : 0.f, up = in ? a.dloss[row] : 0.f;
            const int64_t y = in ? load_id(a.labels, a.wide, row, a.V) - a.v0 - mw : -1;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int k = 32 * i + 8 * q + e;
                        const float p = ex2((g.acc[i][j][4 * q + e] - lse) * kLog2e);
                        v[e] = in && mw + k < a.M ? up * (y == k ? p - 1.f : p) : 0.f;
                    }
                    const int64_t m = mw + 32 * i + 8 * q;
                    store4(dl + t * a.dl_ld + m, v[0], v[1], v[2], v[3], 4);
                    if (dlt) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) store_one(dlt + (m + e) * a.dlt_ld + t, v[e]);
                    }
                }
        }
    } else {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int64_t n = nw + 32 * j;
            if (n >= N) continue;
            float* o = a.slots ? a.slots + (int64_t(blockIdx.y) * a.slot_rows + n) * a.M : nullptr;
            T* r = a.slots ? nullptr : static_cast<T*>(a.out) + (a.out_rows ? int64_t(a.out_rows[n]) : n) * a.M;
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int64_t m = mw + 32 * i + 8 * q, room = a.M - m;
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = g.acc[i][j][4 * q + e];
                    if (o) {
                        if (a.add) {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (e < room) v[e] += o[m + e];
                        }
                        store4(o + m, v[0], v[1], v[2], v[3], room);
                    } else {
                        store4(r + m, v[0], v[1], v[2], v[3], room);
                    }
                }
        }
    }
}

// The parts of a token's statistics, joined: a token's blocks go by over 32 lanes.
__global__ __launch_bounds__(256) void k_loss(int64_t blocks, const float2* part, int64_t ld, const float* hit,
                                               const int32_t* list, const int32_t* count, float* loss, float* lse) {
    constexpr int P = 32;  // tokens of a workgroup
    __shared__ float2 s[256 / P][P];
    const int x = threadIdx.x % P, y = threadIdx.x / P;
    const int64_t t = int64_t(blockIdx.x) * P + x, n = *count;
    if (int64_t(blockIdx.x) * P >= n) return;
    float top = kNegInf, sum = 0.f;
    if (t < n)
        for (int64_t b = y; b < blocks; b += 256 / P) {
            const float2 p = part[b * ld + t];
            const float m = fmaxf(top, p.x), ref = m == kNegInf ? 0.f : m;
            sum = sum * ex2((top - ref) * kLog2e) + p.y * ex2((p.x - ref) * kLog2e);
            top = m;
        }
    s[y][x] = make_float2(top, sum);
    __syncthreads();
    if (y || t >= n) return;
    top = kNegInf, sum = 0.f;
    for (int k = 0; k < 256 / P; ++k) top = fmaxf(top, s[k][x].x);
    const float ref = top == kNegInf ? 0.f : top;
    for (int k = 0; k < 256 / P; ++k) sum += s[k][x].y * ex2((s[k][x].x - ref) * kLog2e);
    const float l = ref + logf(sum);
    const int64_t i = list[t];
    lse[i] = l;
    loss[i] = l - hit[t];
}

// out[row][c] = the sum of the slots
template <typename T>
__global__ __launch_bounds__(256) void k_sum_slots(int splits, int64_t slot_rows, int64_t R, const int32_t* count,
                                                    int64_t C, const float* slots, const int32_t* rows, T* out) {
    if (count) R = *count;
    const int64_t total = R * C;
    for (int64_t i = blockIdx.x * int64_t(256) + threadIdx.x; i < total; i += int64_t(gridDim.x) * 256) {
        float v = 0.f;
        for (int k = 0; k < splits; ++k) v += slots[int64_t(k) * slot_rows * C + i];
        const int64_t r = i / C;
        store_one(out + (rows ? int64_t(rows[r]) * C + (i - r * C) : i), v);
    }
}

template <typename T, int WHAT>
gt_status product(const LossArgs& a, hipStream_t s) {
#define GT_CALL(WM, WN, TM, TN)                                                                            \
    do {                                                                                                   \
        using G = GemmNT<T, WM, WN, TM, TN>;                                                               \
        const dim3 grid(xcd_grid(cdiv(a.M, G::BM) * cdiv(a.N, G::BN)), unsigned(a.splits));                \
        k_product<T, WHAT, WM, WN, TM, TN><<<grid, G::kThreads, 0, s>>>(a);                                \
    } while (0)
    if (a.M <= 64) {
        if (a.N <= 64) GT_CALL(2, 2, 1, 1);
        else GT_CALL(2, 4, 1, 2);
    } else {
        if (a.N <= 64) GT_CALL(4, 1, 2, 2);
        else GT_CALL(2, 4, 4, 2);
    }
#undef GT_CALL
    GT_LAUNCH_CHECK("class_loss product");
    return GT_OK;
}
// the block sides that product() takes
int64_t block_rows(int64_t x) { return x <= 64 ? 64 : 256; }

int splits_of(int64_t M, int64_t N, int64_t steps) {
    const int64_t blocks = cdiv(M, block_rows(M)) * cdiv(N, block_rows(N));
    int64_t s = kSplitBlocks / blocks;
    if (s > steps / kSplitSteps) s = steps / kSplitSteps;
    return int(s < 1 ? 1 : s);
}

// ----------------------------------------------------------------- workspace

struct Shape {
    int64_t n, V, ldx, ldw;
    int D, size;
    bool pad_x, pad_w;
    int64_t row;   // bytes of a padded row
    int64_t mp;    // tokens, whole blocks
    int64_t piece;  // classes a piece
    int sx, sw;     // splits of dX and dW
    bool slots_x;
};

Shape shape_of(int64_t n, int64_t V, int32_t D, gt_dtype dt, int64_t ldx, int64_t ldw) {
    Shape h = {};
    h.n = n, h.V = V, h.D = D, h.ldx = ldx, h.ldw = ldw;
    h.size = dt == GT_BF16 ? 2 : 4;
    h.row = cdiv(int64_t(D) * h.size, kStepBytes) * kStepBytes;
    const bool whole = h.row == int64_t(D) * h.size;
    h.pad_x = !whole || ldx * h.size % 16 != 0;
    h.pad_w = !whole || ldw * h.size % 16 != 0;
    h.mp = cdiv(n, 256) * 256;
    const int64_t all = cdiv(V, 256) * 256;
    int64_t piece = kPieceBytes / (h.mp * h.size) / 256 * 256;
    if (piece < kMinPiece) piece = kMinPiece;
    h.piece = piece < all ? piece : all;
    h.sx = splits_of(D, n, h.piece * h.size / kStepBytes);
    h.sw = splits_of(D, h.piece < V ? h.piece : V, h.mp * h.size / kStepBytes);
    h.slots_x = h.sx > 1 || h.piece < V;
    return h;
}

struct List {
    int32_t *list, *count, *cnt;
};
List list_ws(Ws& w, int64_t n) {
    List l;
    l.list = w.take<int32_t>(size_t(n));
    l.count = w.take<int32_t>(1);
    l.cnt = w.take<int32_t>(size_t(cdiv(n, kListRows)));
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
    f.x = h.pad_x ? w.take<char>(size_t(h.n * h.row)) : nullptr;
    f.w = h.pad_w ? w.take<char>(size_t(h.V * h.row)) : nullptr;
    f.part = w.take<float>(size_t(2 * h.mp * cdiv(h.V, block_rows(h.V))));
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
    b.x = h.pad_x ? w.take<char>(size_t(h.n * h.row)) : nullptr;
    b.w = h.pad_w ? w.take<char>(size_t(h.V * h.row)) : nullptr;
    b.xt = w.take<char>(size_t(h.D) * size_t(h.mp * h.size));
    b.wt = w.take<char>(size_t(h.D) * size_t(h.piece * h.size));
    b.dl = w.take<char>(size_t(h.mp * h.piece * h.size));
    b.dlt = w.take<char>(size_t(h.mp * h.piece * h.size));
    b.slots_x = h.slots_x ? w.take<float>(size_t(h.sx) * size_t(h.n) * h.D) : nullptr;
    b.slots_w = h.sw > 1 ? w.take<float>(size_t(h.sw) * size_t(h.piece) * h.D) : nullptr;
    return b;
}

gt_status make_list(const Shape& h, bool wide, const void* labels, const List& l, float* loss, float* lse,
                    hipStream_t s) {
    const unsigned blocks = unsigned(cdiv(h.n, kListRows));
    if (blocks > 1) {
        k_list_count<<<blocks, kListThreads, 0, s>>>(h.n, h.V, wide, labels, l.cnt);
        GT_LAUNCH_CHECK("class_loss count");
    }
    k_list_place<<<blocks, kListThreads, 0, s>>>(h.n, h.V, wide, labels, l.cnt, l.list, l.count, loss, lse);
    GT_LAUNCH_CHECK("class_loss list");
    return GT_OK;
}

// X and W as the products take them
template <typename T>
gt_status make_rows(const Shape& h, const void*& X, int64_t& ldx, char* x, const void*& W, int64_t& ldw, char* w,
                    hipStream_t s) {
    const int ldd = int(h.row / h.size);
    if (h.pad_x) {
        k_pad<T><<<grid_for(h.n, 4, 1 << 16), 256, 0, s>>>(h.n, h.D, static_cast<const T*>(X), ldx,
                                                           reinterpret_cast<T*>(x), ldd);
        GT_LAUNCH_CHECK("class_loss pad");
        X = x, ldx = ldd;
    }
    if (h.pad_w) {
        k_pad<T><<<grid_for(h.V, 4, 1 << 16), 256, 0, s>>>(h.V, h.D, static_cast<const T*>(W), ldw,
                                                           reinterpret_cast<T*>(w), ldd);
        GT_LAUNCH_CHECK("class_loss pad");
        W = w, ldw = ldd;
    }
    return GT_OK;
}

template <typename T>
gt_status run_fwd(const Shape& h, const void* X, const void* W, bool wide, const void* labels, float* loss, float* lse,
                  const FwdWs& f, hipStream_t s) {
    gt_status st = make_list(h, wide, labels, f.l, loss, lse, s);
    if (st != GT_OK) return st;
    int64_t ldx = h.ldx, ldw = h.ldw;
    st = make_rows<T>(h, X, ldx, f.x, W, ldw, f.w, s);
    if (st != GT_OK) return st;
    LossArgs a = {};
    a.A = static_cast<const char*>(W), a.lda = ldw * h.size, a.M = h.V;
    a.B = static_cast<const char*>(X), a.ldb = ldx * h.size, a.N = h.n;
    a.n_count = f.l.count, a.rows = f.l.list, a.list = f.l.list;
    a.steps = h.row / kStepBytes, a.splits = 1;
    a.V = h.V, a.labels = labels, a.wide = wide;
    a.part = f.part, a.part_ld = h.mp, a.hit = f.hit;
    st = product<T, kStats>(a, s);
    if (st != GT_OK) return st;
    k_loss<<<unsigned(cdiv(h.n, 32)), 256, 0, s>>>(cdiv(h.V, block_rows(h.V)), reinterpret_cast<float2*>(f.part), h.mp,
                                                   f.hit, f.l.list, f.l.count, loss, lse);
    GT_LAUNCH_CHECK("class_loss join");
    return GT_OK;
}

template <typename T>
gt_status run_bwd(const Shape& h, const void* X0, const void* W0, bool wide, const void* labels, const float* lse,
                  const float* dloss, void* dX, void* dW, const BwdWs& b, hipStream_t s) {
    if (h.n == 0) {
        k_zero<T><<<grid_for(h.V * h.D, 256, 1 << 16), 256, 0, s>>>(h.V * h.D, static_cast<T*>(dW));
        GT_LAUNCH_CHECK("class_loss zero");
        return GT_OK;
    }
    gt_status st = make_list(h, wide, labels, b.l, nullptr, nullptr, s);
    if (st != GT_OK) return st;
    const void *X = X0, *W = W0;
    int64_t ldx = h.ldx, ldw = h.ldw;
    st = make_rows<T>(h, X, ldx, b.x, W, ldw, b.w, s);
    if (st != GT_OK) return st;
    if (dX) {
        k_zero_rows<T><<<grid_for(h.n, 4, 1 << 16), 256, 0, s>>>(h.n, h.D, h.V, wide, labels, static_cast<T*>(dX));
        GT_LAUNCH_CHECK("class_loss zero rows");
    }
    const unsigned turns = unsigned(cdiv(h.D, 64));
    if (dW) {
        k_turn<T><<<dim3(unsigned(cdiv(h.n, 64)), turns), 256, 0, s>>>(
            h.n, b.l.count, b.l.list, h.D, static_cast<const T*>(X), ldx, reinterpret_cast<T*>(b.xt), h.mp);
        GT_LAUNCH_CHECK("class_loss turn");
    }
    for (int64_t v0 = 0; v0 < h.V; v0 += h.piece) {
        const int64_t vn = h.V - v0 < h.piece ? h.V - v0 : h.piece;
        const char* w = static_cast<const char*>(W) + v0 * ldw * h.size;
        LossArgs a = {};
        a.A = w, a.lda = ldw * h.size, a.M = vn;
        a.B = static_cast<const char*>(X), a.ldb = ldx * h.size, a.N = h.n;
        a.n_count = b.l.count, a.rows = b.l.list, a.list = b.l.list;
        a.steps = h.row / kStepBytes, a.splits = 1;
        a.v0 = v0, a.V = h.V, a.labels = labels, a.wide = wide, a.lse = lse, a.dloss = dloss;
        a.dl = b.dl, a.dl_ld = h.piece;
        a.dlt = dW ? b.dlt : nullptr, a.dlt_ld = h.mp;
        st = product<T, kGrad>(a, s);
        if (st != GT_OK) return st;
        if (dX) {
            k_turn<T><<<dim3(unsigned(cdiv(vn, 64)), turns), 256, 0, s>>>(
                vn, nullptr, nullptr, h.D, reinterpret_cast<const T*>(w), ldw, reinterpret_cast<T*>(b.wt), h.piece);
            GT_LAUNCH_CHECK("class_loss turn");
            LossArgs x = {};
            x.A = b.wt, x.lda = h.piece * h.size, x.M = h.D;
            x.B = b.dl, x.ldb = h.piece * h.size, x.N = h.n, x.n_count = b.l.count;
            x.steps = cdiv(vn * h.size, kStepBytes), x.splits = h.sx;
            x.slots = b.slots_x, x.slot_rows = h.n, x.add = v0 > 0;
            x.out = dX, x.out_rows = b.l.list;
            st = product<T, kStore>(x, s);
            if (st != GT_OK) return st;
        }
        if (dW) {
            LossArgs x = {};
            x.A = b.xt, x.lda = h.mp * h.size, x.M = h.D;
            x.B = b.dlt, x.ldb = h.mp * h.size, x.N = vn;
            x.k_count = b.l.count, x.splits = h.sw;
            x.slots = b.slots_w, x.slot_rows = h.piece;
            T* out = static_cast<T*>(dW) + v0 * h.D;
            x.out = out;
            st = product<T, kStore>(x, s);
            if (st != GT_OK) return st;
            if (b.slots_w) {
                k_sum_slots<T><<<grid_for(vn * h.D, 256, 1 << 16), 256, 0, s>>>(h.sw, h.piece, vn, nullptr, h.D,
                                                                                b.slots_w, nullptr, out);
                GT_LAUNCH_CHECK("class_loss sum");
            }
        }
    }
    if (dX && b.slots_x) {
        k_sum_slots<T><<<grid_for(h.n * h.D, 256, 1 << 16), 256, 0, s>>>(h.sx, h.n, h.n, b.l.count, h.D, b.slots_x,
                                                                         b.l.list, static_cast<T*>(dX));
        GT_LAUNCH_CHECK("class_loss sum");
    }
    return GT_OK;
}

bool loss_sizes(int64_t n, int64_t V, int32_t D, gt_dtype dt, int64_t ldx, int64_t ldw) {
    const int64_t most = int64_t(1) << 31;
    return (dt == GT_BF16 || dt == GT_F32) && n >= 0 && n < most && V >= 1 && V < most && D >= 1 && D <= GT_MAX_WIDTH &&
           ldx >= D && ldw >= D && ldx < most && ldw < most;
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
