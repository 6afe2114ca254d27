// The norms between two blocks of a layer, with the gate and the scaled residual
// that lie between them, in one pass over the rows; forward and backward.
//
// Bound by memory: the forward reads x, f (and a gate of rows) and writes y, z;
// the backward reads x, f, (gate), dy, dz and writes dx, df, (dgate).  A row lies
// in the registers of LPR lanes (a part of a wavefront, a wavefront or a
// workgroup), NV 16-byte pieces of each array a lane, so every value is read
// once; a lane keeps its columns from row to row, and with them the parameters
// and the columns' sums of the parameters' gradients.  Workgroups walk the rows
// grid-wide and leave one partial sum per column, which k_norm_sum adds in a
// fixed order.  100,000 rows of 512 in bf16 with a sigmoid gate 110 us forward and
// 195 backward, a million of 256 with a gate vector 410 and 680 (4.7 TB/s).
#include "attn_common.h"
#include "lanes.h"

using namespace gt;

namespace {

constexpr int kMaxD = 8192;
constexpr int64_t kFarBytes = int64_t(256) << 20;  // the last-level cache
constexpr int kSums = 5;  // dw_post, db_post, dw_pre, db_pre, dgate (vector)

struct NormArgs {
    int64_t n;
    int D, norm, gate_kind;
    float eps, res_scale;
    const void *x, *f, *gate, *dy, *dz;
    const float *w_post, *b_post, *w_pre, *b_pre;
    void *y, *z, *dx, *df, *dgate;
    float* stats;
    float* part;  // [blocks][kSums][D]
    uint32_t want;  // bit k: sum k is wanted
    bool far;       // the results go past the last-level cache
};

template <int LPR>
struct RowSum {
    static constexpr int kThreads = LPR > 256 ? LPR : 256;
    static constexpr int kRows = kThreads / LPR;  // rows a workgroup works on together
    // the sums of a and b over the row's lanes, in every lane
    __device__ __forceinline__ static void two(float& a, float& b, float* s) {
        constexpr int W = LPR < kWave ? LPR : kWave;
        if constexpr (W > 1) step<1, W>(a, b);
        if constexpr (LPR > kWave) {
            const int wave = int(threadIdx.x) / kWave;
            __syncthreads();
            if (lane_id() == 0) s[2 * wave] = a, s[2 * wave + 1] = b;
            __syncthreads();
            a = b = 0.f;
#pragma unroll
            for (int w = 0; w < LPR / kWave; ++w) a += s[2 * w], b += s[2 * w + 1];
        }
    }
    template <int O, int W>
    __device__ __forceinline__ static void step(float& a, float& b) {
        if constexpr (O < W) {
            a += __int_as_float(xor_lane<O>(__float_as_int(a)));
            b += __int_as_float(xor_lane<O>(__float_as_int(b)));
            step<2 * O, W>(a, b);
        }
    }
};

// 16 bytes at any element's address (global accesses need no more alignment; a
// load or store for each element instead: rows of 511 in bf16 1,460 GB/s forward
// and 950 backward against 3,700 and 3,850).
template <typename T>
struct Piece {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4)));
    typedef uint32_t word __attribute__((aligned(4)));
};
template <>
struct Piece<uint16_t> {
    typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2)));
    typedef uint32_t word __attribute__((aligned(2)));
};

// A lane's NV pieces of one row: E consecutive features each, LPR pieces apart.
// kWhole: rows are whole pieces; kFull besides: the row fills its lanes.  kRagged:
// the row's last piece is loaded ending with the row and shifted, and stored in
// parts.  kTiny: rows of less than a piece, an element at a time.
enum Rows { kFull, kWhole, kRagged, kTiny };

template <typename T, int LPR, int NV, Rows R>
struct Cols {
    static constexpr int E = 16 / int(sizeof(T));
    static constexpr bool FULL = R == kFull, VEC = R <= kWhole;
    typedef typename Piece<T>::type piece_t;
    int D, lane;  // lane of the row
    __device__ __forceinline__ int col(int v) const { return (lane + LPR * v) * E; }
    __device__ __forceinline__ bool in(int v, int t) const { return FULL || (VEC ? col(v) < D : col(v) + t < D); }
    __device__ __forceinline__ void load(float (&o)[NV][E], const void* p, int64_t row) const {
        const T* r = static_cast<const T*>(p) + row * D;
        if constexpr (R == kTiny) {
#pragma unroll
            for (int t = 0; t < E; ++t) {
                o[0][t] = 0.f;
                if (col(0) + t < D) {
                    if constexpr (E == 8) o[0][t] = bf16_to_f32(r[col(0) + t]);
                    else o[0][t] = r[col(0) + t];
                }
            }
            return;
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            piece_t x = {0, 0, 0, 0};
            const int c = col(v);
            const int over = VEC || c + E <= D ? 0 : c + E - D;  // elements of the piece behind the row's end
            if (FULL || c < D) x = *reinterpret_cast<const piece_t*>(r + c - over);
            uint32_t w[4] = {x[0], x[1], x[2], x[3]};
            if constexpr (!VEC) {  // down by `over` elements, zeros from above
                const int bits = over * 8 * int(sizeof(T));
                if (bits & 64) w[0] = w[2], w[1] = w[3], w[2] = w[3] = 0;
                if (bits & 32) w[0] = w[1], w[1] = w[2], w[2] = w[3], w[3] = 0;
                if constexpr (E == 8) {
                    const uint32_t by = bits & 16;
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_alignbit(i < 3 ? w[i + 1] : 0, w[i], by);
                }
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if constexpr (E == 8) o[v][2 * t] = bf16lo(w[t]), o[v][2 * t + 1] = bf16hi(w[t]);
                else o[v][t] = __uint_as_float(w[t]);
            }
        }
    }
    __device__ __forceinline__ void store(void* p, int64_t row, const float (&o)[NV][E], bool far) const {
        T* r = static_cast<T*>(p) + row * D;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c = col(v);
            if (!FULL && c >= D) continue;
            uint32_t w[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if constexpr (E == 8) w[t] = pack_bf16x2(o[v][2 * t], o[v][2 * t + 1]);
                else w[t] = __float_as_uint(o[v][t]);
            }
            if (VEC || c + E <= D) {
                const piece_t x = {w[0], w[1], w[2], w[3]};
                if (far) __builtin_nontemporal_store(x, reinterpret_cast<piece_t*>(r + c));
                else *reinterpret_cast<piece_t*>(r + c) = x;
            } else {
                constexpr int kWord = 4 / int(sizeof(T));  // elements per 32 bits
                const int left = D - c;
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    if (left >= kWord * (t + 1)) *reinterpret_cast<typename Piece<T>::word*>(r + c + kWord * t) = w[t];
                    else if (kWord == 2 && left > kWord * t) r[c + kWord * t] = T(w[t]);
                }
            }
        }
    }
    __device__ __forceinline__ void param(float (&o)[NV][E], const float* p, float none) const {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int t = 0; t < E; ++t) o[v][t] = p && col(v) + t < D ? p[col(v) + t] : none;
    }
};

// mean and 1 / sqrt(var + eps) of a row (two passes over registers: no
// cancellation of a large mean); mean 0 without layer.
template <int LPR, int NV, int E, typename C>
__device__ __forceinline__ void row_stats(const float (&v)[NV][E], const C& c, bool layer, float eps, float inv_d,
                                          float* s, float& mean, float& rstd) {
    float a = 0.f, b = 0.f;
    mean = 0.f;
    if (layer) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int t = 0; t < E; ++t) a += v[k][t];
        RowSum<LPR>::two(a, b, s);
        mean = a * inv_d;
    }
    a = b = 0.f;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int t = 0; t < E; ++t) {
            const float x = c.in(k, t) ? v[k][t] - mean : 0.f;
            a = fmaf(x, x, a);
        }
    RowSum<LPR>::two(a, b, s);
    rstd = 1.f / sqrtf(fmaf(a, inv_d, eps));
}

__device__ __forceinline__ float sigmoid(float v) { return 1.f / (1.f + __expf(-v)); }

template <typename T, int LPR, int NV, Rows R>
__global__ __launch_bounds__(RowSum<LPR>::kThreads) void k_norm_fwd(NormArgs a) {
    using C = Cols<T, LPR, NV, R>;
    using S = RowSum<LPR>;
    constexpr int E = C::E;
    __shared__ float s_sum[2 * S::kThreads / kWave];
    const int t_row = int(threadIdx.x) / LPR;
    const C c = {a.D, int(threadIdx.x) % LPR};
    const bool layer = a.norm == GT_NORM_LAYER;
    const float inv_d = 1.f / float(a.D);
    float w1[NV][E], b1[NV][E], w2[NV][E], b2[NV][E], g[NV][E];
    c.param(w1, a.w_post, 1.f);
    c.param(b1, a.b_post, 0.f);
    c.param(w2, a.w_pre, 1.f);
    c.param(b2, a.b_pre, 0.f);
    c.param(g, a.gate_kind == GT_GATE_VECTOR ? static_cast<const float*>(a.gate) : nullptr, 1.f);
    for (int64_t r0 = int64_t(blockIdx.x) * S::kRows; r0 < a.n; r0 += int64_t(gridDim.x) * S::kRows) {
        // every lane stays in the exchanges; a lane behind the last row works on the last one and writes nothing
        const int64_t row = r0 + t_row < a.n ? r0 + t_row : a.n - 1;
        const bool own = r0 + t_row < a.n;
        float x[NV][E], f[NV][E];
        c.load(f, a.f, row);
        c.load(x, a.x, row);
        if (a.gate_kind >= GT_GATE_ROWS) c.load(g, a.gate, row);
        float mf, rf, my, ry;
        row_stats<LPR>(f, c, layer, a.eps, inv_d, s_sum, mf, rf);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int t = 0; t < E; ++t) {
                const float u = fmaf((f[v][t] - mf) * rf, w1[v][t], b1[v][t]);
                const float gv = a.gate_kind == GT_GATE_SIGMOID ? sigmoid(g[v][t]) : g[v][t];
                x[v][t] = c.in(v, t) ? fmaf(gv, u, a.res_scale * x[v][t]) : 0.f;
            }
        row_stats<LPR>(x, c, layer, a.eps, inv_d, s_sum, my, ry);
        if (own) {
            c.store(a.y, row, x, a.far);
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int t = 0; t < E; ++t) x[v][t] = fmaf((x[v][t] - my) * ry, w2[v][t], b2[v][t]);
            c.store(a.z, row, x, a.far);
            if (c.lane == 0) *reinterpret_cast<float4*>(a.stats + 4 * row) = make_float4(mf, rf, my, ry);
        }
    }
}

// A lane's parameters: in registers or, one each of a kernel's four, in LDS.
template <typename C, int LPR, int NV, bool LDS>
struct Params {
    static constexpr int E = C::E;
    float v[LDS ? 1 : NV][LDS ? 1 : E];
    float* s;
    __device__ __forceinline__ Params(const C& c, const float* p, float none, float* lds) {
        if constexpr (LDS) {
            s = lds + 4 * int(threadIdx.x);
            float x[NV][E];
            c.param(x, p, none);
#pragma unroll
            for (int k = 0; k < NV * E / 4; ++k)
                *reinterpret_cast<float4*>(s + 4 * LPR * k) = make_float4(x[4 * k / E][4 * k % E], x[4 * k / E][4 * k % E + 1],
                                                                          x[4 * k / E][4 * k % E + 2], x[4 * k / E][4 * k % E + 3]);
        } else {
            c.param(v, p, none);
        }
    }
    // the lane's own writes, in the order of the program
    __device__ __forceinline__ float operator()(int k, int t) const {
        if constexpr (LDS) return s[4 * LPR * ((k * E + t) / 4) + t % 4];
        else return v[k][t];
    }
    __device__ __forceinline__ void get(float (&o)[NV][E]) const {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int t = 0; t < E; ++t) o[k][t] = (*this)(k, t);
    }
};

// With fh = (f - mf) rf, yh = (y - my) ry and <v> a row's mean:
//   t  = dy + ry (dz w2 - <dz w2> - yh <dz w2 yh>)      the gradient of y
//   dx = res_scale t, dg = u t, du = g t
//   df = rf (du w1 - <du w1> - fh <du w1 fh>)
// (without the <dz w2> and <du w1> terms for the root mean square).
// Rows of 512 lanes hold 16 columns a lane, whose parameters and sums do not fit the
// registers together: the parameters lie in LDS (32,768 rows of 8,192 in bf16, a gate
// vector, all parameters: 808 us against 1632 with spilled registers).
template <typename T, int LPR, int NV, Rows R>
__global__ __launch_bounds__(RowSum<LPR>::kThreads) void k_norm_bwd(NormArgs a) {
    using C = Cols<T, LPR, NV, R>;
    using S = RowSum<LPR>;
    constexpr int E = C::E;
    __shared__ float s_sum[2 * S::kThreads / kWave];
    __shared__ float s_part[S::kRows > 1 ? S::kThreads * NV * E : 1];
    const int t_row = int(threadIdx.x) / LPR;
    const C c = {a.D, int(threadIdx.x) % LPR};
    const bool layer = a.norm == GT_NORM_LAYER;
    const float inv_d = 1.f / float(a.D);
    const float* vector = a.gate_kind == GT_GATE_VECTOR ? static_cast<const float*>(a.gate) : nullptr;
    constexpr bool kLds = LPR == 512;
    constexpr int kEach = LPR * NV * E;
    __shared__ __attribute__((aligned(16))) float s_par[kLds ? 4 * kEach : 1];
    const Params<C, LPR, NV, kLds> w1(c, a.w_post, 1.f, s_par), b1(c, a.b_post, 0.f, s_par + kEach),
        w2(c, a.w_pre, 1.f, s_par + 2 * kEach), gv(c, vector, 1.f, s_par + 3 * kEach);
    float g[NV][E], sum[kSums][NV][E];
    gv.get(g);
#pragma unroll
    for (int k = 0; k < kSums; ++k)
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int t = 0; t < E; ++t) sum[k][v][t] = 0.f;
    for (int64_t r0 = int64_t(blockIdx.x) * S::kRows; r0 < a.n; r0 += int64_t(gridDim.x) * S::kRows) {
        const int64_t row = r0 + t_row < a.n ? r0 + t_row : a.n - 1;
        const bool own = r0 + t_row < a.n;
        float x[NV][E], f[NV][E], dy[NV][E], dz[NV][E];
        const float4 st = *reinterpret_cast<const float4*>(a.stats + 4 * row);
        c.load(f, a.f, row);
        c.load(x, a.x, row);
        if (a.gate_kind >= GT_GATE_ROWS) c.load(g, a.gate, row);
        else if constexpr (kLds) gv.get(g);
        c.load(dz, a.dz, row);
        c.load(dy, a.dy, row);
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int t = 0; t < E; ++t) {
                f[v][t] = c.in(v, t) ? (f[v][t] - st.x) * st.y : 0.f;  // fh
                if (a.gate_kind == GT_GATE_SIGMOID) g[v][t] = sigmoid(g[v][t]);
                const float u = fmaf(f[v][t], w1(v, t), b1(v, t));
                x[v][t] = c.in(v, t) ? (fmaf(g[v][t], u, a.res_scale * x[v][t]) - st.z) * st.w : 0.f;  // yh
                const float d = dz[v][t] * w2(v, t);
                s1 += d;
                s2 = fmaf(d, x[v][t], s2);
                if (own) {
                    sum[2][v][t] = fmaf(dz[v][t], x[v][t], sum[2][v][t]);
                    sum[3][v][t] += dz[v][t];
                }
            }
        S::two(s1, s2, s_sum);
        const float m1 = layer ? s1 * inv_d : 0.f, m2 = s2 * inv_d;
        s1 = s2 = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int t = 0; t < E; ++t) {
                const float ty = fmaf(st.w, dz[v][t] * w2(v, t) - m1 - x[v][t] * m2, dy[v][t]);
                const float u = fmaf(f[v][t], w1(v, t), b1(v, t));
                const float du = g[v][t] * ty, dg = u * ty;
                x[v][t] = a.res_scale * ty;
                dy[v][t] = a.gate_kind == GT_GATE_SIGMOID ? dg * (g[v][t] * (1.f - g[v][t])) : dg;
                if (own) {
                    sum[0][v][t] = fmaf(du, f[v][t], sum[0][v][t]);
                    sum[1][v][t] += du;
                    sum[4][v][t] += dg;
                }
                dz[v][t] = c.in(v, t) ? du * w1(v, t) : 0.f;
                s1 += dz[v][t];
                s2 = fmaf(dz[v][t], f[v][t], s2);
            }
        S::two(s1, s2, s_sum);
        const float n1 = layer ? s1 * inv_d : 0.f, n2 = s2 * inv_d;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int t = 0; t < E; ++t) f[v][t] = st.y * (dz[v][t] - n1 - f[v][t] * n2);
        if (own) {
            c.store(a.dx, row, x, a.far);
            c.store(a.df, row, f, a.far);
            if (a.gate_kind >= GT_GATE_ROWS) c.store(a.dgate, row, dy, a.far);
        }
    }
    // the columns' sums over the workgroup's rows
    for (int k = 0; k < kSums; ++k) {
        if (!(a.want >> k & 1)) continue;
        float* out = a.part + (int64_t(blockIdx.x) * kSums + k) * a.D;
        if constexpr (S::kRows > 1) {
            __syncthreads();
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int t = 0; t < E; ++t) s_part[(t_row * LPR * NV + LPR * v + c.lane) * E + t] = sum[k][v][t];
            __syncthreads();
            for (int x = int(threadIdx.x); x < LPR * NV * E && x < a.D; x += S::kThreads) {
                float t = 0.f;
                for (int r = 0; r < S::kRows; ++r) t += s_part[r * (LPR * NV * E) + x];
                out[x] = t;
            }
        } else {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int t = 0; t < E; ++t)
                    if (c.col(v) + t < a.D) out[c.col(v) + t] = sum[k][v][t];
        }
    }
}

// out[k][x] = the sum over the workgroups' partial sums, 16 columns a workgroup:
// 64 threads for each, every one a 64th of the partial sums, then those 64.
struct SumOut {
    float* p[kSums];
};
__global__ __launch_bounds__(1024) void k_norm_sum(int blocks, int D, const float* __restrict__ part, SumOut o) {
    __shared__ float s[1024];
    const int k = int(blockIdx.y), x = int(blockIdx.x) * 16 + int(threadIdx.x & 15);
    float* out = o.p[k];
    if (!out) return;  // uniform
    float t = 0.f;
    if (x < D)
#pragma unroll 8
        for (int b = int(threadIdx.x) / 16; b < blocks; b += 64) t += part[(int64_t(b) * kSums + k) * D + x];
    s[threadIdx.x] = t;
    __syncthreads();
    if (threadIdx.x >= 16 || x >= D) return;
    for (int w = 1; w < 64; ++w) t += s[16 * w + threadIdx.x];
    out[x] = t;
}

// Lanes per row and pieces per lane: the fewest lanes, but no fewer than 8, that
// hold a row at one piece each, and two a lane where a row would only just leave a
// wavefront (or a workgroup of 256 or 512).  Rows of 1 to 4 pieces leave half to
// seven eighths of their lanes without data: 2M rows of 8, 16, 32 and 64 columns in
// bf16 take 120, 127, 140 and 208 us forward (1.1, 2.0, 3.7 and 4.9 TB/s).
#define GT_NORM_SHAPE(pieces, CALL)                 \
    do {                                            \
        if ((pieces) <= 8) { CALL(8, 1); }          \
        else if ((pieces) <= 16) { CALL(16, 1); }   \
        else if ((pieces) <= 32) { CALL(32, 1); }   \
        else if ((pieces) <= 64) { CALL(64, 1); }   \
        else if ((pieces) <= 128) { CALL(64, 2); }  \
        else if ((pieces) <= 256) { CALL(256, 1); } \
        else if constexpr (sizeof(T) == 4) {        \
            if ((pieces) <= 512) { CALL(256, 2); }  \
            else if ((pieces) <= 1024) { CALL(512, 2); } \
            else { CALL(512, 4); }                  \
        } else if ((pieces) <= 512) { CALL(512, 1); } \
        else { CALL(512, 2); }                      \
    } while (0)

int norm_rows(int pieces) { return pieces <= 8 ? 32 : pieces <= 16 ? 16 : pieces <= 32 ? 8 : pieces <= 128 ? 4 : 1; }

constexpr int kNormBlocks = 1024;

int norm_blocks(int64_t n, int32_t D, gt_dtype dt) {
    const int pieces = int(cdiv(D, dt == GT_BF16 ? 8 : 4));
    const int64_t want = cdiv(n, norm_rows(pieces));
    return int(want < kNormBlocks ? want : kNormBlocks);
}

bool off16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

template <typename T>
void run_fwd(const NormArgs& a, int pieces, int blocks, hipStream_t s) {
    constexpr int E = 16 / int(sizeof(T));
    const bool whole = a.D % E == 0;
#define GT_CALL(LPR, NV)                                                                                   \
    do {                                                                                                   \
        constexpr int kThreads = RowSum<LPR>::kThreads;                                                    \
        if (whole && pieces == LPR * NV) k_norm_fwd<T, LPR, NV, kFull><<<blocks, kThreads, 0, s>>>(a);     \
        else if (whole) k_norm_fwd<T, LPR, NV, kWhole><<<blocks, kThreads, 0, s>>>(a);                     \
        else k_norm_fwd<T, LPR, NV, kRagged><<<blocks, kThreads, 0, s>>>(a);                               \
    } while (0)
    if (a.D < E) k_norm_fwd<T, 8, 1, kTiny><<<blocks, RowSum<8>::kThreads, 0, s>>>(a);
    else GT_NORM_SHAPE(pieces, GT_CALL);
#undef GT_CALL
}
template <typename T>
void run_bwd(const NormArgs& a, int pieces, int blocks, hipStream_t s) {
    constexpr int E = 16 / int(sizeof(T));
    const bool whole = a.D % E == 0;
#define GT_CALL(LPR, NV)                                                                                   \
    do {                                                                                                   \
        constexpr int kThreads = RowSum<LPR>::kThreads;                                                    \
        if (whole && pieces == LPR * NV) k_norm_bwd<T, LPR, NV, kFull><<<blocks, kThreads, 0, s>>>(a);     \
        else if (whole) k_norm_bwd<T, LPR, NV, kWhole><<<blocks, kThreads, 0, s>>>(a);                     \
        else k_norm_bwd<T, LPR, NV, kRagged><<<blocks, kThreads, 0, s>>>(a);                               \
    } while (0)
    if (a.D < E) k_norm_bwd<T, 8, 1, kTiny><<<blocks, RowSum<8>::kThreads, 0, s>>>(a);
    else GT_NORM_SHAPE(pieces, GT_CALL);
#undef GT_CALL
}

gt_status norm_check(const char* who, int64_t n, int32_t D, gt_dtype dt, int32_t norm, int32_t gate_kind,
                     const void* gate) {
    const std::string w(who);
    if (n < 0 || n >= (int64_t(1) << 31)) return fail(GT_ERR_INVALID_ARG, w + ": n out of range");
    if ((dt != GT_BF16 && dt != GT_F32) || D < 1 || D > kMaxD) return fail(GT_ERR_UNSUPPORTED, w + ": unsupported (dtype, D)");
    if (norm != GT_NORM_LAYER && norm != GT_NORM_RMS) return fail(GT_ERR_UNSUPPORTED, w + ": unknown norm");
    if (gate_kind < GT_GATE_NONE || gate_kind > GT_GATE_SIGMOID) return fail(GT_ERR_UNSUPPORTED, w + ": unknown gate");
    if ((gate_kind == GT_GATE_VECTOR || (gate_kind != GT_GATE_NONE && n > 0)) && !gate)
        return fail(GT_ERR_INVALID_ARG, w + ": null gate");
    return GT_OK;
}

}  // namespace

extern "C" gt_status gt_block_norm_fwd(int64_t n, int32_t D, gt_dtype dt, int32_t norm, float eps, const void* x,
                                       float res_scale, const void* f, int32_t gate_kind, const void* gate,
                                       const float* w_post, const float* b_post, const float* w_pre,
                                       const float* b_pre, void* y, void* z, float* stats, hipStream_t s) {
    const char* who = "gt_block_norm_fwd";
    const gt_status st = norm_check(who, n, D, dt, norm, gate_kind, gate);
    if (st != GT_OK) return st;
    if (!(eps > 0.f)) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": eps must be positive");
    if (n == 0) return GT_OK;
    if (!x || !f || !y || !z || !stats) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    if (off16(stats)) return fail(GT_ERR_UNSUPPORTED, std::string(who) + ": stats must start at a multiple of 16 bytes");
    NormArgs a = {};
    a.far = n * D * (dt == GT_BF16 ? 2 : 4) > kFarBytes;
    a.n = n, a.D = D, a.norm = norm, a.gate_kind = gate_kind, a.eps = eps, a.res_scale = res_scale;
    a.x = x, a.f = f, a.gate = gate;
    a.w_post = w_post, a.b_post = b_post, a.w_pre = w_pre, a.b_pre = b_pre;
    a.y = y, a.z = z, a.stats = stats;
    const int E = dt == GT_BF16 ? 8 : 4, pieces = int(cdiv(D, E)), blocks = norm_blocks(n, D, dt);
    if (dt == GT_BF16) run_fwd<uint16_t>(a, pieces, blocks, s);
    else run_fwd<float>(a, pieces, blocks, s);
    GT_LAUNCH_CHECK("block_norm_fwd");
    return GT_OK;
}

extern "C" size_t gt_block_norm_bwd_workspace_size(int64_t n, int32_t D, gt_dtype dt) {
    if (n < 0 || D < 1 || D > kMaxD || (dt != GT_BF16 && dt != GT_F32)) return 0;
    Ws w(nullptr);
    w.take<float>(size_t(norm_blocks(n, D, dt)) * kSums * D);
    return w.size();
}

extern "C" gt_status gt_block_norm_bwd(int64_t n, int32_t D, gt_dtype dt, int32_t norm, const void* x,
                                       float res_scale, const void* f, int32_t gate_kind, const void* gate,
                                       const float* w_post, const float* b_post, const float* w_pre,
                                       const float* stats, const void* dy, const void* dz, void* dx, void* df,
                                       void* dgate, float* dw_post, float* db_post, float* dw_pre, float* db_pre,
                                       void* ws, size_t ws_bytes, hipStream_t s) {
    const char* who = "gt_block_norm_bwd";
    const gt_status st = norm_check(who, n, D, dt, norm, gate_kind, gate);
    if (st != GT_OK) return st;
    if (n > 0 && (!x || !f || !stats || !dy || !dz || !dx || !df || (gate_kind != GT_GATE_NONE && !dgate)))
        return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    if (gate_kind == GT_GATE_VECTOR && !dgate) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    if (off16(stats)) return fail(GT_ERR_UNSUPPORTED, std::string(who) + ": stats must start at a multiple of 16 bytes");
    const size_t need = gt_block_norm_bwd_workspace_size(n, D, dt);
    if (ws_bytes < need) return fail(GT_ERR_WORKSPACE, std::string(who) + ": workspace too small");
    if (need > 0 && !ws) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": null pointer");
    Ws w(ws);
    const int E = dt == GT_BF16 ? 8 : 4, pieces = int(cdiv(D, E)), blocks = norm_blocks(n, D, dt);
    NormArgs a = {};
    a.far = n * D * (dt == GT_BF16 ? 2 : 4) > kFarBytes;
    a.n = n, a.D = D, a.norm = norm, a.gate_kind = gate_kind, a.res_scale = res_scale;
    a.x = x, a.f = f, a.gate = gate, a.dy = dy, a.dz = dz;
    a.w_post = w_post, a.b_post = b_post, a.w_pre = w_pre;
    a.dx = dx, a.df = df, a.dgate = dgate;
    a.stats = const_cast<float*>(stats);
    a.part = w.take<float>(size_t(blocks) * kSums * D);
    SumOut o = {{dw_post, db_post, dw_pre, db_pre,
                 gate_kind == GT_GATE_VECTOR ? static_cast<float*>(dgate) : nullptr}};
    for (int k = 0; k < kSums; ++k)
        if (o.p[k]) a.want |= 1u << k;
    if (n > 0) {
        if (dt == GT_BF16) run_bwd<uint16_t>(a, pieces, blocks, s);
        else run_bwd<float>(a, pieces, blocks, s);
        GT_LAUNCH_CHECK("block_norm_bwd");
    }
    if (a.want) {
        k_norm_sum<<<dim3(unsigned(cdiv(D, 16)), kSums), 1024, 0, s>>>(blocks, D, a.part, o);
        GT_LAUNCH_CHECK("block_norm_bwd sum");
    }
    return GT_OK;
}
