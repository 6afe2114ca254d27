// Embedding: the scaled sum of one table row for each id of a token or node, and the
// table's gradient by sorted ids.
//
//   out_i = scale sum_f table[id_if],  dtable_r = scale sum of dout_i over the (i, f) with id_if = r.
//
// Both are bound by memory.  The forward gathers 16-byte pieces, one lane a piece of
// an output row.  The backward sorts the (id, row) pairs by id (stable, so a row's
// terms are added in the order of the tokens), finds each table row's run by binary
// search and sums it; every table row is written, the unused ones with zeros.  A run
// of more than kRun terms is cut: the sorted pairs go by chunks of kRun over the
// grid, each leaves the sums of the (at most two) long runs that it holds, and one
// workgroup a run and 64 columns adds those.  No atomics touch a sum: results are the
// same run to run.
#include "prim.h"
#include "rows.h"

using namespace gt;

namespace {

constexpr int kRun = 64;         // terms one group of lanes adds alone
constexpr int kMergeCols = 64;   // columns of a workgroup that adds partial sums
constexpr unsigned kMergeBlocks = 1024;

// Lanes that share a row: a power of two from 8 to 256.
int lanes_of(int64_t pieces) {
    int l = 8;
    while (l < pieces && l < 256) l *= 2;
    return l;
}

// The first column of a row's piece: the last one ends with the row, so that a width
// of any size goes in whole pieces (two lanes then write the same values there).
template <typename T>
__device__ __forceinline__ int piece_col(int p, int D) {
    constexpr int E = Piece<T>::E;
    return p * E + E <= D ? p * E : D - E;
}

template <typename T, bool ONE>
__global__ __launch_bounds__(256) void k_embed_fwd(int64_t n, int F, int64_t R, int D, bool wide, int lanes,
                                                    const void* ids, const T* table, float scale, T* out, bool far) {
    constexpr int E = Piece<T>::E;
    const int per = 256 / lanes;
    for (int64_t i = int64_t(blockIdx.x) * per + threadIdx.x / lanes; i < n; i += int64_t(gridDim.x) * per) {
        if (D < E) {  // rows of less than a piece, a column a lane
            const int c = threadIdx.x % lanes;
            if (c >= D) continue;
            float acc = 0.f;
            for (int f = 0; f < F; ++f) {
                const int64_t id = load_id(ids, wide, i * F + f, R);
                if (id >= 0) acc += load_one(table + id * D + c);
            }
            store_one(out + i * D + c, acc * scale);
            continue;
        }
        const int pieces = int(cdiv(D, E));
        for (int p = threadIdx.x % lanes; p < pieces; p += lanes) {
            const int c = piece_col<T>(p, D);
            float acc[E];
#pragma unroll
            for (int t = 0; t < E; ++t) acc[t] = 0.f;
            if constexpr (ONE) {
                const int64_t id = load_id(ids, wide, i, R);
                if (id >= 0) load_piece(acc, table + id * D + c);
            } else {
                constexpr int U = 4;  // table rows in flight
                for (int f = 0; f < F; f += U) {
                    int64_t id[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) id[u] = f + u < F ? load_id(ids, wide, i * F + f + u, R) : -1;
                    float v[U][E];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        if (id[u] >= 0) {
                            load_piece(v[u], table + id[u] * D + c);
                        } else {
#pragma unroll
                            for (int t = 0; t < E; ++t) v[u][t] = 0.f;
                        }
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u)
#pragma unroll
                        for (int t = 0; t < E; ++t) acc[t] += v[u][t];
                }
            }
#pragma unroll
            for (int t = 0; t < E; ++t) acc[t] *= scale;
            store_piece(out + i * D + c, acc, far);
        }
    }
}

__global__ __launch_bounds__(256) void k_embed_keys(int64_t pairs, int F, int64_t R, bool wide, const void* ids,
                                                     uint32_t* key, uint32_t* row) {
    const int64_t k = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (k >= pairs) return;
    const int64_t id = load_id(ids, wide, k, R);
    key[k] = uint32_t(id >= 0 ? id : R);  // behind the table: added to nothing
    row[k] = uint32_t(k / F);
}

// start[r] = the first sorted pair of table row r; long runs into a list (its order
// does not matter to any result).
__global__ __launch_bounds__(256) void k_embed_starts(int64_t pairs, int64_t R, const uint32_t* key, int32_t* start) {
    const int64_t r = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (r > R) return;
    int64_t lo = 0, hi = pairs;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (int64_t(key[mid]) < r) lo = mid + 1;
        else hi = mid;
    }
    start[r] = int32_t(lo);
}

__global__ __launch_bounds__(256) void k_embed_list(int64_t R, const int32_t* start, int32_t* list, uint32_t* count) {
    const int64_t r = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (r < R && start[r + 1] - start[r] > kRun) list[atomicAdd(count, 1u)] = int32_t(r);
}

// acc += the pieces at column c of the rows row[a..b)
template <typename T>
__device__ __forceinline__ void sum_rows(float (&acc)[Piece<T>::E], const T* dout, const uint32_t* row, int64_t a,
                                         int64_t b, int64_t step, int D, int c) {
    constexpr int E = Piece<T>::E, U = 4;
    int64_t k = a;
    for (; k + (U - 1) * step < b; k += U * step) {
        float v[U][E];
#pragma unroll
        for (int u = 0; u < U; ++u) load_piece(v[u], dout + int64_t(row[k + u * step]) * D + c);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int t = 0; t < E; ++t) acc[t] += v[u][t];
    }
    for (; k < b; k += step) {
        float v[E];
        load_piece(v, dout + int64_t(row[k]) * D + c);
#pragma unroll
        for (int t = 0; t < E; ++t) acc[t] += v[t];
    }
}

// Table rows of at most kRun terms.
template <typename T>
__global__ __launch_bounds__(256) void k_embed_rows(int64_t R, int D, int lanes, const int32_t* start,
                                                     const uint32_t* row, const T* dout, float scale, T* dtable,
                                                     bool far) {
    constexpr int E = Piece<T>::E;
    const int per = 256 / lanes;
    for (int64_t r = int64_t(blockIdx.x) * per + threadIdx.x / lanes; r < R; r += int64_t(gridDim.x) * per) {
        const int64_t a = start[r], b = start[r + 1];
        if (b - a > kRun) continue;
        if (D < E) {
            const int c = threadIdx.x % lanes;
            if (c >= D) continue;
            float acc = 0.f;
            for (int64_t k = a; k < b; ++k) acc += load_one(dout + int64_t(row[k]) * D + c);
            store_one(dtable + r * D + c, acc * scale);
            continue;
        }
        const int pieces = int(cdiv(D, E));
        for (int p = threadIdx.x % lanes; p < pieces; p += lanes) {
            const int c = piece_col<T>(p, D);
            float acc[E];
#pragma unroll
            for (int t = 0; t < E; ++t) acc[t] = 0.f;
            sum_rows(acc, dout, row, a, b, 1, D, c);
#pragma unroll
            for (int t = 0; t < E; ++t) acc[t] *= scale;
            store_piece(dtable + r * D + c, acc, far);
        }
    }
}

// The long runs' sums inside a chunk of kRun sorted pairs: of the run of its first
// pair (slot 0) and of its last (slot 1, if it is another).
template <typename T>
__global__ __launch_bounds__(256) void k_embed_chunks(int64_t pairs, int64_t R, int D, int lanes, const int32_t* start,
                                                       const uint32_t* key, const uint32_t* row, const T* dout,
                                                       float* part) {
    constexpr int E = Piece<T>::E;
    const int per = 256 / lanes;
    for (int64_t chunk = int64_t(blockIdx.x) * per + threadIdx.x / lanes; chunk * kRun < pairs;
         chunk += int64_t(gridDim.x) * per) {
        const int64_t e0 = chunk * kRun, e1 = e0 + kRun < pairs ? e0 + kRun : pairs;
        for (int s = 0; s < 2; ++s) {
            const int64_t r = key[s ? e1 - 1 : e0];
            if (r >= R || (s && r == int64_t(key[e0]))) continue;
            int64_t a = start[r], b = start[r + 1];
            if (b - a <= kRun) continue;
            a = a > e0 ? a : e0, b = b < e1 ? b : e1;
            float* o = part + (2 * chunk + s) * D;
            if (D < E) {
                const int c = threadIdx.x % lanes;
                if (c >= D) continue;
                float acc = 0.f;
                for (int64_t k = a; k < b; ++k) acc += load_one(dout + int64_t(row[k]) * D + c);
                o[c] = acc;
                continue;
            }
            const int pieces = int(cdiv(D, E));
            for (int p = threadIdx.x % lanes; p < pieces; p += lanes) {
                const int c = piece_col<T>(p, D);
                float acc[E];
#pragma unroll
                for (int t = 0; t < E; ++t) acc[t] = 0.f;
                sum_rows(acc, dout, row, a, b, 1, D, c);
#pragma unroll
                for (int t = 0; t < E; ++t) o[c + t] = acc[t];
            }
        }
    }
}

// The partial sums of each long run, added: 16 groups of lanes take every 16th chunk,
// then one adds the groups.
template <typename T>
__global__ __launch_bounds__(1024) void k_embed_merge(int D, const int32_t* start, const uint32_t* key,
                                                       const int32_t* list, const uint32_t* count, const float* part,
                                                       float scale, T* dtable) {
    constexpr int G = 1024 / kMergeCols;
    __shared__ float s_sum[G][kMergeCols];
    const int g = threadIdx.x / kMergeCols, col = threadIdx.x % kMergeCols, c = blockIdx.y * kMergeCols + col;
    const int64_t runs = *count;
    for (int64_t q = blockIdx.x; q < runs; q += gridDim.x) {
        const int64_t r = list[q];
        const int64_t a = start[r], b = start[r + 1];
        const int64_t first = a / kRun, last = (b - 1) / kRun;
        float acc = 0.f;
        if (c < D) {
#pragma unroll 4
            for (int64_t k = first + g; k <= last; k += G) {
                // slot 1 only where the chunk starts with another row
                const int64_t s = k == first && int64_t(key[k * kRun]) != r;
                acc += part[(2 * k + s) * D + c];
            }
        }
        s_sum[g][col] = acc;
        __syncthreads();
        if (g == 0 && c < D) {
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < G; ++k) sum += s_sum[k][col];
            store_one(dtable + r * D + c, sum * scale);
        }
        __syncthreads();
    }
}

struct BwdWs {
    uint32_t *key, *row, *count;
    int32_t *start, *list;
    SortTmp sort;
    float* part;
};
BwdWs bwd_ws(Ws& w, int64_t pairs, int64_t R, int32_t D) {
    BwdWs b;
    b.key = w.take<uint32_t>(size_t(pairs));
    b.row = w.take<uint32_t>(size_t(pairs));
    b.sort = sort_tmp(w, pairs, 4, true);
    b.start = w.take<int32_t>(size_t(R + 1));
    b.count = w.take<uint32_t>(1);
    b.list = w.take<int32_t>(size_t(pairs / kRun + 1));
    b.part = w.take<float>(size_t(pairs > kRun ? 2 * cdiv(pairs, kRun) : 0) * size_t(D));
    return b;
}

template <typename T>
gt_status run_bwd(int64_t n, int32_t F, int64_t R, int32_t D, bool wide, const void* ids, const void* dout_,
                  float scale, void* dtable_, BwdWs b, hipStream_t s) {
    const int64_t pairs = n * F;
    const T* dout = static_cast<const T*>(dout_);
    T* dtable = static_cast<T*>(dtable_);
    const int lanes = lanes_of(cdiv(D, Piece<T>::E)), per = 256 / lanes;
    const bool far = R * D * int64_t(sizeof(T)) > kFarBytes;
    if (pairs > 0) {
        k_embed_keys<<<unsigned(cdiv(pairs, 256)), 256, 0, s>>>(pairs, F, R, wide, ids, b.key, b.row);
        GT_LAUNCH_CHECK("embed_bwd keys");
        const gt_status st = radix_sort_u32(b.key, b.row, pairs, bits_for(R + 1), b.sort, s);
        if (st != GT_OK) return st;
    }
    k_embed_starts<<<unsigned(cdiv(R + 1, 256)), 256, 0, s>>>(pairs, R, b.key, b.start);
    GT_LAUNCH_CHECK("embed_bwd starts");
    k_embed_rows<T><<<grid_for(R, per), 256, 0, s>>>(R, D, lanes, b.start, b.row, dout, scale, dtable, far);
    GT_LAUNCH_CHECK("embed_bwd rows");
    if (pairs > kRun) {
        const gt_status st = fill_u32(b.count, 1, 0, s);
        if (st != GT_OK) return st;
        k_embed_list<<<unsigned(cdiv(R, 256)), 256, 0, s>>>(R, b.start, b.list, b.count);
        GT_LAUNCH_CHECK("embed_bwd list");
        const int64_t chunks = cdiv(pairs, kRun);
        k_embed_chunks<T><<<grid_for(chunks, per), 256, 0, s>>>(pairs, R, D, lanes, b.start, b.key, b.row, dout,
                                                                      b.part);
        GT_LAUNCH_CHECK("embed_bwd chunks");
        const int64_t most = chunks < R ? chunks : R;
        const dim3 grid(unsigned(most < kMergeBlocks ? most : kMergeBlocks), unsigned(cdiv(D, kMergeCols)));
        k_embed_merge<T><<<grid, 1024, 0, s>>>(D, b.start, b.key, b.list, b.count, b.part, scale, dtable);
        GT_LAUNCH_CHECK("embed_bwd merge");
    }
    return GT_OK;
}

bool embed_sizes(int64_t n, int32_t F, int64_t R, int32_t D) {
    const int64_t most = int64_t(1) << 31;
    return n >= 0 && n < most && F >= 1 && n * F < most && R >= 1 && R < most && D >= 1 &&
           D <= GT_MAX_WIDTH;
}
gt_status embed_check(const char* who, int64_t n, int32_t F, int64_t R, int32_t D, gt_dtype dt, gt_itype it) {
    if ((dt != GT_BF16 && dt != GT_F32) || (it != GT_I32 && it != GT_I64))
        return fail(GT_ERR_UNSUPPORTED, std::string(who) + ": unsupported dtype");
    if (!embed_sizes(n, F, R, D)) return fail(GT_ERR_INVALID_ARG, std::string(who) + ": n, F, R or D out of range");
    return GT_OK;
}

}  // namespace

extern "C" gt_status gt_embed_fwd(int64_t n, int32_t F, int64_t R, int32_t D, gt_dtype dt, gt_itype it,
                                  const void* ids, const void* table, float scale, void* out, hipStream_t s) {
    const gt_status st = embed_check("gt_embed_fwd", n, F, R, D, dt, it);
    if (st != GT_OK) return st;
    if (n == 0) return GT_OK;
    if (!ids || !table || !out) return fail(GT_ERR_INVALID_ARG, "gt_embed_fwd: null pointer");
    const int E = dt == GT_BF16 ? 8 : 4, lanes = lanes_of(cdiv(D, E));
    const unsigned grid = grid_for(n, 256 / lanes);
    const bool far = n * D * (dt == GT_BF16 ? 2 : 4) > kFarBytes, wide = it == GT_I64;
#define GT_CALL(T, ONE)                                                                                      \
    k_embed_fwd<T, ONE><<<grid, 256, 0, s>>>(n, F, R, D, wide, lanes, ids, static_cast<const T*>(table), scale, \
                                             static_cast<T*>(out), far)
    if (dt == GT_BF16) {
        if (F == 1) GT_CALL(uint16_t, true);
        else GT_CALL(uint16_t, false);
    } else {
        if (F == 1) GT_CALL(float, true);
        else GT_CALL(float, false);
    }
#undef GT_CALL
    GT_LAUNCH_CHECK("embed_fwd");
    return GT_OK;
}

extern "C" size_t gt_embed_bwd_workspace_size(int64_t n, int32_t F, int64_t R, int32_t D, gt_dtype dt) {
    if (!embed_sizes(n, F, R, D) || (dt != GT_BF16 && dt != GT_F32)) return 0;
    Ws w(nullptr);
    bwd_ws(w, n * F, R, D);
    return w.size();
}

extern "C" gt_status gt_embed_bwd(int64_t n, int32_t F, int64_t R, int32_t D, gt_dtype dt, gt_itype it,
                                  const void* ids, const void* dout, float scale, void* dtable, void* ws,
                                  size_t ws_bytes, hipStream_t s) {
    const gt_status st = embed_check("gt_embed_bwd", n, F, R, D, dt, it);
    if (st != GT_OK) return st;
    if (!dtable || !ws || (n > 0 && (!ids || !dout))) return fail(GT_ERR_INVALID_ARG, "gt_embed_bwd: null pointer");
    if (ws_bytes < gt_embed_bwd_workspace_size(n, F, R, D, dt))
        return fail(GT_ERR_WORKSPACE, "gt_embed_bwd: workspace too small");
    Ws w(ws);
    const BwdWs b = bwd_ws(w, n * F, R, D);
    if (dt == GT_BF16) return run_bwd<uint16_t>(n, F, R, D, it == GT_I64, ids, dout, scale, dtable, b, s);
    return run_bwd<float>(n, F, R, D, it == GT_I64, ids, dout, scale, dtable, b, s);
}
