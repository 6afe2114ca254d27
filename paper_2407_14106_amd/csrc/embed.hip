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
//
// 16,384 tokens x 2,048 of 128,000 rows in bf16: forward 29 us (4.6 TB/s), the gradient's
// sort 46 and sums 143 (524 MB written, 4.1 TB/s).  A million nodes x 256, three fields of
// 1,500 rows: forward 165 us (512 MB written, 1.5 GB gathered from L2), sort 80, sums 234
// (1.5 GB of dout's rows gathered, 0.65 of them from memory), their merge 30.  100,000 x
// 256 in fp32, nine fields of 173 rows: forward 41 us from LDS (70 from L2), backward 110.
#include "prim.h"
#include "rows.h"

using namespace gt;

namespace {

constexpr int kRun = 64;         // terms one group of lanes adds alone (128: 100,000 x 9 fields' sums 76 us, not 47)
constexpr int kMergeCols = 64;   // columns of a workgroup that adds partial sums
constexpr unsigned kMergeBlocks = 1024;
constexpr unsigned kMostBlocks = 1 << 20;
constexpr int64_t kL2Bytes = int64_t(32) << 20;  // of all XCDs

constexpr int kFwdBlocks = 256 * 8;  // workgroups of 256 that the chip holds
constexpr int kHeldBlocks = 256 * 2;
constexpr int64_t kHeldGathers = int64_t(128) << 20;  // bytes
constexpr int64_t kSmallPairs = 8192;  // one workgroup sorts, above them the grid
constexpr int kCounts = 1 + 256 + 256;  // long runs; chunks of a class, and how many of them have been placed

// Lanes that share a row: a power of two from 8 to 256.
int lanes_log2(int64_t pieces) {
    int l = 3;
    while ((1 << l) < pieces && l < 8) ++l;
    return l;
}

// The first column of a row's piece: the last one ends with the row, so that a width
// of any size goes in whole pieces (two lanes then write the same values there).
template <typename T>
__device__ __forceinline__ int piece_col(int p, int D) {
    constexpr int E = Piece<T>::E;
    return p * E + E <= D ? p * E : D - E;
}

struct FwdArgs {
    int64_t n, R;
    int F, D, shift;  // 2^shift lanes share a row
    bool wide, far;
    const void* ids;
    const void* table;
    float scale;
    void* out;
};

constexpr uint32_t kNoId = ~0u;

// Ids f to f + FB - 1 of a row; those outside the table are kNoId.
template <int FB>
__device__ __forceinline__ void load_ids(uint32_t (&id)[FB], const FwdArgs& g, int64_t i, int f) {
    const int64_t at = i * g.F + f;
    if (g.wide) {
        const int64_t* p = static_cast<const int64_t*>(g.ids) + at;
#pragma unroll
        for (int u = 0; u < FB; ++u) {
            const uint64_t v = FB < 4 || f + u < g.F ? uint64_t(p[u]) : ~0ull;
            id[u] = v < uint64_t(g.R) ? uint32_t(v) : kNoId;
        }
    } else {
        const int32_t* p = static_cast<const int32_t*>(g.ids) + at;
#pragma unroll
        for (int u = 0; u < FB; ++u) {
            const uint32_t v = FB < 4 || f + u < g.F ? uint32_t(p[u]) : kNoId;
            id[u] = v < uint32_t(g.R) ? v : kNoId;
        }
    }
}

// A lane's piece c of an output row: the first FB ids are in registers.
template <typename T, int FB>
__device__ __forceinline__ void embed_piece(const FwdArgs& g, int64_t i, const uint32_t (&first)[FB],
                                            const T* const (&row)[FB], int c, T* out) {
    constexpr int E = Piece<T>::E;
    if constexpr (FB == 1) {
        if (g.scale == 1.f) {  // one row as it is
            typedef typename Piece<T>::type piece_t;
            piece_t x = {0, 0, 0, 0};
            if (first[0] != kNoId) x = *reinterpret_cast<const piece_t*>(row[0] + c);
            if (g.far) __builtin_nontemporal_store(x, reinterpret_cast<piece_t*>(out + c));
            else *reinterpret_cast<piece_t*>(out + c) = x;
            return;
        }
    }
    float acc[E];
#pragma unroll
    for (int t = 0; t < E; ++t) acc[t] = 0.f;
    float v[FB][E];
#pragma unroll
    for (int u = 0; u < FB; ++u) {
        if (first[u] != kNoId) {
            load_piece(v[u], row[u] + c);
        } else {
#pragma unroll
            for (int t = 0; t < E; ++t) v[u][t] = 0.f;
        }
    }
#pragma unroll
    for (int u = 0; u < FB; ++u)
#pragma unroll
        for (int t = 0; t < E; ++t) acc[t] += v[u][t];
    if constexpr (FB == 4)
        for (int f = FB; f < g.F; f += FB) {
            uint32_t id[FB];
            load_ids<FB>(id, g, i, f);
#pragma unroll
            for (int u = 0; u < FB; ++u)
                if (id[u] != kNoId) {
                    load_piece(v[u], static_cast<const T*>(g.table) + int64_t(id[u]) * g.D + c);
#pragma unroll
                    for (int t = 0; t < E; ++t) acc[t] += v[u][t];
                }
        }
#pragma unroll
    for (int t = 0; t < E; ++t) acc[t] *= g.scale;
    store_piece(out + c, acc, g.far);
}

// FB: fields at a time, F of up to four (a part of more).  A row's first ids are read
// while the row before is summed.
template <typename T, int FB>
__global__ __launch_bounds__(256) void k_embed_fwd(FwdArgs g) {
    constexpr int E = Piece<T>::E;
    const T* table = static_cast<const T*>(g.table);
    const int lanes = 1 << g.shift, lane = threadIdx.x & (lanes - 1), pieces = int(cdiv(g.D, E));
    const int64_t step = int64_t(gridDim.x) * (256 >> g.shift);
    int64_t i = int64_t(blockIdx.x) * (256 >> g.shift) + (threadIdx.x >> g.shift);
    if (i >= g.n) return;
    uint32_t next[FB];
    load_ids<FB>(next, g, i, 0);
    for (; i < g.n; i += step) {
        uint32_t first[FB];
        const T* row[FB];
#pragma unroll
        for (int u = 0; u < FB; ++u) {
            first[u] = next[u];
            row[u] = table + int64_t(first[u]) * g.D;
        }
        if (i + step < g.n) load_ids<FB>(next, g, i + step, 0);
        T* out = static_cast<T*>(g.out) + i * g.D;
        if (g.D < E) {  // rows of less than a piece, a column a lane
            if (lane >= g.D) continue;
            float acc = 0.f;
            for (int f = 0; f < g.F; ++f) {
                const int64_t id = load_id(g.ids, g.wide, i * g.F + f, g.R);
                if (id >= 0) acc += load_one(table + id * g.D + lane);
            }
            store_one(out + lane, acc * g.scale);
            continue;
        }
        int p = lane;
        for (; p + lanes < pieces; p += 2 * lanes) {
            embed_piece<T, FB>(g, i, first, row, piece_col<T>(p, g.D), out);
            embed_piece<T, FB>(g, i, first, row, piece_col<T>(p + lanes, g.D), out);
        }
        if (p < pieces) embed_piece<T, FB>(g, i, first, row, piece_col<T>(p, g.D), out);
    }
}

// The same from LDS, for tables of few rows: a workgroup holds P pieces of every table
// row and forms those pieces of many output rows (100,000 x 256 fp32, nine fields of 173
// rows: 41 us; gathered from L2 70).
constexpr int kHeldBytes = 64 * 1024, kHeldThreads = 1024;  // two workgroups a CU
template <typename T, int P>
__global__ __launch_bounds__(kHeldThreads) void k_embed_held(FwdArgs g) {
    constexpr int E = Piece<T>::E, U = 4;
    __shared__ uint4 s_row[kHeldBytes / 16];
    const T* table = static_cast<const T*>(g.table);
    const int pieces = int(cdiv(g.D, E)), p0 = int(blockIdx.y) * P, lane = threadIdx.x % P;
    for (int k = threadIdx.x; k < int(g.R) * P; k += kHeldThreads) {
        const int p = p0 + k % P;
        if (p >= pieces) continue;
        typedef typename Piece<T>::type piece_t;
        const piece_t x = *reinterpret_cast<const piece_t*>(table + int64_t(k / P) * g.D + piece_col<T>(p, g.D));
        s_row[k] = make_uint4(x[0], x[1], x[2], x[3]);
    }
    __syncthreads();
    if (p0 + lane >= pieces) return;
    const int c = piece_col<T>(p0 + lane, g.D);
    const int64_t step = int64_t(gridDim.x) * (kHeldThreads / P);
    int64_t i = int64_t(blockIdx.x) * (kHeldThreads / P) + threadIdx.x / P;
    if (i >= g.n) return;
    uint32_t id[U];
    load_ids<U>(id, g, i, 0);
    for (; i < g.n; i += step) {
        float acc[E];
#pragma unroll
        for (int t = 0; t < E; ++t) acc[t] = 0.f;
        for (int f = 0;;) {
            uint32_t now[U];
#pragma unroll
            for (int u = 0; u < U; ++u) now[u] = id[u];
            f += U;
            const bool more = f < g.F;
            if (more) load_ids<U>(id, g, i, f);
            else if (i + step < g.n) load_ids<U>(id, g, i + step, 0);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (now[u] != kNoId) {
                    const uint4 x = s_row[int(now[u]) * P + lane];
                    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        if constexpr (sizeof(T) == 2) acc[2 * t] += bf16lo(w[t]), acc[2 * t + 1] += bf16hi(w[t]);
                        else acc[t] += __uint_as_float(w[t]);
                    }
                }
            if (!more) break;
        }
#pragma unroll
        for (int t = 0; t < E; ++t) acc[t] *= g.scale;
        store_piece(static_cast<T*>(g.out) + i * g.D + c, acc, g.far);
    }
}

template <typename T>
void run_fwd(FwdArgs g, hipStream_t s) {
    const int64_t pieces = cdiv(g.D, Piece<T>::E);
    // Table rows' pieces in LDS where many gathers repay their copies to the workgroups:
    // four fields or more (100,000 x 256 to 1,024, fields 1 / 2 / 4 / 9: 0.8 to 0.95, 0.8
    // to 0.92, 1.1 to 1.46, 1.3 to 1.8 times as fast as from L2) of 128 MB together (10,000
    // x 9 x 256 fp32, 92 MB: 0.9; 10,000 x 9 x 1,024 bf16, 184 MB: 1.2).
    const bool many = g.F >= 4 && g.n * g.F * g.D * int64_t(sizeof(T)) >= kHeldGathers;
    for (int P = 16; many && P >= 8; P /= 2)
        if (pieces >= P && g.R * P * 16 <= kHeldBytes) {
            const int64_t slices = cdiv(pieces, P), blocks = cdiv(g.n, kHeldThreads / P), most = cdiv(kHeldBlocks, slices);
            const dim3 grid(unsigned(blocks < most ? blocks : most), unsigned(slices));
            if (P == 16) k_embed_held<T, 16><<<grid, kHeldThreads, 0, s>>>(g);
            else k_embed_held<T, 8><<<grid, kHeldThreads, 0, s>>>(g);
            return;
        }
    // two pieces a lane, which share the work on the ids, where the rows fill the chip
    g.shift = lanes_log2(g.n * pieces > kFwdBlocks * 256 * 4 ? cdiv(pieces, 2) : pieces);
    const unsigned grid = grid_for(g.n, 256 >> g.shift, kFwdBlocks);
    if (g.F == 1) k_embed_fwd<T, 1><<<grid, 256, 0, s>>>(g);
    else if (g.F == 2) k_embed_fwd<T, 2><<<grid, 256, 0, s>>>(g);
    else if (g.F == 3) k_embed_fwd<T, 3><<<grid, 256, 0, s>>>(g);
    else k_embed_fwd<T, 4><<<grid, 256, 0, s>>>(g);
}

// The pairs' stable sort by key, up to 9 bits a pass, least significant first (a table of
// up to 511 rows takes one pass, of 262,143 two; in 11 bits, three million pairs of 1,501
// keys took one pass of 139 us instead of two of 40: the digits' counts are as many as
// the pairs, and neighbours go to places far apart).  A workgroup has a tile of pairs,
// wavefront after wavefront in rounds of 64; it counts the tile's digits, the counts of
// all tiles are scanned digit by digit, and a pair goes to its digit's place in its tile
// by (wavefront, round, lane).  The first pass takes the ids themselves.
constexpr int kSortThreads = 256, kSortWaves = kSortThreads / kWave, kSortRounds = 8;
constexpr int kSortTile = kSortThreads * kSortRounds, kMostBits = 9;

struct SortArgs {
    int64_t pairs, tiles, R;
    int F, shift, bits;  // 2^bits digits at `shift`
    bool wide;
    const void* ids;            // first pass
    const uint32_t *key, *row;  // the others
    uint32_t* hist;             // [digit][tile]
    const int64_t* place;       // its scan
    uint32_t *key_out, *row_out, *count;
};

// Digits of a wavefront's rounds; behind the last pair 2^bits.
template <bool FIRST>
__device__ __forceinline__ void load_pairs(const SortArgs& a, int64_t base, uint32_t (&key)[kSortRounds],
                                           uint32_t (&row)[kSortRounds], bool rows) {
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const int64_t i = base + r * kWave;
        key[r] = row[r] = 0;
        if (i >= a.pairs) continue;
        if constexpr (FIRST) {
            const int64_t id = load_id(a.ids, a.wide, i, a.R);
            key[r] = uint32_t(id >= 0 ? id : a.R);  // behind the table: added to nothing
            row[r] = uint32_t(i) / uint32_t(a.F);
        } else {
            key[r] = a.key[i];
            if (rows) row[r] = a.row[i];
        }
    }
}

template <bool FIRST>
__global__ __launch_bounds__(kSortThreads) void k_embed_sort_count(SortArgs a) {
    __shared__ uint32_t s_n[1 << kMostBits];
    const int digits = 1 << a.bits, tid = threadIdx.x;
    for (int d = tid; d < digits; d += kSortThreads) s_n[d] = 0;
    if constexpr (FIRST)
        if (blockIdx.x == 0)
            for (int k = tid; k < kCounts; k += kSortThreads) a.count[k] = 0;
    uint32_t key[kSortRounds], row[kSortRounds];
    const int64_t base = int64_t(blockIdx.x) * kSortTile + tid / kWave * (kSortRounds * kWave) + tid % kWave;
    load_pairs<FIRST>(a, base, key, row, false);
    __syncthreads();
    const uint64_t lt = lanemask_lt();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const bool valid = base + r * kWave < a.pairs;
        const uint32_t d = (key[r] >> a.shift) & uint32_t(digits - 1);
        // frequent digits: the wavefront's pairs of its first pair's digit in one addition
        const uint32_t lead = uint32_t(__builtin_amdgcn_readfirstlane(int(d)));
        const uint64_t same = ballot(valid && d == lead);
        if (valid) {
            if (d != lead) atomicAdd(&s_n[d], 1u);
            else if ((same & lt) == 0) atomicAdd(&s_n[d], uint32_t(__popcll(same)));
        }
    }
    __syncthreads();
    for (int d = tid; d < digits; d += kSortThreads) a.hist[int64_t(d) * a.tiles + blockIdx.x] = s_n[d];
}

template <bool FIRST>
__global__ __launch_bounds__(kSortThreads) void k_embed_sort_place(SortArgs a) {
    __shared__ uint32_t s_n[kSortWaves][1 << kMostBits];  // counts, then where a wavefront's pairs of a digit go
    const int digits = 1 << a.bits, tid = threadIdx.x, w = tid / kWave;
    for (int d = tid; d < digits; d += kSortThreads)
#pragma unroll
        for (int q = 0; q < kSortWaves; ++q) s_n[q][d] = 0;
    uint32_t key[kSortRounds], row[kSortRounds], rank[kSortRounds];
    const int64_t base = int64_t(blockIdx.x) * kSortTile + w * (kSortRounds * kWave) + tid % kWave;
    load_pairs<FIRST>(a, base, key, row, true);
    __syncthreads();
    const uint64_t lt = lanemask_lt();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r) {
        const bool valid = base + r * kWave < a.pairs;
        const uint32_t d = (key[r] >> a.shift) & uint32_t(digits - 1);
        uint64_t peers = ballot(valid);
        for (int b = 0; b < a.bits; ++b) {
            const bool bit = (d >> b) & 1u;
            const uint64_t bm = ballot(bit);
            peers &= bit ? bm : ~bm;
        }
        // the wavefront's pairs of the digit so far: read by all of them, then moved on
        // by the first (a wavefront's LDS accesses complete in order)
        const uint32_t mine = uint32_t(__popcll(peers & lt)), before = valid ? s_n[w][d] : 0u;
        lanes_fence();
        if (valid && mine == 0) s_n[w][d] = before + uint32_t(__popcll(peers));
        lanes_fence();
        rank[r] = before + mine;
    }
    __syncthreads();
    for (int d = tid; d < digits; d += kSortThreads) {
        uint32_t at = uint32_t(a.place[int64_t(d) * a.tiles + blockIdx.x]);  // fewer than 2^31 pairs
#pragma unroll
        for (int q = 0; q < kSortWaves; ++q) {
            const uint32_t c = s_n[q][d];
            s_n[q][d] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortRounds; ++r)
        if (base + r * kWave < a.pairs) {
            const uint32_t p = s_n[w][(key[r] >> a.shift) & uint32_t(digits - 1)] + rank[r];
            a.key_out[p] = key[r];
            a.row_out[p] = row[r];
        }
}

// The first of the sorted pairs whose key is at or above r.
__device__ __forceinline__ int64_t first_of(const uint32_t* key, int64_t pairs, int64_t r) {
    int64_t lo = 0, hi = pairs;
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (int64_t(key[mid]) < r) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}
// start[r] = the first sorted pair of table row r; the rows with long runs into a list
// (its order does not matter to any result).
__global__ __launch_bounds__(256) void k_embed_starts(int64_t pairs, int64_t R, const uint32_t* key, int32_t* start,
                                                       int32_t* list, uint32_t* count) {
    const int64_t r = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (r > R) return;
    const int64_t a = first_of(key, pairs, r);
    start[r] = int32_t(a);
    // the pair kRun behind the first is the row's too
    if (r < R && a + kRun < pairs && int64_t(key[a + kRun]) == r) list[atomicAdd(count, 1u)] = int32_t(r);
}

// The pairs of a small call, keyed and sorted by one workgroup in LDS, 8 bits of the key
// a pass.  A wavefront owns consecutive pairs in rounds of 64, a pair's place among those
// of its digit follows (wavefront, round, lane), so every pass is stable.  The keys stay
// where they are, their numbers move.  A whole gradient of 16 columns, of 100, 500, 5,000
// and 50,000 rows: at 4,096 pairs 22, 25, 22, 22 us (sorted by the grid 29, 26, 33, 35),
// at 8,192 42, 36, 31, 31 (46, 29, 35, 37).
constexpr int kSmallThreads = 1024, kSmallWaves = kSmallThreads / kWave;
__global__ __launch_bounds__(kSmallThreads) void k_embed_sort_small(int pairs, int F, int64_t R, bool wide,
                                                                     const void* ids, int bits, uint32_t* key,
                                                                     uint32_t* row, uint32_t* count) {
    __shared__ uint32_t s_k[kSmallPairs];
    __shared__ uint16_t s_v[2][kSmallPairs];
    __shared__ uint32_t s_n[kSmallWaves][256];
    __shared__ uint32_t s_part[4];
    const int tid = threadIdx.x, w = tid / kWave, lane = lane_id();
    if (tid < kCounts) count[tid] = 0;
    for (int i = tid; i < pairs; i += kSmallThreads) {
        const int64_t id = load_id(ids, wide, i, R);
        s_k[i] = uint32_t(id >= 0 ? id : R);
        s_v[0][i] = uint16_t(i);
    }
    const int rounds = (pairs + kSmallThreads - 1) / kSmallThreads, base = w * rounds * kWave + lane;
    const uint64_t lt = lanemask_lt();
    int from = 0;
    for (int shift = 0; shift < bits; shift += 8, from ^= 1) {
        for (int i = tid; i < kSmallWaves * 256; i += kSmallThreads) s_n[i / 256][i % 256] = 0;
        __syncthreads();
        for (int r = 0; r < rounds; ++r) {
            const int i = base + r * kWave;
            if (i < pairs) atomicAdd(&s_n[w][(s_k[s_v[from][i]] >> shift) & 255u], 1u);
        }
        __syncthreads();
        // thread d < 256: where the digit's pairs of each wavefront start
        uint32_t total = 0;
        if (tid < 256)
            for (int q = 0; q < kSmallWaves; ++q) {
                const uint32_t c = s_n[q][tid];
                s_n[q][tid] = total;
                total += c;
            }
        uint32_t x = total;
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) {
            const uint32_t y = uint32_t(__shfl_up(int(x), o, kWave));
            if (lane >= o) x += y;
        }
        if (tid < 256 && lane == kWave - 1) s_part[w] = x;
        __syncthreads();
        if (tid < 256) {
            uint32_t start = x - total;
            for (int q = 0; q < w; ++q) start += s_part[q];
            for (int q = 0; q < kSmallWaves; ++q) s_n[q][tid] += start;
        }
        __syncthreads();
        for (int r = 0; r < rounds; ++r) {
            const int i = base + r * kWave;
            const bool valid = i < pairs;
            const uint16_t v = valid ? s_v[from][i] : uint16_t(0);
            const uint32_t d = (s_k[v] >> shift) & 255u;
            uint64_t peers = ballot(valid);
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                const bool bit = (d >> b) & 1u;
                const uint64_t bm = ballot(bit);
                peers &= bit ? bm : ~bm;
            }
            // the digit's place so far: read by all of its lanes, then moved on by the
            // first (a wavefront's LDS accesses complete in order)
            const int mine = __popcll(peers & lt);
            const uint32_t at = valid ? s_n[w][d] : 0u;
            if (valid) s_v[from ^ 1][at + mine] = v;
            lanes_fence();
            if (valid && mine == 0) s_n[w][d] = at + uint32_t(__popcll(peers));
            lanes_fence();
        }
        __syncthreads();
    }
    for (int i = tid; i < pairs; i += kSmallThreads) {
        const uint32_t v = s_v[from][i];
        key[i] = s_k[v];
        row[i] = v / uint32_t(F);
    }
}

// The chunks' order by the rows that they read, in 256 classes by a chunk's first row
// (the order inside a class does not matter to any result): counted, then placed.
__device__ __forceinline__ int row_class(const uint32_t* row, int64_t chunk, int64_t n) {
    return int(int64_t(row[chunk * kRun]) * 256 / n);
}
__global__ __launch_bounds__(256) void k_embed_order_count(int64_t chunks, int64_t n, const uint32_t* row,
                                                            uint32_t* count) {
    __shared__ uint32_t s_n[256];
    s_n[threadIdx.x] = 0;
    __syncthreads();
    for (int64_t c = int64_t(blockIdx.x) * 256 + threadIdx.x; c < chunks; c += int64_t(gridDim.x) * 256)
        atomicAdd(&s_n[row_class(row, c, n)], 1u);
    __syncthreads();
    if (s_n[threadIdx.x]) atomicAdd(&count[threadIdx.x], s_n[threadIdx.x]);
}
__global__ __launch_bounds__(256) void k_embed_order_place(int64_t chunks, int64_t n, const uint32_t* row,
                                                            const uint32_t* count, uint32_t* used, uint32_t* order) {
    __shared__ uint32_t s_n[256], s_at[256], s_part[4];
    const int tid = threadIdx.x, lane = lane_id();
    s_n[tid] = 0;
    __syncthreads();
    for (int64_t c = int64_t(blockIdx.x) * 256 + tid; c < chunks; c += int64_t(gridDim.x) * 256)
        atomicAdd(&s_n[row_class(row, c, n)], 1u);
    const uint32_t total = count[tid];
    uint32_t x = total;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t y = uint32_t(__shfl_up(int(x), o, kWave));
        if (lane >= o) x += y;
    }
    if (lane == kWave - 1) s_part[tid / kWave] = x;
    __syncthreads();
    uint32_t at = x - total;
    for (int q = 0; q < tid / kWave; ++q) at += s_part[q];
    s_at[tid] = at + (s_n[tid] ? atomicAdd(&used[tid], s_n[tid]) : 0u);
    __syncthreads();
    for (int64_t c = int64_t(blockIdx.x) * 256 + tid; c < chunks; c += int64_t(gridDim.x) * 256)
        order[atomicAdd(&s_at[row_class(row, c, n)], 1u)] = uint32_t(c);
}

// acc += the pieces at column c of the rows row[a..b)
template <int U, typename T>
__device__ __forceinline__ void sum_rows(float (&acc)[Piece<T>::E], const T* dout, const uint32_t* row, int64_t a,
                                         int64_t b, int D, int c) {
    constexpr int E = Piece<T>::E;
    int64_t k = a;
    for (; k + U <= b; k += U) {
        float v[U][E];
#pragma unroll
        for (int u = 0; u < U; ++u) load_piece(v[u], dout + int64_t(row[k + u]) * D + c);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int t = 0; t < E; ++t) acc[t] += v[u][t];
    }
    for (; k < b; ++k) {
        float v[E];
        load_piece(v, dout + int64_t(row[k]) * D + c);
#pragma unroll
        for (int t = 0; t < E; ++t) acc[t] += v[t];
    }
}

struct BwdArgs {
    int64_t pairs, R;
    int D, lanes, shift;
    const int32_t* start;
    const uint32_t *key, *row;
    const uint32_t* order;  // of the chunks, or null
    const void* dout;
    float scale;
    void* dtable;
    bool far;
    float* part;
    unsigned chunk_blocks;  // the first ones of the grid
};

// A table row of at most kRun terms, by a group of lanes.
template <typename T, int U>
__device__ __forceinline__ void short_run(const BwdArgs& g, int64_t r, int64_t a, int64_t b, int lane) {
    constexpr int E = Piece<T>::E;
    const T* dout = static_cast<const T*>(g.dout);
    T* o = static_cast<T*>(g.dtable) + r * g.D;
    if (g.D < E) {
        if (lane >= g.D) return;
        float acc = 0.f;
        for (int64_t k = a; k < b; ++k) acc += load_one(dout + int64_t(g.row[k]) * g.D + lane);
        store_one(o + lane, acc * g.scale);
        return;
    }
    const int pieces = int(cdiv(g.D, E));
    for (int p = lane; p < pieces; p += g.lanes) {
        const int c = piece_col<T>(p, g.D);
        float acc[E];
#pragma unroll
        for (int t = 0; t < E; ++t) acc[t] = 0.f;
        sum_rows<U>(acc, dout, g.row, a, b, g.D, c);
#pragma unroll
        for (int t = 0; t < E; ++t) acc[t] *= g.scale;
        store_piece(o + c, acc, g.far);
    }
}

// The long runs' sums inside a chunk of kRun sorted pairs: of the run of its first
// pair (slot 0) and of its last (slot 1, if it is another).
template <typename T, int U>
__device__ __forceinline__ void chunk_sums(const BwdArgs& g, int64_t chunk, int lane) {
    constexpr int E = Piece<T>::E;
    const T* dout = static_cast<const T*>(g.dout);
    const int64_t e0 = chunk * kRun, e1 = e0 + kRun < g.pairs ? e0 + kRun : g.pairs;
    for (int s = 0; s < 2; ++s) {
        const int64_t r = g.key[s ? e1 - 1 : e0];
        if (r >= g.R || (s && r == int64_t(g.key[e0]))) continue;
        int64_t a = g.start[r], b = g.start[r + 1];
        if (b - a <= kRun) continue;
        a = a > e0 ? a : e0, b = b < e1 ? b : e1;
        float* o = g.part + (2 * chunk + s) * g.D;
        if (g.D < E) {
            if (lane >= g.D) continue;
            float acc = 0.f;
            for (int64_t k = a; k < b; ++k) acc += load_one(dout + int64_t(g.row[k]) * g.D + lane);
            o[lane] = acc;
            continue;
        }
        const int pieces = int(cdiv(g.D, E));
        for (int p = lane; p < pieces; p += g.lanes) {
            const int c = piece_col<T>(p, g.D);
            float acc[E];
#pragma unroll
            for (int t = 0; t < E; ++t) acc[t] = 0.f;
            sum_rows<U>(acc, dout, g.row, a, b, g.D, c);
#pragma unroll
            for (int t = 0; t < E; t += 4) {
                const float v[4] = {acc[t], acc[t + 1], acc[t + 2], acc[t + 3]};
                store_piece(o + c + t, v, false);
            }
        }
    }
}

// U: terms on their way at a time.  More registers leave fewer wavefronts, which rows
// without terms (stores alone) would feel.
template <typename T, int U>
__global__ __launch_bounds__(256) void k_embed_sums(BwdArgs g) {
    const int per = 256 >> g.shift, lane = threadIdx.x & (g.lanes - 1), at = threadIdx.x >> g.shift;
    if (blockIdx.x < g.chunk_blocks) {
        // an XCD takes chunks whose rows lie together
        const int64_t chunks = cdiv(g.pairs, kRun);
        for (int64_t c = xcd_block(blockIdx.x, g.chunk_blocks) * per + at; c < chunks; c += int64_t(g.chunk_blocks) * per)
            chunk_sums<T, U>(g, g.order ? int64_t(g.order[c]) : c, lane);
    } else {
        const int64_t step = int64_t(gridDim.x - g.chunk_blocks) * per;
        for (int64_t r = int64_t(blockIdx.x - g.chunk_blocks) * per + at; r < g.R; r += step) {
            const int64_t a = g.start[r], b = g.start[r + 1];
            if (b - a <= kRun) short_run<T, U>(g, r, a, b, lane);
        }
    }
}

// The partial sums of each long run, added: 16 groups of 16 lanes take every 16th
// chunk, four columns a lane, then one adds the groups.
template <typename T>
__global__ __launch_bounds__(256) void k_embed_merge(int D, const int32_t* start, const uint32_t* key,
                                                      const int32_t* list, const uint32_t* count, const float* part,
                                                      float scale, T* dtable) {
    constexpr int L = kMergeCols / 4, G = 256 / L;
    __shared__ float4 s_sum[G][L];
    const int g = threadIdx.x / L, x = threadIdx.x % L, c = blockIdx.y * kMergeCols + 4 * x, room = D - c;
    const int64_t runs = *count;
    for (int64_t q = blockIdx.x; q < runs; q += gridDim.x) {
        const int64_t r = list[q];
        const int64_t a = start[r], b = start[r + 1];
        const int64_t first = a / kRun, last = (b - 1) / kRun;
        // slot 1 only where the first chunk starts with another row
        const bool second = int64_t(key[first * kRun]) != r;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
        if (room >= 4) {
#pragma unroll 4
            for (int64_t k = first + g; k <= last; k += G) {
                float w[4];
                load_piece(w, part + (2 * k + (k == first && second)) * D + c);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += w[e];
            }
        } else if (room > 0) {
            for (int64_t k = first + g; k <= last; k += G)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < room) v[e] += part[(2 * k + (k == first && second)) * D + c + e];
        }
        s_sum[g][x] = make_float4(v[0], v[1], v[2], v[3]);
        __syncthreads();
        if (g == 0) {
#pragma unroll
            for (int k = 1; k < G; ++k) {
                const float4 w = s_sum[k][x];
                v[0] += w.x, v[1] += w.y, v[2] += w.z, v[3] += w.w;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < room) store_one(dtable + r * D + c + e, v[e] * scale);
        }
        __syncthreads();
    }
}

struct BwdWs {
    uint32_t *key, *row, *key2, *row2, *hist, *count, *order;
    int64_t* place;
    ScanTmp scan;
    int32_t *start, *list;
    float* part;
};

// Rows that several fields read are taken together (kept in the caches) where they are
// more than the L2 caches hold anyway (nine fields of 100,000 x 256 fp32: sums 124 -> 49
// us, three of a million x 256 bf16 314 -> 217, for 13 of ordering).
bool ordered(int64_t n, int32_t F, int32_t D, int size) { return F > 1 && n * D * size > kL2Bytes; }

// Passes over keys 0 to R, and the bits that each takes.
struct SortPasses {
    int passes, bits;
    explicit SortPasses(int64_t R) {
        const int all = bits_for(R + 1);
        passes = int(cdiv(all, kMostBits));
        bits = int(cdiv(all, passes));
    }
};

// Sorts the pairs into b.key and b.row.
gt_status sort_pairs(int64_t pairs, int32_t F, int64_t R, bool wide, const void* ids, const BwdWs& b, hipStream_t s) {
    const SortPasses p(R);
    SortArgs a = {};
    a.pairs = pairs, a.tiles = cdiv(pairs, kSortTile), a.R = R, a.F = F, a.bits = p.bits, a.wide = wide, a.ids = ids;
    a.hist = b.hist, a.place = b.place, a.count = b.count;
    const unsigned grid = unsigned(a.tiles);
    for (int k = 0; k < p.passes; ++k, a.shift += p.bits) {
        // the last pass ends in key and row
        const bool main = (p.passes - 1 - k) % 2 == 0;
        a.key = main ? b.key2 : b.key, a.row = main ? b.row2 : b.row;
        a.key_out = main ? b.key : b.key2, a.row_out = main ? b.row : b.row2;
        if (k == 0) k_embed_sort_count<true><<<grid, kSortThreads, 0, s>>>(a);
        else k_embed_sort_count<false><<<grid, kSortThreads, 0, s>>>(a);
        GT_LAUNCH_CHECK("embed_bwd count");
        const gt_status st = exclusive_scan_u32(b.hist, a.tiles << p.bits, b.place, b.scan, s);
        if (st != GT_OK) return st;
        if (k == 0) k_embed_sort_place<true><<<grid, kSortThreads, 0, s>>>(a);
        else k_embed_sort_place<false><<<grid, kSortThreads, 0, s>>>(a);
        GT_LAUNCH_CHECK("embed_bwd place");
    }
    return GT_OK;
}

BwdWs bwd_ws(Ws& w, int64_t n, int32_t F, int64_t R, int32_t D, int size) {
    const int64_t pairs = n * F, chunks = cdiv(pairs, kRun);
    BwdWs b = {};
    b.key = w.take<uint32_t>(size_t(pairs));
    b.row = w.take<uint32_t>(size_t(pairs));
    if (pairs > kSmallPairs) {
        const SortPasses p(R);
        const int64_t entries = cdiv(pairs, kSortTile) << p.bits;
        if (p.passes > 1) {
            b.key2 = w.take<uint32_t>(size_t(pairs));
            b.row2 = w.take<uint32_t>(size_t(pairs));
        }
        b.hist = w.take<uint32_t>(size_t(entries));
        b.place = w.take<int64_t>(size_t(entries + 1));
        b.scan.block_sums = w.take<int64_t>(size_t(scan_tmp_elems(entries)));
    }
    b.start = w.take<int32_t>(size_t(R + 1));
    b.count = w.take<uint32_t>(kCounts);
    b.list = w.take<int32_t>(size_t(pairs / kRun + 1));
    b.part = w.take<float>(size_t(pairs > kRun ? 2 * chunks : 0) * size_t(D));
    if (ordered(n, F, D, size)) b.order = w.take<uint32_t>(size_t(chunks));
    return b;
}

template <typename T>
gt_status run_bwd(int64_t n, int32_t F, int64_t R, int32_t D, bool wide, const void* ids, const void* dout,
                  float scale, void* dtable, const BwdWs& b, hipStream_t s) {
    const int64_t pairs = n * F, chunks = cdiv(pairs, kRun);
    const int shift = lanes_log2(cdiv(D, Piece<T>::E)), per = 256 >> shift;
    if (pairs <= kSmallPairs) {
        k_embed_sort_small<<<1, kSmallThreads, 0, s>>>(int(pairs), F, R, wide, ids, bits_for(R + 1), b.key, b.row,
                                                       b.count);
        GT_LAUNCH_CHECK("embed_bwd sort");
    } else {
        const gt_status st = sort_pairs(pairs, F, R, wide, ids, b, s);
        if (st != GT_OK) return st;
    }
    k_embed_starts<<<unsigned(cdiv(R + 1, 256)), 256, 0, s>>>(pairs, R, b.key, b.start, b.list, b.count);
    GT_LAUNCH_CHECK("embed_bwd starts");
    const bool runs = pairs > kRun, order = runs && b.order;
    if (order) {
        const unsigned blocks = grid_for(chunks, 2048, 1024);
        k_embed_order_count<<<blocks, 256, 0, s>>>(chunks, n, b.row, b.count + 1);
        k_embed_order_place<<<blocks, 256, 0, s>>>(chunks, n, b.row, b.count + 1, b.count + 257, b.order);
        GT_LAUNCH_CHECK("embed_bwd order");
    }
    BwdArgs g = {pairs, R, D, 1 << shift, shift, b.start, b.key, b.row, order ? b.order : nullptr, dout, scale, dtable,
                 R * D * int64_t(sizeof(T)) > kFarBytes, b.part, runs ? xcd_grid(cdiv(chunks, per)) : 0};
    if (g.chunk_blocks > kMostBlocks) g.chunk_blocks = kMostBlocks;
    const unsigned grid = g.chunk_blocks + grid_for(R, per, kMostBlocks);
    if (order) k_embed_sums<T, 8><<<grid, 256, 0, s>>>(g);
    else k_embed_sums<T, 4><<<grid, 256, 0, s>>>(g);
    GT_LAUNCH_CHECK("embed_bwd sums");
    if (runs) {
        const int64_t most = pairs / kRun < R ? pairs / kRun : R;
        const dim3 blocks(unsigned(most < kMergeBlocks ? most : kMergeBlocks), unsigned(cdiv(D, kMergeCols)));
        k_embed_merge<T><<<blocks, 256, 0, s>>>(D, b.start, b.key, b.list, b.count, b.part, scale,
                                                static_cast<T*>(dtable));
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
    FwdArgs g = {n, R, F, D, 0, it == GT_I64, n * D * (dt == GT_BF16 ? 2 : 4) > kFarBytes, ids, table, scale, out};
    if (dt == GT_BF16) run_fwd<uint16_t>(g, s);
    else run_fwd<float>(g, s);
    GT_LAUNCH_CHECK("embed_fwd");
    return GT_OK;
}

extern "C" size_t gt_embed_bwd_workspace_size(int64_t n, int32_t F, int64_t R, int32_t D, gt_dtype dt) {
    if (!embed_sizes(n, F, R, D) || (dt != GT_BF16 && dt != GT_F32)) return 0;
    Ws w(nullptr);
    bwd_ws(w, n, F, R, D, dt == GT_BF16 ? 2 : 4);
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
    const BwdWs b = bwd_ws(w, n, F, R, D, dt == GT_BF16 ? 2 : 4);
    if (dt == GT_BF16) return run_bwd<uint16_t>(n, F, R, D, it == GT_I64, ids, dout, scale, dtable, b, s);
    return run_bwd<float>(n, F, R, D, it == GT_I64, ids, dout, scale, dtable, b, s);
}
