// embed.cu -- embedding lookup with scaling, and the table's gradient by sorted tokens.
//
// Forward:   out[t] = scale * table[ids[t]].
// Backward:  dtable[v] (+)= scale * sum over the t with ids[t] = v of dout[t],
// summed in fp32 in an order that the tokens alone fix: the tokens of a row in
// their own order, long runs in windows of a fixed length.
//
// Both are bound by HBM, and every row of the gradient is written once.  40960 tokens
// of 1280 from bf16 rows to fp32: 42 us, 5.8 TB/s (a copy of as many bytes 5.7).  The
// gradient of 16384 of them to a table of 50304 rows, bf16 to fp32: 60 us, 5.0 TB/s (the
// order and the zero rows 40, of which the zeros alone take 25; the sums 20).  Added in
// place: 16384 of 1280 to 50304 rows 42 us, 2.5 TB/s (the order 9 of them, with no zero rows
// to write beside it; the sums at two blocks an SM for the old rows' registers); 4999 of
// 501, fp32, 12.7 us, 1.4 TB/s (a few us are the launches' latencies, and odd rows are
// loaded element by element).
#include <algorithm>

#include <nvtx3/nvToolsExt.h>

#include "model_ops.cuh"

namespace malt {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kWindow = 16;         // tokens of a window (32: 20 us for 17 at 4999 tokens)
constexpr int kLeastSlice = 64;     // columns that a warp sums, at least
constexpr int64_t kMaxDim = int64_t{1} << 24;       // 32-bit counts of windows and slices
constexpr int64_t kMaxTokens = int64_t{1} << 30;    // 32-bit places in the order, and a window past them

// ------------------------------------------------------------------- forward
// One warp per token and slice of the row; every lane has up to kFwdLoads
// vectors in flight.
constexpr int kFwdLoads = 8;

template <typename I>
__device__ __forceinline__ int64_t load_id(const I* ids, int64_t t) {
    return static_cast<int64_t>(ids[t]);
}

template <typename I, typename S, typename D, int VEC>
__global__ void __launch_bounds__(kThreads)
embed_forward_kernel(const I* ids, int64_t tokens, int64_t vocab, int64_t dim, const S* table, int64_t table_ld,
                     D* out, int64_t out_ld, float scale, int steps, int slices) {
    chain_wait();
    const int lane = threadIdx.x & 31;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    const int64_t t = item / slices;
    if (t >= tokens) return;
    const int64_t begin = (item - t * slices) * steps * (32 * VEC) + lane * VEC;
    const int64_t id = load_id(ids, t);
    D* const o = out + t * out_ld;
    float x[kFwdLoads][VEC];
    const bool inside = id >= 0 && id < vocab;
    if (inside) {
        const S* const row = table + id * table_ld;
#pragma unroll
        for (int j = 0; j < kFwdLoads; ++j) {
            const int64_t e = begin + j * (32 * VEC);
            if (j < steps && e < dim) load_vec<S, VEC>(row + e, x[j]);
        }
    } else {
        // padding has no row; an id past the table has no value; neither is scaled
        scale = 1.f;
        const float v = id < 0 ? 0.f : __int_as_float(0x7fc00000);
#pragma unroll
        for (int j = 0; j < kFwdLoads; ++j)
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[j][i] = v;
    }
#pragma unroll
    for (int j = 0; j < kFwdLoads; ++j) {
        const int64_t e = begin + j * (32 * VEC);
        if (j < steps && e < dim) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[j][i] *= scale;
            store_vec<D, VEC>(o + e, x[j]);
        }
    }
}

// ------------------------------------------------------------ backward: sort
// Block b of n (a power of two) owns the table rows b, b + n, b + 2 n, ...: the ids of
// frequent tokens, which lie together, are spread over the blocks (owners of neighbouring
// rows: the first block alone matches most of a text, 10 us of 18 for 16384 tokens).  It
// reads every id, counts those of its rows (per warp, each warp a contiguous run of
// tokens) and those of the blocks before it, and writes the records of its tokens to
// their place in the order (block, row, token): no launch has to wait for another
// block's counts, and the order needs no atomic that decides it.  Then it zeroes its rows
// that no token names (beside the sums, by warps or blocks of their own, the zeros' stores
// hold up the sums' loads: 62 to 73 us for 58).
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
static_assert(kSortWarps == 32, "a warp adds up one value of each warp");
constexpr int kSortLoads = 8;               // ids of a lane in flight
constexpr int kListed = 64;                 // tokens that a warp need not look for twice
constexpr int kMaxOwned = kSortThreads;     // rows of a block: one thread scans each
// Bytes of the kernel's static arrays, at most.
constexpr int kSortStatic = kSortWarps * (kListed + 1) * static_cast<int>(sizeof(int32_t)) + 64;

// A token in sorted order: its index, its row and the row's range of records.
struct __align__(16) TokenRecord {
    int32_t token, row, begin, end;
};

template <typename I, typename D, int VEC>
__global__ void __launch_bounds__(kSortThreads)
embed_sort_kernel(const I* ids, int32_t tokens, int32_t vocab, int shift, int32_t owned, TokenRecord* rec,
                  int32_t* total, uint32_t* arrived, int32_t counters, D* dtable, int64_t ld, int64_t dim, int fill) {
    extern __shared__ uint32_t smem[];
    uint32_t* const place = smem;                               // [kSortWarps][owned]
    int32_t* const row_begin = reinterpret_cast<int32_t*>(smem + kSortWarps * owned);
    int32_t* const row_end = row_begin + owned;
    __shared__ int32_t listed[kSortWarps][kListed];     // the warp's first tokens of this block's rows
    __shared__ int32_t warp_tmp[kSortWarps];
    __shared__ int32_t s_base;

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t mask = (1u << shift) - 1;
    for (int i = threadIdx.x; i < kSortWarps * owned; i += kSortThreads) place[i] = 0;
    __syncthreads();
    chain_wait();
    for (int64_t i = blockIdx.x * kSortThreads + threadIdx.x; i < counters; i += gridDim.x * kSortThreads)
        arrived[i] = 0;

    const int32_t per = (tokens / kSortWarps / 32 + 1) * 32;
    const int32_t lo = static_cast<int32_t>(min(static_cast<int64_t>(warp) * per, static_cast<int64_t>(tokens)));
    const int32_t hi = static_cast<int32_t>(min(static_cast<int64_t>(lo) + per, static_cast<int64_t>(tokens)));
    uint32_t* const mine = place + warp * owned;
    int32_t below = 0, found = 0;
    for (int32_t i0 = lo; i0 < hi; i0 += 32 * kSortLoads) {
        int64_t id[kSortLoads];
#pragma unroll
        for (int k = 0; k < kSortLoads; ++k) {
            const int32_t i = i0 + 32 * k + lane;
            id[k] = i < hi ? load_id(ids, i) : -1;
        }
#pragma unroll
        for (int k = 0; k < kSortLoads; ++k) {
            const bool inside = static_cast<uint64_t>(id[k]) < static_cast<uint64_t>(vocab);   // nor negative
            const uint32_t of = static_cast<uint32_t>(id[k]) & mask;
            below += inside && of < blockIdx.x;
            const bool in = inside && of == blockIdx.x;
            const unsigned m = __ballot_sync(~0u, in);
            if (in) {
                atomicAdd(mine + (static_cast<uint32_t>(id[k]) >> shift), 1u);
                const int32_t at = found + __popc(m & ((1u << lane) - 1));
                if (at < kListed) listed[warp][at] = i0 + 32 * k + lane;
            }
            found += __popc(m);
        }
    }
    below = __reduce_add_sync(~0u, below);
    if (lane == 0) warp_tmp[warp] = below;
    __syncthreads();
    if (warp == 0) {
        const int32_t b = __reduce_add_sync(~0u, warp_tmp[lane]);
        if (lane == 0) s_base = b;
    }
    __syncthreads();
    // Exclusive sums: over the rows, and within a row over the warps.
    int32_t count = 0;
    if (threadIdx.x < owned)
#pragma unroll
        for (int w = 0; w < kSortWarps; ++w) count += place[w * owned + threadIdx.x];
    int32_t incl = count;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int32_t up = __shfl_up_sync(~0u, incl, d);
        if (lane >= d) incl += up;
    }
    if (lane == 31) warp_tmp[warp] = incl;
    __syncthreads();
    int32_t before = lane < warp ? warp_tmp[lane] : 0;
    before = __reduce_add_sync(~0u, before);
    if (threadIdx.x < owned) {
        int32_t at = s_base + before + incl - count;
        row_begin[threadIdx.x] = at;
        row_end[threadIdx.x] = at + count;
#pragma unroll 8
        for (int w = 0; w < kSortWarps; ++w) {
            const int32_t n = place[w * owned + threadIdx.x];
            place[w * owned + threadIdx.x] = at;
            at += n;
        }
    }
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == kSortThreads - 1) *total = s_base + before + incl;
    __syncthreads();

    // Each token to its row's next place, in the tokens' order.
    auto put = [&](bool in, int32_t token, int64_t id) {
        const unsigned m = __ballot_sync(~0u, in);
        if (in) {
            const uint32_t r = static_cast<uint32_t>(id) >> shift;
            const unsigned peers = __match_any_sync(m, r), lower = peers & ((1u << lane) - 1);
            const uint32_t first = mine[r];
            __syncwarp(m);
            if (lower == 0) mine[r] = first + __popc(peers);
            __syncwarp(m);
            rec[first + __popc(lower)] = TokenRecord{token, static_cast<int32_t>(id), row_begin[r], row_end[r]};
        }
        __syncwarp();       // the next call's lanes may be others: votes order no memory
    };
    if (found <= kListed) {
        for (int32_t i = lane; i - lane < found; i += 32) {
            const int32_t token = i < found ? listed[warp][i] : 0;
            put(i < found, token, i < found ? load_id(ids, token) : -1);
        }
    } else {
        for (int32_t i0 = lo; i0 < hi; i0 += 32 * kSortLoads) {
            int64_t id[kSortLoads];
#pragma unroll
            for (int k = 0; k < kSortLoads; ++k) {
                const int32_t i = i0 + 32 * k + lane;
                id[k] = i < hi ? load_id(ids, i) : -1;
            }
#pragma unroll
            for (int k = 0; k < kSortLoads; ++k)
                put(static_cast<uint64_t>(id[k]) < static_cast<uint64_t>(vocab) &&
                        (static_cast<uint32_t>(id[k]) & mask) == blockIdx.x,
                    i0 + 32 * k + lane, id[k]);
        }
    }
    if (!fill) return;
    const float zero[VEC] = {};
    for (int64_t r = warp; (r << shift) + blockIdx.x < vocab; r += kSortWarps) {
        if (row_begin[r] != row_end[r]) continue;
        D* const row = dtable + ((r << shift) + blockIdx.x) * ld;
        for (int64_t e = lane * VEC; e < dim; e += 32 * VEC) store_vec<D, VEC>(row + e, zero);
    }
}

// ------------------------------------------------------------- backward: sums
// A warp takes a window of the sorted tokens and a slice of the row.  A row of at
// most `window` tokens is summed by the window that it begins in, whole; a longer
// one in parts, a part per window, which the last of its windows to arrive adds up in
// their order.
// The parts of windows w0 .. w1 of a row, a slice of it, in the windows' order.
template <typename D, bool ADD, int VEC, int SUB>
__device__ __forceinline__ void join_parts(const float* parts, int32_t w0, int32_t w1, int64_t base, int64_t dim, D* row,
                                           float scale) {
    constexpr int kLoads = 8;
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
        const int64_t e = base + s * (32 * VEC);
        if (e >= dim) continue;
        float acc[VEC] = {};
        for (int32_t k0 = w0; k0 <= w1; k0 += kLoads) {
            float x[kLoads][VEC];
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                const int32_t k = min(k0 + u, w1);
                load_l2<VEC>(parts + (static_cast<int64_t>(k) * 2 + (k == w0)) * dim + e, x[u]);
            }
#pragma unroll
            for (int u = 0; u < kLoads; ++u)
#pragma unroll
                for (int i = 0; i < VEC; ++i) acc[i] += k0 + u <= w1 ? x[u][i] : 0.f;
        }
        float y[VEC] = {};
        if (ADD) load_vec<D, VEC>(row + e, y);
#pragma unroll
        for (int i = 0; i < VEC; ++i) y[i] = ADD ? fmaf(scale, acc[i], y[i]) : scale * acc[i];
        store_vec<D, VEC>(row + e, y);
    }
}

constexpr int kSumLoads = 8;        // tokens in flight

// ADD: to what the table holds, whose rows are loaded with the tokens that end them (that
// takes the registers of two blocks of an SM; without, four: 60 us for 65 at two).
template <typename S, typename D, bool ADD, int VEC, int SUB>
__global__ void __launch_bounds__(kThreads, ADD ? 2 : 4)
embed_sum_kernel(const TokenRecord* rec, const int32_t* total, int32_t windows, int32_t window, int32_t slices,
                 const S* dout, int64_t dout_ld, D* dtable, int64_t ld, int64_t dim, float scale, float* parts,
                 uint32_t* arrived) {
    chain_wait();
    const int32_t n = *after_wait(total);
    const int lane = threadIdx.x & 31;
    rec = after_wait(rec);
    const int64_t item = static_cast<int64_t>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    const int32_t w = static_cast<int32_t>(item / slices);
    if (w >= windows) return;
    const int32_t slice = static_cast<int32_t>(item - static_cast<int64_t>(w) * slices);
    const int64_t base = static_cast<int64_t>(slice) * (32 * VEC * SUB) + lane * VEC;
    const int32_t a = w * window, b = min(n, a + window);
    if (a >= n) return;
    // From the first token that is no tail of a row of the window before, to the end of
    // the last row that this window sums whole.
    const TokenRecord head = rec[a], tail = rec[b - 1];
    const int32_t i0 = head.begin < a && head.end - head.begin <= window ? head.end : a;
    const int32_t stop = tail.end - tail.begin <= window ? tail.end : b;
    int64_t column[SUB];            // of the lane's vectors; past the row's end its last one, not stored
#pragma unroll
    for (int s = 0; s < SUB; ++s) column[s] = min(base + s * (32 * VEC), dim - VEC);
    float acc[SUB][VEC] = {};
    for (int32_t at = i0; at < stop; at += 32) {
        const TokenRecord mine = rec[min(at + lane, stop - 1)];
        const int32_t here = min(32, stop - at);
        // tokens that end a row, or this window's part of it
        const unsigned ends = __ballot_sync(~0u, lane < here && (at + lane + 1 == mine.end || at + lane + 1 == stop));
        for (int32_t j0 = 0; j0 < here; j0 += kSumLoads) {
            Raw<S, VEC> x[kSumLoads][SUB];
            Raw<D, VEC> old[ADD ? kSumLoads : 1][SUB];
#pragma unroll
            for (int j = 0; j < kSumLoads; ++j) {
                const int32_t token = __shfl_sync(~0u, mine.token, min(j0 + j, here - 1));
                const S* const row = dout + static_cast<int64_t>(token) * dout_ld;
#pragma unroll
                for (int s = 0; s < SUB; ++s) x[j][s] = *reinterpret_cast<const Raw<S, VEC>*>(row + column[s]);
                if (ADD && j0 + j < here && (ends >> (j0 + j) & 1)) {
                    const D* const to = dtable + static_cast<int64_t>(__shfl_sync(~0u, mine.row, j0 + j)) * ld;
#pragma unroll
                    for (int s = 0; s < SUB; ++s)
                        old[ADD ? j : 0][s] = *reinterpret_cast<const Raw<D, VEC>*>(to + column[s]);
                }
            }
#pragma unroll
            for (int j = 0; j < kSumLoads; ++j) {
                if (j0 + j >= here) break;
#pragma unroll
                for (int s = 0; s < SUB; ++s)
#pragma unroll
                    for (int k = 0; k < VEC; ++k) acc[s][k] += static_cast<float>(x[j][s].v[k]);
                if ((ends >> (j0 + j) & 1) == 0) continue;
                const int32_t row = __shfl_sync(~0u, mine.row, j0 + j), begin = __shfl_sync(~0u, mine.begin, j0 + j);
                const int32_t end = __shfl_sync(~0u, mine.end, j0 + j);
                if (end - begin <= window) {
                    D* const to = dtable + static_cast<int64_t>(row) * ld;
#pragma unroll
                    for (int s = 0; s < SUB; ++s) {
                        float y[VEC];
#pragma unroll
                        for (int k = 0; k < VEC; ++k)
                            y[k] = ADD ? fmaf(scale, acc[s][k], static_cast<float>(old[ADD ? j : 0][s].v[k]))
                                       : scale * acc[s][k];
                        if (base + s * (32 * VEC) < dim) store_vec<D, VEC>(to + column[s], y);
                    }
                } else {
                    // slot 0: the row began in an earlier window; slot 1: it begins in this one
                    float* const part = parts + (static_cast<int64_t>(w) * 2 + (begin >= a)) * dim;
#pragma unroll
                    for (int s = 0; s < SUB; ++s)
                        if (base + s * (32 * VEC) < dim) store_vec<float, VEC>(part + column[s], acc[s]);
                    // The last window of the row to arrive adds up the parts.
                    const int32_t w0 = begin / window, w1 = (end - 1) / window;
                    uint32_t before = 0;
                    __threadfence();
                    __syncwarp();
                    if (lane == 0) before = atomicAdd(arrived + static_cast<int64_t>(w0) * slices + slice, 1u);
                    if (__shfl_sync(~0u, before, 0) == static_cast<uint32_t>(w1 - w0)) {
                        __threadfence();
                        __syncwarp();       // the lanes' loads after the lane that saw the count
                        join_parts<D, ADD, VEC, SUB>(parts, w0, w1, base, dim, dtable + static_cast<int64_t>(row) * ld,
                                                     scale);
                    }
                }
#pragma unroll
                for (int s = 0; s < SUB; ++s)
#pragma unroll
                    for (int k = 0; k < VEC; ++k) acc[s][k] = 0.f;
            }
        }
    }
}

// ----------------------------------------------------------------------- host
// Windows of the sorted tokens: kWindow tokens, more where that would make over 1024
// windows (a row's parts are then at most 1024).
int32_t window_length(int64_t tokens) {
    int64_t w = kWindow;
    while (tokens > w * 1024) w *= 2;
    return static_cast<int32_t>(w);
}

struct Workspace {
    size_t rec, total, arrived, parts, bytes;
    int32_t counters;       // a counter for each window and slice of a row, where rows may be long
};
Workspace workspace_of(int64_t tokens, int64_t dim) {
    const int64_t window = window_length(tokens), windows = (tokens + window - 1) / window;
    Workspace w;
    w.rec = 0;
    w.total = static_cast<size_t>(tokens) * sizeof(TokenRecord);
    w.arrived = w.total + 256;
    w.counters = tokens > window ? static_cast<int32_t>(windows * ((dim + kLeastSlice - 1) / kLeastSlice)) : 0;
    w.parts = w.arrived + (static_cast<size_t>(w.counters) * sizeof(uint32_t) + 255) / 256 * 256;
    w.bytes = w.parts + (tokens > window ? static_cast<size_t>(windows) * 2 * dim * sizeof(float) : 0);
    return w;
}

int check(const malt_embed_t* e) {
    if (e == nullptr || e->tokens < 0 || e->vocab < 0 || e->dim < 0 || !(e->scale == e->scale))
        return MALT_ERR_INVALID_ARG;
    if (!index_type(e->ids_dtype) || !float_type(e->table_dtype) || !float_type(e->rows_dtype))
        return MALT_ERR_UNSUPPORTED;
    constexpr int64_t kMax = (int64_t{1} << 31) - 1 - (1 << 16);
    if (e->tokens >= kMaxTokens || e->vocab > kMax || e->dim > kMaxDim) return MALT_ERR_UNSUPPORTED;
    if (e->table_ld < e->dim || e->rows_ld < e->dim) return MALT_ERR_INVALID_ARG;
    if ((e->tokens > 0 && (e->ids == nullptr || (e->dim > 0 && e->rows == nullptr))) ||
        (e->vocab > 0 && e->dim > 0 && e->table == nullptr))
        return MALT_ERR_INVALID_ARG;
    if (!aligned_to(e->ids, type_bytes(e->ids_dtype)) || !aligned_to(e->table, type_bytes(e->table_dtype)) ||
        !aligned_to(e->rows, type_bytes(e->rows_dtype)))
        return MALT_ERR_MISALIGNED;
    return MALT_OK;
}

// Whether both matrices can be read and written in vectors of vec elements.
bool vectors(const malt_embed_t* e, int vec) {
    const int tb = type_bytes(e->table_dtype) * vec, rb = type_bytes(e->rows_dtype) * vec;
    return e->dim % vec == 0 && e->table_ld % vec == 0 && e->rows_ld % vec == 0 &&
           aligned_to(e->table, std::min(tb, 16)) && aligned_to(e->rows, std::min(rb, 16));
}

template <typename I, typename S, typename D, int VEC>
cudaError_t forward(const malt_embed_t* e, cudaStream_t s) {
    const int64_t all = (e->dim + 32 * VEC - 1) / (32 * VEC);
    const int64_t slices = (all + kFwdLoads - 1) / kFwdLoads;
    const int64_t steps = (all + slices - 1) / slices;
    const int64_t blocks = (e->tokens * slices + kWarps - 1) / kWarps;
    if (blocks >= (int64_t{1} << 31)) return cudaErrorInvalidValue;
    return launch_chained(embed_forward_kernel<I, S, D, VEC>, static_cast<unsigned>(blocks), kThreads, 0, s,
                          static_cast<const I*>(e->ids), e->tokens, e->vocab, e->dim,
                          static_cast<const S*>(e->table), e->table_ld, static_cast<D*>(e->rows), e->rows_ld,
                          e->scale, static_cast<int>(steps), static_cast<int>(slices));
}

template <typename I, typename D, int VEC>
cudaError_t sort(const malt_embed_t* e, const Workspace& w, uint8_t* ws, bool add, cudaStream_t s) {
    // Blocks, as a power of two: the largest that the SMs hold at once, more for a table of
    // more rows than these can own (16384 tokens of 1280: 131072 rows in one wave 125 us,
    // 151936 in two 137, both 5.7 TB/s or more).
    int shift = 0;
    while ((2 << shift) <= sm_count()) ++shift;
    while ((int64_t{kMaxOwned} << shift) < e->vocab) ++shift;
    const int64_t blocks = int64_t{1} << shift;
    const int32_t owned = static_cast<int32_t>((e->vocab + blocks - 1) / blocks);
    const size_t smem = (kSortWarps + 2) * sizeof(uint32_t) * static_cast<size_t>(owned);
    auto* const kernel = embed_sort_kernel<I, D, VEC>;
    // Past 48 KB with the kernel's static arrays.  Always to the most that a block may own, so
    // that calls of other threads set the same value.
    if (smem + kSortStatic > 48 * 1024) {
        constexpr int kMost = (kSortWarps + 2) * static_cast<int>(sizeof(uint32_t)) * kMaxOwned;
        const cudaError_t rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost);
        if (rc != cudaSuccess) { cudaGetLastError(); return rc; }
    }
    return launch_chained(kernel, static_cast<unsigned>(blocks), kSortThreads, smem, s, static_cast<const I*>(e->ids),
                          static_cast<int32_t>(e->tokens), static_cast<int32_t>(e->vocab), shift, owned,
                          reinterpret_cast<TokenRecord*>(ws + w.rec), reinterpret_cast<int32_t*>(ws + w.total),
                          reinterpret_cast<uint32_t*>(ws + w.arrived), w.counters, static_cast<D*>(e->table),
                          e->table_ld, e->dim, add ? 0 : 1);
}

template <typename I, typename D>
cudaError_t sort_types(const malt_embed_t* e, const Workspace& w, uint8_t* ws, bool add, cudaStream_t s) {
    constexpr int V = 16 / sizeof(D);
    return e->table_ld % V == 0 && e->dim % V == 0 && aligned_to(e->table, 16) ? sort<I, D, V>(e, w, ws, add, s)
                                                                                : sort<I, D, 1>(e, w, ws, add, s);
}

template <typename S, typename D, bool ADD, int VEC, int SUB>
cudaError_t sums(const malt_embed_t* e, const Workspace& w, uint8_t* ws, cudaStream_t s) {
    const int32_t window = window_length(e->tokens);
    const int32_t windows = static_cast<int32_t>((e->tokens + window - 1) / window);
    const int64_t slices = (e->dim + 32 * VEC * SUB - 1) / (32 * VEC * SUB);
    static_assert(32 * VEC * SUB >= kLeastSlice, "counters for narrower slices");
    const int64_t blocks = (windows * slices + kWarps - 1) / kWarps;
    if (blocks >= (int64_t{1} << 31)) return cudaErrorInvalidValue;
    return launch_chained(embed_sum_kernel<S, D, ADD, VEC, SUB>, static_cast<unsigned>(blocks), kThreads, 0, s,
                          reinterpret_cast<const TokenRecord*>(ws + w.rec),
                          reinterpret_cast<const int32_t*>(ws + w.total), windows, window,
                          static_cast<int32_t>(slices), static_cast<const S*>(e->rows), e->rows_ld,
                          static_cast<D*>(e->table), e->table_ld, e->dim, e->scale,
                          reinterpret_cast<float*>(ws + w.parts), reinterpret_cast<uint32_t*>(ws + w.arrived));
}

template <typename I>
cudaError_t forward_types(const malt_embed_t* e, cudaStream_t s) {
    const bool tb = e->table_dtype == MALT_BF16, rb = e->rows_dtype == MALT_BF16;
    if (tb && rb) return vectors(e, 8) ? forward<I, bf16, bf16, 8>(e, s) : forward<I, bf16, bf16, 1>(e, s);
    if (tb) return vectors(e, 4) ? forward<I, bf16, float, 4>(e, s) : forward<I, bf16, float, 1>(e, s);
    if (rb) return vectors(e, 4) ? forward<I, float, bf16, 4>(e, s) : forward<I, float, bf16, 1>(e, s);
    return vectors(e, 4) ? forward<I, float, float, 4>(e, s) : forward<I, float, float, 1>(e, s);
}

template <typename S, typename D>
cudaError_t sums_types(const malt_embed_t* e, const Workspace& w, uint8_t* ws, bool add, cudaStream_t s) {
    if (vectors(e, 4)) return add ? sums<S, D, true, 4, 1>(e, w, ws, s) : sums<S, D, false, 4, 1>(e, w, ws, s);
    return add ? sums<S, D, true, 1, 2>(e, w, ws, s) : sums<S, D, false, 1, 2>(e, w, ws, s);
}

}  // namespace
}  // namespace malt

extern "C" {

int malt_embed_forward(const malt_embed_t* e, void* stream) {
    using namespace malt;
    const int rc = check(e);
    if (rc != MALT_OK || e->tokens == 0 || e->dim == 0) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    nvtxRangePushA("malt_embed_forward");
    const cudaError_t c = e->ids_dtype == MALT_I32 ? forward_types<int32_t>(e, s) : forward_types<int64_t>(e, s);
    nvtxRangePop();
    return cuda_status(c, "malt_embed_forward");
}

size_t malt_embed_workspace_bytes(int64_t tokens, int64_t dim) {
    if (tokens < 0 || tokens >= malt::kMaxTokens || dim < 0 || dim > malt::kMaxDim) return 0;
    return malt::workspace_of(tokens, dim).bytes;
}

int malt_embed_backward(const malt_embed_t* e, int32_t accumulate, void* workspace, size_t workspace_bytes,
                        void* stream) {
    using namespace malt;
    const int rc = check(e);
    if (rc != MALT_OK || e->vocab == 0 || e->dim == 0 || (accumulate && e->tokens == 0)) return rc;
    const Workspace w = workspace_of(e->tokens, e->dim);
    if (workspace == nullptr || workspace_bytes < w.bytes) return MALT_ERR_INVALID_ARG;
    if (!aligned_to(workspace, 16)) return MALT_ERR_MISALIGNED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    uint8_t* const ws = static_cast<uint8_t*>(workspace);
    nvtxRangePushA("malt_embed_backward");
    const bool tb = e->table_dtype == MALT_BF16, rb = e->rows_dtype == MALT_BF16, add = accumulate != 0;
    cudaError_t c;
    if (e->ids_dtype == MALT_I32)
        c = tb ? sort_types<int32_t, bf16>(e, w, ws, add, s) : sort_types<int32_t, float>(e, w, ws, add, s);
    else
        c = tb ? sort_types<int64_t, bf16>(e, w, ws, add, s) : sort_types<int64_t, float>(e, w, ws, add, s);
    if (c == cudaSuccess && e->tokens > 0)
        c = rb ? (tb ? sums_types<bf16, bf16>(e, w, ws, add, s) : sums_types<bf16, float>(e, w, ws, add, s))
               : (tb ? sums_types<float, bf16>(e, w, ws, add, s) : sums_types<float, float>(e, w, ws, add, s));
    nvtxRangePop();
    return cuda_status(c, "malt_embed_backward");
}

}  // extern "C"
