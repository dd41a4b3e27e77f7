// distill.cu -- distillation from a teacher's top logits: loss, its gradient, and
// both in one pass.
//
// Per row with student logits s (all of the vocabulary) and the teacher's entries
// (idx_j, t_j), temperature tau and weight w:
//   p = softmax over the listed entries of t_j / tau,  q = softmax(s / tau),
//   loss = w tau^2 sum_j p_j (log p_j - log q[idx_j]),
//   d loss / d s_v = w tau (q_v - sum over j with idx_j = v of p_j).
// A row of weight 0, or one with no listed entry, has loss 0 and gradient 0
// whatever its logits hold.
//
// A thread block takes a row, or a cluster of blocks where there are few rows.  One
// sweep finds the row's maximum m and sum of 2^((s - m) c), c = log2(e) / tau, each
// thread with a running maximum over batches of vectors; the second writes the
// gradient and finds the row in L2.  One warp more takes the teacher's entries
// meanwhile.  Bound by HBM: the logits once, their gradient once.  8192 rows of 50304
// bf16 logits: 251 us, 6.26 TB/s of what has to move (loss alone 123 us, 6.7 TB/s;
// gradient alone 253 us, 6.5 TB/s).  Rows kept in shared memory instead, by blocks that
// stay and copy the next row meanwhile, took 276 us: a block's barriers then stand
// between its sweeps with no other block on the SM to fill them.
//
// An exponent s c - m c is one fused multiply-add of the rounded product m c, whose
// rounding is the same for every entry and is taken out of the sum again at its end.
// Where that product is so large that its rounding is no small exponent (a cold
// temperature, or a row of the type's lowest values, which is a uniform one) the
// difference is taken first.
#include <algorithm>
#include <cooperative_groups.h>

#include <nvtx3/nvToolsExt.h>

#include "model_ops.cuh"

namespace malt {
namespace {

constexpr int kMaxTop = 1024;
// Threads that sweep a row, blocks that an SM holds and vectors of a thread in flight.
// Wide: rows of both sweeps, few blocks, so that all their rows stay in L2 from the first
// sweep to the second (8192 rows of 50304 bf16: 251 us, medium 343).  Medium: single
// sweeps, and both sweeps of parts up to kMediumPart, whose blocks spend their time at
// barriers (16384 rows of 8192 bf16: 105 us, wide 175; 8000 of 16384 fp32: 218, wide
// 157).  Short and narrow: more rows at a time, for rows whose time is latency (16384 of
// 8192 bf16: short 88 us; 6000 of 16384: short 76, medium 68; 16384 of 4000: narrow 49,
// short 55; of 2000: narrow 35, 46 at 96 threads).
struct Shape {
    int threads, blocks, batch;
};
enum Width { kNarrow, kShort, kMedium, kWide };
__host__ __device__ constexpr Shape shape_of(int width) {
    return width == kNarrow ? Shape{64, 20, 4} : width == kShort ? Shape{128, 12, 4}
         : width == kMedium ? Shape{224, 7, 4} : Shape{480, 3, 5};
}
constexpr int64_t kNarrowRow = 9 * 1024, kShortRow = 17 * 1024, kMediumPart = 56 * 1024;
// Bytes of a row that one block takes, at most, in clusters of up to kSizeCluster.  With
// a forward sweep larger parts push one another out of L2 (2048 rows of 131072 bf16: two
// parts 198 us, one 233), smaller ones wait for one another.  The gradient alone waits
// for nothing, needs no clusters (104 us with them for 102), and small parts fill the
// last wave (1531 fp32 rows of 50257: 102 us at 70 KB, 104 at 140; 8192 bf16 rows of
// 50304: 253 and 264).  Clusters of 8 leave more SMs without one (300 fp32 rows of
// 150000: 88 us, 75 in fours).
constexpr int64_t kSweptPart = 140 * 1024, kWrittenPart = 70 * 1024;
constexpr int kSizeCluster = 4;
// While a row's blocks leave SMs idle: up to the largest portable cluster.
constexpr int kMaxCluster = 8;
constexpr float kLog2e = 1.4426950408889634f;

struct Params {
    const void* logits;
    int64_t ld;
    int64_t rows, vocab;
    const void* top_ids;
    const void* top_logits;
    int64_t top_ids_ld, top_logits_ld;
    int32_t top, ids_i64, top_bf16;
    const float* weight;
    float temperature;
    float* loss;                // forward
    float* stats;               // forward: written (may be null); gradient alone: read
    const float* dloss;         // gradient: d (the caller's value) / d loss, or null for 1
    void* dlogits;
    int64_t dlogits_ld;
    int32_t parts;              // blocks of a row: with a forward sweep a cluster
};

// Max and sum of 2^((x - max) c) of a set of values.
struct MaxSum {
    float m, s;
};
__device__ __forceinline__ float rescale(float from, float to, float c) {
    return from == to ? 1.f : exp2_fast((from - to) * c);      // equal infinities too
}
// Over the warp's lanes, each with its own.
__device__ __forceinline__ MaxSum warp_merge(MaxSum a, float c) {
    const float m = warp_max(a.m);
    return MaxSum{m, warp_sum(a.s * rescale(a.m, m, c))};
}
// Over n of them in shared memory, the same in every lane of a warp.
__device__ __forceinline__ MaxSum merge_all(const MaxSum* of, int n, float c) {
    const int lane = threadIdx.x & 31;
    float m = -INFINITY, s = 0.f;
    for (int k = lane; k < n; k += 32) m = fmaxf(m, of[k].m);
    m = warp_max(m);
    for (int k = lane; k < n; k += 32) s += of[k].s * rescale(of[k].m, m, c);
    return MaxSum{m, warp_sum(s)};
}

// One vector of logits (16 bytes) as pairs of fp32, and its largest entry.
template <typename T>
__device__ __forceinline__ f32x2 pair_of(const uint4& u, int i) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    if constexpr (sizeof(T) == 4) return pack2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    else return pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
template <typename T, int N>
__device__ __forceinline__ float largest(const uint4 (&u)[N]) {
    if constexpr (sizeof(T) == 4) {
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < N; ++i)
            m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(u[i].x), __uint_as_float(u[i].y)),
                               fmaxf(__uint_as_float(u[i].z), __uint_as_float(u[i].w))));
        return m;
    } else {
        auto h = [](uint32_t w) { return *reinterpret_cast<const __nv_bfloat162*>(&w); };
        __nv_bfloat162 m = h(u[0].x);
#pragma unroll
        for (int i = 0; i < N; ++i)
            m = __hmax2(m, __hmax2(__hmax2(h(u[i].x), h(u[i].y)), __hmax2(h(u[i].z), h(u[i].w))));
        return fmaxf(__low2float(m), __high2float(m));      // NaN only where all are
    }
}

// A product m c whose rounding (half an ulp, 2^-5 here at most) is a small exponent that
// the sum can be corrected by; past it, and past fp32's range, differences come first.
__device__ __forceinline__ bool in_range(float product) { return fabsf(product) < 0x1p20f; }

// Running maximum and sum of a thread, the sum in two halves relative to `ref`, the
// rounded product m c, or past the range to m c itself.
struct Running {
    float m = -INFINITY, ref = -INFINITY;
    f32x2 s = 0;
    __device__ __forceinline__ void raise(float to, float c) {
        if (!(to > m)) return;
        const float next = to * c;
        const bool was = in_range(ref), is = in_range(next);
        // Past the range the sum is relative to m c itself: on crossing, the rounding of the
        // side in range comes in.
        const float f = was && is ? exp2_fast(ref - next)
                                  : exp2_fast(fmaf(m - to, c, was ? -fmaf(m, c, -ref) : is ? fmaf(to, c, -next) : 0.f));
        s = mul2(s, pack2(f, f));       // from -inf: nothing summed yet, times 0
        m = to;
        ref = next;
    }
    template <typename T, int N>
    __device__ __forceinline__ void add(const uint4 (&u)[N], float c) {
        constexpr int kPairs = 8 / sizeof(T);
        raise(largest<T>(u), c);
        if (in_range(ref)) {
            const f32x2 cc = pack2(c, c), rr = pack2(-ref, -ref);
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int k = 0; k < kPairs; ++k) {
                    const float2 e = unpack2(fma2(pair_of<T>(u[i], k), cc, rr));
                    s = add2(s, pack2(exp2_fast(e.x), exp2_fast(e.y)));
                }
        } else {
            const float base = m == -INFINITY ? 0.f : m;        // nothing but -inf (or NaN) so far
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int k = 0; k < kPairs; ++k) {
                    const float2 x = unpack2(pair_of<T>(u[i], k));
                    s = add2(s, pack2(exp2_fast((x.x - base) * c), exp2_fast((x.y - base) * c)));
                }
        }
    }
    __device__ __forceinline__ void add1(float x, float c) {
        raise(x, c);
        const float base = m == -INFINITY ? 0.f : m;
        s = add2(s, pack2(in_range(ref) ? exp2_fast(fmaf(x, c, -ref)) : exp2_fast((x - base) * c), 0.f));
    }
    __device__ __forceinline__ MaxSum sum(float c) const {
        const float2 h = unpack2(s);
        return MaxSum{m, (h.x + h.y) * (in_range(ref) ? exp2_fast(-fmaf(m, c, -ref)) : 1.f)};
    }
};

// The teacher's entries of a row in shared memory, and what their softmax takes.
struct Top {
    int32_t* id;        // -1: not listed; filled up to a multiple of 4, aligned to 16 bytes
    float* t;           // teacher's logits, then log-probabilities
    float* x;           // student's logits
    float* p;           // probabilities
};
__host__ __device__ __forceinline__ int padded_top(int top) { return (top + 3) / 4 * 4; }
// One warp reads the entries of a row; those that do not count get id -1.
template <typename T>
__device__ __forceinline__ void list_entries(const Params& P, int64_t row, const Top& top) {
    const int lane = threadIdx.x & 31, padded = padded_top(P.top);
    for (int j = lane; j < padded; j += 32) {
        int64_t id = -1;
        float t[1] = {-INFINITY};
        if (j < P.top) {
            const int64_t id_at = row * P.top_ids_ld + j, at = row * P.top_logits_ld + j;
            id = P.ids_i64 ? static_cast<const int64_t*>(P.top_ids)[id_at]
                           : static_cast<const int32_t*>(P.top_ids)[id_at];
            if (P.top_bf16) load_vec<bf16, 1>(static_cast<const bf16*>(P.top_logits) + at, t);
            else load_vec<float, 1>(static_cast<const float*>(P.top_logits) + at, t);
        }
        const bool here = id >= 0 && id < P.vocab && t[0] != -INFINITY;     // a probability of 0 lists nothing
        top.id[j] = here ? static_cast<int32_t>(id) : -1;
        top.t[j] = here ? t[0] : -INFINITY;
    }
    __syncwarp();
}
// The student's logits of those in [begin, end).
template <typename T>
__device__ __forceinline__ void look_up(const Params& P, const T* x, int begin, int end, const Top& top) {
    for (int j = threadIdx.x & 31; j < P.top; j += 32) {
        float v[1] = {0.f};
        if (top.id[j] >= begin && top.id[j] < end) load_vec<T, 1>(x + top.id[j], v);
        top.x[j] = v[0];
    }
}

// Probabilities of a row's entries, by one warp; whether any is listed.
__device__ __forceinline__ int softmax_of(const Params& P, const Top& top, float inv_tau) {
    const int lane = threadIdx.x & 31;
    float max = -INFINITY, sum = 0.f;
    bool any = false;           // by the ids: the maximum passes NaN over
    for (int j = lane; j < P.top; j += 32) {
        max = fmaxf(max, top.t[j]);
        any |= top.id[j] >= 0;
    }
    max = warp_max(max);
    for (int j = lane; j < P.top; j += 32) {
        const float t = (top.t[j] - max) * inv_tau, e = top.id[j] >= 0 ? expf(t) : 0.f;
        top.t[j] = t;
        top.p[j] = e;
        sum += e;
    }
    sum = warp_sum(sum);
    const float log_t = logf(sum), f = 1.f / sum;
    for (int j = lane; j < P.top; j += 32) {
        top.t[j] -= log_t;
        top.p[j] *= f;
    }
    return __any_sync(~0u, any);
}

// Loss and statistics of a row, by one warp.
__device__ __forceinline__ void store_loss(const Params& P, int64_t row, float w, float inv_tau, const Top& top,
                                           const MaxSum& all) {
    const int lane = threadIdx.x & 31;
    const float log_q = logf(all.s);
    float l = 0.f;
    for (int j = lane; j < P.top; j += 32) {
        if (top.id[j] < 0) continue;
        const float p = top.p[j];
        if (p != 0.f) l += p * (top.t[j] - ((top.x[j] - all.m) * inv_tau - log_q));
    }
    l = warp_sum(l);
    if (lane == 0) {
        P.loss[row] = w * P.temperature * P.temperature * l;
        if (P.stats != nullptr) {
            P.stats[2 * row] = all.m;
            P.stats[2 * row + 1] = all.s;
        }
    }
}

// 16 bytes of results, which leave the logits' place in L2 alone; SAME: their address is
// a multiple of 16.
template <typename T, bool SAME, int VEC>
__device__ __forceinline__ void put(T* at, const float (&v)[VEC]) {
    if constexpr (SAME) {
        uint4 u;
        if constexpr (sizeof(T) == 4)
            u = make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        else
            u = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
        __stcs(reinterpret_cast<uint4*>(at), u);
    } else {
#pragma unroll
        for (int k = 0; k < VEC; ++k) {
            const float one[1] = {v[k]};
            store_vec<T, 1>(at + k, one);
        }
    }
}

// The gradient's term scale * q of a logit.
struct Gradient {
    float scale, f, ref, m, c;
    bool fast;
    __device__ __forceinline__ Gradient(float scale_, const MaxSum& all, float c_) : scale(scale_), m(all.m), c(c_) {
        ref = m * c;
        fast = in_range(ref);
        f = scale / all.s * (fast ? exp2_fast(-fmaf(m, c, -ref)) : 1.f);
    }
    __device__ __forceinline__ float at(float v) const {
        return f * (fast ? exp2_fast(fmaf(v, c, -ref)) : exp2_fast((v - m) * c));
    }
    template <typename T, bool SAME>
    __device__ __forceinline__ void store(const uint4& u, T* to) const {
        constexpr int VEC = 16 / sizeof(T);
        float v[VEC];
        if (fast) {
            const f32x2 cc = pack2(c, c), rr = pack2(-ref, -ref), ff = pack2(f, f);
#pragma unroll
            for (int k = 0; k < VEC / 2; ++k) {
                const float2 e = unpack2(fma2(pair_of<T>(u, k), cc, rr));
                const float2 g = unpack2(mul2(pack2(exp2_fast(e.x), exp2_fast(e.y)), ff));
                v[2 * k] = g.x;
                v[2 * k + 1] = g.y;
            }
        } else {
            unpack<T>(u, v);
#pragma unroll
            for (int k = 0; k < VEC; ++k) v[k] = at(v[k]);
        }
        put<T, SAME, VEC>(to, v);
    }
    template <typename T>
    __device__ __forceinline__ void store1(const T* from, T* to) const {
        float v[1];
        load_vec<T, 1>(from, v);
        v[0] = at(v[0]);
        store_vec<T, 1>(to, v);
    }
};

// The listed entries of [begin, end), written again with their target by `threads`
// threads.  An entry listed twice is written twice with the same sum.
template <typename T>
__device__ __forceinline__ void store_targets(const Params& P, const Gradient& g, const Top& top, int begin, int end,
                                              T* dx, int first, int threads) {
    for (int j = first; j < P.top; j += threads) {
        const int32_t id = top.id[j];
        if (id < begin || id >= end) continue;
        float p = 0.f;
        for (int k = 0; k < P.top; k += 4) {
            const int4 four = *reinterpret_cast<const int4*>(top.id + k);
            const float4 q = *reinterpret_cast<const float4*>(top.p + k);
            p += four.x == id ? q.x : 0.f;
            p += four.y == id ? q.y : 0.f;
            p += four.z == id ? q.z : 0.f;
            p += four.w == id ? q.w : 0.f;
        }
        const float v[1] = {g.at(top.x[j]) - g.scale * p};
        store_vec<T, 1>(dx + id, v);
    }
}

// A part of a row: where its vectors and the entries outside them lie.
template <typename T>
struct Part {
    static constexpr int VEC = 16 / sizeof(T);
    int begin, end;     // its entries
    int first;          // the first of its vectors' entries
    int odd;            // this thread's entry outside the row's vectors, or -1
    int count;          // its vectors
    // part of 2^shift
    __device__ __forceinline__ Part(const T* x, int vocab, int part, int shift, bool sweeps) {
        // Vectors start on 16-byte addresses: `lead` entries come before the first one.
        const int parts = 1 << shift;
        const int past = static_cast<int>(reinterpret_cast<uintptr_t>(x) % 16 / sizeof(T));
        const int lead = min(vocab, (VEC - past) % VEC);
        const int vectors = (vocab - lead) / VEC;
        const int v_begin = static_cast<int>(static_cast<int64_t>(vectors) * part >> shift);
        const int v_end = static_cast<int>(static_cast<int64_t>(vectors) * (part + 1) >> shift);
        begin = part == 0 ? 0 : lead + v_begin * VEC;
        end = part == parts - 1 ? vocab : lead + v_end * VEC;
        first = lead + v_begin * VEC;
        count = v_end - v_begin;
        // Fewer than 2 VEC entries of a row lie outside: one thread each.
        const int tail = lead + vectors * VEC, t = threadIdx.x;
        odd = -1;
        if (part == 0 && t < lead) odd = t;
        if (part == parts - 1 && t >= 32 && t - 32 < vocab - tail) odd = tail + t - 32;
        if (!sweeps) odd = -1;
    }
};

// FWD: loss (and statistics).  GRAD: gradient, from the statistics where FWD is
// false.  SAME: the gradient's rows start as far from a 16-byte boundary as the
// logits' (else it is stored element by element).  Threads 0 .. N-1 sweep the row, the
// warp after them takes the teacher's entries.
template <typename T, bool FWD, bool GRAD, bool SAME, int WIDTH>
__global__ void __launch_bounds__(shape_of(WIDTH).threads + 32, shape_of(WIDTH).blocks)
distill_kernel(const __grid_constant__ Params P) {
    static_assert(shape_of(WIDTH).threads >= 64, "a row's odd entries fall to threads 0..7 and 32..39");
    constexpr int N = shape_of(WIDTH).threads, kBatch = shape_of(WIDTH).batch;
    namespace cg = cooperative_groups;
    constexpr int VEC = 16 / sizeof(T), kWarps = N / 32, kAll = N + 32;
    __shared__ MaxSum of_warp[kWarps];
    __shared__ MaxSum of_block;
    __shared__ int listed;
    extern __shared__ uint4 entries[];      // the teacher's
    const cg::cluster_group cluster = cg::this_cluster();
    const int parts = FWD ? static_cast<int>(cluster.num_blocks()) : P.parts;
    const int part = FWD ? static_cast<int>(cluster.block_rank()) : static_cast<int>(blockIdx.x & (parts - 1));
    const int64_t row = blockIdx.x / parts;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool teacher = warp == kWarps;
    chain_wait();

    const T* const x = static_cast<const T*>(P.logits) + row * P.ld;
    T* const dx = GRAD ? static_cast<T*>(P.dlogits) + row * P.dlogits_ld : nullptr;
    const Part<T> here(x, static_cast<int>(P.vocab), part, 31 - __clz(parts), !teacher);
    const int begin = here.begin, end = here.end, odd = here.odd, count = here.count;
    const T* const xv = x + here.first;
    T* const dxv = GRAD ? dx + here.first : nullptr;

    const float w = P.weight != nullptr ? P.weight[row] : 1.f;
    const float up = GRAD && P.dloss != nullptr ? P.dloss[row] : 1.f;
    const float inv_tau = 1.f / P.temperature;
    const float c = kLog2e / P.temperature;
    const int padded = padded_top(P.top);
    float* const tops = reinterpret_cast<float*>(entries);
    const Top top{reinterpret_cast<int32_t*>(tops), tops + padded, tops + 2 * padded, tops + 3 * padded};
    bool on = w != 0.f && (FWD || up != 0.f);       // the same for every block of the row

    // The first batch is on its way before anything is known of the row.
    Running mine;
    uint4 u[kBatch];
    auto load = [&](int i) {        // past the part's end: entries of -inf
        constexpr uint32_t kNone = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
        const T* const at = xv + static_cast<int64_t>(i) * VEC;
#pragma unroll
        for (int k = 0; k < kBatch; ++k)
            u[k] = i + k * N < count ? *reinterpret_cast<const uint4*>(at + k * N * VEC)
                                     : make_uint4(kNone, kNone, kNone, kNone);
    };
    if (!teacher) load(threadIdx.x);
    if (teacher) {
        list_entries<T>(P, row, top);
        look_up(P, x, FWD ? 0 : begin, FWD ? static_cast<int>(P.vocab) : end, top);
        const int any = softmax_of(P, top, inv_tau);
        if (lane == 0) listed = any;
    }
    if (FWD && on && !teacher) {
        for (int i = threadIdx.x; i < count; i += kBatch * N) {
            if (i != threadIdx.x) load(i);
            mine.add<T>(u, c);
        }
        if (odd >= 0) {
            float v[1];
            load_vec<T, 1>(x + odd, v);
            mine.add1(v[0], c);
        }
        const MaxSum a = warp_merge(mine.sum(c), c);
        if (lane == 0) of_warp[warp] = a;
    }
    __syncthreads();
    on = on && listed != 0;
    if (!on) {      // the same for every block of the row
        if (FWD && part == 0 && threadIdx.x == 0) {
            P.loss[row] = 0.f;
            if (P.stats != nullptr) P.stats[2 * row] = P.stats[2 * row + 1] = 0.f;
        }
        if (GRAD) {
            const float zero[VEC] = {}, none[1] = {};
            if (odd >= 0) store_vec<T, 1>(dx + odd, none);
            for (int i = threadIdx.x; i < count; i += kAll)
                put<T, SAME, VEC>(dxv + static_cast<int64_t>(i) * VEC, zero);
        }
        return;
    }
    MaxSum all;
    if (FWD) {
        all = merge_all(of_warp, kWarps, c);
        if (parts > 1) {
            if (threadIdx.x == 0) of_block = all;
            cluster.sync();
            all = warp_merge(lane < parts ? *cluster.map_shared_rank(&of_block, lane) : MaxSum{-INFINITY, 0.f}, c);
            cluster.sync();         // no block leaves while another reads its part
        }
    } else {
        all = MaxSum{P.stats[2 * row], P.stats[2 * row + 1]};
    }

    if (FWD && part == 0 && teacher) store_loss(P, row, w, inv_tau, top, all);
    if (!GRAD) return;
    const Gradient g(w * up * P.temperature, all, c);
    if (!teacher) {
        for (int i = threadIdx.x; i < count; i += kBatch * N) {
            if (FWD || i != threadIdx.x) load(i);
            T* const to = dxv + static_cast<int64_t>(i) * VEC;
#pragma unroll
            for (int k = 0; k < kBatch; ++k)
                if (i + k * N < count) g.store<T, SAME>(u[k], to + k * N * VEC);
        }
        if (odd >= 0) g.store1(x + odd, dx + odd);
    }
    __syncthreads();
    store_targets(P, g, top, begin, end, dx, threadIdx.x, kAll);
}

// ----------------------------------------------------------------------- host
int check(const malt_distill_t* d) {
    if (d == nullptr || d->rows < 0 || d->vocab < 1 || d->top < 0 || !(d->temperature >= 1e-15f) ||
        !(d->temperature <= 1e15f))
        return MALT_ERR_INVALID_ARG;
    if (!float_type(d->dtype) || !float_type(d->top_dtype) || !index_type(d->ids_dtype)) return MALT_ERR_UNSUPPORTED;
    if (d->top > kMaxTop || d->rows >= (int64_t{1} << 27) || d->vocab >= (int64_t{1} << 31))
        return MALT_ERR_UNSUPPORTED;
    if (d->ld < d->vocab || d->top_ids_ld < d->top || d->top_logits_ld < d->top) return MALT_ERR_INVALID_ARG;
    if (d->rows > 0 && (d->logits == nullptr || (d->top > 0 && (d->top_ids == nullptr || d->top_logits == nullptr))))
        return MALT_ERR_INVALID_ARG;
    if (!aligned_to(d->logits, type_bytes(d->dtype)) || !aligned_to(d->top_ids, type_bytes(d->ids_dtype)) ||
        !aligned_to(d->top_logits, type_bytes(d->top_dtype)) || !aligned_to(d->weight, 4))
        return MALT_ERR_MISALIGNED;
    return MALT_OK;
}

// Shared memory of one row's entries.
int64_t entries_bytes(int64_t top) { return 16 * padded_top(static_cast<int>(top)); }

template <typename T, bool FWD, bool GRAD, int WIDTH>
cudaError_t launch_width(const malt_distill_t* d, Params P, int parts, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    P.parts = parts;
    auto past = [](const void* p) { return reinterpret_cast<uintptr_t>(p) % 16; };
    const bool same = !GRAD || (past(P.logits) == past(P.dlogits) && (P.ld - P.dlogits_ld) % V == 0);
    return launch_clusters(same ? distill_kernel<T, FWD, GRAD, true, WIDTH>
                                : distill_kernel<T, FWD, GRAD, !GRAD, WIDTH>,
                           static_cast<unsigned>(d->rows * parts), FWD ? parts : 1, shape_of(WIDTH).threads + 32,
                           entries_bytes(d->top), s, P);
}

template <typename T, bool FWD, bool GRAD>
cudaError_t launch(const malt_distill_t* d, const Params& P, cudaStream_t s) {
    const int64_t bytes = d->vocab * static_cast<int64_t>(sizeof(T)), part = FWD ? kSweptPart : kWrittenPart;
    int parts = 1;
    while (parts < kSizeCluster && bytes > parts * part) parts *= 2;
    // More while a row's blocks leave SMs idle and its parts keep a vector for each thread.
    while (parts < kMaxCluster && d->rows * parts < sm_count() &&
           bytes / (2 * parts) >= shape_of(kMedium).threads * 16)
        parts *= 2;
    // Short rows leave most of a wide block waiting for its barriers; a single sweep has
    // nothing to keep in L2.
    if (bytes <= kNarrowRow) return launch_width<T, FWD, GRAD, kNarrow>(d, P, parts, s);
    if (bytes <= kShortRow) return launch_width<T, FWD, GRAD, kShort>(d, P, parts, s);
    if constexpr (FWD && GRAD)
        if (bytes / parts > kMediumPart) return launch_width<T, FWD, GRAD, kWide>(d, P, parts, s);
    return launch_width<T, FWD, GRAD, kMedium>(d, P, parts, s);
}

Params params_of(const malt_distill_t* d) {
    Params P = {};
    P.logits = d->logits;
    P.ld = d->ld;
    P.rows = d->rows;
    P.vocab = d->vocab;
    P.top_ids = d->top_ids;
    P.top_logits = d->top_logits;
    P.top_ids_ld = d->top_ids_ld;
    P.top_logits_ld = d->top_logits_ld;
    P.top = static_cast<int32_t>(d->top);
    P.ids_i64 = d->ids_dtype == MALT_I64;
    P.top_bf16 = d->top_dtype == MALT_BF16;
    P.weight = d->weight;
    P.temperature = d->temperature;
    return P;
}

int check_gradient(const malt_distill_t* d, const void* dlogits, int64_t ld) {
    if (ld < d->vocab || (d->rows > 0 && dlogits == nullptr)) return MALT_ERR_INVALID_ARG;
    return aligned_to(dlogits, type_bytes(d->dtype)) ? MALT_OK : MALT_ERR_MISALIGNED;
}

template <bool FWD, bool GRAD>
int run(const malt_distill_t* d, const Params& P, void* stream, const char* name) {
    if (d->rows == 0) return MALT_OK;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    nvtxRangePushA(name);
    const cudaError_t c = d->dtype == MALT_BF16 ? launch<bf16, FWD, GRAD>(d, P, s) : launch<float, FWD, GRAD>(d, P, s);
    nvtxRangePop();
    return cuda_status(c, name);
}

}  // namespace
}  // namespace malt

extern "C" {

int malt_distill_forward(const malt_distill_t* d, float* loss, float* stats, void* stream) {
    using namespace malt;
    const int rc = check(d);
    if (rc != MALT_OK) return rc;
    if (d->rows > 0 && loss == nullptr) return MALT_ERR_INVALID_ARG;
    if (!aligned_to(loss, 4) || !aligned_to(stats, 4)) return MALT_ERR_MISALIGNED;
    Params P = params_of(d);
    P.loss = loss;
    P.stats = stats;
    return run<true, false>(d, P, stream, "malt_distill_forward");
}

int malt_distill_backward(const malt_distill_t* d, const float* stats, const float* dloss, void* dlogits,
                          int64_t dlogits_ld, void* stream) {
    using namespace malt;
    int rc = check(d);
    if (rc == MALT_OK) rc = check_gradient(d, dlogits, dlogits_ld);
    if (rc != MALT_OK) return rc;
    if (d->rows > 0 && stats == nullptr) return MALT_ERR_INVALID_ARG;
    if (!aligned_to(stats, 4) || !aligned_to(dloss, 4)) return MALT_ERR_MISALIGNED;
    Params P = params_of(d);
    P.stats = const_cast<float*>(stats);
    P.dloss = dloss;
    P.dlogits = dlogits;
    P.dlogits_ld = dlogits_ld;
    return run<false, true>(d, P, stream, "malt_distill_backward");
}

int malt_distill_forward_backward(const malt_distill_t* d, float* loss, float* stats, void* dlogits,
                                  int64_t dlogits_ld, void* stream) {
    using namespace malt;
    int rc = check(d);
    if (rc == MALT_OK) rc = check_gradient(d, dlogits, dlogits_ld);
    if (rc != MALT_OK) return rc;
    if (d->rows > 0 && loss == nullptr) return MALT_ERR_INVALID_ARG;
    if (!aligned_to(loss, 4) || !aligned_to(stats, 4)) return MALT_ERR_MISALIGNED;
    Params P = params_of(d);
    P.loss = loss;
    P.stats = stats;
    P.dlogits = dlogits;
    P.dlogits_ld = dlogits_ld;
    return run<true, true>(d, P, stream, "malt_distill_forward_backward");
}

}  // extern "C"
