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
// meanwhile.  Bound by HBM: the logits once, their gradient once.
//
// An exponent s c - m c is one fused multiply-add of the rounded product m c, whose
// rounding is the same for every entry and is taken out of the sum again at its end.
// Where that product leaves fp32's range (a row of the type's lowest values is a
// uniform one) the difference is taken first.
#include <algorithm>
#include <cooperative_groups.h>

#include <nvtx3/nvToolsExt.h>

#include "model_ops.cuh"

namespace malt {
namespace {

constexpr int kMaxTop = 1024;
constexpr int kWide = 512, kNarrow = 128;      // threads that sweep a row
constexpr int kBatch = 4;           // vectors of a thread in flight
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
};

// Max and sum of 2^((x - max) c) of a set of values.
struct MaxSum {
    float m, s;
};
__device__ __forceinline__ float rescale(float from, float to, float c) {
    return from == to ? 1.f : exp2_fast((from - to) * c);      // equal infinities too
}
__device__ __forceinline__ MaxSum merge(MaxSum a, MaxSum b, float c) {
    const float m = fmaxf(a.m, b.m);
    return MaxSum{m, a.s * rescale(a.m, m, c) + b.s * rescale(b.m, m, c)};
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

// The products that exponents are taken from stay far inside fp32's range.
__device__ __forceinline__ bool in_range(float product) { return fabsf(product) < 1e30f; }

// Running maximum and sum of a thread, the sum in two halves relative to `ref`, the
// rounded product m c.
struct Running {
    float m = -INFINITY, ref = -INFINITY;
    f32x2 s = 0;
    __device__ __forceinline__ void raise(float to, float c) {
        if (!(to > m)) return;
        const float next = to * c;
        const float f = in_range(ref) && in_range(next) ? exp2_fast(ref - next) : exp2_fast((m - to) * c);
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

// FWD: loss (and statistics).  GRAD: gradient, from the statistics where FWD is
// false.  SAME: the gradient's rows start as far from a 16-byte boundary as the
// logits' (else it is stored element by element).  Threads 0 .. N-1 sweep the row, the
// warp after them takes the teacher's entries.
template <typename T, bool FWD, bool GRAD, bool SAME, int N>
__global__ void __launch_bounds__(N + 32, N == kWide ? 3 : 10)
distill_kernel(const __grid_constant__ Params P) {
    namespace cg = cooperative_groups;
    constexpr int VEC = 16 / sizeof(T), kWarps = N / 32, kAll = N + 32;
    auto put = [](T* at, const float (&v)[VEC]) {
        if constexpr (SAME) {
            store_vec<T, VEC>(at, v);
        } else {
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                const float one[1] = {v[k]};
                store_vec<T, 1>(at + k, one);
            }
        }
    };
    __shared__ MaxSum of_warp[kWarps];
    __shared__ MaxSum of_block;
    __shared__ float t_max_s, t_sum_s;
    __shared__ int listed_s;
    __shared__ int32_t top_id[kMaxTop];
    __shared__ float top_p[kMaxTop];
    __shared__ float top_x[kMaxTop];
    const cg::cluster_group cluster = cg::this_cluster();
    const int parts = static_cast<int>(cluster.num_blocks()), part = static_cast<int>(cluster.block_rank());
    const int64_t row = blockIdx.x / parts;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const bool teacher = warp == kWarps;
    chain_wait();

    const T* const x = static_cast<const T*>(P.logits) + row * P.ld;
    T* const dx = GRAD ? static_cast<T*>(P.dlogits) + row * P.dlogits_ld : nullptr;
    // The row's parts start on vectors of its address: `lead` entries come before the
    // first one.
    const int64_t lead = min(P.vocab, static_cast<int64_t>((VEC - reinterpret_cast<uintptr_t>(x) / sizeof(T) % VEC) % VEC));
    const int64_t vectors = (P.vocab - lead) / VEC;
    const int64_t v_begin = vectors * part / parts, v_end = vectors * (part + 1) / parts;
    const int64_t begin = part == 0 ? 0 : lead + v_begin * VEC;
    const int64_t end = part == parts - 1 ? P.vocab : lead + v_end * VEC;
    const T* const xv = x + lead + v_begin * VEC;
    T* const dxv = GRAD ? dx + lead + v_begin * VEC : nullptr;
    const int count = static_cast<int>(v_end - v_begin);        // vectors of this part
    const int64_t tail = lead + vectors * VEC;      // first entry past the vectors
    // Entries outside the vectors (fewer than 2 VEC of a row): one thread each.
    int64_t odd = -1;
    if (part == 0 && threadIdx.x < lead) odd = threadIdx.x;
    if (part == parts - 1 && threadIdx.x >= 32 && tail + threadIdx.x - 32 < P.vocab) odd = tail + threadIdx.x - 32;
    if (teacher) odd = -1;

    const float w = P.weight != nullptr ? P.weight[row] : 1.f;
    const float up = GRAD && P.dloss != nullptr ? P.dloss[row] : 1.f;
    const float inv_tau = 1.f / P.temperature;
    const float c = kLog2e / P.temperature;
    bool on = w != 0.f && (FWD || up != 0.f);       // the same for every block of the row

    Running mine;
    if (on && teacher) {
        // The student's logits of the entries are read before any block of the row
        // writes its gradient, which may take their place.
        int listed = 0;
        float t_max = -INFINITY;
        for (int j = lane; j < P.top; j += 32) {
            const int64_t id_at = row * P.top_ids_ld + j, at = row * P.top_logits_ld + j;
            const int64_t id = P.ids_i64 ? static_cast<const int64_t*>(P.top_ids)[id_at]
                                         : static_cast<const int32_t*>(P.top_ids)[id_at];
            float t[1] = {-INFINITY}, v[1] = {0.f};
            if (id >= 0 && id < P.vocab) {
                if (P.top_bf16) load_vec<bf16, 1>(static_cast<const bf16*>(P.top_logits) + at, t);
                else load_vec<float, 1>(static_cast<const float*>(P.top_logits) + at, t);
            }
            const bool here = t[0] != -INFINITY;    // a probability of 0 lists nothing
            if (here) {
                listed = 1;
                if (FWD || (id >= begin && id < end)) load_vec<T, 1>(x + id, v);
            }
            top_id[j] = here ? static_cast<int32_t>(id) : -1;
            top_p[j] = t[0];
            top_x[j] = v[0];
            t_max = fmaxf(t_max, t[0]);
        }
        t_max = warp_max(t_max);
        float t_sum = 0.f;
        for (int j = lane; j < P.top; j += 32)
            if (top_id[j] >= 0) t_sum += expf((top_p[j] - t_max) * inv_tau);
        t_sum = warp_sum(t_sum);
        listed = __any_sync(~0u, listed);
        if (lane == 0) {
            listed_s = listed;
            t_max_s = t_max;
            t_sum_s = t_sum;
        }
    }
    if (FWD && on && !teacher) {
        int i = threadIdx.x;
        for (; i + (kBatch - 1) * N < count; i += kBatch * N) {
            uint4 u[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) u[k] = *reinterpret_cast<const uint4*>(xv + static_cast<int64_t>(i + k * N) * VEC);
            mine.add<T>(u, c);
        }
        for (; i < count; i += N) {
            const uint4 u[1] = {*reinterpret_cast<const uint4*>(xv + static_cast<int64_t>(i) * VEC)};
            mine.add<T>(u, c);
        }
        if (odd >= 0) {
            float v[1];
            load_vec<T, 1>(x + odd, v);
            mine.add1(v[0], c);
        }
        MaxSum a = mine.sum(c);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1)
            a = merge(a, MaxSum{__shfl_xor_sync(~0u, a.m, d), __shfl_xor_sync(~0u, a.s, d)}, c);
        if (lane == 0) of_warp[warp] = a;
    }
    __syncthreads();
    on = on && listed_s != 0;
    if (!on) {      // the same for every block of the row
        if (FWD && part == 0 && threadIdx.x == 0) {
            P.loss[row] = 0.f;
            if (P.stats != nullptr) P.stats[2 * row] = P.stats[2 * row + 1] = 0.f;
        }
        if (GRAD) {
            const float zero[VEC] = {}, none[1] = {};
            if (odd >= 0) store_vec<T, 1>(dx + odd, none);
            for (int i = threadIdx.x; i < count; i += kAll) put(dxv + static_cast<int64_t>(i) * VEC, zero);
        }
        return;
    }
    MaxSum all;
    if (FWD) {
        all = lane < kWarps ? of_warp[lane] : MaxSum{-INFINITY, 0.f};
#pragma unroll
        for (int d = 16; d > 0; d >>= 1)
            all = merge(all, MaxSum{__shfl_xor_sync(~0u, all.m, d), __shfl_xor_sync(~0u, all.s, d)}, c);
        if (parts > 1) {
            if (threadIdx.x == 0) of_block = all;
            cluster.sync();
            all = MaxSum{-INFINITY, 0.f};
            for (int k = 0; k < parts; ++k) all = merge(all, *cluster.map_shared_rank(&of_block, k), c);
            cluster.sync();         // no block leaves while another reads its part
        }
    } else {
        all = MaxSum{P.stats[2 * row], P.stats[2 * row + 1]};
    }

    const float t_max = t_max_s, t_sum = t_sum_s;
    if (FWD && part == 0 && teacher) {
        const float log_q = logf(all.s), log_t = logf(t_sum);
        float l = 0.f;
        for (int j = lane; j < P.top; j += 32) {
            if (top_id[j] < 0) continue;
            const float log_p = (top_p[j] - t_max) * inv_tau - log_t;
            const float p = expf(log_p);
            if (p != 0.f) l += p * (log_p - ((top_x[j] - all.m) * inv_tau - log_q));
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
    if (!GRAD) return;
    const float scale = w * up * P.temperature;
    const float ref = all.m * c;
    const bool fast = in_range(ref);
    const float f = scale / all.s * (fast ? exp2_fast(-fmaf(all.m, c, -ref)) : 1.f);
    auto q_of = [&](float v) { return f * (fast ? exp2_fast(fmaf(v, c, -ref)) : exp2_fast((v - all.m) * c)); };
    if (!teacher) {
        const f32x2 cc = pack2(c, c), rr = pack2(-ref, -ref), ff = pack2(f, f);
        auto grad = [&](const uint4& u, int i) {
            float v[VEC];
            if (fast) {
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
                for (int k = 0; k < VEC; ++k) v[k] = q_of(v[k]);
            }
            put(dxv + static_cast<int64_t>(i) * VEC, v);
        };
        int i = threadIdx.x;
        for (; i + (kBatch - 1) * N < count; i += kBatch * N) {
            uint4 u[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) u[k] = *reinterpret_cast<const uint4*>(xv + static_cast<int64_t>(i + k * N) * VEC);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) grad(u[k], i + k * N);
        }
        for (; i < count; i += N) grad(*reinterpret_cast<const uint4*>(xv + static_cast<int64_t>(i) * VEC), i);
        if (odd >= 0) {
            float v[1];
            load_vec<T, 1>(x + odd, v);
            v[0] = q_of(v[0]);
            store_vec<T, 1>(dx + odd, v);
        }
    } else {
        for (int j = lane; j < P.top; j += 32)
            if (top_id[j] >= 0) top_p[j] = expf((top_p[j] - t_max) * inv_tau) / t_sum;
    }
    // The listed entries of this block's part, written again with their target.
    __syncthreads();
    for (int j = threadIdx.x; j < P.top; j += kAll) {
        const int32_t id = top_id[j];
        if (id < begin || id >= end) continue;
        float p = 0.f;          // an entry listed twice: both write the same sum
        for (int k = 0; k < P.top; ++k)
            if (top_id[k] == id) p += top_p[k];
        const float v[1] = {q_of(top_x[j]) - scale * p};
        store_vec<T, 1>(dx + id, v);
    }
}

// ----------------------------------------------------------------------- host
int check(const malt_distill_t* d) {
    if (d == nullptr || d->rows < 0 || d->vocab < 1 || d->top < 0 || !(d->temperature >= 1e-15f) ||
        !(d->temperature <= 1e15f))
        return MALT_ERR_INVALID_ARG;
    if (!float_type(d->dtype) || !float_type(d->top_dtype) || !index_type(d->ids_dtype)) return MALT_ERR_UNSUPPORTED;
    if (d->top > kMaxTop || d->rows >= (int64_t{1} << 27) || d->vocab >= (int64_t{1} << 31)) return MALT_ERR_UNSUPPORTED;
    if (d->ld < d->vocab || d->top_ids_ld < d->top || d->top_logits_ld < d->top) return MALT_ERR_INVALID_ARG;
    if (d->rows > 0 && (d->logits == nullptr || (d->top > 0 && (d->top_ids == nullptr || d->top_logits == nullptr))))
        return MALT_ERR_INVALID_ARG;
    if (!aligned_to(d->logits, type_bytes(d->dtype)) || !aligned_to(d->top_ids, type_bytes(d->ids_dtype)) ||
        !aligned_to(d->top_logits, type_bytes(d->top_dtype)) || !aligned_to(d->weight, 4))
        return MALT_ERR_MISALIGNED;
    return MALT_OK;
}

template <typename T, bool FWD, bool GRAD>
cudaError_t launch(const malt_distill_t* d, const Params& P, cudaStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const bool same = !GRAD || (reinterpret_cast<uintptr_t>(P.logits) % 16 == reinterpret_cast<uintptr_t>(P.dlogits) % 16 &&
                                (P.ld - P.dlogits_ld) % V == 0);
    // A row is split while its blocks leave SMs idle and its parts keep a batch of vectors.
    int parts = 1;
    while (parts < kMaxCluster && d->rows * parts < sm_count() && d->vocab / (2 * parts) >= kWide * V) parts *= 2;
    auto go = [&](auto* kernel, int threads) {
        return launch_clusters(kernel, static_cast<unsigned>(d->rows * parts), parts, threads + 32, 0, s, P);
    };
    // Short rows leave most of a wide block waiting for its barriers.
    if (d->vocab <= kNarrow * V * kBatch)
        return same ? go(distill_kernel<T, FWD, GRAD, true, kNarrow>, kNarrow)
                    : go(distill_kernel<T, FWD, GRAD, !GRAD, kNarrow>, kNarrow);
    return same ? go(distill_kernel<T, FWD, GRAD, true, kWide>, kWide)
                : go(distill_kernel<T, FWD, GRAD, !GRAD, kWide>, kWide);
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
