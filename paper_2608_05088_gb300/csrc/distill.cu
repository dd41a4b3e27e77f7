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
// sweep finds the row's maximum m and sum of 2^((s - m) log2(e) / tau), each thread
// with a running maximum over batches of vectors; the second writes the gradient and
// finds the row in L2.  Bound by HBM: the logits once, their gradient once.
// Differences are taken before the product with log2(e) / tau, so that a row of the
// type's lowest values is a uniform one and not an overflow.
#include <algorithm>
#include <cooperative_groups.h>

#include <nvtx3/nvToolsExt.h>

#include "model_ops.cuh"

namespace malt {
namespace {

constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxTop = 1024;
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

__device__ __forceinline__ float block_sum(float v, float* tmp) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) tmp[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_sum((threadIdx.x & 31) < kWarps ? tmp[threadIdx.x & 31] : 0.f);
}
__device__ __forceinline__ float block_max(float v, float* tmp) {
    v = warp_max(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) tmp[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_max((threadIdx.x & 31) < kWarps ? tmp[threadIdx.x & 31] : -INFINITY);
}

// FWD: loss (and statistics).  GRAD: gradient, from the statistics where FWD is
// false.  SAME: the gradient's rows start as far from a 16-byte boundary as the
// logits' (else it is stored element by element).
template <typename T, bool FWD, bool GRAD, bool SAME>
__global__ void __launch_bounds__(kThreads)
distill_kernel(const __grid_constant__ Params P) {
    namespace cg = cooperative_groups;
    constexpr int VEC = 16 / sizeof(T);
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
    __shared__ float tmp[kWarps];
    __shared__ float tmp_s[kWarps];
    __shared__ MaxSum of_block;
    __shared__ int32_t top_id[kMaxTop];
    __shared__ float top_p[kMaxTop];
    __shared__ float top_x[kMaxTop];
    const cg::cluster_group cluster = cg::this_cluster();
    const int parts = static_cast<int>(cluster.num_blocks()), part = static_cast<int>(cluster.block_rank());
    const int64_t row = blockIdx.x / parts;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
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
    const T* const xv = x + lead;
    const int64_t tail = lead + vectors * VEC;      // first entry past the vectors

    // The teacher's entries, with the student's logit of each read before any block
    // of the row writes its gradient (which may take the logits' place).
    const float w = P.weight != nullptr ? P.weight[row] : 1.f;
    const float up = GRAD && P.dloss != nullptr ? P.dloss[row] : 1.f;
    const float inv_tau = 1.f / P.temperature;
    const float c = kLog2e / P.temperature;
    bool on = w != 0.f && (FWD || up != 0.f);
    int listed = 0;
    if (on) {
        for (int j = threadIdx.x; j < P.top; j += kThreads) {
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
        }
    }
    on = __syncthreads_or(listed) != 0;
    if (!on) {      // the same for every block of the row
        if (FWD && part == 0 && threadIdx.x == 0) {
            P.loss[row] = 0.f;
            if (P.stats != nullptr) P.stats[2 * row] = P.stats[2 * row + 1] = 0.f;
        }
        if (GRAD) {
            const float zero[VEC] = {}, none[1] = {};
            if (part == 0)
                for (int64_t i = threadIdx.x; i < lead; i += kThreads) store_vec<T, 1>(dx + i, none);
            for (int64_t i = v_begin + threadIdx.x; i < v_end; i += kThreads) put(dx + lead + i * VEC, zero);
            if (part == parts - 1)
                for (int64_t i = tail + threadIdx.x; i < P.vocab; i += kThreads) store_vec<T, 1>(dx + i, none);
        }
        return;
    }
    float t_max = -INFINITY;
    for (int j = threadIdx.x; j < P.top; j += kThreads) t_max = fmaxf(t_max, top_p[j]);
    t_max = block_max(t_max, tmp);
    float t_sum = 0.f;
    for (int j = threadIdx.x; j < P.top; j += kThreads)
        if (top_id[j] >= 0) t_sum += expf((top_p[j] - t_max) * inv_tau);
    t_sum = block_sum(t_sum, tmp);
    const float log_t = logf(t_sum);

    MaxSum all;
    if (FWD) {
        MaxSum a = {-INFINITY, 0.f};
        for (int64_t i = v_begin + threadIdx.x; i < v_end; i += kBatch * kThreads) {
            float v[kBatch][VEC];
            float m = a.m;
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const bool in = i + u * kThreads < v_end;
                if (in) load_vec<T, VEC>(xv + (i + u * kThreads) * VEC, v[u]);
#pragma unroll
                for (int k = 0; k < VEC; ++k)
                    if (!in) v[u][k] = -INFINITY;
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
#pragma unroll
                for (int k = 0; k < VEC; ++k) m = fmaxf(m, v[u][k]);
            a.s *= rescale(a.m, m, c);
            a.m = m;
            const float ref = m == -INFINITY ? 0.f : m;     // nothing but -inf so far: 2^-inf = 0
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
#pragma unroll
                for (int k = 0; k < VEC; ++k) a.s += exp2_fast((v[u][k] - ref) * c);
        }
        auto one = [&](int64_t i) {
            float v[1];
            load_vec<T, 1>(x + i, v);
            const float m = fmaxf(a.m, v[0]);
            a.s = a.s * rescale(a.m, m, c) + exp2_fast((v[0] - (m == -INFINITY ? 0.f : m)) * c);
            a.m = m;
        };
        if (part == 0)
            for (int64_t i = threadIdx.x; i < lead; i += kThreads) one(i);
        if (part == parts - 1)
            for (int64_t i = tail + threadIdx.x; i < P.vocab; i += kThreads) one(i);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1)
            a = merge(a, MaxSum{__shfl_xor_sync(~0u, a.m, d), __shfl_xor_sync(~0u, a.s, d)}, c);
        __syncthreads();
        if (lane == 0) {
            tmp[warp] = a.m;
            tmp_s[warp] = a.s;
        }
        __syncthreads();
        all = lane < kWarps ? MaxSum{tmp[lane], tmp_s[lane]} : MaxSum{-INFINITY, 0.f};
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

    if (FWD && part == 0) {
        const float log_q = logf(all.s);
        float l = 0.f;
        for (int j = threadIdx.x; j < P.top; j += kThreads) {
            if (top_id[j] < 0) continue;
            const float log_p = (top_p[j] - t_max) * inv_tau - log_t;
            const float p = expf(log_p);
            if (p != 0.f) l += p * (log_p - ((top_x[j] - all.m) * inv_tau - log_q));
        }
        l = block_sum(l, tmp);
        if (threadIdx.x == 0) {
            P.loss[row] = w * P.temperature * P.temperature * l;
            if (P.stats != nullptr) {
                P.stats[2 * row] = all.m;
                P.stats[2 * row + 1] = all.s;
            }
        }
    }
    if (GRAD) {
        const float scale = w * up * P.temperature;
        const float f = scale / all.s, m = all.m;
        for (int64_t i = v_begin + threadIdx.x; i < v_end; i += kBatch * kThreads) {
            float v[kBatch][VEC];
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (i + u * kThreads < v_end) load_vec<T, VEC>(xv + (i + u * kThreads) * VEC, v[u]);
#pragma unroll
            for (int u = 0; u < kBatch; ++u)
                if (i + u * kThreads < v_end) {
#pragma unroll
                    for (int k = 0; k < VEC; ++k) v[u][k] = f * exp2_fast((v[u][k] - m) * c);
                    put(dx + lead + (i + u * kThreads) * VEC, v[u]);
                }
        }
        auto one = [&](int64_t i) {
            float v[1];
            load_vec<T, 1>(x + i, v);
            v[0] = f * exp2_fast((v[0] - m) * c);
            store_vec<T, 1>(dx + i, v);
        };
        if (part == 0)
            for (int64_t i = threadIdx.x; i < lead; i += kThreads) one(i);
        if (part == parts - 1)
            for (int64_t i = tail + threadIdx.x; i < P.vocab; i += kThreads) one(i);
        // The listed entries of this block's part, written again with their target.
        for (int j = threadIdx.x; j < P.top; j += kThreads)
            if (top_id[j] >= 0) top_p[j] = expf((top_p[j] - t_max) * inv_tau) / t_sum;
        __syncthreads();
        for (int j = threadIdx.x; j < P.top; j += kThreads) {
            const int32_t id = top_id[j];
            if (id < begin || id >= end) continue;
            float p = 0.f;          // an entry listed twice: both write the same sum
            for (int k = 0; k < P.top; ++k)
                if (top_id[k] == id) p += top_p[k];
            const float v[1] = {f * exp2_fast((top_x[j] - m) * c) - scale * p};
            store_vec<T, 1>(dx + id, v);
        }
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
    while (parts < kMaxCluster && d->rows * parts < sm_count() && d->vocab / (2 * parts) >= kThreads * V) parts *= 2;
    return launch_clusters(same ? distill_kernel<T, FWD, GRAD, true> : distill_kernel<T, FWD, GRAD, !GRAD>,
                           static_cast<unsigned>(d->rows * parts), parts, kThreads, 0, s, P);
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
