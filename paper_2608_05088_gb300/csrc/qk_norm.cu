// qk_norm.cu -- RMS norms of queries and keys for each head, with the position
// rotation in the same pass, and the gradient of both.
//
// Per row x (one head of one token, D entries), gain g and angles of the token's
// position, the first R entries in pairs (a, b):
//   r = 1 / sqrt(mean(x^2) + eps),  n = x r g,
//   y_a = n_a cos - n_b sin,  y_b = n_b cos + n_a sin,  y = n past entry R.
// Gradient, from dy and the same x (nothing else is kept from the forward pass):
//   dn = dy rotated back,  dg = sum over rows of dn x r,  u = dn g,
//   dx = r (u - x r^2 mean(u x)).
//
// Bound by HBM: x is read once (and dy), y (dx) written once.  A row is held by a few
// neighbouring lanes, both partners of a pair in one lane, so the norm takes a
// shuffle or two and the rotation none.
#include <algorithm>

#include <nvtx3/nvToolsExt.h>

#include "model_ops.cuh"

namespace malt {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxHeadDim = 1024;

struct Rows {           // heads of the tokens of a [batch, seq, heads, dim] view
    void* data;
    int64_t batch_stride, seq_stride, head_stride;
    __device__ __forceinline__ int64_t at(int64_t b, int64_t s, int64_t h) const {
        return b * batch_stride + s * seq_stride + h * head_stride;
    }
};

struct Kind {           // queries or keys
    Rows x, y, dy, dx;  // forward: x -> y; backward: dy, x -> dx
    const void* gain;
    float* dgain;
    float* parts;       // [blocks][dim] partial gain gradients
    int32_t heads;
    int32_t blocks;
    uint32_t split;     // slots of a token: slot j takes heads j, j + split, ...
    uint32_t slots;     // of all tokens
    int32_t gain_vectors;   // the gains are fp32 and aligned to 16 bytes
};

struct Params {
    Kind kind[2];
    const void* positions;
    int64_t positions_batch_stride;
    const float* cosines;
    const float* sines;
    int64_t table_rows, batch, seq;
    int32_t positions_i64, gain_bf16;
    int32_t dim, rot;
    float eps;
};

__device__ __forceinline__ float gain_at(const Params& P, const Kind& K, int i) {
    if (K.gain == nullptr) return 1.f;
    return P.gain_bf16 ? __bfloat162float(static_cast<const bf16*>(K.gain)[i]) : static_cast<const float*>(K.gain)[i];
}

__device__ __forceinline__ int64_t position_of(const Params& P, int64_t b, int64_t s) {
    if (P.positions == nullptr) return s;
    const int64_t i = b * P.positions_batch_stride + s;
    return P.positions_i64 ? static_cast<const int64_t*>(P.positions)[i] : static_cast<const int32_t*>(P.positions)[i];
}

// Entries of pair p of a row, and of the unpaired rest.
template <bool INTER>
__device__ __forceinline__ void pair_at(int p, int rot, int* a, int* b) {
    *a = INTER ? 2 * p : p;
    *b = INTER ? 2 * p + 1 : rot / 2 + p;
}

// Cosine and sine of pair p: a position outside the tables has no angle.
__device__ __forceinline__ float2 angle(const Params& P, int64_t pos, int p) {
    if (pos < 0 || pos >= P.table_rows) return make_float2(__int_as_float(0x7fc00000), __int_as_float(0x7fc00000));
    const int64_t i = pos * (P.rot / 2) + p;
    return make_float2(P.cosines[i], P.sines[i]);
}

// --------------------------------------------------------------- aligned rows
// A row is held by LPR neighbouring lanes, 2 V entries each (V: 16 bytes of them):
// the V pairs that the lane turns, partners in the lane, so that one lane needs V
// cosines and V sines.  These lanes are a slot, which keeps its token's angles and
// the gains in registers and walks over heads; neighbouring slots take neighbouring
// heads of a token, so that a warp's loads are contiguous.
template <typename T, bool INTER>
struct Chunk {
    static constexpr int V = 16 / sizeof(T);
    int a, b;           // first entries of the lane's two vectors
    bool turned;
    __device__ __forceinline__ Chunk(int c, int rot) {
        turned = c * 2 * V < rot;
        if (INTER || !turned) {
            a = c * 2 * V;
            b = a + V;
        } else {
            a = c * V;
            b = rot / 2 + c * V;
        }
    }
    // entry of the lane's value i of 2 V, and the two values of its pair p
    __device__ __forceinline__ int entry(int i) const { return i < V ? a + i : b + i - V; }
    static __device__ __forceinline__ constexpr int first(int p) { return INTER ? 2 * p : p; }
    static __device__ __forceinline__ constexpr int second(int p) { return INTER ? 2 * p + 1 : V + p; }
};

template <int V>
struct Angles {
    float c[V], s[V];
    __device__ __forceinline__ void load(const Params& P, int64_t pos, int chunk, bool turned) {
        const bool in = pos >= 0 && pos < P.table_rows;
        if (turned && in) {
            const int64_t at = pos * (P.rot / 2) + chunk * V;
            load_vec<float, V>(P.cosines + at, c);
            load_vec<float, V>(P.sines + at, s);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                c[i] = turned ? __int_as_float(0x7fc00000) : 1.f;
                s[i] = turned ? __int_as_float(0x7fc00000) : 0.f;
            }
        }
    }
};

template <int LPR>
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int d = LPR / 2; d > 0; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
    return v;
}

template <typename T>
__device__ __forceinline__ uint4 load16(const T* p) { return *reinterpret_cast<const uint4*>(p); }

// Gains of the lane's entries.
template <typename C, int N>
__device__ __forceinline__ void load_gains(const Params& P, const Kind& K, const C& chunk, float (&g)[N]) {
    constexpr int V = N / 2;
    if (K.gain_vectors) {
        float lo[V], hi[V];
        load_vec<float, V>(static_cast<const float*>(K.gain) + chunk.a, lo);
        load_vec<float, V>(static_cast<const float*>(K.gain) + chunk.b, hi);
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = lo[i], g[V + i] = hi[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) g[i] = gain_at(P, K, chunk.entry(i));
    }
}

constexpr int kFwdHeads = 4;        // rows of a slot in flight
constexpr int kBwdHeads = 2;

template <typename T, bool INTER, int LPR>
__global__ void __launch_bounds__(kThreads)
qk_forward_kernel(const __grid_constant__ Params P) {
    using C = Chunk<T, INTER>;
    constexpr int V = C::V, N = 2 * V, U = kFwdHeads;
    const bool keys = blockIdx.x >= P.kind[0].blocks;
    const Kind& K = P.kind[keys];
    const uint32_t block = blockIdx.x - (keys ? P.kind[0].blocks : 0);
    const int lane = threadIdx.x & 31, sub = lane % LPR;
    const uint32_t slot = (block * kWarps + (threadIdx.x >> 5)) * (32 / LPR) + lane / LPR;
    const bool live = slot < K.slots && sub * N < P.dim;
    const uint32_t token = slot / K.split, j = slot - token * K.split;
    const int64_t b = token / static_cast<uint32_t>(P.seq), s = token - b * P.seq;
    const C chunk(sub, P.rot);
    const T* const x = static_cast<const T*>(K.x.data) + K.x.at(b, s, 0);
    T* const y = static_cast<T*>(K.y.data) + K.y.at(b, s, 0);
    float g[N];
    Angles<V> t;
    chain_wait();
    for (int h0 = 0; h0 < K.heads; h0 += U * K.split) {
        uint4 raw[U][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * K.split + j;
            raw[u][0] = raw[u][1] = make_uint4(0, 0, 0, 0);
            if (live && h < K.heads) {
                raw[u][0] = load16(x + h * K.x.head_stride + chunk.a);
                raw[u][1] = load16(x + h * K.x.head_stride + chunk.b);
            }
        }
        if (h0 == 0 && live) {
            t.load(P, position_of(P, b, s), sub, chunk.turned);
            load_gains(P, K, chunk, g);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int h = h0 + u * K.split + j;
            float v[N];
            unpack<T>(raw[u][0], v);
            unpack<T>(raw[u][1], v + V);
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < N; ++i) ss = fmaf(v[i], v[i], ss);
            const float r = rsqrtf(row_sum<LPR>(ss) / static_cast<float>(P.dim) + P.eps);
            if (!live || h >= K.heads) continue;
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] *= r * g[i];
            float o[2][V];
#pragma unroll
            for (int p = 0; p < V; ++p) {
                const int ia = C::first(p), ib = C::second(p);
                o[ia / V][ia % V] = v[ia] * t.c[p] - v[ib] * t.s[p];
                o[ib / V][ib % V] = v[ib] * t.c[p] + v[ia] * t.s[p];
            }
            store_vec<T, V>(y + h * K.y.head_stride + chunk.a, o[0]);
            store_vec<T, V>(y + h * K.y.head_stride + chunk.b, o[1]);
        }
    }
}

// The blocks stay and walk over the slots, with the gain gradient of their lanes'
// entries in registers; each leaves its sum for the join launch.
template <typename T, bool INTER, int LPR>
__global__ void __launch_bounds__(kThreads, 2)
qk_backward_kernel(const __grid_constant__ Params P) {
    using C = Chunk<T, INTER>;
    constexpr int V = C::V, N = 2 * V, U = kBwdHeads, kSlots = 32 / LPR;
    extern __shared__ float sums[];         // [kWarps][dim]
    const bool keys = blockIdx.x >= P.kind[0].blocks;
    const Kind& K = P.kind[keys];
    const uint32_t block = blockIdx.x - (keys ? P.kind[0].blocks : 0);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % LPR;
    const bool mine = sub * N < P.dim;
    const C chunk(sub, P.rot);
    float g[N], acc[N] = {};
    Angles<V> t;
    chain_wait();
    if (mine) load_gains(P, K, chunk, g);
    const float n = static_cast<float>(P.dim);
    for (uint64_t first = (static_cast<uint64_t>(block) * kWarps + warp) * kSlots; first < K.slots;
         first += static_cast<uint64_t>(K.blocks) * kWarps * kSlots) {
        const uint64_t slot = first + lane / LPR;
        const bool live = slot < K.slots && mine;
        const uint32_t token = static_cast<uint32_t>(slot) / K.split, j = static_cast<uint32_t>(slot) - token * K.split;
        const int64_t b = token / static_cast<uint32_t>(P.seq), s = token - b * P.seq;
        const T* const x = static_cast<const T*>(K.x.data) + K.x.at(b, s, 0);
        const T* const dy = static_cast<const T*>(K.dy.data) + K.dy.at(b, s, 0);
        T* const dx = static_cast<T*>(K.dx.data) + K.dx.at(b, s, 0);
        for (int h0 = 0; h0 < K.heads; h0 += U * K.split) {
            uint4 rx[U][2], ry[U][2];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + u * K.split + j;
                rx[u][0] = rx[u][1] = ry[u][0] = ry[u][1] = make_uint4(0, 0, 0, 0);
                if (live && h < K.heads) {
                    rx[u][0] = load16(x + h * K.x.head_stride + chunk.a);
                    rx[u][1] = load16(x + h * K.x.head_stride + chunk.b);
                    ry[u][0] = load16(dy + h * K.dy.head_stride + chunk.a);
                    ry[u][1] = load16(dy + h * K.dy.head_stride + chunk.b);
                }
            }
            if (h0 == 0 && live) t.load(P, position_of(P, b, s), sub, chunk.turned);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int h = h0 + u * K.split + j;
                const bool here = live && h < K.heads;
                float v[N], d[N];
                unpack<T>(rx[u][0], v);
                unpack<T>(rx[u][1], v + V);
                unpack<T>(ry[u][0], d);
                unpack<T>(ry[u][1], d + V);
                float ss = 0.f, ux = 0.f;
                if (here) {
#pragma unroll
                    for (int p = 0; p < V; ++p) {       // rotated back
                        const int ia = C::first(p), ib = C::second(p);
                        const float da = d[ia] * t.c[p] + d[ib] * t.s[p], db = d[ib] * t.c[p] - d[ia] * t.s[p];
                        d[ia] = da;
                        d[ib] = db;
                    }
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        ss = fmaf(v[i], v[i], ss);
                        ux = fmaf(d[i] * g[i], v[i], ux);
                    }
                }
                const float r = rsqrtf(row_sum<LPR>(ss) / n + P.eps);
                const float c = r * r * (row_sum<LPR>(ux) / n);
                if (!here) continue;
                float o[2][V];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    acc[i] = fmaf(d[i], v[i] * r, acc[i]);
                    o[i / V][i % V] = r * (d[i] * g[i] - v[i] * c);
                }
                store_vec<T, V>(dx + h * K.dx.head_stride + chunk.a, o[0]);
                store_vec<T, V>(dx + h * K.dx.head_stride + chunk.b, o[1]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int d = LPR; d < 32; d <<= 1) acc[i] += __shfl_xor_sync(~0u, acc[i], d);
    if (lane < LPR && mine) {
#pragma unroll
        for (int i = 0; i < N; ++i) sums[warp * P.dim + chunk.entry(i)] = acc[i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < P.dim; i += kThreads) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) t += sums[w * P.dim + i];
        K.parts[block * static_cast<int64_t>(P.dim) + i] = t;
    }
}

// ------------------------------------------------------- any size and alignment
// One warp per row, element by element.
template <typename T, bool INTER>
__global__ void __launch_bounds__(kThreads)
qk_forward_any_kernel(const __grid_constant__ Params P) {
    chain_wait();
    const bool second = blockIdx.x >= P.kind[0].blocks;
    const Kind& K = P.kind[second];
    const int64_t block = blockIdx.x - (second ? P.kind[0].blocks : 0);
    const int lane = threadIdx.x & 31;
    const int64_t row = block * kWarps + (threadIdx.x >> 5);
    const int64_t token = row / K.heads, h = row - token * K.heads;
    if (token >= P.batch * P.seq) return;
    const int64_t b = token / P.seq, s = token - b * P.seq;
    const T* const x = static_cast<const T*>(K.x.data) + K.x.at(b, s, h);
    T* const y = static_cast<T*>(K.y.data) + K.y.at(b, s, h);
    const int64_t pos = position_of(P, b, s);
    float ss = 0.f;
    for (int i = lane; i < P.dim; i += 32) {
        float v[1];
        load_vec<T, 1>(x + i, v);
        ss = fmaf(v[0], v[0], ss);
    }
    const float r = rsqrtf(warp_sum(ss) / static_cast<float>(P.dim) + P.eps);
    for (int p = lane; p < P.rot / 2; p += 32) {
        int ia, ib;
        pair_at<INTER>(p, P.rot, &ia, &ib);
        const float2 cs = angle(P, pos, p);
        float a[1], c[1];
        load_vec<T, 1>(x + ia, a);
        load_vec<T, 1>(x + ib, c);
        a[0] *= r * gain_at(P, K, ia);
        c[0] *= r * gain_at(P, K, ib);
        const float ya[1] = {a[0] * cs.x - c[0] * cs.y}, yb[1] = {c[0] * cs.x + a[0] * cs.y};
        store_vec<T, 1>(y + ia, ya);
        store_vec<T, 1>(y + ib, yb);
    }
    for (int i = P.rot + lane; i < P.dim; i += 32) {
        float v[1];
        load_vec<T, 1>(x + i, v);
        v[0] *= r * gain_at(P, K, i);
        store_vec<T, 1>(y + i, v);
    }
}

template <typename T, bool INTER>
__global__ void __launch_bounds__(kThreads)
qk_backward_any_kernel(const __grid_constant__ Params P) {
    extern __shared__ float acc_all[];          // [kWarps][dim] gain gradients of a warp's rows
    const bool second = blockIdx.x >= P.kind[0].blocks;
    const Kind& K = P.kind[second];
    const int64_t block = blockIdx.x - (second ? P.kind[0].blocks : 0);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float* const acc = acc_all + warp * P.dim;
    for (int i = lane; i < P.dim; i += 32) acc[i] = 0.f;
    __syncwarp();
    chain_wait();
    const int64_t rows = P.batch * P.seq * K.heads;
    for (int64_t row = block * kWarps + warp; row < rows; row += static_cast<int64_t>(K.blocks) * kWarps) {
        const int64_t token = row / K.heads, h = row - token * K.heads;
        const int64_t b = token / P.seq, s = token - b * P.seq;
        const T* const x = static_cast<const T*>(K.x.data) + K.x.at(b, s, h);
        const T* const dy = static_cast<const T*>(K.dy.data) + K.dy.at(b, s, h);
        T* const dx = static_cast<T*>(K.dx.data) + K.dx.at(b, s, h);
        const int64_t pos = position_of(P, b, s);
        float ss = 0.f, ux = 0.f;
        for (int p = lane; p < P.rot / 2; p += 32) {
            int ia, ib;
            pair_at<INTER>(p, P.rot, &ia, &ib);
            const float2 cs = angle(P, pos, p);
            float xa[1], xb[1], ya[1], yb[1];
            load_vec<T, 1>(x + ia, xa);
            load_vec<T, 1>(x + ib, xb);
            load_vec<T, 1>(dy + ia, ya);
            load_vec<T, 1>(dy + ib, yb);
            ss = fmaf(xa[0], xa[0], fmaf(xb[0], xb[0], ss));
            const float na = ya[0] * cs.x + yb[0] * cs.y, nb = yb[0] * cs.x - ya[0] * cs.y;
            ux = fmaf(na * gain_at(P, K, ia), xa[0], fmaf(nb * gain_at(P, K, ib), xb[0], ux));
        }
        for (int i = P.rot + lane; i < P.dim; i += 32) {
            float v[1], d[1];
            load_vec<T, 1>(x + i, v);
            load_vec<T, 1>(dy + i, d);
            ss = fmaf(v[0], v[0], ss);
            ux = fmaf(d[0] * gain_at(P, K, i), v[0], ux);
        }
        const float n = static_cast<float>(P.dim);
        const float r = rsqrtf(warp_sum(ss) / n + P.eps);
        const float c = r * r * (warp_sum(ux) / n);
        for (int p = lane; p < P.rot / 2; p += 32) {
            int ia, ib;
            pair_at<INTER>(p, P.rot, &ia, &ib);
            const float2 cs = angle(P, pos, p);
            float xa[1], xb[1], ya[1], yb[1];
            load_vec<T, 1>(x + ia, xa);
            load_vec<T, 1>(x + ib, xb);
            load_vec<T, 1>(dy + ia, ya);
            load_vec<T, 1>(dy + ib, yb);
            const float na = ya[0] * cs.x + yb[0] * cs.y, nb = yb[0] * cs.x - ya[0] * cs.y;
            acc[ia] = fmaf(na, xa[0] * r, acc[ia]);
            acc[ib] = fmaf(nb, xb[0] * r, acc[ib]);
            const float da[1] = {r * (na * gain_at(P, K, ia) - xa[0] * c)}, db[1] = {r * (nb * gain_at(P, K, ib) - xb[0] * c)};
            store_vec<T, 1>(dx + ia, da);
            store_vec<T, 1>(dx + ib, db);
        }
        for (int i = P.rot + lane; i < P.dim; i += 32) {
            float v[1], d[1];
            load_vec<T, 1>(x + i, v);
            load_vec<T, 1>(dy + i, d);
            acc[i] = fmaf(d[0], v[0] * r, acc[i]);
            const float o[1] = {r * (d[0] * gain_at(P, K, i) - v[0] * c)};
            store_vec<T, 1>(dx + i, o);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < P.dim; i += kThreads) {
        float t = 0.f;
        for (int w = 0; w < kWarps; ++w) t += acc_all[w * P.dim + i];
        K.parts[block * P.dim + i] = t;
    }
}

// Gain gradients: block 0 adds up the parts of the queries, block 1 of the keys,
// for 32 entries at a time, every warp a run of the parts.
__global__ void __launch_bounds__(1024)
qk_gain_kernel(const __grid_constant__ Params P) {
    __shared__ float sums[32][33];
    chain_wait();
    const Kind& K = P.kind[blockIdx.y];
    if (K.dgain == nullptr) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int i = blockIdx.x * 32 + lane;
    const float* const parts = after_wait(K.parts);
    float t = 0.f;
    if (i < P.dim)
        for (int k = warp; k < K.blocks; k += 32) t += parts[static_cast<int64_t>(k) * P.dim + i];
    sums[warp][lane] = t;
    __syncthreads();
    if (warp == 0 && i < P.dim) {
        float u = 0.f;
#pragma unroll
        for (int w = 0; w < 32; ++w) u += sums[w][lane];
        K.dgain[i] = u;
    }
}

// ----------------------------------------------------------------------- host
int64_t tokens_of(const malt_qk_norm_t* p) { return p->batch * p->seq; }

int check(const malt_qk_norm_t* p) {
    if (p == nullptr || p->batch < 0 || p->seq < 0 || p->table_rows < 0 || !(p->eps >= 0.f)) return MALT_ERR_INVALID_ARG;
    if (!float_type(p->dtype) || !float_type(p->gain_dtype)) return MALT_ERR_UNSUPPORTED;
    if (p->head_dim < 1 || p->head_dim > kMaxHeadDim) return MALT_ERR_UNSUPPORTED;
    if (p->rot_dim < 0 || p->rot_dim > p->head_dim || p->rot_dim % 2 != 0) return MALT_ERR_INVALID_ARG;
    constexpr int64_t kMax = int64_t{1} << 31;
    if (p->batch >= kMax || p->seq >= kMax || p->batch * p->seq >= kMax) return MALT_ERR_UNSUPPORTED;
    if (p->rot_dim > 0 && p->table_rows > 0 && (p->cosines == nullptr || p->sines == nullptr)) return MALT_ERR_INVALID_ARG;
    if (p->positions != nullptr && !index_type(p->positions_dtype)) return MALT_ERR_UNSUPPORTED;
    if (!aligned_to(p->cosines, 4) || !aligned_to(p->sines, 4) ||
        (p->positions != nullptr && !aligned_to(p->positions, type_bytes(p->positions_dtype))) ||
        !aligned_to(p->q_gain, type_bytes(p->gain_dtype)) || !aligned_to(p->k_gain, type_bytes(p->gain_dtype)))
        return MALT_ERR_MISALIGNED;
    return MALT_OK;
}

int check_heads(const malt_qk_norm_t* p, const malt_heads_t* h, const malt_heads_t* like) {
    if (h == nullptr || h->heads < 0 || h->heads != like->heads) return MALT_ERR_INVALID_ARG;
    if (h->heads >= (1 << 20)) return MALT_ERR_UNSUPPORTED;
    if (h->heads > 0 && tokens_of(p) > 0 && h->data == nullptr) return MALT_ERR_INVALID_ARG;
    if (!aligned_to(h->data, type_bytes(p->dtype))) return MALT_ERR_MISALIGNED;
    return MALT_OK;
}

Rows rows_of(const malt_heads_t* h) { return Rows{h->data, h->batch_stride, h->seq_stride, h->head_stride}; }

Params params_of(const malt_qk_norm_t* p) {
    Params P = {};
    P.positions = p->positions;
    P.positions_batch_stride = p->positions_batch_stride;
    P.cosines = p->cosines;
    P.sines = p->sines;
    P.table_rows = p->table_rows;
    P.batch = p->batch;
    P.seq = p->seq;
    P.positions_i64 = p->positions_dtype == MALT_I64;
    P.gain_bf16 = p->gain_dtype == MALT_BF16;
    P.dim = p->head_dim;
    P.rot = p->rot_dim;
    P.eps = p->eps;
    P.kind[0].gain = p->q_gain;
    P.kind[1].gain = p->k_gain;
    return P;
}

// Blocks of a backward launch, and the most that its two kinds round up to: each
// leaves a part of a gain gradient in the workspace.
int32_t backward_blocks() { return sm_count() * 6; }
int32_t backward_parts() { return backward_blocks() + 2; }

// Whether the rows of a view can be read in 16-byte vectors.
template <typename T>
bool vectors(const Params& P, const Rows& r) {
    constexpr int64_t V = 16 / sizeof(T);
    return aligned_to(r.data, 16) && (P.batch == 1 || r.batch_stride % V == 0) &&
           (P.seq == 1 || r.seq_stride % V == 0) && r.head_stride % V == 0;
}

// Lanes of a row in the aligned kernels, 0 where they do not apply.
template <typename T>
int lanes_of(const Params& P, bool backward) {
    constexpr int N = 32 / sizeof(T);
    if (P.dim % N != 0 || P.rot % N != 0 || P.dim / N > 32) return 0;
    if (!aligned_to(P.cosines, 16) || !aligned_to(P.sines, 16)) return 0;
    for (const Kind& K : P.kind) {
        if (K.heads == 0) continue;
        if (!vectors<T>(P, K.x)) return 0;
        if (backward ? !vectors<T>(P, K.dy) || !vectors<T>(P, K.dx) : !vectors<T>(P, K.y)) return 0;
    }
    int lanes = 2;
    while (lanes * N < P.dim) lanes *= 2;
    return lanes;
}

// Slots of a token for each kind: a few batches of heads a slot, which spreads the
// angles' cost, but enough slots to fill the GPU.
void split_heads(Params& P, int lanes, int batch) {
    const int64_t tokens = P.batch * P.seq;
    const int64_t wanted = sm_count() * 64ll * (32 / lanes);
    for (Kind& K : P.kind) {
        K.gain_vectors = K.gain != nullptr && !P.gain_bf16 && aligned_to(K.gain, 16);
        int64_t rounds = 2, split;
        do {
            split = std::max<int64_t>(1, (K.heads + batch * rounds - 1) / (batch * rounds));
        } while (--rounds > 0 && tokens * split < wanted);
        if (tokens * K.heads < wanted) split = std::max(K.heads, 1);
        if (tokens * split >= (int64_t{1} << 31)) split = 1;
        K.split = static_cast<uint32_t>(split);
        K.slots = K.heads == 0 ? 0 : static_cast<uint32_t>(tokens * split);
    }
}

template <typename T, bool INTER, int LPR>
cudaError_t forward_rows(Params& P, cudaStream_t s) {
    constexpr int64_t kSlots = kWarps * (32 / LPR);
    for (Kind& K : P.kind) K.blocks = static_cast<int32_t>((K.slots + kSlots - 1) / kSlots);
    return launch_chained(qk_forward_kernel<T, INTER, LPR>, P.kind[0].blocks + P.kind[1].blocks, kThreads, 0, s, P);
}

template <typename T, bool INTER, int LPR>
cudaError_t backward_rows(Params& P, cudaStream_t s) {
    constexpr int64_t kSlots = kWarps * (32 / LPR);
    const int64_t heads = P.kind[0].heads + P.kind[1].heads;
    for (Kind& K : P.kind) {
        const int64_t share = K.heads > 0 ? std::max<int64_t>(1, static_cast<int64_t>(sm_count()) * 2 * K.heads / heads) : 0;
        K.blocks = static_cast<int32_t>(std::min<int64_t>((K.slots + kSlots - 1) / kSlots, share));
    }
    P.kind[1].parts = P.kind[0].parts + static_cast<int64_t>(P.kind[0].blocks) * P.dim;
    return launch_chained(qk_backward_kernel<T, INTER, LPR>, P.kind[0].blocks + P.kind[1].blocks, kThreads,
                          kWarps * P.dim * sizeof(float), s, P);
}

template <typename T, bool INTER>
cudaError_t rows_kernel(Params& P, int lanes, bool backward, cudaStream_t s) {
    split_heads(P, lanes, backward ? kBwdHeads : kFwdHeads);
    switch (lanes) {
        case 2: return backward ? backward_rows<T, INTER, 2>(P, s) : forward_rows<T, INTER, 2>(P, s);
        case 4: return backward ? backward_rows<T, INTER, 4>(P, s) : forward_rows<T, INTER, 4>(P, s);
        case 8: return backward ? backward_rows<T, INTER, 8>(P, s) : forward_rows<T, INTER, 8>(P, s);
        case 16: return backward ? backward_rows<T, INTER, 16>(P, s) : forward_rows<T, INTER, 16>(P, s);
        default: return backward ? backward_rows<T, INTER, 32>(P, s) : forward_rows<T, INTER, 32>(P, s);
    }
}

template <typename T>
cudaError_t forward(Params& P, bool inter, cudaStream_t s) {
    if (const int lanes = lanes_of<T>(P, false))
        return inter ? rows_kernel<T, true>(P, lanes, false, s) : rows_kernel<T, false>(P, lanes, false, s);
    for (Kind& K : P.kind) {
        const int64_t blocks = (P.batch * P.seq * K.heads + kWarps - 1) / kWarps;
        if (blocks >= (int64_t{1} << 30)) return cudaErrorInvalidValue;
        K.blocks = static_cast<int32_t>(blocks);
    }
    return launch_chained(inter ? qk_forward_any_kernel<T, true> : qk_forward_any_kernel<T, false>,
                          P.kind[0].blocks + P.kind[1].blocks, kThreads, 0, s, P);
}

template <typename T>
cudaError_t backward(Params& P, bool inter, cudaStream_t s) {
    if (const int lanes = lanes_of<T>(P, true))
        return inter ? rows_kernel<T, true>(P, lanes, true, s) : rows_kernel<T, false>(P, lanes, true, s);
    const int64_t heads = P.kind[0].heads + P.kind[1].heads;
    for (Kind& K : P.kind) {
        const int64_t blocks = (P.batch * P.seq * K.heads + kWarps - 1) / kWarps;
        const int64_t share = K.heads > 0 ? std::max<int64_t>(1, static_cast<int64_t>(backward_blocks()) * K.heads / heads) : 0;
        K.blocks = static_cast<int32_t>(std::min(blocks, share));
    }
    P.kind[1].parts = P.kind[0].parts + static_cast<int64_t>(P.kind[0].blocks) * P.dim;
    return launch_chained(inter ? qk_backward_any_kernel<T, true> : qk_backward_any_kernel<T, false>,
                          P.kind[0].blocks + P.kind[1].blocks, kThreads, kWarps * P.dim * sizeof(float), s, P);
}

}  // namespace
}  // namespace malt

extern "C" {

int malt_qk_norm_forward(const malt_qk_norm_t* p, const malt_heads_t* q, const malt_heads_t* k,
                         const malt_heads_t* q_out, const malt_heads_t* k_out, void* stream) {
    using namespace malt;
    int rc = check(p);
    if (rc != MALT_OK) return rc;
    if (q == nullptr || k == nullptr) return MALT_ERR_INVALID_ARG;
    const malt_heads_t* const all[4] = {q, k, q_out, k_out};
    for (int i = 0; i < 4; ++i)
        if ((rc = check_heads(p, all[i], i % 2 ? k : q)) != MALT_OK) return rc;
    if (tokens_of(p) == 0 || q->heads + k->heads == 0) return MALT_OK;
    Params P = params_of(p);
    P.kind[0].x = rows_of(q);
    P.kind[1].x = rows_of(k);
    P.kind[0].y = rows_of(q_out);
    P.kind[1].y = rows_of(k_out);
    P.kind[0].heads = static_cast<int32_t>(q->heads);
    P.kind[1].heads = static_cast<int32_t>(k->heads);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    nvtxRangePushA("malt_qk_norm_forward");
    const cudaError_t c = p->dtype == MALT_BF16 ? forward<bf16>(P, p->interleaved != 0, s)
                                                : forward<float>(P, p->interleaved != 0, s);
    nvtxRangePop();
    return cuda_status(c, "malt_qk_norm_forward");
}

size_t malt_qk_norm_workspace_bytes(int32_t head_dim) {
    if (head_dim < 1 || head_dim > malt::kMaxHeadDim) return 0;
    return static_cast<size_t>(malt::backward_parts()) * head_dim * sizeof(float);
}

int malt_qk_norm_backward(const malt_qk_norm_t* p, const malt_heads_t* dq_out, const malt_heads_t* dk_out,
                          const malt_heads_t* q, const malt_heads_t* k, const malt_heads_t* dq,
                          const malt_heads_t* dk, float* dq_gain, float* dk_gain, void* workspace,
                          size_t workspace_bytes, void* stream) {
    using namespace malt;
    int rc = check(p);
    if (rc != MALT_OK) return rc;
    if (q == nullptr || k == nullptr) return MALT_ERR_INVALID_ARG;
    const malt_heads_t* const all[6] = {q, k, dq_out, dk_out, dq, dk};
    for (int i = 0; i < 6; ++i)
        if ((rc = check_heads(p, all[i], i % 2 ? k : q)) != MALT_OK) return rc;
    if (!aligned_to(dq_gain, 4) || !aligned_to(dk_gain, 4) || !aligned_to(workspace, 16)) return MALT_ERR_MISALIGNED;
    if (workspace == nullptr || workspace_bytes < malt_qk_norm_workspace_bytes(p->head_dim)) return MALT_ERR_INVALID_ARG;
    Params P = params_of(p);
    P.kind[0].x = rows_of(q);
    P.kind[1].x = rows_of(k);
    P.kind[0].dy = rows_of(dq_out);
    P.kind[1].dy = rows_of(dk_out);
    P.kind[0].dx = rows_of(dq);
    P.kind[1].dx = rows_of(dk);
    P.kind[0].heads = static_cast<int32_t>(q->heads);
    P.kind[1].heads = static_cast<int32_t>(k->heads);
    P.kind[0].dgain = dq_gain;
    P.kind[1].dgain = dk_gain;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    nvtxRangePushA("malt_qk_norm_backward");
    cudaError_t c = cudaSuccess;
    P.kind[0].parts = static_cast<float*>(workspace);
    if (tokens_of(p) > 0 && q->heads + k->heads > 0)
        c = p->dtype == MALT_BF16 ? backward<bf16>(P, p->interleaved != 0, s)
                                  : backward<float>(P, p->interleaved != 0, s);
    if (c == cudaSuccess && (dq_gain != nullptr || dk_gain != nullptr)) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((P.dim + 31) / 32, 2);
        cfg.blockDim = dim3(1024);
        cfg.stream = s;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        c = cudaLaunchKernelEx(&cfg, qk_gain_kernel, P);
        if (c != cudaSuccess) cudaGetLastError();
    }
    nvtxRangePop();
    return cuda_status(c, "malt_qk_norm_backward");
}

}  // extern "C"
