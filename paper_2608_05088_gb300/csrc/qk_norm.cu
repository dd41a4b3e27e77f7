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
// shuffle or two and the rotation none.  16384 tokens of 2 x 20 heads of 64 in bf16:
// forward 31 us, 5.4 TB/s, gradient 46 us, 5.5 TB/s (a plain copy of as many bytes runs
// at 5.6 and 5.75).
//
// That asks for heads and rotated parts of whole lanes, multiples of 16 entries in bf16 and
// of 8 in fp32, on 16-byte addresses (lanes_of).  All other rows take one warp each, element
// by element, and six to twelve times as long: 16384 tokens of 2 x 16 heads of 80 in bf16, 80
// rotated 33 and 60 us, 40 rotated 338 and 390; heads of 64, all rotated, 25 and 39, of 72
// 318 and 514; in fp32 72 of 72 52 and 82, 68 of 68 332 and 494.
#include <algorithm>

#include <nvtx3/nvToolsExt.h>

#include "model_ops.cuh"

namespace malt {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxHeadDim = 1024;
constexpr int kMaxSplit = 256;
constexpr int64_t kMaxRows = int64_t{1} << 33;      // of a forward launch, a warp each

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
    int32_t lanes;              // of a row, aligned rows only
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
// A row is held by neighbouring lanes, 2 V entries each: the V pairs that the lane turns,
// partners in the lane, in two vectors of V, so that one lane needs V cosines and V
// sines.  These lanes are a slot, which keeps its token's angles and the gains in
// registers and walks over heads; neighbouring slots take neighbouring heads of a token,
// so that a warp's loads are contiguous.  Arithmetic is on two pairs at once: A holds the
// first members, B the second ones.
template <int V, bool INTER>
struct Chunk {
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
    // entry of the lane's value i of 2 V, and the values of pair p
    __device__ __forceinline__ int entry(int i) const { return i < V ? a + i : b + i - V; }
    static __device__ __forceinline__ constexpr int first(int p) { return INTER ? 2 * p : p; }
    static __device__ __forceinline__ constexpr int second(int p) { return INTER ? 2 * p + 1 : V + p; }
};

// A lane's vectors of a row as they are in memory.
template <typename T, int V>
struct RawRow {
    static constexpr int W = V * sizeof(T) / 4;     // words of a vector
    uint32_t w[2][W];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 2 * W; ++i) w[i / W][i % W] = 0;
    }
    __device__ __forceinline__ void load(const T* row, int a, int b) {
        const Raw<uint32_t, W> lo = *reinterpret_cast<const Raw<uint32_t, W>*>(row + a);
        const Raw<uint32_t, W> hi = *reinterpret_cast<const Raw<uint32_t, W>*>(row + b);
#pragma unroll
        for (int i = 0; i < W; ++i) w[0][i] = lo.v[i], w[1][i] = hi.v[i];
    }
    // value i of the vector
    __device__ __forceinline__ float at(int vector, int i) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[vector][i]);
        else return __uint_as_float(i % 2 ? w[vector][i / 2] & 0xffff0000u : w[vector][i / 2] << 16);
    }
};

// A lane's 2 V values as its pairs' members.
template <int V, bool INTER>
struct Members {
    using C = Chunk<V, INTER>;
    f32x2 a[V / 2], b[V / 2];
    __device__ __forceinline__ Members() {}
    template <typename T>
    __device__ __forceinline__ explicit Members(const RawRow<T, V>& raw) {
        float v[2 * V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[i] = raw.at(0, i);
            v[V + i] = raw.at(1, i);
        }
        from(v);
    }
    __device__ __forceinline__ void from(const float (&v)[2 * V]) {
#pragma unroll
        for (int p = 0; p < V; p += 2) {
            a[p / 2] = pack2(v[C::first(p)], v[C::first(p + 1)]);
            b[p / 2] = pack2(v[C::second(p)], v[C::second(p + 1)]);
        }
    }
    __device__ __forceinline__ void to(float (&v)[2 * V]) const {
#pragma unroll
        for (int p = 0; p < V; p += 2) {
            const float2 x = unpack2(a[p / 2]), y = unpack2(b[p / 2]);
            v[C::first(p)] = x.x;
            v[C::first(p + 1)] = x.y;
            v[C::second(p)] = y.x;
            v[C::second(p + 1)] = y.y;
        }
    }
    template <typename T>
    __device__ __forceinline__ void store(T* row, const C& chunk) const {
        float v[2 * V], lo[V], hi[V];
        to(v);
#pragma unroll
        for (int i = 0; i < V; ++i) lo[i] = v[i], hi[i] = v[V + i];
        store_vec<T, V>(row + chunk.a, lo);
        store_vec<T, V>(row + chunk.b, hi);
    }
};

// The token's cosines and sines of the lane's pairs.
template <int V>
struct Angles {
    f32x2 c[V / 2], s[V / 2];
    __device__ __forceinline__ void load(const Params& P, int64_t pos, int chunk, bool turned) {
        const bool in = pos >= 0 && pos < P.table_rows;
        float x[V], y[V];
        if (turned && in) {
            const int64_t at = pos * (P.rot / 2) + chunk * V;
            load_vec<float, V>(P.cosines + at, x);
            load_vec<float, V>(P.sines + at, y);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                x[i] = turned ? __int_as_float(0x7fc00000) : 1.f;
                y[i] = turned ? __int_as_float(0x7fc00000) : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            c[i / 2] = pack2(x[i], x[i + 1]);
            s[i / 2] = pack2(y[i], y[i + 1]);
        }
    }
};

// Lanes of a warp by slots of `lanes` neighbours each (LANES: a power of two known here;
// 0: any number, the warp's last lanes may belong to no slot).
template <int LANES>
struct Slots {
    int lanes, per_warp, slot, sub;
    __device__ __forceinline__ explicit Slots(int n) {
        const int lane = threadIdx.x & 31;
        lanes = LANES > 0 ? LANES : n;
        per_warp = 32 / lanes;
        slot = lane / lanes;
        sub = lane - slot * lanes;
        if (LANES == 0 && slot >= per_warp) sub = 32;      // holds nothing
    }
    __device__ __forceinline__ float sum(float v) const {
        if constexpr (LANES > 0) {
#pragma unroll
            for (int d = LANES / 2; d > 0; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
            return v;
        } else {
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const float up = __shfl_down_sync(~0u, v, d);
                if (sub + d < lanes) v += up;
            }
            return __shfl_sync(~0u, v, slot * lanes);
        }
    }
};

// Gains of the lane's entries.
template <int V, bool INTER>
__device__ __forceinline__ Members<V, INTER> load_gains(const Params& P, const Kind& K, const Chunk<V, INTER>& chunk) {
    float g[2 * V];
    if (K.gain_vectors) {
        float lo[V], hi[V];
        load_vec<float, V>(static_cast<const float*>(K.gain) + chunk.a, lo);
        load_vec<float, V>(static_cast<const float*>(K.gain) + chunk.b, hi);
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = lo[i], g[V + i] = hi[i];
    } else {
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) g[i] = gain_at(P, K, chunk.entry(i));
    }
    Members<V, INTER> m;
    m.from(g);
    return m;
}

__device__ __forceinline__ float sum2(f32x2 v) {
    const float2 h = unpack2(v);
    return h.x + h.y;
}
__device__ __forceinline__ f32x2 twice(float v) { return pack2(v, v); }

// Entries of a lane's vectors: 16 bytes.
template <typename T>
__host__ __device__ constexpr int vector_of() { return 16 / sizeof(T); }

// Forward: rows of a slot in flight, and blocks of an SM (four rows at two blocks: 34 us
// for 31).
constexpr int kFwdHeads = 2;
constexpr int kFwdBlocks = 3;
// Backward: the rows of a slot on their way and the one at work, in shared memory (rows
// in registers, two at a time: 55 us for 46; two blocks of 256 threads 49, three blocks a
// SM spill).
constexpr int kBwdThreads = 128;
constexpr int kBwdWarps = kBwdThreads / 32;
constexpr int kBwdStages = 4;
constexpr int kBwdBlocks = 4;

// y_a = r (x_a (g_a cos) - x_b (g_b sin)),  y_b = r (x_b (g_b cos) + x_a (g_a sin)): the
// products in brackets are the token's.
template <typename T, bool INTER, int LANES>
__global__ void __launch_bounds__(kThreads, kFwdBlocks)
qk_forward_kernel(const __grid_constant__ Params P) {
    constexpr int V = vector_of<T>(), N = 2 * V, U = kFwdHeads;
    using C = Chunk<V, INTER>;
    const bool keys = blockIdx.x >= P.kind[0].blocks;
    const Kind& K = P.kind[keys];
    const uint32_t block = blockIdx.x - (keys ? P.kind[0].blocks : 0);
    const Slots<LANES> slots(P.lanes);
    const uint32_t slot = (block * kWarps + (threadIdx.x >> 5)) * slots.per_warp + slots.slot;
    const bool live = slot < K.slots && slots.sub * N < P.dim;
    const uint32_t token = slot / K.split, j = slot - token * K.split;
    const int64_t b = token / static_cast<uint32_t>(P.seq), s = token - b * P.seq;
    const C chunk(slots.sub, P.rot);
    const T* x = static_cast<const T*>(K.x.data) + K.x.at(b, s, j);
    T* y = static_cast<T*>(K.y.data) + K.y.at(b, s, j);
    const int64_t x_step = K.split * K.x.head_stride, y_step = K.split * K.y.head_stride;
    const float inv_n = 1.f / static_cast<float>(P.dim);
    f32x2 ac[V / 2], as[V / 2], bc[V / 2], bs[V / 2];
    chain_wait();
    for (int h = j; h - static_cast<int>(j) < K.heads; h += U * K.split, x += U * x_step, y += U * y_step) {
        RawRow<T, V> raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            raw[u].clear();
            if (live && h + u * static_cast<int>(K.split) < K.heads) raw[u].load(x + u * x_step, chunk.a, chunk.b);
        }
        if (h == j && live) {
            Angles<V> t;
            t.load(P, position_of(P, b, s), slots.sub, chunk.turned);
            const Members<V, INTER> g = load_gains(P, K, chunk);
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                ac[i] = mul2(g.a[i], t.c[i]);
                as[i] = mul2(g.a[i], t.s[i]);
                bc[i] = mul2(g.b[i], t.c[i]);
                bs[i] = mul2(g.b[i], mul2(t.s[i], twice(-1.f)));
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            Members<V, INTER> v(raw[u]);
            f32x2 ss = 0;
#pragma unroll
            for (int i = 0; i < V / 2; ++i) ss = fma2(v.a[i], v.a[i], fma2(v.b[i], v.b[i], ss));
            const f32x2 r = twice(rsqrtf(fmaf(slots.sum(sum2(ss)), inv_n, P.eps)));
            if (!live || h + u * static_cast<int>(K.split) >= K.heads) continue;
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const f32x2 a = mul2(v.a[i], r), b = mul2(v.b[i], r);
                v.a[i] = fma2(a, ac[i], mul2(b, bs[i]));
                v.b[i] = fma2(b, bc[i], mul2(a, as[i]));
            }
            v.store(y + u * y_step, chunk);
        }
    }
}

// The blocks stay and walk over the slots, with the gain gradient of their lanes'
// entries in registers; each leaves its sum for the join launch.  Every lane copies its
// own vectors of the rows to come to shared memory, in the background: a copy concerns
// no other lane, and rows on their way take no registers.
template <typename T, bool INTER, int LANES>
__global__ void __launch_bounds__(kBwdThreads, kBwdBlocks)
qk_backward_kernel(const __grid_constant__ Params P) {
    constexpr int V = vector_of<T>(), N = 2 * V;
    using C = Chunk<V, INTER>;
    using M = Members<V, INTER>;
    extern __shared__ uint4 stage[];        // [kBwdStages][4][kBwdThreads]; at the end the slots' sums
    __shared__ int64_t place[kBwdStages][kBwdThreads];     // positions
    const bool keys = blockIdx.x >= P.kind[0].blocks;
    const Kind& K = P.kind[keys];
    const uint32_t block = blockIdx.x - (keys ? P.kind[0].blocks : 0);
    const int warp = threadIdx.x >> 5;
    const Slots<LANES> slots(P.lanes);
    const bool mine = slots.sub * N < P.dim;
    const C chunk(slots.sub, P.rot);
    M g, acc;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) g.a[i] = g.b[i] = acc.a[i] = acc.b[i] = 0;
    Angles<V> t;
    chain_wait();
    if (mine) g = load_gains(P, K, chunk);
    const float inv_n = 1.f / static_cast<float>(P.dim);
    const uint32_t per_block = kBwdWarps * slots.per_warp;
    const uint64_t begin = static_cast<uint64_t>(block) * per_block + warp * slots.per_warp;
    const uint64_t step = static_cast<uint64_t>(K.blocks) * per_block;
    const int rows = static_cast<int>((K.heads + K.split - 1) / K.split);      // of a slot, at most
    const int64_t x_step = K.split * K.x.head_stride, dy_step = K.split * K.dy.head_stride;
    const int64_t dx_step = K.split * K.dx.head_stride;

    // The lane's slot of a group: whether there is one, its first head and its token.
    struct Where {
        bool live;
        uint32_t j;
        int64_t b, s;
    };
    auto where = [&](uint64_t first) {
        const uint64_t slot = first + slots.slot;
        const uint32_t token = static_cast<uint32_t>(slot) / K.split;
        const int64_t b = token / static_cast<uint32_t>(P.seq);
        return Where{slot < K.slots && mine, static_cast<uint32_t>(slot) - token * K.split, b, token - b * P.seq};
    };
    // The copies' place in the sequence of rows.
    uint64_t ahead = begin;
    int ahead_row = 0, ahead_slot = 0, ahead_stage = 0;
    bool to_live = false;
    int to_h = 0;
    const T *from_x = nullptr, *from_dy = nullptr;
    auto fetch = [&] {
        if (ahead < K.slots) {
            if (ahead_row == 0) {
                const Where to = where(ahead);
                to_live = to.live;
                to_h = to.j;
                from_x = static_cast<const T*>(K.x.data) + K.x.at(to.b, to.s, to.j);
                from_dy = static_cast<const T*>(K.dy.data) + K.dy.at(to.b, to.s, to.j);
                if (to.live && P.positions != nullptr) {
                    const int64_t i = to.b * P.positions_batch_stride + to.s;
                    int64_t* const at = &place[ahead_slot % kBwdStages][threadIdx.x];
                    if (P.positions_i64) copy_async<8>(at, static_cast<const int64_t*>(P.positions) + i);
                    else copy_async<4>(at, static_cast<const int32_t*>(P.positions) + i);
                }
            }
            if (to_live && to_h < K.heads) {
                uint4* const at = stage + ahead_stage * 4 * kBwdThreads + threadIdx.x;
                copy_async<16>(at, from_x + chunk.a);
                copy_async<16>(at + kBwdThreads, from_x + chunk.b);
                copy_async<16>(at + 2 * kBwdThreads, from_dy + chunk.a);
                copy_async<16>(at + 3 * kBwdThreads, from_dy + chunk.b);
            }
            from_x += x_step;
            from_dy += dy_step;
            to_h += K.split;
            if (++ahead_row == rows) {
                ahead_row = 0;
                ahead += step;
                ++ahead_slot;
            }
        }
        copies_commit();
        if (++ahead_stage == kBwdStages) ahead_stage = 0;
    };
#pragma unroll 1
    for (int k = 0; k < kBwdStages - 1; ++k) fetch();

    int at_stage = 0, at_slot = 0;
    for (uint64_t first = begin; first < K.slots; first += step, ++at_slot) {
        const Where w = where(first);
        T* dx = static_cast<T*>(K.dx.data) + K.dx.at(w.b, w.s, w.j);
#pragma unroll 1
        for (int i = 0, h = w.j; i < rows; ++i, h += K.split, dx += dx_step) {
            fetch();
            copies_wait<kBwdStages - 1>();
            if (i == 0 && w.live) {
                const int64_t* const p = &place[at_slot % kBwdStages][threadIdx.x];
                const int64_t pos = P.positions == nullptr ? w.s
                                    : P.positions_i64      ? *p
                                                           : *reinterpret_cast<const int32_t*>(p);
                t.load(P, pos, slots.sub, chunk.turned);
            }
            const bool here = w.live && h < K.heads;
            f32x2 ss = 0, ux = 0;
            M v, d;
            if (here) {
                const uint4* const at = stage + at_stage * 4 * kBwdThreads + threadIdx.x;
                float f[N];
                unpack<T>(at[0], f);
                unpack<T>(at[kBwdThreads], f + V);
                v.from(f);
                unpack<T>(at[2 * kBwdThreads], f);
                unpack<T>(at[3 * kBwdThreads], f + V);
                d.from(f);
#pragma unroll
                for (int k = 0; k < V / 2; ++k) {       // rotated back
                    const f32x2 da = fma2(d.b[k], t.s[k], mul2(d.a[k], t.c[k]));
                    const f32x2 db = fma2(mul2(d.a[k], twice(-1.f)), t.s[k], mul2(d.b[k], t.c[k]));
                    d.a[k] = da;
                    d.b[k] = db;
                    ss = fma2(v.a[k], v.a[k], fma2(v.b[k], v.b[k], ss));
                    ux = fma2(mul2(da, g.a[k]), v.a[k], fma2(mul2(db, g.b[k]), v.b[k], ux));
                }
            }
            if (++at_stage == kBwdStages) at_stage = 0;
            const float r1 = rsqrtf(fmaf(slots.sum(sum2(ss)), inv_n, P.eps));
            const f32x2 r = twice(r1), c = twice(-(r1 * (slots.sum(sum2(ux)) * inv_n)));
            if (here) {
#pragma unroll
                for (int k = 0; k < V / 2; ++k) {
                    const f32x2 a = mul2(v.a[k], r), b = mul2(v.b[k], r);     // normalised
                    acc.a[k] = fma2(d.a[k], a, acc.a[k]);
                    acc.b[k] = fma2(d.b[k], b, acc.b[k]);
                    v.a[k] = mul2(r, fma2(a, c, mul2(d.a[k], g.a[k])));
                    v.b[k] = mul2(r, fma2(b, c, mul2(d.b[k], g.b[k])));
                }
                v.store(dx, chunk);
            }
        }
    }
    copies_wait<0>();
    __syncthreads();
    float* const sums = reinterpret_cast<float*>(stage);
    if (mine) {
        float v[N];
        acc.to(v);
        float* const at = sums + (warp * slots.per_warp + slots.slot) * P.dim;
#pragma unroll
        for (int i = 0; i < N; ++i) at[chunk.entry(i)] = v[i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < P.dim; i += kBwdThreads) {
        float t = 0.f;
        for (int w = 0; w < kBwdWarps * slots.per_warp; ++w) t += sums[w * P.dim + i];
        K.parts[block * static_cast<int64_t>(P.dim) + i] = t;
    }
}

// ------------------------------------------------------- any size and alignment
// One warp per row, element by element: bound by instructions (a lane loads 2 or 4 bytes at
// a time, and a token's angles and the gains again for every head).
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
            const float da[1] = {r * (na * gain_at(P, K, ia) - xa[0] * c)};
            const float db[1] = {r * (nb * gain_at(P, K, ib) - xb[0] * c)};
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

// Gain gradients: a block adds up the parts of the queries or the keys for 32 entries,
// every warp each 32nd part.
__global__ void __launch_bounds__(1024)
qk_gain_kernel(const __grid_constant__ Params P) {
    __shared__ float sums[32][33];
    chain_wait();
    const Kind& K = P.kind[blockIdx.y];
    if (K.dgain == nullptr) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int i = blockIdx.x * 32 + lane;
    const float* const parts = after_wait(K.parts);
    constexpr int kLoads = 10;      // parts of a warp in flight
    float t = 0.f;
    for (int k0 = warp; k0 < K.blocks; k0 += 32 * kLoads) {
        float x[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int k = k0 + 32 * u;
            x[u] = k < K.blocks && i < P.dim ? parts[static_cast<int64_t>(k) * P.dim + i] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kLoads; ++u) t += x[u];
    }
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
    if (p == nullptr || p->batch < 0 || p->seq < 0 || p->table_rows < 0 || !(p->eps >= 0.f))
        return MALT_ERR_INVALID_ARG;
    if (!float_type(p->dtype) || !float_type(p->gain_dtype)) return MALT_ERR_UNSUPPORTED;
    if (p->head_dim < 1 || p->head_dim > kMaxHeadDim) return MALT_ERR_UNSUPPORTED;
    if (p->rot_dim < 0 || p->rot_dim > p->head_dim || p->rot_dim % 2 != 0) return MALT_ERR_INVALID_ARG;
    constexpr int64_t kMax = int64_t{1} << 31;
    if (p->batch >= kMax || p->seq >= kMax || p->batch * p->seq >= kMax) return MALT_ERR_UNSUPPORTED;
    if (p->rot_dim > 0 && p->table_rows > 0 && (p->cosines == nullptr || p->sines == nullptr))
        return MALT_ERR_INVALID_ARG;
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

// Whether the rows of a view can be read in vectors of V entries.
template <typename T, int V>
bool vectors(const Params& P, const Rows& r) {
    return aligned_to(r.data, V * sizeof(T)) && (P.batch == 1 || r.batch_stride % V == 0) &&
           (P.seq == 1 || r.seq_stride % V == 0) && r.head_stride % V == 0;
}

// Lanes of a row in the aligned kernels, 0 where they do not apply: a lane holds two vectors
// of 16 bytes, all turned or none.
template <typename T, int V>
int lanes_of(const Params& P, bool backward) {
    constexpr int N = 2 * V;
    if (P.dim % N != 0 || P.rot % N != 0 || P.dim / N > 32) return 0;
    if (!aligned_to(P.cosines, 16) || !aligned_to(P.sines, 16)) return 0;
    for (const Kind& K : P.kind) {
        if (K.heads == 0) continue;
        if (!vectors<T, V>(P, K.x)) return 0;
        if (backward ? !vectors<T, V>(P, K.dy) || !vectors<T, V>(P, K.dx) : !vectors<T, V>(P, K.y)) return 0;
    }
    return P.dim / N;
}

// Slots of a token for each kind.  Enough to give every SM `warps` warps; of these the
// number that costs least, a slot taking its heads in batches and, once, its token's
// place and angles, which cost about as much as kSlotCost heads.
constexpr double kSlotCost = 1.5;
void split_heads(Params& P, int lanes, int batch, int warps) {
    P.lanes = lanes;
    const int64_t tokens = P.batch * P.seq;
    const int64_t wanted = static_cast<int64_t>(sm_count()) * warps * (32 / lanes);
    for (Kind& K : P.kind) {
        K.gain_vectors = K.gain != nullptr && !P.gain_bf16 && aligned_to(K.gain, 16);
        int64_t best = std::max<int64_t>(K.heads, 1);
        double least = 1e30;
        for (int64_t split = 1; split <= K.heads && split <= kMaxSplit; ++split) {
            if (tokens * split < wanted && split < K.heads) continue;
            const int64_t heads = (K.heads + split - 1) / split;
            const double cost = split * ((heads + batch - 1) / batch * batch + kSlotCost);
            if (cost < least) least = cost, best = split;
        }
        if (tokens * best >= (int64_t{1} << 31)) best = 1;
        K.split = static_cast<uint32_t>(best);
        K.slots = K.heads == 0 ? 0 : static_cast<uint32_t>(tokens * best);
    }
}

template <typename T, bool INTER, int LANES>
cudaError_t forward_rows(Params& P, cudaStream_t s) {
    const int64_t kSlots = kWarps * (32 / P.lanes);
    for (Kind& K : P.kind) K.blocks = static_cast<int32_t>((K.slots + kSlots - 1) / kSlots);
    return launch_chained(qk_forward_kernel<T, INTER, LANES>, P.kind[0].blocks + P.kind[1].blocks, kThreads, 0, s, P);
}

template <typename T, bool INTER, int LANES>
cudaError_t backward_rows(Params& P, cudaStream_t s) {
    const int64_t kSlots = kBwdWarps * (32 / P.lanes);
    const int64_t heads = P.kind[0].heads + P.kind[1].heads;
    for (Kind& K : P.kind) {
        const int64_t all = static_cast<int64_t>(sm_count()) * kBwdBlocks;
        const int64_t share = K.heads > 0 ? std::max<int64_t>(1, all * K.heads / heads) : 0;
        K.blocks = static_cast<int32_t>(std::min<int64_t>((K.slots + kSlots - 1) / kSlots, share));
    }
    P.kind[1].parts = P.kind[0].parts + static_cast<int64_t>(P.kind[0].blocks) * P.dim;
    constexpr int kSmem = kBwdStages * 4 * kBwdThreads * 16;
    static_assert(kSmem >= kBwdThreads * 2 * vector_of<T>() * static_cast<int>(sizeof(float)),
                  "the sums of every lane's entries take the stages' place");
    static_assert(kBwdBlocks <= 6, "the workspace has a part for each block");
    auto* const kernel = qk_backward_kernel<T, INTER, LANES>;
    const cudaError_t rc = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (rc != cudaSuccess) { cudaGetLastError(); return rc; }
    return launch_chained(kernel, P.kind[0].blocks + P.kind[1].blocks, kBwdThreads, kSmem, s, P);
}

template <typename T, bool INTER>
cudaError_t forward_lanes(Params& P, int lanes, cudaStream_t s) {
    split_heads(P, lanes, kFwdHeads, 32);
    switch (lanes) {
        case 2: return forward_rows<T, INTER, 2>(P, s);
        case 4: return forward_rows<T, INTER, 4>(P, s);
        case 8: return forward_rows<T, INTER, 8>(P, s);
        case 16: return forward_rows<T, INTER, 16>(P, s);
        case 32: return forward_rows<T, INTER, 32>(P, s);
        default: return forward_rows<T, INTER, 0>(P, s);
    }
}

template <typename T, bool INTER>
cudaError_t backward_lanes(Params& P, int lanes, cudaStream_t s) {
    split_heads(P, lanes, 1, kBwdBlocks * kBwdWarps);
    switch (lanes) {
        case 2: return backward_rows<T, INTER, 2>(P, s);
        case 4: return backward_rows<T, INTER, 4>(P, s);
        case 8: return backward_rows<T, INTER, 8>(P, s);
        case 16: return backward_rows<T, INTER, 16>(P, s);
        case 32: return backward_rows<T, INTER, 32>(P, s);
        default: return backward_rows<T, INTER, 0>(P, s);
    }
}

template <typename T>
cudaError_t forward(Params& P, bool inter, cudaStream_t s) {
    if (const int lanes = lanes_of<T, vector_of<T>()>(P, false))
        return inter ? forward_lanes<T, true>(P, lanes, s) : forward_lanes<T, false>(P, lanes, s);
    for (Kind& K : P.kind) {
        static_assert(kMaxRows / kWarps <= int64_t{1} << 30, "the blocks of both kinds are a 32-bit number");
        K.blocks = static_cast<int32_t>((P.batch * P.seq * K.heads + kWarps - 1) / kWarps);
    }
    return launch_chained(inter ? qk_forward_any_kernel<T, true> : qk_forward_any_kernel<T, false>,
                          P.kind[0].blocks + P.kind[1].blocks, kThreads, 0, s, P);
}

template <typename T>
cudaError_t backward(Params& P, bool inter, cudaStream_t s) {
    if (const int lanes = lanes_of<T, vector_of<T>()>(P, true))
        return inter ? backward_lanes<T, true>(P, lanes, s) : backward_lanes<T, false>(P, lanes, s);
    const int64_t heads = P.kind[0].heads + P.kind[1].heads;
    for (Kind& K : P.kind) {
        const int64_t blocks = (P.batch * P.seq * K.heads + kWarps - 1) / kWarps;
        const int64_t all = backward_blocks();
        const int64_t share = K.heads > 0 ? std::max<int64_t>(1, all * K.heads / heads) : 0;
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
    if (tokens_of(p) * std::max(q->heads, k->heads) >= kMaxRows - kWarps) return MALT_ERR_UNSUPPORTED;
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
    if (workspace == nullptr || workspace_bytes < malt_qk_norm_workspace_bytes(p->head_dim))
        return MALT_ERR_INVALID_ARG;
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
