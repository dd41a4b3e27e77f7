// rms_norm.cu -- the RMS norm of a residual stream: the stream's addition, the norm (also
// to 8 bits with scales) and the gradient.
//
// Per row of dim entries, with sublayer output x, stream s and gain g:
//   h = x + s, rounded to the stream's type (h = x without a stream),
//   r = 1 / sqrt(mean(h^2) + eps),  y = h r g,
//   8 bits: per 128 entries scale = max(max |y|, 1e-30) / 448, code = e4m3(y / scale);
//   backward, u = dy g:  dx = r (u - h r mean(u h r)) + dh,  dg = sum over rows of dy h r.
//
// Bound by HBM: every operand once.  A row lies in the registers of one or more warps,
// loaded at once, so that it is read a single time; statistics go through shuffles, and
// between the warps of a row through shared memory.  16384 rows of 1280, bf16 added to an fp32
// stream: 37.5 us, 6.7 TB/s; to 8 bits from bf16: 28, 5.3 TB/s, by instructions.  Entries of a thread lie in vectors of
// eight, or one by one where rows are no multiple of eight or not aligned.
#include <cuda_fp8.h>

#include <algorithm>
#include <initializer_list>

#include <nvtx3/nvToolsExt.h>

#include "model_ops.cuh"

namespace malt {
namespace {

constexpr int kGroup = 128;             // entries that share a scale
constexpr float kMaxE4m3 = 448.f, kLeast = 1e-30f;
constexpr int kBlockWarps = 4;          // of a block whose rows take fewer
constexpr int kMaxWarps = 16;           // of a row
constexpr int kLoopThreads = 256;       // of a block of the loops over long or mixed rows
// Threads of a backward block whose threads hold K vectors of a row's three operands.
constexpr int grad_threads(int K) { return K <= 2 ? 512 : 128; }
constexpr int kGainBlocks = 2;          // blocks of the backward pass on an SM
constexpr int kMostSms = 256;           // that workspaces count on
constexpr int kGainSplit = 32;          // warps that add up the parts of 32 entries of dg

struct Rows {
    void* p;
    int64_t ld;
};

struct Params {
    Rows x, s, h, y;            // backward: dy, dh, h, dx
    const void* gain;
    float* scales;              // 8 bits
    int64_t scales_ld;
    float* parts;               // backward: [gridDim.x][dim] sums of dg, or null
    int32_t tokens, dim;
    int32_t warps;              // of a row
    float eps, inv_dim;
    int32_t gain_bf16, x_bf16, s_bf16, y_type;     // types of the loops over long or mixed rows
};

// VEC entries from p on as they are in memory.
template <typename T, int VEC>
struct Chunk {
    uint32_t w[VEC * sizeof(T) < 4 ? 1 : VEC * sizeof(T) / 4];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (VEC == 1) {
            if constexpr (sizeof(T) == 4) w[0] = __float_as_uint(*p);
            else w[0] = static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(p)) << 16;
        } else {
#pragma unroll
            for (int i = 0; i < VEC * static_cast<int>(sizeof(T)) / 16; ++i) {
                const uint4 u = reinterpret_cast<const uint4*>(p)[i];
                w[4 * i] = u.x, w[4 * i + 1] = u.y, w[4 * i + 2] = u.z, w[4 * i + 3] = u.w;
            }
        }
    }
    __device__ __forceinline__ float at(int i) const {
        if constexpr (sizeof(T) == 4 || VEC == 1) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
};

template <typename T>
__device__ __forceinline__ float rounded(float v) {
    if constexpr (sizeof(T) == 2) return __bfloat162float(__float2bfloat16_rn(v));
    else return v;
}

__device__ __forceinline__ float gain_at(const Params& P, int i) {
    if (P.gain == nullptr) return 1.f;
    return P.gain_bf16 ? __bfloat162float(static_cast<const bf16*>(P.gain)[i]) : static_cast<const float*>(P.gain)[i];
}

// The sum over the warps of a row, the same in all its threads.  `part` holds the warps of
// the block; every row of the block comes here equally often.
__device__ __forceinline__ float row_sum(float v, int warps, float* part) {
    v = warp_sum(v);
    if (warps == 1) return v;
    const int warp = threadIdx.x >> 5, first = warp - warp % warps;
    if ((threadIdx.x & 31) == 0) part[warp] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < warps; ++i) v += part[first + i];
    __syncthreads();
    return v;
}

// The larger by size, NaN last of all.
__device__ __forceinline__ float larger(float a, float b) { return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b))); }

__device__ __forceinline__ float scale_of(float largest) { return larger(largest, kLeast) / kMaxE4m3; }
__device__ __forceinline__ uint32_t code_pair(float a, float b) {
    return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}

// Y: bf16, float, or uint8_t for 8 bits.  K: vectors of a thread.
template <typename X, typename S, typename Y, int VEC, int K>
__global__ void __launch_bounds__(kMaxWarps * 32) rms_norm_kernel(const __grid_constant__ Params P) {
    __shared__ float part[kMaxWarps];
    const int span = P.warps * 32, t = threadIdx.x % span;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * (blockDim.x / span) + threadIdx.x / span;
    const bool on = row < P.tokens;
    chain_wait();
    const bool add = P.s.p != nullptr;
    const X* const x = static_cast<const X*>(P.x.p) + row * P.x.ld;
    const S* const s = static_cast<const S*>(P.s.p) + row * P.s.ld;
    Chunk<X, VEC> cx[K];
    Chunk<S, VEC> cs[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = (t + k * span) * VEC;
        cx[k] = {}, cs[k] = {};
        if (on && e < P.dim) {
            cx[k].load(x + e);
            if (add) cs[k].load(s + e);
        }
    }
    float sum = 0.f;
    float h[K][VEC];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            h[k][i] = add ? rounded<S>(cx[k].at(i) + cs[k].at(i)) : cx[k].at(i);
            sum = fmaf(h[k][i], h[k][i], sum);
        }
    if (on && add) {
        S* const to = static_cast<S*>(P.h.p) + row * P.h.ld;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = (t + k * span) * VEC;
            if (e < P.dim) store_vec<S, VEC>(to + e, h[k]);
        }
    }
    const float r = 1.f / sqrtf(row_sum(sum, P.warps, part) / P.dim + P.eps);
    Y* const y = static_cast<Y*>(P.y.p) + row * P.y.ld;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = (t + k * span) * VEC;
        const bool here = on && e < P.dim;
        float v[VEC] = {};
        if (here) {
            float g[VEC];
            if (P.gain == nullptr || VEC == 1) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) g[i] = gain_at(P, e + i);
            } else if (P.gain_bf16) {
                load_vec<bf16, VEC>(static_cast<const bf16*>(P.gain) + e, g);
            } else {
                load_vec<float, VEC>(static_cast<const float*>(P.gain) + e, g);
            }
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = h[k][i] * r * g[i];
        }
        if constexpr (sizeof(Y) > 1) {
            if (here) store_vec<Y, VEC>(y + e, v);
        } else {
            static_assert(VEC == 8, "16 lanes of eight entries share a scale");
            float a = fabsf(v[0]);
#pragma unroll
            for (int i = 1; i < VEC; ++i) a = larger(a, fabsf(v[i]));
#pragma unroll
            for (int d = 8; d > 0; d >>= 1) a = larger(a, __shfl_xor_sync(~0u, a, d));
            const float scale = scale_of(a), inv = 1.f / scale;     // (a quotient each: 6 us more)
            if (here) {
                uint2 u;
                u.x = code_pair(v[0] * inv, v[1] * inv) | code_pair(v[2] * inv, v[3] * inv) << 16;
                u.y = code_pair(v[4] * inv, v[5] * inv) | code_pair(v[6] * inv, v[7] * inv) << 16;
                *reinterpret_cast<uint2*>(y + e) = u;
                if (e % kGroup == 0) P.scales[row * P.scales_ld + e / kGroup] = scale;
            }
        }
    }
}

// A value of a type that the host gives.
__device__ __forceinline__ float load_as(const void* p, int64_t i, int is_bf16) {
    return is_bf16 ? __bfloat162float(static_cast<const bf16*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store_as(void* p, int64_t i, int is_bf16, float v) {
    if (is_bf16) static_cast<bf16*>(p)[i] = __float2bfloat16_rn(v);
    else static_cast<float*>(p)[i] = v;
}

__device__ __forceinline__ float block_sum(float v, float* part) {
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = 0.f;
    for (int i = 0; i < kLoopThreads / 32; ++i) v += part[i];
    __syncthreads();
    return v;
}

// Rows of any length, types and alignment, read a second time after their statistics.
__global__ void __launch_bounds__(kLoopThreads) rms_norm_loop_kernel(const __grid_constant__ Params P) {
    __shared__ float part[kLoopThreads / 32];
    const int64_t row = blockIdx.x;
    chain_wait();
    const bool add = P.s.p != nullptr;
    float sum = 0.f;
    for (int i = threadIdx.x; i < P.dim; i += kLoopThreads) {
        float h = load_as(P.x.p, row * P.x.ld + i, P.x_bf16);
        if (add) {
            h += load_as(P.s.p, row * P.s.ld + i, P.s_bf16);
            if (P.s_bf16) h = rounded<bf16>(h);
            store_as(P.h.p, row * P.h.ld + i, P.s_bf16, h);
        }
        sum = fmaf(h, h, sum);
    }
    const float r = 1.f / sqrtf(block_sum(sum, part) / P.dim + P.eps);
    const Rows& from = add ? P.h : P.x;
    const int from_bf16 = add ? P.s_bf16 : P.x_bf16;
    auto y_at = [&](int i) {
        return i < P.dim ? load_as(from.p, row * from.ld + i, from_bf16) * r * gain_at(P, i) : 0.f;
    };
    if (P.scales == nullptr) {
        for (int i = threadIdx.x; i < P.dim; i += kLoopThreads) store_as(P.y.p, row * P.y.ld + i, P.y_type == MALT_BF16, y_at(i));
        return;
    }
    uint8_t* const y = static_cast<uint8_t*>(P.y.p) + row * P.y.ld;
    const int lane = threadIdx.x & 31;
    for (int group = threadIdx.x >> 5; group * kGroup < P.dim; group += kLoopThreads / 32) {
        float v[kGroup / 32], a = 0.f;
#pragma unroll
        for (int k = 0; k < kGroup / 32; ++k) {
            v[k] = y_at(group * kGroup + k * 32 + lane);
            a = larger(a, fabsf(v[k]));
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) a = larger(a, __shfl_xor_sync(~0u, a, d));
        const float scale = scale_of(a), inv = 1.f / scale;
#pragma unroll
        for (int k = 0; k < kGroup / 32; ++k) {
            const int i = group * kGroup + k * 32 + lane;
            if (i < P.dim) y[i] = static_cast<uint8_t>(code_pair(v[k] * inv, 0.f));
        }
        if (lane == 0) P.scales[row * P.scales_ld + group] = scale;
    }
}

// Two sums over the warps of a row at once, with one barrier: `part` holds the warps' of two
// rows in turn.
__device__ __forceinline__ float2 row_sums(float2 v, int warps, float2* part) {
    v = make_float2(warp_sum(v.x), warp_sum(v.y));
    if (warps == 1) return v;
    const int warp = threadIdx.x >> 5, first = warp - warp % warps;
    if ((threadIdx.x & 31) == 0) part[warp] = v;
    __syncthreads();
    v = make_float2(0.f, 0.f);
    for (int i = 0; i < warps; ++i) v.x += part[first + i].x, v.y += part[first + i].y;
    return v;
}

// The sums of dg of a block's rows, one part per entry.
template <int VEC, int K>
__device__ __forceinline__ void store_parts(const Params& P, const float (&dg)[K][VEC], float* of_row, int t, int span,
                                            int per, int mine) {
    float* const out = P.parts + static_cast<int64_t>(blockIdx.x) * P.dim;
    if (per == 1) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const int e = (t + k * span) * VEC + i;
                if (e < P.dim) out[e] = dg[k][i];
            }
        return;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const int e = (t + k * span) * VEC + i;
            if (e < P.dim) of_row[mine * P.dim + e] = dg[k][i];
        }
    __syncthreads();
    for (int e = threadIdx.x; e < P.dim; e += blockDim.x) {
        float v = 0.f;
        for (int j = 0; j < per; ++j) v += of_row[j * P.dim + e];
        out[e] = v;
    }
}

// Eight gains from entry e on.
__device__ __forceinline__ void load_gains(const Params& P, int e, float (&g)[8]) {
    if (P.gain == nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = 1.f;
    } else if (P.gain_bf16) {
        load_vec<bf16, 8>(static_cast<const bf16*>(P.gain) + e, g);
    } else {
        load_vec<float, 8>(static_cast<const float*>(P.gain) + e, g);
    }
}

// Backward.  Blocks stay and take every gridDim.x-th set of rows; a row's operands and the sums
// of dg lie in registers, in as few warps as hold them: what a row costs apart from its
// entries (shuffles, a root, a barrier) comes once a warp.  16384 rows of 1280, bf16 dy, fp32
// h and dh: 57 us in one warp a row (5.1 TB/s), 61 in five with two barriers a row, 57 to 95
// with the next rows in shared memory, copied in the background by threads or in bulk.
template <typename D, typename H, int K>
__global__ void __launch_bounds__(grad_threads(K), 1) rms_norm_grad_kernel(const __grid_constant__ Params P) {
    constexpr int VEC = 8;
    __shared__ float2 part[2][kMaxWarps];
    extern __shared__ uint4 dynamic[];      // [rows of the block][dim] sums of dg
    const int span = P.warps * 32, t = threadIdx.x % span, per = blockDim.x / span, mine = threadIdx.x / span;
    chain_wait();
    float dg[K][VEC] = {};
    const int64_t step = static_cast<int64_t>(gridDim.x) * per;
    int turn = 0;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * per; first < P.tokens; first += step, turn ^= 1) {
        const int64_t row = first + mine;
        const bool on = row < P.tokens;
        const D* const pd = static_cast<const D*>(P.x.p) + row * P.x.ld;
        const H* const ph = static_cast<const H*>(P.h.p) + row * P.h.ld;
        const H* const pr = static_cast<const H*>(P.s.p) + row * P.s.ld;
        Chunk<D, VEC> cd[K];
        Chunk<H, VEC> ch[K], cr[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = (t + k * span) * VEC;
            cd[k] = {}, ch[k] = {}, cr[k] = {};
            if (on && e < P.dim) {
                ch[k].load(ph + e);
                cd[k].load(pd + e);
                if (P.s.p != nullptr) cr[k].load(pr + e);
            }
        }
        float2 sums = make_float2(0.f, 0.f);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = (t + k * span) * VEC;
            float g[VEC] = {};
            if (e < P.dim) load_gains(P, e, g);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float h = ch[k].at(i);
                sums.x = fmaf(h, h, sums.x);
                sums.y = fmaf(cd[k].at(i) * g[i], h, sums.y);
            }
        }
        sums = row_sums(sums, P.warps, part[turn]);
        const float r = rsqrtf(fmaf(sums.x, P.inv_dim, P.eps));
        const float c = sums.y * r * P.inv_dim;     // mean of u h r
        if (!on) continue;                          // (rows end with the last set)
        H* const dx = static_cast<H*>(P.y.p) + row * P.y.ld;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = (t + k * span) * VEC;
            if (e >= P.dim) continue;
            float g[VEC], v[VEC];
            load_gains(P, e, g);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float n = ch[k].at(i) * r, dy = cd[k].at(i);
                v[i] = fmaf(r, fmaf(-n, c, dy * g[i]), cr[k].at(i));
                dg[k][i] = fmaf(dy, n, dg[k][i]);
            }
            store_vec<H, VEC>(dx + e, v);
        }
    }
    if (P.parts != nullptr) store_parts<VEC, K>(P, dg, reinterpret_cast<float*>(dynamic), t, span, per, mine);
}

// The same one entry at a time, for rows off the vectors.
template <typename D, typename H, int K>
__global__ void __launch_bounds__(kMaxWarps * 32) rms_norm_grad_single_kernel(const __grid_constant__ Params P) {
    __shared__ float2 part[2][kMaxWarps];
    extern __shared__ uint4 dynamic[];      // [rows of the block][dim] sums of dg
    const int span = P.warps * 32, t = threadIdx.x % span, per = blockDim.x / span, mine = threadIdx.x / span;
    chain_wait();
    float dg[K][1] = {};
    const int64_t step = static_cast<int64_t>(gridDim.x) * per;
    int turn = 0;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * per; first < P.tokens; first += step, turn ^= 1) {
        const int64_t row = first + mine;
        const bool on = row < P.tokens;
        const D* const pd = static_cast<const D*>(P.x.p) + row * P.x.ld;
        const H* const ph = static_cast<const H*>(P.h.p) + row * P.h.ld;
        const H* const pr = static_cast<const H*>(P.s.p) + row * P.s.ld;
        Chunk<D, 1> cd[K];
        Chunk<H, 1> ch[K], cr[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = t + k * span;
            cd[k] = {}, ch[k] = {}, cr[k] = {};
            if (on && e < P.dim) {
                ch[k].load(ph + e);
                cd[k].load(pd + e);
                if (P.s.p != nullptr) cr[k].load(pr + e);
            }
        }
        float2 sums = make_float2(0.f, 0.f);
        float u[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = t + k * span;
            u[k] = e < P.dim ? cd[k].at(0) * gain_at(P, e) : 0.f;
            sums.x = fmaf(ch[k].at(0), ch[k].at(0), sums.x);
            sums.y = fmaf(u[k], ch[k].at(0), sums.y);
        }
        sums = row_sums(sums, P.warps, part[turn]);
        const float r = 1.f / sqrtf(sums.x / P.dim + P.eps);
        const float c = sums.y * r / P.dim;
        if (!on) continue;
        H* const dx = static_cast<H*>(P.y.p) + row * P.y.ld;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = t + k * span;
            if (e >= P.dim) continue;
            const float n = ch[k].at(0) * r;
            const float v[1] = {fmaf(r, fmaf(-n, c, u[k]), cr[k].at(0))};
            dg[k][0] = fmaf(cd[k].at(0), n, dg[k][0]);
            store_vec<H, 1>(dx + e, v);
        }
    }
    if (P.parts != nullptr) store_parts<1, K>(P, dg, reinterpret_cast<float*>(dynamic), t, span, per, mine);
}

// Rows past the registers: a block keeps its part of dg in global memory.
__global__ void __launch_bounds__(kLoopThreads) rms_norm_grad_loop_kernel(const __grid_constant__ Params P) {
    __shared__ float part[kLoopThreads / 32];
    chain_wait();
    float* const out = P.parts + static_cast<int64_t>(blockIdx.x) * P.dim;
    if (P.parts != nullptr)
        for (int i = threadIdx.x; i < P.dim; i += kLoopThreads) out[i] = 0.f;
    for (int64_t row = blockIdx.x; row < P.tokens; row += gridDim.x) {
        float sum = 0.f, dot = 0.f;
        for (int i = threadIdx.x; i < P.dim; i += kLoopThreads) {
            const float h = load_as(P.h.p, row * P.h.ld + i, P.s_bf16);
            sum = fmaf(h, h, sum);
            dot = fmaf(load_as(P.x.p, row * P.x.ld + i, P.x_bf16) * gain_at(P, i), h, dot);
        }
        sum = block_sum(sum, part);
        dot = block_sum(dot, part);
        const float r = 1.f / sqrtf(sum / P.dim + P.eps);
        const float c = dot * r / P.dim;
        for (int i = threadIdx.x; i < P.dim; i += kLoopThreads) {
            const float n = load_as(P.h.p, row * P.h.ld + i, P.s_bf16) * r;
            const float dy = load_as(P.x.p, row * P.x.ld + i, P.x_bf16);
            const float dh = P.s.p != nullptr ? load_as(P.s.p, row * P.s.ld + i, P.s_bf16) : 0.f;
            store_as(P.y.p, row * P.y.ld + i, P.s_bf16, fmaf(r, fmaf(-n, c, dy * gain_at(P, i)), dh));
            if (P.parts != nullptr) out[i] = fmaf(dy, n, out[i]);
        }
    }
}

// dg: the blocks' parts added up, 32 entries a block, its warps a share of the parts each (304
// parts of 1280: 32 warps instead of 8 took 1.6 us off).
__global__ void __launch_bounds__(32 * kGainSplit)
rms_norm_gain_kernel(const float* __restrict__ parts, int n, int dim, float* __restrict__ dgain) {
    __shared__ float of_warp[kGainSplit][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e = blockIdx.x * 32 + lane;
    chain_wait();
    parts = after_wait(parts);
    float v = 0.f;
    if (e < dim) {
#pragma unroll 8
        for (int j = warp; j < n; j += kGainSplit) v += parts[static_cast<int64_t>(j) * dim + e];
    }
    of_warp[warp][lane] = v;
    __syncthreads();
    if (warp == 0 && e < dim) {
#pragma unroll
        for (int j = 1; j < kGainSplit; ++j) v += of_warp[j][lane];
        dgain[e] = v;
    }
}

// ----------------------------------------------------------------------- host
int check_rows(const malt_rows_t* r, const malt_rms_norm_t* p, bool bytes = false) {
    if (r == nullptr || r->ld < p->dim || (p->tokens > 0 && r->data == nullptr)) return MALT_ERR_INVALID_ARG;
    if (bytes ? r->dtype != MALT_E4M3 : !float_type(r->dtype)) return MALT_ERR_UNSUPPORTED;
    return bytes || aligned_to(r->data, type_bytes(r->dtype)) ? MALT_OK : MALT_ERR_MISALIGNED;
}

Extent place_of(const malt_rows_t* r, const malt_rms_norm_t* p) {
    if (r == nullptr) return {};
    return extent_of(r->data, p->tokens, p->dim, r->ld, r->dtype == MALT_E4M3 ? 1 : type_bytes(r->dtype));
}
// Whether an output may lie where an input does: elsewhere, or entry on entry.
bool may_share(const malt_rows_t* out, const malt_rows_t* in, const malt_rms_norm_t* p) {
    if (out == nullptr || in == nullptr) return true;
    if (out->data == in->data && out->ld == in->ld && out->dtype == in->dtype) return true;
    return !overlap(place_of(out, p), place_of(in, p));
}
// Whether what is written beside them lies apart from all of them.
bool apart(const Extent& e, std::initializer_list<const malt_rows_t*> rows, const malt_rms_norm_t* p) {
    for (const malt_rows_t* r : rows)
        if (overlap(e, place_of(r, p))) return false;
    return true;
}
Extent gain_extent(const malt_rms_norm_t* p) { return extent_of(p->gain, p->dim * type_bytes(p->gain_dtype)); }

int check(const malt_rms_norm_t* p) {
    if (p == nullptr || p->tokens < 0 || p->dim < 1 || !(p->eps >= 0.f)) return MALT_ERR_INVALID_ARG;
    if (p->tokens >= (int64_t{1} << 31) - 64 || p->dim > (int64_t{1} << 24)) return MALT_ERR_UNSUPPORTED;
    if (p->gain != nullptr && !float_type(p->gain_dtype)) return MALT_ERR_UNSUPPORTED;
    return p->gain == nullptr || aligned_to(p->gain, type_bytes(p->gain_dtype)) ? MALT_OK : MALT_ERR_MISALIGNED;
}

// Rows whose vectors of eight entries lie on 16-byte addresses (8-bit ones on 8).
bool vectors(const malt_rows_t* r, int bytes) {
    return r == nullptr || (aligned_to(r->data, std::min(16, 8 * bytes)) && r->ld % 8 == 0);
}
bool vectors(const malt_rms_norm_t* p) {
    return p->dim % 8 == 0 && (p->gain == nullptr || aligned_to(p->gain, 16));
}

Params params_of(const malt_rms_norm_t* p) {
    Params P = {};
    P.gain = p->gain;
    P.gain_bf16 = p->gain_dtype == MALT_BF16;
    P.tokens = static_cast<int32_t>(p->tokens);
    P.dim = static_cast<int32_t>(p->dim);
    P.eps = p->eps;
    P.inv_dim = 1.f / static_cast<float>(p->dim);
    return P;
}
Rows rows_of(const malt_rows_t* r) { return r == nullptr ? Rows{} : Rows{r->data, r->ld}; }

// How a row of n vectors is split: into warps, with `each` vectors a thread.
struct Split {
    int warps, each;
    unsigned rows() const { return std::max(1, kBlockWarps / warps); }          // of a block
    unsigned threads() const { return rows() * static_cast<unsigned>(warps) * 32; }
};
// The one that leaves the fewest vectors unused, of those the one of fewest warps; no warps
// where none holds the row with `most` vectors a thread.
Split split_of(int64_t n, int most, int most_warps = kMaxWarps) {
    Split best{0, 0};
    int64_t least = INT64_MAX;
    for (int w = 1; w <= most_warps; ++w) {
        const int64_t each = (n + w * 32 - 1) / (w * 32);
        if (each <= most && w * each < least) {
            least = w * each;
            best = Split{w, static_cast<int>(each)};
        }
    }
    return best;
}
// Vectors of a thread.
constexpr int kForwardVectors = 5, kSingles = 16;

template <typename X, typename S, typename Y, int VEC, int K>
cudaError_t launch_forward(const Params& P, const Split& by, cudaStream_t s) {
    return launch_chained(rms_norm_kernel<X, S, Y, VEC, K>, (P.tokens + by.rows() - 1) / by.rows(), by.threads(), 0, s, P);
}

template <typename X, typename S, typename Y, int VEC>
cudaError_t forward_of(Params P, cudaStream_t s, bool* done) {
    const Split by = split_of(P.dim / VEC, VEC == 8 ? kForwardVectors : kSingles);
    P.warps = by.warps;
    *done = by.warps != 0;
    if (!*done) return cudaSuccess;
    if constexpr (VEC == 8) {
        switch (by.each) {
            case 1: return launch_forward<X, S, Y, VEC, 1>(P, by, s);
            case 2: return launch_forward<X, S, Y, VEC, 2>(P, by, s);
            case 3: return launch_forward<X, S, Y, VEC, 3>(P, by, s);
            case 4: return launch_forward<X, S, Y, VEC, 4>(P, by, s);
            default: return launch_forward<X, S, Y, VEC, 5>(P, by, s);
        }
    } else {
        if (by.each <= 4) return launch_forward<X, S, Y, VEC, 4>(P, by, s);
        if (by.each <= 8) return launch_forward<X, S, Y, VEC, 8>(P, by, s);
        return launch_forward<X, S, Y, VEC, 16>(P, by, s);
    }
}

template <typename X, typename S>
cudaError_t forward_of(const Params& P, int y_type, bool fast, cudaStream_t s, bool* done) {
    if (P.scales != nullptr) return fast ? forward_of<X, S, uint8_t, 8>(P, s, done) : cudaSuccess;
    if (y_type == MALT_BF16)
        return fast ? forward_of<X, S, bf16, 8>(P, s, done) : forward_of<X, S, bf16, 1>(P, s, done);
    return fast ? forward_of<X, S, float, 8>(P, s, done) : forward_of<X, S, float, 1>(P, s, done);
}

int forward(const malt_rms_norm_t* p, const malt_rows_t* x, const malt_rows_t* residual, const malt_rows_t* h,
            const malt_rows_t* y, float* scales, int64_t scales_ld, void* stream, const char* name) {
    int rc = check(p);
    if (rc == MALT_OK) rc = check_rows(x, p);
    if (rc == MALT_OK && (residual == nullptr) != (h == nullptr)) rc = MALT_ERR_INVALID_ARG;
    if (rc == MALT_OK && residual != nullptr) rc = check_rows(residual, p);
    if (rc == MALT_OK && h != nullptr) rc = check_rows(h, p);
    if (rc == MALT_OK && h != nullptr && h->dtype != residual->dtype) rc = MALT_ERR_UNSUPPORTED;
    if (rc == MALT_OK) rc = check_rows(y, p, scales != nullptr);
    if (rc != MALT_OK) return rc;
    if (p->tokens == 0) return MALT_OK;
    const Extent gain = gain_extent(p);
    const Extent of_scales = extent_of(scales, p->tokens, (p->dim + kGroup - 1) / kGroup, scales_ld, 4);
    if (!may_share(h, x, p) || !may_share(h, residual, p) || !may_share(y, x, p) || !may_share(y, residual, p) ||
        !apart(place_of(y, p), {h}, p) || !apart(gain, {h, y}, p) || !apart(of_scales, {x, residual, h, y}, p) ||
        overlap(of_scales, gain))
        return MALT_ERR_INVALID_ARG;
    Params P = params_of(p);
    P.x = rows_of(x), P.s = rows_of(residual), P.h = rows_of(h), P.y = rows_of(y);
    P.scales = scales;
    P.scales_ld = scales_ld;
    const int s_type = residual != nullptr ? residual->dtype : x->dtype;
    P.x_bf16 = x->dtype == MALT_BF16;
    P.s_bf16 = s_type == MALT_BF16;
    P.y_type = y->dtype;
    const bool fast = vectors(p) && vectors(x, type_bytes(x->dtype)) && vectors(residual, type_bytes(s_type)) &&
                      vectors(h, type_bytes(s_type)) && vectors(y, scales != nullptr ? 1 : type_bytes(y->dtype));
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    nvtxRangePushA(name);
    bool done = false;
    cudaError_t e = cudaSuccess;
    if (P.x_bf16 && P.s_bf16) e = forward_of<bf16, bf16>(P, y->dtype, fast, s, &done);
    else if (P.x_bf16) e = forward_of<bf16, float>(P, y->dtype, fast, s, &done);
    else if (!P.s_bf16) e = forward_of<float, float>(P, y->dtype, fast, s, &done);
    // Longer rows, fp32 rows added to a bf16 stream, and rows to 8 bits off the vectors.
    if (!done) e = launch_chained(rms_norm_loop_kernel, P.tokens, kLoopThreads, 0, s, P);
    nvtxRangePop();
    return cuda_status(e, name);
}

// Blocks of the backward pass: what the SMs hold, or one for each set of rows.
int64_t grad_blocks(int64_t tokens, int64_t per) {
    return std::min<int64_t>((tokens + per - 1) / per, kGainBlocks * std::min(sm_count(), kMostSms));
}

template <typename D, typename H, int K>
cudaError_t launch_grad(const Params& P, const Split& by, cudaStream_t s, unsigned blocks) {
    return launch_chained(rms_norm_grad_kernel<D, H, K>, blocks, by.threads(),
                          by.rows() > 1 ? by.rows() * P.dim * sizeof(float) : 0, s, P);
}

template <typename D, typename H, int K>
cudaError_t launch_single(const Params& P, const Split& by, unsigned blocks, cudaStream_t s) {
    return launch_chained(rms_norm_grad_single_kernel<D, H, K>, blocks, by.threads(),
                          by.rows() > 1 ? by.rows() * P.dim * sizeof(float) : 0, s, P);
}

template <typename D, typename H>
cudaError_t grad_of(const Params& P, const Split& by, bool fast, unsigned blocks, cudaStream_t s) {
    if (fast) {
        switch (by.each) {
            case 1: return launch_grad<D, H, 1>(P, by, s, blocks);
            case 2: return launch_grad<D, H, 2>(P, by, s, blocks);
            case 3: return launch_grad<D, H, 3>(P, by, s, blocks);
            case 4: return launch_grad<D, H, 4>(P, by, s, blocks);
            default: return launch_grad<D, H, 5>(P, by, s, blocks);
        }
    }
    if (by.each <= 4) return launch_single<D, H, 4>(P, by, blocks, s);
    if (by.each <= 8) return launch_single<D, H, 8>(P, by, blocks, s);
    return launch_single<D, H, 16>(P, by, blocks, s);
}

}  // namespace
}  // namespace malt

extern "C" {

int malt_rms_norm_forward(const malt_rms_norm_t* p, const malt_rows_t* x, const malt_rows_t* residual,
                          const malt_rows_t* h, const malt_rows_t* y, void* stream) {
    return malt::forward(p, x, residual, h, y, nullptr, 0, stream, "malt_rms_norm_forward");
}

int malt_rms_norm_forward_8bit(const malt_rms_norm_t* p, const malt_rows_t* x, const malt_rows_t* residual,
                               const malt_rows_t* h, const malt_rows_t* y, float* scales, int64_t scales_ld,
                               void* stream) {
    using namespace malt;
    if (p == nullptr || (p->tokens > 0 && scales == nullptr)) return MALT_ERR_INVALID_ARG;
    if (p->dim >= 1 && scales_ld < (p->dim + kGroup - 1) / kGroup) return MALT_ERR_INVALID_ARG;
    if (!aligned_to(scales, 4)) return MALT_ERR_MISALIGNED;
    // (a call for no rows may leave the scales out, and writes none)
    float dummy;
    return forward(p, x, residual, h, y, scales != nullptr ? scales : &dummy, scales_ld, stream,
                   "malt_rms_norm_forward_8bit");
}

size_t malt_rms_norm_workspace_bytes(int64_t tokens, int64_t dim) {
    if (tokens < 0 || dim < 1 || tokens >= (int64_t{1} << 31) - 64 || dim > (int64_t{1} << 24)) return 0;
    const int64_t blocks = std::max<int64_t>(1, std::min<int64_t>(tokens, malt::kGainBlocks * malt::kMostSms));
    return static_cast<size_t>(blocks * dim * 4);
}

int malt_rms_norm_backward(const malt_rms_norm_t* p, const malt_rows_t* dy, const malt_rows_t* h,
                           const malt_rows_t* dh, const malt_rows_t* dx, float* dgain, void* workspace,
                           size_t workspace_bytes, void* stream) {
    using namespace malt;
    int rc = check(p);
    if (rc == MALT_OK) rc = check_rows(dy, p);
    if (rc == MALT_OK) rc = check_rows(h, p);
    if (rc == MALT_OK && dh != nullptr) rc = check_rows(dh, p);
    if (rc == MALT_OK) rc = check_rows(dx, p);
    if (rc != MALT_OK) return rc;
    if (dx->dtype != h->dtype || (dh != nullptr && dh->dtype != h->dtype)) return MALT_ERR_UNSUPPORTED;
    if (!may_share(dx, dy, p) || !may_share(dx, h, p) || !may_share(dx, dh, p)) return MALT_ERR_INVALID_ARG;
    if (!aligned_to(dgain, 4)) return MALT_ERR_MISALIGNED;
    if (dgain != nullptr) {
        if (workspace == nullptr || workspace_bytes < malt_rms_norm_workspace_bytes(p->tokens, p->dim))
            return MALT_ERR_INVALID_ARG;
        if (!aligned_to(workspace, 16)) return MALT_ERR_MISALIGNED;
    }
    const Extent gain = gain_extent(p), of_gain = extent_of(dgain, p->dim * 4);
    const Extent parts =
        extent_of(dgain != nullptr ? workspace : nullptr, static_cast<int64_t>(malt_rms_norm_workspace_bytes(p->tokens, p->dim)));
    if (!apart(gain, {dx}, p) || !apart(of_gain, {dy, h, dh, dx}, p) || !apart(parts, {dy, h, dh, dx}, p) ||
        overlap(gain, of_gain) || overlap(gain, parts) || overlap(of_gain, parts))
        return MALT_ERR_INVALID_ARG;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (p->tokens == 0) {
        if (dgain == nullptr) return MALT_OK;
        return cuda_status(cudaMemsetAsync(dgain, 0, p->dim * sizeof(float), s), "malt_rms_norm_backward");
    }
    Params P = params_of(p);
    P.x = rows_of(dy), P.h = rows_of(h), P.s = rows_of(dh), P.y = rows_of(dx);
    P.parts = dgain != nullptr ? static_cast<float*>(workspace) : nullptr;
    P.x_bf16 = dy->dtype == MALT_BF16;
    P.s_bf16 = h->dtype == MALT_BF16;
    const int bytes = type_bytes(h->dtype);
    const bool fast = vectors(p) && vectors(dy, type_bytes(dy->dtype)) && vectors(h, bytes) && vectors(dh, bytes) &&
                      vectors(dx, bytes);
    Split by = fast ? split_of(p->dim / 8, 5, kBlockWarps) : split_of(p->dim, kSingles);
    if (fast && by.warps == 0) by = split_of(p->dim / 8, 2);
    P.warps = by.warps;
    const unsigned blocks = static_cast<unsigned>(grad_blocks(p->tokens, by.warps == 0 ? 1 : by.rows()));
    nvtxRangePushA("malt_rms_norm_backward");
    cudaError_t e;
    if (by.warps == 0) e = launch_chained(rms_norm_grad_loop_kernel, blocks, kLoopThreads, 0, s, P);
    else if (P.x_bf16 && P.s_bf16) e = grad_of<bf16, bf16>(P, by, fast, blocks, s);
    else if (P.x_bf16) e = grad_of<bf16, float>(P, by, fast, blocks, s);
    else if (P.s_bf16) e = grad_of<float, bf16>(P, by, fast, blocks, s);
    else e = grad_of<float, float>(P, by, fast, blocks, s);
    if (e == cudaSuccess && dgain != nullptr)
        e = launch_chained(rms_norm_gain_kernel, static_cast<unsigned>((p->dim + 31) / 32), 32 * kGainSplit, 0, s,
                           static_cast<const float*>(workspace), static_cast<int>(blocks), P.dim, dgain);
    nvtxRangePop();
    return cuda_status(e, "malt_rms_norm_backward");
}

}  // extern "C"
