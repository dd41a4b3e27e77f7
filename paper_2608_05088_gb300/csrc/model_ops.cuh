// model_ops.cuh -- what the model operators (embed.cu, qk_norm.cu, distill.cu) share:
// element access in fp32, reductions, argument checks and launches.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <cstdio>
#include <utility>

#include "../../include/malt.h"
#include "chain.cuh"
#include "extent.h"

namespace malt {

using bf16 = __nv_bfloat16;

// ------------------------------------------------------------ element access
// VEC consecutive elements as fp32.  The address is aligned to VEC elements
// (at most 16 bytes at once).
template <typename T, int VEC>
__device__ __forceinline__ void load_vec(const T* p, float (&x)[VEC]) {
    constexpr int kBytes = sizeof(T) * VEC;
    if constexpr (sizeof(T) == 4) {
        if constexpr (kBytes == 4) {
            x[0] = *p;
        } else if constexpr (kBytes == 8) {
            const float2 a = *reinterpret_cast<const float2*>(p);
            x[0] = a.x, x[1] = a.y;
        } else {
#pragma unroll
            for (int i = 0; i < VEC; i += 4) {
                const float4 a = *reinterpret_cast<const float4*>(p + i);
                x[i] = a.x, x[i + 1] = a.y, x[i + 2] = a.z, x[i + 3] = a.w;
            }
        }
    } else if constexpr (VEC == 1) {
        x[0] = __bfloat162float(*p);
    } else {
        uint32_t u[VEC / 2];
        if constexpr (kBytes == 4) {
            u[0] = *reinterpret_cast<const uint32_t*>(p);
        } else if constexpr (kBytes == 8) {
            const uint2 a = *reinterpret_cast<const uint2*>(p);
            u[0] = a.x, u[1] = a.y;
        } else {
            const uint4 a = *reinterpret_cast<const uint4*>(p);
            u[0] = a.x, u[1] = a.y, u[2] = a.z, u[3] = a.w;
        }
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {     // a bf16 is the upper half of its fp32
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
}

// N elements as they are in memory, loaded at once.
template <typename T, int N>
struct alignas(sizeof(T) * N) Raw {
    T v[N];
};

// 16 bytes of T as fp32.
template <typename T>
__device__ __forceinline__ void unpack(const uint4& u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            x[i] = __uint_as_float(w[i]);
        } else {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

template <typename T, int VEC>
__device__ __forceinline__ void store_vec(T* p, const float (&x)[VEC]) {
    constexpr int kBytes = sizeof(T) * VEC;
    if constexpr (sizeof(T) == 4) {
        if constexpr (kBytes == 4) {
            *p = x[0];
        } else if constexpr (kBytes == 8) {
            *reinterpret_cast<float2*>(p) = make_float2(x[0], x[1]);
        } else {
#pragma unroll
            for (int i = 0; i < VEC; i += 4)
                *reinterpret_cast<float4*>(p + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
        }
    } else if constexpr (VEC == 1) {
        *p = __float2bfloat16_rn(x[0]);
    } else if constexpr (kBytes == 4) {
        *reinterpret_cast<uint32_t*>(p) = pack_bf16(x[0], x[1]);
    } else if constexpr (kBytes == 8) {
        *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
    } else {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]),
                                                  pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    }
}

// VEC (1 or 4) floats that another SM may have written in this launch: from L2.
template <int VEC>
__device__ __forceinline__ void load_l2(const float* p, float (&x)[VEC]) {
    static_assert(VEC == 1 || VEC == 4);
    if constexpr (VEC == 1) {
        x[0] = __ldcg(p);
    } else {
        const float4 a = __ldcg(reinterpret_cast<const float4*>(p));
        x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w;
    }
}

// ---------------------------------------------------------------- reductions
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(~0u, v, d);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, d));
    return v;
}

// 2^x; the hardware's approximation (relative error about 2^-22), 2^-inf = 0.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// BYTES (4, 8 or 16, both addresses aligned to them) from global to shared memory in the
// background.  The copies since the last commit are a group; copies_wait<N> waits for all
// groups of this thread but the last N, and makes them visible to it alone.
template <int BYTES>
__device__ __forceinline__ void copy_async(void* to, const void* from) {
    const uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(to));
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Two floats in a 64-bit register: the packed arithmetic issues one instruction for both.
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pack2(float a, float b) {
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 unpack2(f32x2 v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
    f32x2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// --------------------------------------------------------------- host checks
inline bool float_type(int32_t t) { return t == MALT_F32 || t == MALT_BF16; }
inline bool index_type(int32_t t) { return t == MALT_I32 || t == MALT_I64; }
inline int type_bytes(int32_t t) { return t == MALT_BF16 ? 2 : t == MALT_I64 ? 8 : 4; }
inline bool aligned_to(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

inline int cuda_status(cudaError_t e, const char* what) {
    if (e == cudaSuccess) return MALT_OK;
    std::fprintf(stderr, "malt: %s failed: %s\n", what, cudaGetErrorString(e));
    return MALT_ERR_CUDA;
}

// SMs of the current device (looked up once per device).
inline int sm_count() {
    constexpr int kDevices = 64;
    static std::atomic<int> counts[kDevices] = {};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return 1; }
    const bool known = dev >= 0 && dev < kDevices;
    if (known && counts[dev].load(std::memory_order_relaxed) > 0) return counts[dev].load(std::memory_order_relaxed);
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return 1;
    }
    if (known) counts[dev].store(n, std::memory_order_relaxed);
    return n;
}

// launch_chained with clusters of `cluster` blocks along x.  A cluster of one is launched as
// no cluster: those blocks start more slowly (16384 distillation rows of 2000: 53 us as
// clusters, 46 without).
template <typename... Params, typename... Args>
cudaError_t launch_clusters(void (*kernel)(Params...), unsigned blocks, unsigned cluster, unsigned threads,
                            size_t smem, cudaStream_t s, Args&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, std::forward<Args>(args)...);
    if (e != cudaSuccess) cudaGetLastError();
    return e;
}

}  // namespace malt
