// adamw8.cu -- the AdamW update of many tensors with its two moments in 8 bits each.
//
// Per tensor, at step t, with m and v as they are kept:
//   m' = b1 m + (1 - b1) g,  v' = b2 v + (1 - b2) g^2,
//   w <- (1 - lr wd) w - (lr / (1 - b1^t)) m' / (sqrt(v') / sqrt(1 - b2^t) + eps),
// and m' and s' = sqrt(v') are kept.  Blocks of 256 entries share an exponent E for each of
// the two, so that the largest is at most 1.9375 2^E; entries are 8-bit floats of 2^E:
//   m: sign, 3 bits of exponent, 4 of mantissa (1.9375 .. 2^-6, then steps of 2^-10),
//   s: 3 bits of exponent, 5 of mantissa (then steps of 2^-11).
// The root is kept, not v: its eight binades are sixteen of v.  An entry is rounded up with
// the probability of its remainder: to the nearest, an average would not move while a step
// changes it by less than half a code (b2 = 0.999 never, b1 = 0.9 within 60% of its goal).
// A root that is not zero never becomes zero: what divides the update stays above 2^-11 of
// the block's largest.  The random bits are a hash of seed, t, tensor and entry, so that a
// run repeats and replicas agree.
//
// A scale is a power of two: scaling is exact, an entry's code is the upper bits of its
// fp32 pattern once the exponent field holds the code's, and a carry out of the remainder is
// an integer addition.  m', v' and s' are rounded as IEEE says, fused only where written so.
//
// One warp takes a block: twice four neighbouring entries a lane, in registers from the loads
// to the stores.  Thread blocks stay and take an equal run of the blocks of all tensors each.
// Bound by HBM: 14 to 18 bytes an entry (w 8, moments 4, g 2 or 4, copy 2), 30 with fp32
// moments.  66 M entries of 219 tensors, bf16 gradients and copies: 179 us, 5.9 TB/s.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <vector>

#include <nvtx3/nvToolsExt.h>

#include "model_ops.cuh"

namespace {

using malt::bf16;

constexpr int kBlock = 256;                 // entries that share an exponent
constexpr int kEntries = kBlock / 32;       // of a lane
constexpr int kWarps = 8;                   // of a thread block
constexpr int kStages = 4;                  // blocks of a warp in shared memory
constexpr int kResident = 2;                // thread blocks of an SM
constexpr int kBindChunk = 400;             // tensors of a bind launch
constexpr uint32_t kLeastExponent = 27, kMostExponent = 254;
// The largest finite value's bits (its block's exponent would be 255 above).
constexpr uint32_t kMostBits = 0x7f780000u;
constexpr uint32_t kNan = 0xffu;            // a root's code, past every block's largest: both moments are NaN
constexpr float kUp = 0x1p120f, kDown = 0x1p-120f;      // a code's exponent field to a float's

struct Ptrs {
    float* w;
    void* copy;
    const void* g;
    uint8_t *m, *m_scale, *v, *v_scale;
    float decay;
    int32_t pad_;
};

struct Desc {
    int64_t numel;
    int64_t first;          // blocks of the tensors before
    int32_t g_bf16;
    int32_t pad_;
};

struct Hyper {
    float lr, beta1, beta2, eps;
};

// Of a step, computed once on the device.
struct Clock {
    long long t;
    float step, root_scale;     // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    uint32_t key;
    float beta1, beta2;         // what the powers are of, at step `powers_t`
    uint32_t pad_;
    long long powers_t;
    double power1, power2;
};

// N: of 32, 128 and kBindChunk the first that holds the launch's tensors (parameters are copied twice on
// their way: a step of 15 tensors and their moments 25 -> 22 us).
template <int N>
struct Bind {
    Ptrs p[N];
    Hyper h;
    Clock* clock;               // advanced by the first launch of a step, or null
    int32_t count, offset;
    uint32_t seed;
};
static_assert(sizeof(Bind<kBindChunk>) <= 32700, "a kernel's parameters");

// A hash of 32 bits: two multiplications by the fractions of the roots of 2 and 3.
__host__ __device__ __forceinline__ uint32_t mix(uint32_t x) {
    x = (x ^ x >> 16) * 0x6A09E667u;
    x = (x ^ x >> 15) * 0xBB67AE85u;
    return x ^ x >> 16;
}

template <int N>
__global__ void __launch_bounds__(N) bind_kernel(const __grid_constant__ Bind<N> B, Ptrs* __restrict__ table) {
    malt::chain_wait();
    const int i = malt::after_wait(static_cast<int>(threadIdx.x));
    if (i < B.count) table[B.offset + i] = B.p[i];
    if (i == 0 && B.clock != nullptr) {
        Clock c = *B.clock;
        c.t += 1;
        if (c.powers_t == c.t - 1 && c.powers_t > 0 && c.beta1 == B.h.beta1 && c.beta2 == B.h.beta2) {
            c.power1 *= static_cast<double>(B.h.beta1);     // (pow takes the one thread some 8 us)
            c.power2 *= static_cast<double>(B.h.beta2);
        } else {
            const double t = static_cast<double>(c.t);
            c.power1 = pow(static_cast<double>(B.h.beta1), t);
            c.power2 = pow(static_cast<double>(B.h.beta2), t);
        }
        c.powers_t = c.t;
        c.beta1 = B.h.beta1;
        c.beta2 = B.h.beta2;
        c.step = static_cast<float>(static_cast<double>(B.h.lr) / (1.0 - c.power1));
        c.root_scale = static_cast<float>(1.0 / sqrt(1.0 - c.power2));
        c.key = mix(mix(B.seed) ^ static_cast<uint32_t>(c.t));
        *B.clock = c;
    }
}

// Where a warp stands in the blocks of all tensors.
struct Place {
    const Desc* desc;
    const Ptrs* ptrs;
    int n, k;                   // tensors, the present one
    Desc d;
    Ptrs p;
    int64_t end;                // its last block's successor
    __device__ __forceinline__ void take() {
        d = desc[k];
        p = ptrs[k];
        end = d.first + (d.numel + kBlock - 1) / kBlock;
    }
    __device__ __forceinline__ Place(const Desc* desc_, const Ptrs* ptrs_, int n_, int k_)
        : desc(desc_), ptrs(ptrs_), n(n_), k(k_) {
        take();
    }
    __device__ __forceinline__ void go_to(int64_t block) {
        while (block >= end && k + 1 < n) {
            ++k;
            take();
        }
    }
};
// Where a run of blocks starts: the host divides the tensors' costs evenly.  A thread block of
// a step takes kRuns of them, one that reads or sets moments (of which an SM holds more) one.
constexpr int kRuns = 4;
struct Start {
    int64_t block;
    int32_t tensor;
    int32_t pad_;
};
// What changing to a tensor costs a thread block, in blocks of 256 (its descriptor, pointers and
// first operands are waited for).  Without it the thread blocks that the hundreds of vectors
// of a model fall to take 70 us longer than the others.
constexpr int64_t kTensorCost = 12;

// 2^(exponent - 127), for the bytes that a scale holds; 0 for 0 (states before their first step).
__device__ __forceinline__ float unit_of(uint32_t exponent) { return __uint_as_float(exponent << 23); }
__device__ __forceinline__ float m_value(uint32_t code, uint32_t root_code, float unit) {
    const float x = __uint_as_float((code & 0x7fu) << 19) * kUp * unit;
    return root_code == kNan ? __uint_as_float(0x7fffffffu) : code & 0x80u ? -x : x;
}
__device__ __forceinline__ float root_value(uint32_t code, float unit) {
    return code == kNan ? __uint_as_float(0x7fffffffu) : __uint_as_float(code << 18) * kUp * unit;
}

__device__ __forceinline__ uint32_t size_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ bool kept(uint32_t bits) { return bits <= kMostBits; }
// The exponent byte of a block from the bits of its largest finite value.
__device__ __forceinline__ uint32_t exponent_of(uint32_t bits) { return max((bits + 0x7ffffu) >> 23, kLeastExponent); }
__device__ __forceinline__ float inverse_unit(uint32_t exponent) {
    return __uint_as_float(exponent == kMostExponent ? 0x00400000u : (kMostExponent - exponent) << 23);
}
// Codes of values that are `kept`; random: 16 bits.
__device__ __forceinline__ uint32_t m_code(float m, float inverse, uint32_t random) {
    const uint32_t code = (__float_as_uint(fabsf(m) * inverse * kDown) + (random << 3)) >> 19;
    return code == 0 ? 0u : code | (__float_as_uint(m) >> 24 & 0x80u);
}
__device__ __forceinline__ uint32_t root_code(float root, float inverse, uint32_t random) {
    const uint32_t code = (__float_as_uint(fabsf(root) * inverse * kDown) + (random << 2)) >> 18;     // (-0: 0)
    return code == 0 && root > 0.f ? 1u : code;
}

// Exponent and codes of a block's eight values of this lane, in one of the two moments; those
// whose `fine` is not set are NaN.
struct Coded {
    uint32_t code[kEntries];
    uint32_t exponent;
};
template <bool ROOT>
__device__ __forceinline__ Coded encode(const float (&x)[kEntries], const bool (&fine)[kEntries],
                                        const uint32_t (&random)[kEntries]) {
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kEntries; ++i) most = max(most, fine[i] ? size_bits(x[i]) : 0u);
    most = __reduce_max_sync(~0u, most);
    Coded c;
    c.exponent = exponent_of(most);
    const float inverse = inverse_unit(c.exponent);
#pragma unroll
    for (int i = 0; i < kEntries; ++i) {
        if constexpr (ROOT) c.code[i] = fine[i] ? root_code(x[i], inverse, random[i] & 0xffffu) : kNan;
        else c.code[i] = fine[i] ? m_code(x[i], inverse, random[i] >> 16) : 0u;
    }
    return c;
}

__device__ __forceinline__ uint2 pack_codes(const uint32_t (&c)[kEntries]) {
    return make_uint2(c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24, c[4] | c[5] << 8 | c[6] << 16 | c[7] << 24);
}
__device__ __forceinline__ uint32_t code_at(const uint2& u, int i) { return (i < 4 ? u.x >> 8 * i : u.y >> 8 * (i - 4)) & 0xffu; }

// A lane's eight entries of a block: four from its first on, and four half a block later.
__device__ __forceinline__ constexpr int entry_of(int i) { return i < 4 ? i : kBlock / 2 - 4 + i; }
struct Entries {
    float w[kEntries], g[kEntries];
    uint2 m, v;                 // codes
    float m_unit, v_unit;
    uint32_t m_exponent, v_exponent;        // of the new codes
};

__device__ __forceinline__ float reciprocal(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// One at a time: blocks that hold or get values that are not finite.
__device__ __noinline__ void update_slow(Entries& x, const Hyper& h, float step, float root_scale, float decay,
                                         uint32_t first, uint32_t key) {
    float m[kEntries], root[kEntries];
    uint32_t random[kEntries];
    bool fine[kEntries];
    for (int i = 0; i < kEntries; ++i) {
        random[i] = mix((first + entry_of(i)) ^ key);
        m[i] = fmaf(h.beta1, m_value(code_at(x.m, i), code_at(x.v, i), x.m_unit), (1.f - h.beta1) * x.g[i]);
        const float s = root_value(code_at(x.v, i), x.v_unit);
        root[i] = sqrtf(fmaf(h.beta2, s * s, ((1.f - h.beta2) * x.g[i]) * x.g[i]));
        x.w[i] = fmaf(-step, m[i] * reciprocal(fmaf(root[i], root_scale, h.eps)), decay * x.w[i]);
        fine[i] = kept(size_bits(m[i])) && kept(size_bits(root[i]));
    }
    const Coded cm = encode<false>(m, fine, random), cv = encode<true>(root, fine, random);
    x.m = pack_codes(cm.code);
    x.v = pack_codes(cv.code);
    x.m_exponent = cm.exponent;
    x.v_exponent = cv.exponent;
}

__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// The uppermost bytes of four words.
__device__ __forceinline__ uint32_t upper_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return __byte_perm(__byte_perm(a, b, 0x0073), __byte_perm(c, d, 0x0073), 0x5410);
}
// The codes of four sums: magnitudes in bits 19 to 25, signs on top.
__device__ __forceinline__ uint32_t signed_codes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    return upper_bytes(a << 5, b << 5, c << 5, d << 5) | (upper_bytes(a, b, c, d) & 0x80808080u);
}
// Whether a byte is 0xff.
__device__ __forceinline__ bool has_nan(uint32_t u) { return (((u & 0x7f7f7f7fu) + 0x01010101u) & u & 0x80808080u) != 0; }

// The same in pairs: the same weights, moments' values and exponents (a negative m that rounds
// to zero has code 0x80 here, 0 there); the quotient that w takes is an approximate one, within
// 2 ulp.  The instructions per entry decide the kernel's time (66 M entries: 288 us with 106 of
// them, 179 with 69 and operands copied ahead).
__device__ __forceinline__ void update(Entries& x, const Hyper& h, float step, float root_scale, float decay,
                                       uint32_t first, uint32_t key) {
    using malt::add2;
    using malt::f32x2;
    using malt::fma2;
    using malt::mul2;
    using malt::pack2;
    using malt::unpack2;
    auto both = [](float v) { return pack2(v, v); };
    constexpr int kPairs = kEntries / 2;
    f32x2 m[kPairs], root[kPairs];
    float most_m = 0.f, most_root = 0.f;
#pragma unroll
    for (int p = 0; p < kPairs; ++p) {
        uint32_t mb[2], vb[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int i = 2 * p + j;
            // the code's byte on top: its sign in place, its magnitude five bits above a float's
            const uint32_t top = __byte_perm(i < 4 ? x.m.x : x.m.y, 0, 0x0444 | (i & 3) << 12);
            mb[j] = static_cast<uint32_t>(static_cast<int32_t>(top) >> 5) & 0x83f80000u;
            vb[j] = __byte_perm(i < 4 ? x.v.x : x.v.y, 0, 0x4044 | (i & 3) << 8) << 2;
        }
        const f32x2 g = pack2(x.g[2 * p], x.g[2 * p + 1]);
        const f32x2 old = mul2(mul2(pack2(__uint_as_float(mb[0]), __uint_as_float(mb[1])), both(kUp)), both(x.m_unit));
        const f32x2 s = mul2(mul2(pack2(__uint_as_float(vb[0]), __uint_as_float(vb[1])), both(kUp)), both(x.v_unit));
        m[p] = fma2(both(h.beta1), old, mul2(both(1.f - h.beta1), g));
        const float2 v = unpack2(fma2(both(h.beta2), mul2(s, s), mul2(mul2(both(1.f - h.beta2), g), g)));
        const float2 r = make_float2(sqrtf(v.x), sqrtf(v.y)), f = unpack2(m[p]);
        root[p] = pack2(r.x, r.y);
        most_m = max_nan(most_m, max_nan(fabsf(f.x), fabsf(f.y)));
        most_root = max_nan(most_root, max_nan(r.x, r.y));
    }
    if (has_nan(x.v.x) || has_nan(x.v.y)) most_root = INFINITY;
    const uint32_t mm = __reduce_max_sync(~0u, __float_as_uint(most_m));
    const uint32_t mr = __reduce_max_sync(~0u, __float_as_uint(most_root));
    if (!kept(mm) || !kept(mr)) {           // the same for all lanes
        Entries y = x;                      // (x itself stays in registers)
        update_slow(y, h, step, root_scale, decay, first, key);
        x = y;
        return;
    }
    x.m_exponent = exponent_of(mm);
    x.v_exponent = exponent_of(mr);
    const f32x2 im = both(inverse_unit(x.m_exponent)), iv = both(inverse_unit(x.v_exponent));
    uint32_t cm[kEntries], cv[kEntries];
#pragma unroll
    for (int p = 0; p < kPairs; ++p) {
        const float2 r = unpack2(root[p]), f = unpack2(m[p]);
        const float2 d = unpack2(fma2(root[p], both(root_scale), both(h.eps)));
        const f32x2 q = mul2(pack2(f.x, f.y), pack2(reciprocal(d.x), reciprocal(d.y)));
        const float2 w = unpack2(fma2(both(-step), q, mul2(both(decay), pack2(x.w[2 * p], x.w[2 * p + 1]))));
        x.w[2 * p] = w.x, x.w[2 * p + 1] = w.y;
        const float2 zm = unpack2(mul2(mul2(m[p], im), both(kDown))), zv = unpack2(mul2(mul2(root[p], iv), both(kDown)));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t random = mix((first + entry_of(2 * p + j)) ^ key);
            cm[2 * p + j] = (random >> 16) * 8 + __float_as_uint(j ? zm.y : zm.x);
            // (a root that is not 0 has a float's pattern above one code)
            cv[2 * p + j] = max((random & 0xffffu) * 4 + __float_as_uint(j ? zv.y : zv.x),
                                min(__float_as_uint(j ? r.y : r.x), 1u << 18)) << 6;
        }
    }
    x.m = make_uint2(signed_codes(cm[0], cm[1], cm[2], cm[3]), signed_codes(cm[4], cm[5], cm[6], cm[7]));
    x.v = make_uint2(upper_bytes(cv[0], cv[1], cv[2], cv[3]), upper_bytes(cv[4], cv[5], cv[6], cv[7]));
}

// Four entries from e on, those below `left` only; whole fours lie on 16 bytes (codes on 4).
template <typename T>
__device__ __forceinline__ void load_four(const T* p, int64_t left, float* x) {
    float v[4] = {};
    if (left >= 4) malt::load_vec<T, 4>(p, v);
    else
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            float one[1] = {0.f};
            if (i < left) malt::load_vec<T, 1>(p + i, one);
            v[i] = one[0];
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = v[i];
}
template <typename T>
__device__ __forceinline__ void store_four(T* p, int64_t left, const float* x) {
    const float v[4] = {x[0], x[1], x[2], x[3]};
    if (left >= 4) malt::store_vec<T, 4>(p, v);
    else
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const float one[1] = {v[i]};
            if (i < left) malt::store_vec<T, 1>(p + i, one);
        }
}
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, int64_t left) {
    if (left >= 4) return *reinterpret_cast<const uint32_t*>(p);
    uint32_t u = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i)
        if (i < left) u |= static_cast<uint32_t>(p[i]) << 8 * i;
    return u;
}
__device__ __forceinline__ void store_codes(uint8_t* p, int64_t left, uint32_t u) {
    if (left >= 4) *reinterpret_cast<uint32_t*>(p) = u;
    else
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < left) p[i] = static_cast<uint8_t>(u >> 8 * i);
}

// A tensor's last block, which is not whole: straight from memory.
__device__ __noinline__ void update_part(const Place& at, int64_t b, int lane, const Hyper& h, float step,
                                         float root_scale, uint32_t key) {
    const Ptrs& p = at.p;
    const int64_t e = b * kBlock + lane * 4;
    Entries x;
    uint32_t m[2], v[2];
    for (int q = 0; q < 2; ++q) {
        const int64_t i = e + q * (kBlock / 2), left = at.d.numel - i;
        load_four(p.w + i, left, x.w + 4 * q);
        if (at.d.g_bf16) load_four(static_cast<const bf16*>(p.g) + i, left, x.g + 4 * q);
        else load_four(static_cast<const float*>(p.g) + i, left, x.g + 4 * q);
        m[q] = load_codes(p.m + i, left);
        v[q] = load_codes(p.v + i, left);
    }
    x.m = make_uint2(m[0], m[1]);
    x.v = make_uint2(v[0], v[1]);
    x.m_unit = unit_of(p.m_scale[b]);
    x.v_unit = unit_of(p.v_scale[b]);
    update(x, h, step, root_scale, p.decay, static_cast<uint32_t>(e), key);
    for (int q = 0; q < 2; ++q) {
        const int64_t i = e + q * (kBlock / 2), left = at.d.numel - i;
        store_four(p.w + i, left, x.w + 4 * q);
        if (p.copy != nullptr) store_four(static_cast<bf16*>(p.copy) + i, left, x.w + 4 * q);
        store_codes(p.m + i, left, q ? x.m.y : x.m.x);
        store_codes(p.v + i, left, q ? x.v.y : x.v.x);
    }
    if (lane == 0) {
        p.m_scale[b] = static_cast<uint8_t>(x.m_exponent);
        p.v_scale[b] = static_cast<uint8_t>(x.v_exponent);
    }
}

// A block's operands in shared memory, copied there while the blocks before are computed.
struct Staged {
    float w[kBlock];
    float g[kBlock];            // bf16: the first half
    uint8_t m[kBlock], v[kBlock];
};
__device__ __forceinline__ void stage(Staged& to, const Place& at, int64_t b, int lane) {
    const Ptrs& p = at.p;
    const int64_t e = b * kBlock;
#pragma unroll
    for (int q = 0; q < 2; ++q) malt::copy_async<16>(to.w + 4 * lane + 128 * q, p.w + e + 4 * lane + 128 * q);
    if (at.d.g_bf16) {
        malt::copy_async<16>(reinterpret_cast<bf16*>(to.g) + 8 * lane, static_cast<const bf16*>(p.g) + e + 8 * lane);
    } else {
#pragma unroll
        for (int q = 0; q < 2; ++q)
            malt::copy_async<16>(to.g + 4 * lane + 128 * q, static_cast<const float*>(p.g) + e + 4 * lane + 128 * q);
    }
    const int part = 16 * (lane & 15);
    malt::copy_async<16>((lane < 16 ? to.m : to.v) + part, (lane < 16 ? p.m : p.v) + e + part);
}

__global__ void __launch_bounds__(kWarps * 32, kResident)
adamw8_kernel(const Desc* __restrict__ desc, const Ptrs* __restrict__ ptrs, int n, const Start* __restrict__ starts,
              const Clock* __restrict__ clock, Hyper h) {
    extern __shared__ uint4 staged_raw[];
    const Start start = starts[kRuns * blockIdx.x];
    const int64_t last = starts[kRuns * (blockIdx.x + 1)].block;
    int64_t at = start.block + (threadIdx.x >> 5);
    malt::chain_wait();
    if (at >= last) return;
    const int lane = threadIdx.x & 31;
    Staged* const ring = reinterpret_cast<Staged*>(staged_raw) + (threadIdx.x >> 5) * kStages;
    const Clock c = *malt::after_wait(clock);
    Place place(malt::after_wait(desc), malt::after_wait(ptrs), n, start.tensor);
    while (at < last) {
        place.go_to(at);
        const Ptrs& p = place.p;
        const uint32_t tensor_key = mix(c.key ^ static_cast<uint32_t>(place.k));
        // This warp's whole blocks of the tensor, 32 at most: a lane has the exponents of one.
        int64_t b = at - place.d.first;
        const int64_t end = min(last - place.d.first, place.d.numel / kBlock);
        const int count = static_cast<int>(min(static_cast<int64_t>(32), (end - b + kWarps - 1) / kWarps));
        if (count <= 0) {
            update_part(place, b, lane, h, c.step, c.root_scale,
                        mix(tensor_key + static_cast<uint32_t>((b * kBlock) >> 32)));
            at += kWarps;
            continue;
        }
        uint32_t m_scales = 0, v_scales = 0;
        if (lane < count) {
            m_scales = p.m_scale[b + lane * kWarps];
            v_scales = p.v_scale[b + lane * kWarps];
        }
#pragma unroll
        for (int j = 0; j < kStages - 1; ++j) {
            if (j < count) stage(ring[j], place, b + j * kWarps, lane);
            malt::copies_commit();
        }
        int slot = 0;
        uint32_t high = static_cast<uint32_t>((b * kBlock) >> 32), key = mix(tensor_key + high);
        for (int j = 0; j < count; ++j, b += kWarps) {
            malt::copies_wait<kStages - 2>();
            __syncwarp();                       // everyone's copies are there, and its last reads of the next slot done
            const Staged& from = ring[slot];
            Entries x;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const float4 w = *reinterpret_cast<const float4*>(from.w + 4 * lane + 128 * q);
                float* const xw = x.w + 4 * q;
                xw[0] = w.x, xw[1] = w.y, xw[2] = w.z, xw[3] = w.w;
                float* const xg = x.g + 4 * q;
                if (place.d.g_bf16) {
                    const uint2 g = *reinterpret_cast<const uint2*>(reinterpret_cast<const bf16*>(from.g) + 4 * lane + 128 * q);
                    xg[0] = __uint_as_float(g.x << 16), xg[1] = __uint_as_float(g.x & 0xffff0000u);
                    xg[2] = __uint_as_float(g.y << 16), xg[3] = __uint_as_float(g.y & 0xffff0000u);
                } else {
                    const float4 g = *reinterpret_cast<const float4*>(from.g + 4 * lane + 128 * q);
                    xg[0] = g.x, xg[1] = g.y, xg[2] = g.z, xg[3] = g.w;
                }
            }
            x.m = make_uint2(*reinterpret_cast<const uint32_t*>(from.m + 4 * lane),
                             *reinterpret_cast<const uint32_t*>(from.m + 4 * lane + 128));
            x.v = make_uint2(*reinterpret_cast<const uint32_t*>(from.v + 4 * lane),
                             *reinterpret_cast<const uint32_t*>(from.v + 4 * lane + 128));
            x.m_unit = unit_of(__shfl_sync(~0u, m_scales, j));
            x.v_unit = unit_of(__shfl_sync(~0u, v_scales, j));
            if (j + kStages - 1 < count)
                stage(ring[slot == 0 ? kStages - 1 : slot - 1], place, b + (kStages - 1) * kWarps, lane);
            malt::copies_commit();
            if (++slot == kStages) slot = 0;
            const int64_t e = b * kBlock + lane * 4;
            if (static_cast<uint32_t>(e >> 32) != high) {
                high = static_cast<uint32_t>(e >> 32);
                key = mix(tensor_key + high);
            }
            update(x, h, c.step, c.root_scale, p.decay, static_cast<uint32_t>(e), key);
            // the lane of this block keeps its new exponents
            if (lane == j) m_scales = x.m_exponent, v_scales = x.v_exponent;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const float* const w = x.w + 4 * q;
                reinterpret_cast<float4*>(p.w + e)[q * 32] = make_float4(w[0], w[1], w[2], w[3]);
                reinterpret_cast<uint32_t*>(p.m + e)[q * 32] = q ? x.m.y : x.m.x;
                reinterpret_cast<uint32_t*>(p.v + e)[q * 32] = q ? x.v.y : x.v.x;
                if (p.copy != nullptr)
                    reinterpret_cast<uint2*>(static_cast<bf16*>(p.copy) + e)[q * 32] =
                        make_uint2(malt::pack_bf16(w[0], w[1]), malt::pack_bf16(w[2], w[3]));
            }
        }
        b -= count * kWarps;
        if (lane < count) {
            p.m_scale[b + lane * kWarps] = static_cast<uint8_t>(m_scales);
            p.v_scale[b + lane * kWarps] = static_cast<uint8_t>(v_scales);
        }
        at += count * kWarps;
        __syncwarp();
    }
}

// The values of all states, tensor after tensor, each on a multiple of 256 with zeros behind
// its entries.  A warp takes a block, eight codes a lane, and all thread blocks are resident
// at once: 69 us for 66 M entries to bf16 (5.8 TB/s); 77 with sixteen codes a lane (each store
// half a sector) and as many blocks as 48 registers let in.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32, kRuns * kResident)
get_moments_kernel(const Desc* __restrict__ desc, const Ptrs* __restrict__ ptrs, int n, const Start* __restrict__ starts, T* m_values,
                   T* root_values) {
    const Start start = starts[blockIdx.x];
    const int64_t last = starts[blockIdx.x + 1].block;
    int64_t at = start.block + (threadIdx.x >> 5);
    malt::chain_wait();
    if (at >= last) return;
    const int part = 8 * (threadIdx.x & 31);
    Place place(malt::after_wait(desc), malt::after_wait(ptrs), n, start.tensor);
    for (; at < last; at += kWarps) {
        place.go_to(at);
        const Ptrs& p = place.p;
        const int64_t b = at - place.d.first, e = b * kBlock + part, left = place.d.numel - e;
        uint2 mc, vc;
        const uint8_t m_scale = p.m_scale[b], v_scale = p.v_scale[b];
        if (left >= 8) {
            mc = *reinterpret_cast<const uint2*>(p.m + e);
            vc = *reinterpret_cast<const uint2*>(p.v + e);
        } else {
            mc = make_uint2(load_codes(p.m + e, left), load_codes(p.m + e + 4, left - 4));
            vc = make_uint2(load_codes(p.v + e, left), load_codes(p.v + e + 4, left - 4));
        }
        const float m_unit = unit_of(m_scale), v_unit = unit_of(v_scale);
        const int64_t to = at * kBlock + part;
        float m[8], root[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[i] = m_value(code_at(mc, i), code_at(vc, i), m_unit);
            root[i] = root_value(code_at(vc, i), v_unit);
        }
        malt::store_vec<T, 8>(m_values + to, m);
        malt::store_vec<T, 8>(root_values + to, root);
    }
}

// The states of such values, rounded to the nearest code.
template <typename T>
__global__ void __launch_bounds__(kWarps * 32)
set_moments_kernel(const Desc* __restrict__ desc, const Ptrs* __restrict__ ptrs, int n, const Start* __restrict__ starts,
                   const T* m_values, const T* root_values) {
    const Start start = starts[blockIdx.x];
    const int64_t last = starts[blockIdx.x + 1].block;
    int64_t at = start.block + (threadIdx.x >> 5);
    malt::chain_wait();
    if (at >= last) return;
    const int lane = threadIdx.x & 31;
    Place place(malt::after_wait(desc), malt::after_wait(ptrs), n, start.tensor);
    for (; at < last; at += kWarps) {
        place.go_to(at);
        const Ptrs& p = place.p;
        const int64_t b = at - place.d.first, e = b * kBlock + lane * 4, from = at * kBlock + lane * 4;
        float m[kEntries], root[kEntries];
        uint32_t half[kEntries];
        bool fine[kEntries];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            load_four(m_values + from + q * (kBlock / 2), 4, m + 4 * q);
            load_four(root_values + from + q * (kBlock / 2), 4, root + 4 * q);
        }
#pragma unroll
        for (int i = 0; i < kEntries; ++i) {
            half[i] = 0x80008000u;
            if (e + entry_of(i) >= place.d.numel) m[i] = root[i] = 0.f;
            fine[i] = kept(size_bits(m[i])) && kept(size_bits(root[i])) && root[i] >= 0.f;
        }
        const Coded cm = encode<false>(m, fine, half), cv = encode<true>(root, fine, half);
        const uint2 mc = pack_codes(cm.code), vc = pack_codes(cv.code);
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            const int64_t i = e + q * (kBlock / 2), left = place.d.numel - i;
            store_codes(p.m + i, left, q ? mc.y : mc.x);
            store_codes(p.v + i, left, q ? vc.y : vc.x);
        }
        if (lane == 0) {
            p.m_scale[b] = static_cast<uint8_t>(cm.exponent);
            p.v_scale[b] = static_cast<uint8_t>(cv.exponent);
        }
    }
}

template <bool GET, typename T>
cudaError_t launch_moments(const Desc* desc, const Ptrs* ptrs, int n, unsigned grid, const Start* starts, void* m,
                           void* root, cudaStream_t s) {
    if constexpr (GET)
        return malt::launch_chained(get_moments_kernel<T>, grid, kWarps * 32, 0, s, desc, ptrs, n, starts,
                                    static_cast<T*>(m), static_cast<T*>(root));
    else
        return malt::launch_chained(set_moments_kernel<T>, grid, kWarps * 32, 0, s, desc, ptrs, n, starts,
                                    static_cast<const T*>(m), static_cast<const T*>(root));
}

constexpr size_t kSmem = sizeof(Staged) * kStages * kWarps;

#define ADAMW8_CUDA(call, what)                                 \
    do {                                                        \
        const int rc_ = malt::cuda_status((call), (what));      \
        if (rc_ != MALT_OK) return rc_;                         \
    } while (0)

bool aligned16(const void* p) { return malt::aligned_to(p, 16); }

int validate(const malt_adamw8_param_t& p) {
    if (p.w == nullptr || p.g == nullptr || p.m == nullptr || p.v == nullptr || p.m_scale == nullptr ||
        p.v_scale == nullptr)
        return MALT_ERR_INVALID_ARG;
    if (p.numel <= 0 || !malt::float_type(p.g_dtype)) return MALT_ERR_UNSUPPORTED;
    if (!(p.weight_decay == p.weight_decay)) return MALT_ERR_INVALID_ARG;
    if (!aligned16(p.w) || !aligned16(p.g) || !aligned16(p.m) || !aligned16(p.v) || !aligned16(p.w_copy))
        return MALT_ERR_MISALIGNED;
    return MALT_OK;
}

int64_t blocks_of(int64_t numel) { return numel / kBlock + (numel % kBlock != 0); }

}  // namespace

struct malt_adamw8_state {
    int device = 0;
    int n = 0;
    uint32_t seed = 0;
    std::vector<malt_adamw8_param_t> shape0;    // sizes and gradient types fixed at init
    void* ws = nullptr;
    Desc* d_desc = nullptr;
    Ptrs* d_ptrs = nullptr;         // of steps
    Ptrs* d_moment_ptrs = nullptr;  // of read-outs and sets: they may run beside a step's two launches
    Clock* d_clock = nullptr;
    Start* d_starts = nullptr;
    int32_t grid = 0;
    cudaStream_t last_stream = nullptr, moments_stream = nullptr;
};

namespace {

// The caller's tensors against those of init, and their pointers to the device.
int check_same(const malt_adamw8_state* st, const malt_adamw8_param_t* params, int32_t n) {
    if (n != st->n) return MALT_ERR_SHAPE_CHANGED;
    if (n > 0 && params == nullptr) return MALT_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        const int rc = validate(params[i]);
        if (rc != MALT_OK) return rc;
        if (params[i].numel != st->shape0[i].numel || params[i].g_dtype != st->shape0[i].g_dtype)
            return MALT_ERR_SHAPE_CHANGED;
    }
    return MALT_OK;
}

// hp: of a step, which the device's clock counts; null for the moments' table.
template <int N>
cudaError_t bind_some(const malt_adamw8_state* st, const malt_adamw8_param_t* params, int off, int count,
                      const malt_adamw_hparams_t* hp, cudaStream_t s) {
    Bind<N> B;
    B.count = count;
    B.offset = off;
    B.seed = st->seed;
    B.clock = hp != nullptr && off == 0 ? st->d_clock : nullptr;
    B.h = hp != nullptr ? Hyper{hp->lr, hp->beta1, hp->beta2, hp->eps} : Hyper{};
    for (int i = 0; i < count; ++i) {
        const malt_adamw8_param_t& p = params[off + i];
        const float decay = hp != nullptr ? 1.f - hp->lr * p.weight_decay : 1.f;
        B.p[i] = Ptrs{p.w, p.w_copy, p.g, p.m, p.m_scale, p.v, p.v_scale, decay, 0};
    }
    for (int i = count; i < N; ++i) B.p[i] = Ptrs{};
    return malt::launch_chained(bind_kernel<N>, 1, N, 0, s, B, hp != nullptr ? st->d_ptrs : st->d_moment_ptrs);
}
int bind(malt_adamw8_state* st, const malt_adamw8_param_t* params, const malt_adamw_hparams_t* hp, cudaStream_t s) {
    (hp != nullptr ? st->last_stream : st->moments_stream) = s;
    ADAMW8_CUDA(cudaSetDevice(st->device), "cudaSetDevice");
    for (int off = 0; off == 0 || off < st->n; off += kBindChunk) {
        const int count = std::min(kBindChunk, st->n - off);
        ADAMW8_CUDA(count <= 32 ? bind_some<32>(st, params, off, count, hp, s)
                    : count <= 128 ? bind_some<128>(st, params, off, count, hp, s)
                                   : bind_some<kBindChunk>(st, params, off, count, hp, s), "adamw8 bind_kernel");
    }
    return MALT_OK;
}

template <bool GET>
int moments(malt_adamw8_state* st, const malt_adamw8_param_t* params, int32_t n, void* m, void* root, int32_t dtype,
            void* stream, const char* name) {
    if (st == nullptr) return MALT_ERR_INVALID_ARG;
    int rc = check_same(st, params, n);
    if (rc != MALT_OK) return rc;
    if (!malt::float_type(dtype)) return MALT_ERR_UNSUPPORTED;
    if (st->grid == 0) return MALT_OK;
    if (m == nullptr || root == nullptr) return MALT_ERR_INVALID_ARG;
    if (!aligned16(m) || !aligned16(root)) return MALT_ERR_MISALIGNED;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    nvtxRangePushA(name);
    rc = bind(st, params, nullptr, s);
    if (rc == MALT_OK) {
        const cudaError_t e =
            dtype == MALT_BF16
                ? launch_moments<GET, bf16>(st->d_desc, st->d_moment_ptrs, n, kRuns * st->grid, st->d_starts, m, root, s)
                : launch_moments<GET, float>(st->d_desc, st->d_moment_ptrs, n, kRuns * st->grid, st->d_starts, m, root, s);
        rc = malt::cuda_status(e, name);
    }
    nvtxRangePop();
    return rc;
}

}  // namespace

extern "C" {

int malt_adamw8_init_state(malt_adamw8_state_t** out, const malt_adamw8_param_t* params, int32_t n, uint32_t seed,
                           void* stream) {
    if (out == nullptr) return MALT_ERR_INVALID_ARG;
    *out = nullptr;
    if (n < 0 || (n > 0 && params == nullptr)) return MALT_ERR_INVALID_ARG;
    int64_t total = 0;
    for (int i = 0; i < n; ++i) {
        const int rc = validate(params[i]);
        if (rc != MALT_OK) return rc;
        total += blocks_of(params[i].numel);
        if (total >= (int64_t{1} << 40)) return MALT_ERR_UNSUPPORTED;
    }
    malt_adamw8_state* st = nullptr;
    try {
        std::vector<Desc> desc(n);
        int64_t first = 0;
        for (int i = 0; i < n; ++i) {
            desc[i] = Desc{params[i].numel, first, params[i].g_dtype == MALT_BF16 ? 1 : 0, 0};
            first += blocks_of(params[i].numel);
        }
        st = new malt_adamw8_state();
        st->n = n;
        st->seed = seed;
        st->shape0.assign(params, params + n);
        st->grid = static_cast<int32_t>(std::min<int64_t>((total + kWarps - 1) / kWarps, kResident * malt::sm_count()));
        // Runs of equal cost: of a tensor kTensorCost, then its blocks.
        const int runs = kRuns * st->grid;
        std::vector<Start> starts(runs + 1);
        const int64_t cost = total + kTensorCost * n;
        int64_t before = 0;             // cost of the tensors before
        for (int i = 0, c = 0; c < runs; ++c) {
            const int64_t want = static_cast<int64_t>(static_cast<double>(cost) * c / runs);
            auto of = [&](int k) { return kTensorCost + blocks_of(params[k].numel); };
            while (i + 1 < n && before + of(i) <= want) before += of(i++);
            const int64_t inside = std::min(std::max<int64_t>(want - before - kTensorCost, 0), blocks_of(params[i].numel));
            starts[c] = Start{desc[i].first + inside, i, 0};
        }
        starts[runs] = Start{total, n > 0 ? n - 1 : 0, 0};
        auto fail = [&](int rc) {
            if (st->ws != nullptr) cudaFree(st->ws);
            delete st;
            return rc;
        };
        if (cudaGetDevice(&st->device) != cudaSuccess) {
            cudaGetLastError();
            return fail(MALT_ERR_CUDA);
        }
        const size_t nn = static_cast<size_t>(std::max(n, 1));
        auto aligned = [](size_t x) { return (x + 255) & ~size_t(255); };
        const size_t o_ptrs = aligned(sizeof(Desc) * nn), o_moment_ptrs = aligned(o_ptrs + sizeof(Ptrs) * nn);
        const size_t o_clock = aligned(o_moment_ptrs + sizeof(Ptrs) * nn);
        const size_t o_starts = o_clock + 256, bytes = aligned(o_starts + sizeof(Start) * (kRuns * st->grid + 1));
        if (cudaMalloc(&st->ws, bytes) != cudaSuccess) {
            st->ws = nullptr;
            cudaGetLastError();
            return fail(MALT_ERR_OUT_OF_MEMORY);
        }
        uint8_t* const base = static_cast<uint8_t*>(st->ws);
        st->d_desc = reinterpret_cast<Desc*>(base);
        st->d_ptrs = reinterpret_cast<Ptrs*>(base + o_ptrs);
        st->d_moment_ptrs = reinterpret_cast<Ptrs*>(base + o_moment_ptrs);
        st->d_clock = reinterpret_cast<Clock*>(base + o_clock);
        st->d_starts = reinterpret_cast<Start*>(base + o_starts);
        cudaStream_t s = static_cast<cudaStream_t>(stream);
        int rc = malt::cuda_status(cudaFuncSetAttribute(adamw8_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                        static_cast<int>(kSmem)), "cudaFuncSetAttribute(adamw8_kernel)");
        if (rc == MALT_OK) rc = malt::cuda_status(cudaMemset(st->ws, 0, bytes), "cudaMemset(state)");
        if (rc == MALT_OK && n > 0)
            rc = malt::cuda_status(cudaMemcpy(st->d_desc, desc.data(), sizeof(Desc) * n, cudaMemcpyHostToDevice),
                                   "cudaMemcpy(desc)");
        if (rc == MALT_OK)
            rc = malt::cuda_status(cudaMemcpy(st->d_starts, starts.data(), sizeof(Start) * starts.size(),
                                              cudaMemcpyHostToDevice), "cudaMemcpy(starts)");
        // The algorithm's m_0 = v_0 = 0.
        for (int i = 0; rc == MALT_OK && i < n; ++i) {
            const size_t k = static_cast<size_t>(params[i].numel), b = static_cast<size_t>(blocks_of(params[i].numel));
            void* const states[4] = {params[i].m, params[i].v, params[i].m_scale, params[i].v_scale};
            for (int j = 0; rc == MALT_OK && j < 4; ++j)
                rc = malt::cuda_status(cudaMemsetAsync(states[j], 0, j < 2 ? k : b, s), "cudaMemsetAsync(states)");
        }
        // (streams that do not wait for the default one may step next)
        if (rc == MALT_OK) rc = malt::cuda_status(cudaStreamSynchronize(nullptr), "cudaStreamSynchronize");
        if (rc != MALT_OK) return fail(rc);
        st->last_stream = st->moments_stream = s;
    } catch (...) {         // no host memory: no exception leaves a C entry
        delete st;
        return MALT_ERR_OUT_OF_MEMORY;
    }
    *out = st;
    return MALT_OK;
}

int malt_adamw8_step(malt_adamw8_state_t* st, const malt_adamw8_param_t* params, int32_t n,
                     const malt_adamw_hparams_t* hp, void* stream) {
    if (st == nullptr || hp == nullptr) return MALT_ERR_INVALID_ARG;
    if (!(hp->beta1 >= 0.f && hp->beta1 < 1.f) || !(hp->beta2 >= 0.f && hp->beta2 < 1.f) || !(hp->eps >= 0.f) ||
        !(hp->lr == hp->lr))
        return MALT_ERR_INVALID_ARG;
    int rc = check_same(st, params, n);
    if (rc != MALT_OK) return rc;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    nvtxRangePushA("malt_adamw8_step");
    rc = bind(st, params, hp, s);
    if (rc == MALT_OK && st->grid > 0)
        rc = malt::cuda_status(malt::launch_chained(adamw8_kernel, st->grid, kWarps * 32, kSmem, s, st->d_desc, st->d_ptrs,
                                                    n, st->d_starts, st->d_clock,
                                                    Hyper{hp->lr, hp->beta1, hp->beta2, hp->eps}), "adamw8_kernel");
    nvtxRangePop();
    return rc;
}

int malt_adamw8_get_moments(malt_adamw8_state_t* st, const malt_adamw8_param_t* params, int32_t n, void* m, void* root,
                            int32_t dtype, void* stream) {
    return moments<true>(st, params, n, m, root, dtype, stream, "malt_adamw8_get_moments");
}

int malt_adamw8_set_moments(malt_adamw8_state_t* st, const malt_adamw8_param_t* params, int32_t n, const void* m,
                            const void* root, int32_t dtype, void* stream) {
    return moments<false>(st, params, n, const_cast<void*>(m), const_cast<void*>(root), dtype, stream,
                          "malt_adamw8_set_moments");
}

int malt_adamw8_get_step(malt_adamw8_state_t* st, int64_t* t_host) {
    if (st == nullptr || t_host == nullptr) return MALT_ERR_INVALID_ARG;
    ADAMW8_CUDA(cudaStreamSynchronize(st->last_stream), "cudaStreamSynchronize");
    long long t = 0;
    ADAMW8_CUDA(cudaMemcpy(&t, &st->d_clock->t, sizeof(t), cudaMemcpyDeviceToHost), "cudaMemcpy(t)");
    *t_host = t;
    return MALT_OK;
}

int malt_adamw8_set_step(malt_adamw8_state_t* st, int64_t t_host) {
    if (st == nullptr || t_host < 0) return MALT_ERR_INVALID_ARG;
    ADAMW8_CUDA(cudaStreamSynchronize(st->last_stream), "cudaStreamSynchronize");
    const long long t = t_host;
    ADAMW8_CUDA(cudaMemcpy(&st->d_clock->t, &t, sizeof(t), cudaMemcpyHostToDevice), "cudaMemcpy(t)");
    ADAMW8_CUDA(cudaStreamSynchronize(nullptr), "cudaStreamSynchronize");
    return MALT_OK;
}

void malt_adamw8_destroy_state(malt_adamw8_state_t* st) {
    if (st == nullptr) return;
    cudaStreamSynchronize(st->last_stream);
    cudaStreamSynchronize(st->moments_stream);
    if (st->ws != nullptr) cudaFree(st->ws);
    delete st;
}

}  // extern "C"
