// head.cu -- softmax cross entropy of an output head, and its gradients, without keeping
// the logits.
//
// With hidden rows h_n (dim entries), table W (vocab x dim), labels y_n and weights w_n:
//   l_nv = h_n . W_v,  m_n = max_v l_nv,  s_n = sum_v exp(l_nv - m_n),
//   loss_n = w_n (log s_n + m_n - l_n,y_n),
//   dl_nv = w_n (exp(l_nv - m_n) / s_n - [v = y_n]),
//   dh_n = sum_v dl_nv W_v,  dW_v (+)= sum_n dl_nv h_n.
//
// Every product runs on the tensor cores (tcgen05, two SMs a tile of 256 x 256, fp32
// accumulators in TMEM).  Forward, a tile of logits leaves TMEM as a maximum and a sum per
// row.  Backward, the logits are formed again, a piece of the vocabulary at a time: dl of a
// piece leaves TMEM in bf16, stays in L2, and is read from there by the tiles of dh and dW.
// head_plan.h has the order of the work; a tile waits on device counters for what it reads,
// so that the three products overlap and leave no tail between pieces.
//
// Rows that do not count (negative labels, weight 0) are left out: the others are gathered
// first, which also gives them the layout that TMA wants.
//
// Precision.  bf16 operands: their products are exact, dl is rounded once to bf16, as the
// operand of the two products that it goes into (of up to 128 rows to the sum of two planes:
// with few terms an entry their roundings do not average out; 3 to 6 us).  With fp32 operands
// each operand is the sum of three bf16 planes (24 bits), dl too, and a product is the six of
// planes i and j with i + j <= 2: what is left out is below 2^-24 of the result's terms.
//
// Bound by the tensor cores: 2 N V D flop forward, 8 N V D with the gradients (6 with the
// logits kept), and for few rows by reading the table.  8192 rows of 1280 against 50304, a tenth
// left out: 2.39 to 2.72 ms for loss and gradients, 1.40 to 1.59 PFLOP/s at the power cap
// (the forward product alone 495 us, 1.94 PFLOP/s).
#include <cuda.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <cstring>
#include <mutex>
#include <type_traits>

#include <nvtx3/nvToolsExt.h>

#include "head_plan.h"
#include "model_ops.cuh"
#include "ptx.cuh"

namespace malt {
namespace {

constexpr int kTile = kHeadTile;
constexpr int kHalf = kTile / 2;                    // rows of a tile in one CTA
constexpr int kSlice = 64;                          // reduction of a slice: one 128-byte row
constexpr int kSlices = 6, kGroup = 2, kRing = kSlices / kGroup;
constexpr uint32_t kABytes = kHalf * kSlice * 2, kBox = kSlice * kSlice * 2;
constexpr uint32_t kSliceBytes = 2 * kABytes;
constexpr int kEpiWarps = 8;
constexpr int kChunks = kTile / 2 / 32;             // of 32 columns, of an epilogue warp
constexpr uint32_t kOutBox = 32 * 32 * 2;
constexpr size_t kSmem = static_cast<size_t>(kSlices) * kSliceBytes + 2 * kEpiWarps * kOutBox + 1024;
constexpr int kThreads = 64 + 32 * kEpiWarps + 32;  // producer, MMA, epilogue, signals
constexpr int kItemSlots = 3, kSigSlots = 4;
constexpr uint32_t kItemReaders = 5 + 2 * kEpiWarps;
constexpr uint32_t kSignals = 2;                    // of a finished tile: one a CTA
constexpr float kLog2 = 1.4426950408889634f;
constexpr int32_t kEnd = -1;
constexpr int kMostPairs = 80;                      // that a launch has
constexpr int kPlanes = 3;                          // of an fp32 operand
constexpr int64_t kTurnedRows = 128;                // up to which the gradient's products are turned
// Slices after which a sum leaves TMEM for fp32 sums in memory: TMEM's are cut off, not rounded, at every 16
// terms, by up to 2^-23 of what they have reached (sums of one sign, whose products reach far below it, by up to
// three times that).  A logit's part ends after 2048 terms, so that what is lost does not grow with the dimension
// (loss of 4096 rows of 4096 against 32000, bf16: 650 us in one part, 730 in two, a maximum 1.5e-6 and 8e-7 off);
// with fp32 operands after 512 (loss of 1000 rows of 1600 against 16000: 238 us with 2048, 254 with 1024, 275 with
// 512; m + log s of rows of 4096 are off by 7.3e-6, 4.7e-6 and 2.6e-6 on the average, those of fp32 products 2.5e-6).
constexpr int kLogitPart = 32, kExactLogitPart = 8, kSumPart = 16;
// What a sum of n such steps loses on the average: its partial sums lie, on the average, on the
// line from 0 to the result x whatever their path, and a step loses half a unit in the last
// place of them, 0.72 2^-24 of their size: n / 2 * 0.72 * 2^-24 x in all, which is put back.  A
// step of 16 zeros loses nothing: of a logit, n is at most the steps in which its hidden row has
// entries, so that a sum of one term is that term.
constexpr float kLostPerStep = 0.36f * 0x1p-24f;

// Planes (i, j) of the products that a product is the sum of, four bits each.
struct Pairs {
    uint32_t a, b;
    int32_t n;
};

struct Gemm {
    CUtensorMap h_k, h_mn, w_k, w_mn, d_k, d_mn, d_out, acc_out, t_out;
    HeadPlan plan;
    Pairs logits, hidden, table;
    int32_t backward, d_planes;
    int32_t dim, dim_ld, vocab;
    int32_t row_ld;                 // compact rows that buffers hold
    const int32_t* live;            // their number
    const int32_t* labels;          // of compact rows
    const float* weights;
    const float2* stats;            // backward: (m, s)
    float2* parts;                  // forward: [2 vocab_tiles][row_ld] (m, s)
    const float* label_logits;
    void* dtable;
    int64_t dtable_ld;
    int32_t dtable_bf16, accumulate;
    int32_t dtable_boxes;           // dW goes out by t_out
    int32_t exact;                  // gradients' sums leave TMEM in parts, logits in shorter ones
    const int32_t* steps;           // of compact rows: 16s of the dimension in which they are not 0
    float* scratch;                 // of the logits' parts: [CTAs][kTile / 2 x kTile]
    int32_t columns;                // TURNED: of the products, 64 or 128
    int32_t abreast;                // TURNED: dl's two planes side by side in dH's product
    uint32_t *queue, *row_done, *col_done, *hidden_done, *piece_done;
    int32_t* status;
    uint64_t budget_ns;
};

using Mn = std::true_type;
using Kn = std::false_type;

template <bool A_MN, bool B_MN>
__device__ __forceinline__ void mma_slice(uint32_t d, uint32_t sa, uint32_t idesc, bool first) {
    const uint32_t sb = sa + kABytes;
    const uint64_t da = A_MN ? smem_desc_mn_sw128(sa, kBox) : smem_desc_k_sw128(sa);
    const uint64_t db = B_MN ? smem_desc_mn_sw128(sb, kBox) : smem_desc_k_sw128(sb);
    // per 16 of the reduction: 32 bytes of a K-major row, or two atoms of 8 rows (1 KB)
    constexpr uint32_t kStepA = A_MN ? 2048u >> 4 : 2u, kStepB = B_MN ? 2048u >> 4 : 2u;
#pragma unroll
    for (int k = 0; k < kSlice / 16; ++k)
        tc_mma_16bit_pair(d, da + kStepA * k, db + kStepB * k, idesc | idesc_majors(A_MN, B_MN),
                          first && k == 0 ? 0u : 1u);
}

__device__ __forceinline__ void give_up(const Gemm& P, volatile int* abort_flag) {
    atomicOr(P.status, 1);
    *abort_flag = 1;
}

// What an item's tile multiplies: slices of `kb` per pair of planes, columns of its B side,
// and the parts of the reduction that leave TMEM one by one, `part` slices each.
struct Shape {
    Pairs pairs;
    int32_t kb, parts, part;
    int32_t subs;               // tiles of the dimension that the item takes one by one
    __device__ __forceinline__ int slices(int p) const { return min(part, kb - p * part); }
};
// Columns of the product of a tile of the dimension.
template <bool TURNED>
__device__ __forceinline__ int columns_of(const Gemm& P, const HeadItem& it, int dt) {
    if (TURNED && it.kind != kHeadTable) return it.kind == kHeadHidden && P.abreast ? 2 * P.columns : P.columns;
    return it.kind > kHeadLogits && P.dim - dt * kTile <= kHalf ? kHalf : kTile;
}
__device__ __forceinline__ Shape shape_of(const Gemm& P, const HeadItem& it, int live) {
    Shape s;
    s.subs = it.kind == kHeadTable && P.plan.wide ? P.plan.dim_tiles : 1;
    if (it.kind <= kHeadLogits) {
        s.pairs = P.logits;
        s.kb = (P.dim + kSlice - 1) / kSlice;
        s.part = P.exact ? kExactLogitPart : kLogitPart;
        s.parts = (s.kb + s.part - 1) / s.part;
        return s;
    }
    if (it.kind == kHeadHidden) {
        s.pairs = P.hidden;
        const int from = it.piece * P.plan.piece_tiles, to = min(P.plan.vocab_tiles, from + P.plan.piece_tiles);
        s.kb = (min(P.vocab, to * kTile) - from * kTile + kSlice - 1) / kSlice;
    } else {
        s.pairs = P.table;
        s.kb = (live + kSlice - 1) / kSlice;
    }
    // (a bf16 dW holds no sums in parts, and needs none)
    s.part = P.exact && !(it.kind == kHeadTable && P.dtable_bf16) ? kSumPart : max(1, s.kb);
    s.parts = max(1, (s.kb + s.part - 1) / s.part);
    return s;
}

__device__ __forceinline__ HeadItem item_of(const Gemm& P, int mt, int index) {
    if (P.backward) return head_item(P.plan, mt, index);
    HeadItem it;
    it.kind = kHeadStats;
    it.piece = 0;
    it.vt = index / mt;
    it.mt = index - it.vt * mt;
    it.dt = 0;
    return it;
}

// Max and sum of exp2((v - max) c) of a row's 32 columns, those from `cols` on left out.
struct RowSum {
    float m = -INFINITY, s = 0.f;
    __device__ __forceinline__ void add(const float (&v)[32], int cols) {
        float top = v[0];
        if (cols < 32) {
            top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 32; ++j) top = j < cols ? fmaxf(top, v[j]) : top;
        } else {
#pragma unroll
            for (int j = 1; j < 32; ++j) top = fmaxf(top, v[j]);
        }
        const float next = fmaxf(m, top);
        if (next > m) {
            s *= exp2_fast((m - next) * kLog2);
            m = next;
        }
        const float base = m == -INFINITY ? 0.f : m;
        const f32x2 nm = pack2(-base, -base), c = pack2(kLog2, kLog2);
        f32x2 sum = pack2(s, 0.f);
        if (cols >= 32) {
#pragma unroll
            for (int j = 0; j < 32; j += 2) {
                const float2 e = unpack2(mul2(add2(pack2(v[j], v[j + 1]), nm), c));
                sum = add2(sum, pack2(exp2_fast(e.x), exp2_fast(e.y)));
            }
            const float2 h = unpack2(sum);
            s = h.x + h.y;
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if (j < cols) s += exp2_fast((v[j] - base) * kLog2);
        }
    }
};

// 32 rows of 16 floats from shared memory to, or added to, the box of a tensor at (c0, c1, c2).
template <bool ADD>
__device__ __forceinline__ void store_box(const CUtensorMap* map, const void* box, int c0, int c1, int c2) {
    if constexpr (ADD)
        asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2, %3}], [%4];"
                     ::"l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(box)) : "memory");
    else
        tma_store_3d(map, box, c0, c1, c2);
}

// What a row's logits need; the loads of compact row n.
struct RowData {
    int label = -1;             // entry of the table
    int steps = 0;
    float weight = 0.f, m = 0.f, inv = 0.f, of_label = 0.f;
    template <bool BACKWARD>
    __device__ __forceinline__ void load(const Gemm& P, int n) {
        of_label = P.label_logits[n];
        label = P.labels[n];
        steps = P.steps[n];
        if (BACKWARD) {
            weight = P.weights[n];
            const float2 st = P.stats[n];
            m = st.x;
            inv = weight / st.y;
        }
    }
};

// dl of 32 logits of a row from column 0 of the chunk on: label's column, or -1; those from
// `cols` on are no entries of the table.
__device__ __forceinline__ void logits_gradient(float (&v)[32], float m, float inv, float weight, int label, int cols) {
    const f32x2 nm = pack2(-m, -m), c = pack2(kLog2, kLog2), ii = pack2(inv, inv);
#pragma unroll
    for (int j = 0; j < 32; j += 2) {
        const float2 e = unpack2(mul2(add2(pack2(v[j], v[j + 1]), nm), c));
        const float2 g = unpack2(mul2(pack2(exp2_fast(e.x), exp2_fast(e.y)), ii));
        v[j] = g.x, v[j + 1] = g.y;
    }
    if (__any_sync(~0u, label >= 0)) {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j == label) v[j] -= weight;
    }
    if (cols < 32) {
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (j >= cols) v[j] = 0.f;
    }
}

// A lane's row of 32 in bf16 into the box of a store with 64-byte swizzle; v keeps what the
// rounding left, which the next plane holds.
__device__ __forceinline__ void stage_bf16(float (&v)[32], uint8_t* box, int lane, bool keep) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float& a = v[8 * q + 2 * j];
            float& b = v[8 * q + 2 * j + 1];
            w[j] = pack_bf16(a, b);
            if (keep) {
                a -= __uint_as_float(w[j] << 16);
                b -= __uint_as_float(w[j] & 0xffff0000u);
            }
        }
        *reinterpret_cast<uint4*>(box + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// 32 x 32 floats, a lane's row each, to (or added to, in L2) a tensor of `cols` columns at (c0, c1,
// c2), in two boxes of 16 columns; obuf: the next of the warp's two boxes in shared memory.
__device__ __forceinline__ void store_square(const CUtensorMap* map, const float (&v)[32], uint8_t* boxes, int& obuf,
                                             bool add, int cols, int c0, int c1, int c2, int lane) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (c0 + 16 * half >= cols) continue;
        uint8_t* const box = boxes + obuf * kOutBox;
        if (lane == 0) bulk_wait_group_read<1>();       // the box's last store has read it
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float* const f = v + 16 * half + 4 * q;
            *reinterpret_cast<float4*>(box + lane * 64 + ((q ^ ((lane >> 1) & 3)) << 4)) = make_float4(f[0], f[1], f[2], f[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
            if (add) store_box<true>(map, box, c0 + 16 * half, c1, c2);
            else store_box<false>(map, box, c0 + 16 * half, c1, c2);
            bulk_commit_group();
        }
        obuf ^= 1;
    }
}

// The same in bf16, stored, in one box; v keeps what the rounding left if `keep`.
__device__ __forceinline__ void store_square_bf16(const CUtensorMap* map, float (&v)[32], uint8_t* boxes, int& obuf,
                                                  bool keep, int c0, int c1, int c2, int lane) {
    uint8_t* const box = boxes + obuf * kOutBox;
    if (lane == 0) bulk_wait_group_read<1>();
    __syncwarp();
    stage_bf16(v, box, lane, keep);
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
        tma_store_3d(map, box, c0, c1, c2);
        bulk_commit_group();
    }
    obuf ^= 1;
}

// 32 x 32 of dW where no box can go: rows that start anywhere, bf16 ones that are added to.  The
// warp turns the square in shared memory (4 KB, no store reading it) and takes it row by row
// (1454 rows of 501 added to 32003: a third of the time of each lane on its row).
__device__ __forceinline__ void store_table(const Gemm& P, const float (&v)[32], int row0, int col0, bool add,
                                            uint8_t* square, int lane) {
    if (lane == 0) bulk_wait_group_read<0>();
    __syncwarp();
    float* const sq = reinterpret_cast<float*>(square);
#pragma unroll
    for (int j = 0; j < 32; ++j) sq[lane * 32 + (j ^ lane)] = v[j];
    __syncwarp();
    const int rows = min(32, P.vocab - row0);
    if (col0 + lane >= P.dim) return;
    const int64_t first = static_cast<int64_t>(row0) * P.dtable_ld + col0 + lane;
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += 16) {
        float x[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            x[r] = 0.f;
            if (add && r0 + r < rows) {
                const int64_t i = first + (r0 + r) * P.dtable_ld;
                x[r] = P.dtable_bf16 ? __bfloat162float(static_cast<const bf16*>(P.dtable)[i])
                                     : static_cast<const float*>(P.dtable)[i];
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (r0 + r >= rows) continue;
            const int64_t i = first + (r0 + r) * P.dtable_ld;
            x[r] += sq[(r0 + r) * 32 + (lane ^ (r0 + r))];
            if (P.dtable_bf16) static_cast<bf16*>(P.dtable)[i] = __float2bfloat16_rn(x[r]);
            else static_cast<float*>(P.dtable)[i] = x[r];
        }
    }
}

// dl of a table entry (a lane's) and 32 rows, whose m, weight / s, weight, label and its logit lie
// in the lanes; entry: of the table, or -1 past its end.
__device__ __forceinline__ void logits_gradient_turned(float (&v)[32], const RowData& r, int entry) {
    const int first = __shfl_sync(~0u, entry, 0);       // (of a warp's entries; -1 if none counts)
    const unsigned labelled = __ballot_sync(~0u, first >= 0 && r.label >= first && r.label < first + 32);
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const float m = __shfl_sync(~0u, r.m, j), inv = __shfl_sync(~0u, r.inv, j);
        float off = 0.f;
        if (labelled >> j & 1) {
            const int label = __shfl_sync(~0u, r.label, j);
            const float of_label = __shfl_sync(~0u, r.of_label, j), weight = __shfl_sync(~0u, r.weight, j);
            if (label == entry) v[j] = of_label, off = weight;
        }
        v[j] = entry >= 0 ? fmaf(exp2_fast((v[j] - m) * kLog2), inv, -off) : 0.f;
    }
}

// store_square_bf16 of a square whose lanes have its columns.
__device__ __forceinline__ void store_turned_bf16(const CUtensorMap* map, float (&v)[32], uint8_t* boxes, int& obuf,
                                                  bool keep, int c0, int c1, int c2, int lane) {
    uint8_t* const box = boxes + obuf * kOutBox;
    if (lane == 0) bulk_wait_group_read<1>();
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 32; ++j) {
        const bf16 b = __float2bfloat16_rn(v[j]);
        if (keep) v[j] -= __bfloat162float(b);
        *reinterpret_cast<bf16*>(box + j * 64 + (((lane >> 3) ^ ((j >> 1) & 3)) << 4) + (lane & 7) * 2) = b;
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
        tma_store_3d(map, box, c0, c1, c2);
        bulk_commit_group();
    }
    obuf ^= 1;
}

// TURNED (up to kTurnedRows rows, backward): the products of logits and dH the other way round, table
// entries or the dimension as their rows and hidden rows as their columns, so that they cost what
// there is of them (loss and gradients of 24 rows of 1280 against 50304: 149 -> 137 us).
template <bool BACKWARD, bool TURNED = false>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
head_gemm_kernel(const __grid_constant__ Gemm P) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[kRing], empty_bar[kRing], tfull_bar[2], tempty_bar[2], drain_bar;
    __shared__ __align__(8) uint64_t item_full[kItemSlots], item_empty[kItemSlots], sig_bar[kSigSlots];
    __shared__ __align__(16) int4 item_ring[kItemSlots];
    // TURNED: what puts back the loss of a logit's part, and of its last one, per compact row
    __shared__ __align__(16) float back_of[TURNED ? 2 : 1][TURNED ? kTurnedRows : 4];
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_sh;
    volatile int* abort_flag = &abort_sh;
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                               ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = static_cast<int>(cluster_ctarank());
    const bool leader = rank == 0;
    const uint64_t budget = P.budget_ns;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kRing; ++s) {
            mbar_init(&full_bar[s], 2);         // both producers
            mbar_init(&empty_bar[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(&tfull_bar[a], 1);
            mbar_init(&tempty_bar[a], 2 * kEpiWarps);
        }
        mbar_init(&drain_bar, 1);
        for (int s = 0; s < kItemSlots; ++s) {
            mbar_init(&item_full[s], 1);
            mbar_init(&item_empty[s], kItemReaders - (BACKWARD ? 0 : 2));
        }
        for (int s = 0; s < kSigSlots; ++s) mbar_init(&sig_bar[s], kEpiWarps);
        abort_sh = 0;
        fence_barrier_init();
        fence_proxy_async_smem();
    }
    if (warp == 0 && lane == 0) {
        tma_prefetch_desc(&P.h_k);
        tma_prefetch_desc(&P.w_k);
        if (BACKWARD) {
            tma_prefetch_desc(&P.h_mn);
            tma_prefetch_desc(&P.w_mn);
            tma_prefetch_desc(&P.d_k);
            tma_prefetch_desc(&P.d_mn);
            tma_prefetch_desc(&P.d_out);
            tma_prefetch_desc(&P.acc_out);
        }
    }
    if (warp == 1) {
        tmem_alloc_pair(&tmem_slot, 2 * kTile);
        tmem_relinquish_pair();
    }
    chain_wait();
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem_base = tmem_slot;
    const int live = *after_wait(P.live);
    const int mt = (live + kTile - 1) / kTile;
    const uint32_t items = BACKWARD ? head_items(P.plan, mt) : static_cast<uint32_t>(mt * P.plan.vocab_tiles);

    // Item number `seq` of this pair, from the ring that the odd CTA's scheduler fills: its
    // index in the order of work, or kEnd; false when the wait gave up.
    auto ring_free = [&](int seq) {
        mbar_arrive_cluster_relaxed(mapa_shared(smem_u32(&item_empty[seq % kItemSlots]), 1));
    };
    auto ring_peek = [&](int seq, int& index) -> bool {
        const int slot = seq % kItemSlots;
        if (!mbar_wait_cluster_bounded(&item_full[slot], static_cast<uint32_t>(seq / kItemSlots) & 1u, budget, abort_flag))
            return false;
        index = ld_shared_v4(&item_ring[slot]).x;
        return true;
    };
    auto ring_item = [&](int seq, int& index) -> bool {
        if (!ring_peek(seq, index)) return false;
        if (index >= kEnd) ring_free(seq);      // (always: the branch keeps the read before the release)
        return true;
    };
    auto reached = [&](const uint32_t* counter, uint32_t target) -> bool {
        return counter_wait_bounded(counter, target, budget, P.status, 1, abort_flag);
    };
    auto piece_tiles = [&](int piece) {
        return min(P.plan.piece_tiles, P.plan.vocab_tiles - piece * P.plan.piece_tiles);
    };
    // Whether what the item's operands were computed from is in memory.
    auto operands_done = [&](const HeadItem& it) -> bool {
        if (it.kind == kHeadHidden)
            return reached(P.row_done + it.piece * P.plan.row_tiles + it.mt, kSignals * piece_tiles(it.piece));
        if (it.kind == kHeadTable) return reached(P.col_done + it.vt, kSignals * mt);
        return true;
    };

    if (warp == 0) {
        // ---------------------------------------------------- TMA producer
        if (lane == 0) {
            uint32_t stage = 0, phase = 0;
            for (int seq = 0;; ++seq) {
                int index;
                if (!ring_item(seq, index)) { give_up(P, abort_flag); break; }
                if (index == kEnd) break;
                const HeadItem it = item_of(P, mt, index);
                if (BACKWARD) {
                    if (!operands_done(it)) { give_up(P, abort_flag); break; }
                    fence_proxy_async_global();
                }
                const Shape s = shape_of(P, it, live);
                // The odd CTA's rows of A may all lie past the live ones: nothing reads what they give.
                const bool rows = TURNED || it.kind == kHeadTable || it.mt * kTile + rank * kHalf < live;
                const bool rows2 = TURNED || it.kind == kHeadTable || it.mt * kTile + kHalf < live;
                const int row0 = rank * kHalf, buffer = BACKWARD ? it.piece % P.plan.buffers * P.d_planes : 0;
                const int piece_col = BACKWARD ? it.piece * P.plan.piece_tiles * kTile : 0;     // its first entry
                int boxes = 0, n0 = 0;              // of B, 64 columns each (of logits one of 128 rows), from column n0 on
                uint32_t bytes = 0;
                auto load_part = [&](int first, int kb) -> bool {
                    int pair = 0, k = 0;
                    for (int q0 = 0; q0 < kb * s.pairs.n; q0 += kGroup) {
                        if (!mbar_wait_cluster_bounded(&empty_bar[stage], phase ^ 1u, budget, abort_flag)) return false;
                        const int nsub = min(kGroup, kb * s.pairs.n - q0);
                        const uint32_t fb = mapa_shared(smem_u32(&full_bar[stage]), 0);
                        if (leader) mbar_arrive_expect_tx(&full_bar[stage], nsub * bytes);
                        for (int j = 0; j < nsub; ++j) {
                            uint8_t* const sa = smem + (stage * kGroup + j) * kSliceBytes;
                            uint8_t* const sb = sa + kABytes;
                            const int pa = s.pairs.a >> 4 * pair & 15, pb = s.pairs.b >> 4 * pair & 15;
                            const int kx = (first + k) * kSlice;
                            if (TURNED && it.kind <= kHeadLogits) {
                                tma_load_3d_pair(sa, &P.w_k, kx, it.vt * kTile + row0, pb, fb);
                                tma_load_3d_pair(sb, &P.h_k, kx, rank * P.columns / 2, pa, fb);
                            } else if (TURNED && it.kind == kHeadHidden) {
                                for (int b = 0; b < kHalf / kSlice; ++b)
                                    tma_load_3d_pair(sa + b * kBox, &P.w_mn, it.dt * kTile + row0 + b * kSlice, piece_col + kx,
                                                     pb, fb);
                                tma_load_3d_pair(sb, &P.d_k, kx, P.abreast ? 0 : rank * P.columns / 2,
                                                 buffer + (P.abreast ? rank : pa), fb);
                            } else if (it.kind <= kHeadLogits) {
                                if (rows) tma_load_3d_pair(sa, &P.h_k, kx, it.mt * kTile + row0, pa, fb);
                                tma_load_3d_pair(sb, &P.w_k, kx, it.vt * kTile + row0, pb, fb);
                            } else if (it.kind == kHeadHidden) {
                                if (rows) tma_load_3d_pair(sa, &P.d_k, kx, it.mt * kTile + row0, buffer + pa, fb);
                                for (int b = 0; b < boxes; ++b)
                                    tma_load_3d_pair(sb + b * kBox, &P.w_mn, n0 + b * kSlice, piece_col + kx, pb, fb);
                            } else {
                                const int v0 = it.vt * kTile - piece_col + row0;
                                for (int b = 0; b < kHalf / kSlice; ++b)
                                    tma_load_3d_pair(sa + b * kBox, &P.d_mn, v0 + b * kSlice, kx, buffer + pa, fb);
                                for (int b = 0; b < boxes; ++b)
                                    tma_load_3d_pair(sb + b * kBox, &P.h_mn, n0 + b * kSlice, kx, pb, fb);
                            }
                            if (++k == kb) k = 0, ++pair;
                        }
                        if (!leader) mbar_arrive_cluster_relaxed(fb);
                        if (++stage == kRing) stage = 0, phase ^= 1u;
                    }
                    return true;
                };
                bool ok = true;
                for (int sub = 0; sub < s.subs && ok; ++sub) {
                    const int dt = it.dt + sub, cols = columns_of<TURNED>(P, it, dt);
                    boxes = cols / 2 / kSlice;
                    n0 = dt * kTile + rank * (cols / 2);
                    bytes = (rows2 ? 2 : 1) * kABytes + cols * kSlice * 2;
                    for (int part = 0; part < s.parts && ok; ++part) ok = load_part(part * s.part, s.slices(part));
                }
                if (!ok) { give_up(P, abort_flag); break; }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && !leader) {
            // ------------------------------------------ scheduler (odd CTA)
            uint32_t claimed = atomicAdd(P.queue, 1u);
            for (int seq = 0;; ++seq) {
                const int index = claimed < items ? static_cast<int>(claimed) : kEnd;
                const int slot = seq % kItemSlots;
                if (!mbar_wait_cluster_bounded(&item_empty[slot], (static_cast<uint32_t>(seq / kItemSlots) & 1u) ^ 1u,
                                               budget, abort_flag)) {
                    give_up(P, abort_flag);
                    break;
                }
                for (uint32_t r = 0; r < 2; ++r) {
                    const uint32_t bar = mapa_shared(smem_u32(&item_full[slot]), r);
                    mbar_arrive_expect_tx_cluster(bar, 16u);
                    st_async_v4(mapa_shared(smem_u32(&item_ring[slot]), r), index, 0, 0, 0, bar);
                }
                if (index == kEnd) break;
                // One more item is claimed while this one waits for its operands, no more: others may run
                // them sooner.
                claimed = atomicAdd(P.queue, 1u);
                if (BACKWARD && !operands_done(item_of(P, mt, index))) {
                    give_up(P, abort_flag);
                    break;
                }
            }
        }
        // ------------------------------------------- MMA issuer (even CTA)
        if (lane == 0 && leader) {
            uint32_t stage = 0, phase = 0;
            int turn = 0;                       // accumulators filled so far
            for (int seq = 0;; ++seq) {
                int index;
                if (!ring_item(seq, index)) { give_up(P, abort_flag); break; }
                if (index == kEnd) break;
                const HeadItem it = item_of(P, mt, index);
                const Shape s = shape_of(P, it, live);
                // The slices of one part into one accumulator.
                auto run = [&](auto a_mn, auto b_mn, uint32_t idesc, uint32_t d, int total) -> bool {
                    for (int q0 = 0; q0 < total; q0 += kGroup) {
                        if (!mbar_wait_cluster_bounded(&full_bar[stage], phase, budget, abort_flag)) return false;
                        tc_fence_after();
                        const int nsub = min(kGroup, total - q0);
                        for (int j = 0; j < nsub; ++j)
                            mma_slice<decltype(a_mn)::value, decltype(b_mn)::value>(
                                d, smem_u32(smem + (stage * kGroup + j) * kSliceBytes), idesc, q0 + j == 0);
                        tc_commit_pair_multicast(&empty_bar[stage], 0x3);
                        if (++stage == kRing) stage = 0, phase ^= 1u;
                    }
                    return true;
                };
                bool ok = true;
                for (int sub = 0, part = 0; sub < s.subs && ok; ++turn) {
                    const uint32_t idesc = idesc_16bit_f32(kTile, columns_of<TURNED>(P, it, it.dt + sub), false);
                    const uint32_t acc = turn & 1, d = tmem_base + acc * kTile;
                    ok = mbar_wait_cluster_bounded(&tempty_bar[acc], ((turn >> 1) & 1u) ^ 1u, budget, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    const int total = s.slices(part) * s.pairs.n;
                    if (it.kind <= kHeadLogits) ok = run(Kn{}, Kn{}, idesc, d, total);
                    else if (it.kind == kHeadHidden)
                        ok = run(std::bool_constant<TURNED>{}, std::bool_constant<!TURNED>{}, idesc, d, total);
                    else ok = run(Mn{}, Mn{}, idesc, d, total);
                    if (ok) tc_commit_pair_multicast(&tfull_bar[acc], 0x3);
                    if (++part == s.parts) part = 0, ++sub;
                }
                if (!ok) { give_up(P, abort_flag); break; }
            }
            // No TMEM is freed while MMAs may be in flight.
            tc_commit_pair_multicast(&drain_bar, 0x1);
            if (!mbar_wait_cluster_bounded(&drain_bar, 0, budget, nullptr)) give_up(P, abort_flag);
        }
    } else if (warp == 2 + kEpiWarps) {
        // ---------------------------------------------------------- signals
        if (BACKWARD && lane == 0) {
            for (int seq = 0;; ++seq) {
                int index;
                if (!ring_peek(seq, index)) { give_up(P, abort_flag); break; }
                if (index == kEnd) break;
                const HeadItem it = head_item(P.plan, mt, index);
                if (!mbar_wait_bounded(&sig_bar[seq % kSigSlots], (seq / kSigSlots) & 1, budget, abort_flag)) {
                    give_up(P, abort_flag);
                    break;
                }
                ring_free(seq);
                if (it.kind == kHeadLogits) {
                    red_release_gpu_add(P.row_done + it.piece * P.plan.row_tiles + it.mt, 1);
                    red_release_gpu_add(P.col_done + it.vt, 1);
                } else {
                    if (it.kind == kHeadHidden)
                        red_release_gpu_add(P.hidden_done + (it.piece % P.plan.splits * P.plan.row_tiles + it.mt) *
                                                                P.plan.dim_tiles + it.dt, 1);
                    red_release_gpu_add(P.piece_done + it.piece, 1);
                }
            }
        }
    } else {
        // -------------------------------------------------------- epilogue
        uint8_t* const stage_out = smem + kSlices * kSliceBytes;
        const int ew = warp - 2, quarter = warp & 3;
        const uint32_t tempty[2] = {mapa_shared(smem_u32(&tempty_bar[0]), 0), mapa_shared(smem_u32(&tempty_bar[1]), 0)};
        int obuf = 0, turn = 0;
        if constexpr (TURNED) {
            static_assert(32 * kEpiWarps == 2 * kTurnedRows, "a thread has a row's factor of one kind");
            const int n = 32 * ew + lane, of_row = n % kTurnedRows, slices = (P.dim + kSlice - 1) / kSlice;
            const int whole = P.exact ? kExactLogitPart : kLogitPart, last = slices - (slices - 1) / whole * whole;
            back_of[n / kTurnedRows][of_row] =
                1.f + kLostPerStep * min((kSlice / 16) * (n < kTurnedRows ? whole : last), P.steps[of_row]);
            asm volatile("bar.sync 1, %0;" ::"n"(32 * kEpiWarps) : "memory");
        }
        for (int seq = 0;; ++seq) {
            int index = kEnd, ok = 1;
            if (lane == 0) ok = ring_item(seq, index) ? 1 : 0;
            ok = __shfl_sync(~0u, ok, 0);
            index = __shfl_sync(~0u, index, 0);
            if (!ok) {
                if (lane == 0) give_up(P, abort_flag);
                break;
            }
            if (index == kEnd) break;
            const HeadItem it = item_of(P, mt, index);
            const Shape shape = shape_of(P, it, live);
            const int parts = shape.parts;
            const int in_tile = rank * kHalf + quarter * 32;            // this warp's first row of the tile

            // What the tile's rows need, while the product is still running.
            const int row = it.mt * kTile + in_tile + lane;             // compact row (not kHeadTable)
            // (columns of the tile that this warp has: half of them)
            const bool turned = TURNED && it.kind != kHeadTable;
            const int col_w = (ew >> 2) * ((turned ? P.columns : kTile) / 2);
            RowData data;
            if (it.kind <= kHeadLogits) data.load<BACKWARD>(P, turned ? col_w + lane : row);
            const int label = data.label - it.vt * kTile - col_w;
            if (BACKWARD) {
                // The buffer of a piece is free once the tiles that read the piece before in it are
                // done; a part of dH has the earlier pieces in it.
                const uint32_t* counter = nullptr;
                uint32_t target = 0;
                if (it.kind == kHeadLogits && it.piece >= P.plan.buffers) {
                    counter = P.piece_done + it.piece - P.plan.buffers;
                    target = kSignals * (mt * P.plan.dim_tiles + P.plan.piece_tiles * P.plan.table_items());
                } else if (it.kind == kHeadHidden && it.piece >= P.plan.splits) {
                    counter = P.hidden_done + (it.piece % P.plan.splits * P.plan.row_tiles + it.mt) * P.plan.dim_tiles +
                              it.dt;
                    target = kSignals * (it.piece / P.plan.splits);
                }
                if (counter != nullptr) {
                    if (lane == 0) ok = reached(counter, target) ? 1 : 0;
                    if (!__shfl_sync(~0u, ok, 0)) {
                        if (lane == 0) give_up(P, abort_flag);
                        break;
                    }
                    __syncwarp();
                    if (lane == 0) fence_proxy_async_global();
                }
            }
            RowSum sum;
            const bool adds = it.kind == kHeadHidden && it.piece >= P.plan.splits;
            // This thread's sums of the logits' parts, 32 bytes of a lane after another's.
            float* const sums = P.scratch + (static_cast<int64_t>(blockIdx.x) * kEpiWarps + ew) * (kChunks * 32 * 32) + lane * 8;
            uint8_t* const boxes = stage_out + ew * 2 * kOutBox;
            for (int sub = 0, part = 0; sub < shape.subs && ok; ++turn) {
                const int dt = it.dt + sub;
                // columns of the tile that this warp has, and those that count
                const int cols_end = it.kind <= kHeadLogits ? P.vocab - it.vt * kTile : P.dim_ld - dt * kTile;
                // (of dl whole slices of 64: what is read of it is written)
                const int chunks = turned ? P.columns / 64
                                          : max(0, min(kChunks, it.kind == kHeadLogits ? (cols_end - col_w + 63) / 64 * 2
                                                                                       : (cols_end - col_w + 31) / 32));
                const uint32_t acc = turn & 1;
                const uint32_t tbase = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + acc * kTile + col_w;
                if (!mbar_wait_cluster_bounded_sleep(&tfull_bar[acc], (turn >> 1) & 1u, budget, abort_flag, 128)) ok = 0;
                ok = __all_sync(~0u, ok);
                if (!ok) break;
                tc_fence_after();
                uint32_t rv[32];
                if (chunks > 0) {
                    tmem_ld_issue(tbase, rv);
                    tmem_ld_wait(rv);
                }
                const int most = (kSlice / 16) * shape.slices(part);
                const bool of_columns = TURNED && it.kind == kHeadLogits;
                const float back = 1.f + kLostPerStep * (it.kind <= kHeadLogits ? min(most, data.steps) : most);
                for (int ch = 0; ch < chunks; ++ch) {
                    float v[32];
                    if (of_columns) {
                        const float4* const of_row = reinterpret_cast<const float4*>(back_of[TURNED && part + 1 == parts] + col_w + ch * 32);
#pragma unroll
                        for (int j = 0; j < 32; j += 4) {
                            const float4 b = of_row[j / 4];
                            v[j] = __uint_as_float(rv[j]) * b.x, v[j + 1] = __uint_as_float(rv[j + 1]) * b.y;
                            v[j + 2] = __uint_as_float(rv[j + 2]) * b.z, v[j + 3] = __uint_as_float(rv[j + 3]) * b.w;
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const float2 f = unpack2(mul2(pack2(__uint_as_float(rv[j]), __uint_as_float(rv[j + 1])),
                                                          pack2(back, back)));
                            v[j] = f.x, v[j + 1] = f.y;
                        }
                    }
                    if (turned && it.kind == kHeadHidden && P.abreast) {
                        tmem_ld_issue(tbase + P.columns + ch * 32, rv);
                        tmem_ld_wait(rv);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] += __uint_as_float(rv[j]);
                    }
                    if (ch + 1 < chunks) tmem_ld_issue(tbase + (ch + 1) * 32, rv);
                    const int here = cols_end - col_w - ch * 32;        // columns from here on that count
                    bool whole = true;
                    if (it.kind <= kHeadLogits && parts > 1) {
                        float* const at = sums + ch * 1024;
                        whole = part + 1 == parts;
                        if (part > 0) {
                            float old[4][8];
#pragma unroll
                            for (int q = 0; q < 4; ++q) load_vec<float, 8>(at + q * 256, old[q]);
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] += old[j / 8][j % 8];
                        }
                        if (!whole) {
#pragma unroll
                            for (int q = 0; q < 4; ++q)
                                store_vec<float, 8>(at + q * 256, *reinterpret_cast<const float (*)[8]>(v + 8 * q));
                        }
                    }
                    if (turned && it.kind == kHeadLogits) {
                        if (whole) {
                            const int entry = it.vt * kTile + in_tile + lane;
                            logits_gradient_turned(v, data, entry < P.vocab ? entry : -1);
                            for (int plane = 0; plane < P.d_planes; ++plane)
                                store_turned_bf16(&P.d_out, v, boxes, obuf, P.d_planes > 1,
                                                  (it.vt - it.piece * P.plan.piece_tiles) * kTile + in_tile, col_w + ch * 32,
                                                  it.piece % P.plan.buffers * P.d_planes + plane, lane);
                            if (ch + 1 < chunks) data.load<BACKWARD>(P, col_w + (ch + 1) * 32 + lane);
                        }
                    } else if (turned) {
                        const int c1 = dt * kTile + in_tile;            // the dimension's, dH's rows
                        if (part > 0 && ch == 0 && lane == 0) bulk_wait_group_all();
                        if (c1 < P.dim_ld)
                            store_square(&P.acc_out, v, boxes, obuf, adds || part > 0, P.columns, col_w + ch * 32, c1,
                                         it.piece % P.plan.splits, lane);
                    } else if (it.kind <= kHeadLogits && whole) {
                        const int at_label = label - ch * 32;
                        const bool labelled = __any_sync(~0u, at_label >= 0 && at_label < 32);
                        if (labelled) {
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (j == at_label) v[j] = data.of_label;
                        }
                        if (!BACKWARD) {
                            sum.add(v, here);
                        } else {
                            logits_gradient(v, data.m, data.inv, data.weight, labelled ? at_label : -1, here);
                            for (int plane = 0; plane < P.d_planes; ++plane)
                                store_square_bf16(&P.d_out, v, boxes, obuf, P.d_planes > 1,
                                                  (it.vt - it.piece * P.plan.piece_tiles) * kTile + col_w + ch * 32,
                                                  it.mt * kTile + in_tile, it.piece % P.plan.buffers * P.d_planes + plane, lane);
                        }
                    } else if (BACKWARD && it.kind == kHeadHidden) {
                        // Stored, or added in L2 to what the pieces and parts before have left.
                        if (part > 0 && ch == 0 && lane == 0) bulk_wait_group_all();        // the part before is there
                        store_square(&P.acc_out, v, boxes, obuf, adds || part > 0, P.dim_ld, dt * kTile + col_w + ch * 32,
                                     it.mt * kTile + in_tile, it.piece % P.plan.splits, lane);
                    } else if (BACKWARD && it.kind == kHeadTable) {
                        if (live == 0) {
#pragma unroll
                            for (int j = 0; j < 32; ++j) v[j] = 0.f;
                        }
                        const int c0 = dt * kTile + col_w + ch * 32, c1 = it.vt * kTile + in_tile;
                        const bool add = P.accumulate || part > 0;
                        if (!P.dtable_boxes) {
                            store_table(P, v, c1, c0, add, boxes, lane);        // (a thread adds to what it wrote itself)
                        } else if (P.dtable_bf16) {
                            if (c0 < P.dim) store_square_bf16(&P.t_out, v, boxes, obuf, false, c0, c1, 0, lane);
                        } else {
                            if (part > 0 && ch == 0 && lane == 0) bulk_wait_group_all();
                            store_square(&P.t_out, v, boxes, obuf, add, P.dim, c0, c1, 0, lane);
                        }
                    }
                    __syncwarp();
                    if (ch + 1 < chunks) tmem_ld_wait(rv);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_remote(tempty[acc]);
                if (++part == parts) part = 0, ++sub;
            }
            if (!ok) {
                if (lane == 0) give_up(P, abort_flag);
                break;
            }
            if (!BACKWARD) {
                P.parts[static_cast<int64_t>(2 * it.vt + (ew >> 2)) * P.row_ld + row] = make_float2(sum.m, sum.s);
            } else if (lane == 0) {
                if (it.kind != kHeadTable) {
                    bulk_wait_group_all();
                    fence_proxy_async_global();
                }
                mbar_arrive(&sig_bar[seq % kSigSlots]);
            }
        }
        if (lane == 0) bulk_wait_group_all();
    }
    tc_fence_before();
    cluster_sync();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, 2 * kTile);
    }
}

// Two (max, sum of exponentials) as one.
__device__ __forceinline__ float2 joined(float2 a, float2 b) {
    // (NaN in a sum stays; a maximum passes it over)
    const float m = fmaxf(a.x, b.x), base = m == -INFINITY ? 0.f : m;
    return make_float2(m, a.y * exp2_fast((a.x - base) * kLog2) + b.y * exp2_fast((b.x - base) * kLog2));
}

// ------------------------------------------------------------------ few rows, forward
// Logits of up to 128 rows the other way round: entries of the table are the products' rows,
// hidden rows their columns, so that the products cost what there is of them (24 rows of 1280
// against 50304: 52 us a call as 256 rows, 37 so, of which 27 here, reading the table).  Pairs of CTAs take the
// table's tiles in turn; a thread has an entry's logits, and a warp turns 32 x 32 of them by
// shuffles into a maximum and a sum a row, which stay in its lanes from tile to tile: every
// CTA leaves one part a row.  A product's reduction goes to up to four sums in TMEM, which are
// added in fp32: each cuts off a fourth as often, from sums a fourth as large.
constexpr int kFewRows = 128;
constexpr int kFewSlices = 8, kFewGroup = 2, kFewRing = kFewSlices / kFewGroup;
constexpr uint32_t kFewSliceBytes = kABytes + kFewRows / 2 * kSlice * 2;
constexpr size_t kFewSmem = static_cast<size_t>(kFewSlices) * kFewSliceBytes + 1024;
constexpr int kFewSums = 4;                          // of a product
constexpr int kFewWarps = 4, kFewThreads = 64 + 32 * kFewWarps;
constexpr int64_t kPrefetchBytes = 64ll << 20;      // of the table, half of L2

struct Few {
    CUtensorMap w_k, h_n;           // boxes of 128 entries; of columns / 2 rows
    int32_t dim, vocab, vocab_tiles;
    int32_t columns;                // of the products: rows, in whole 32s
    int32_t each;                   // slices of one of a product's sums
    int32_t row_ld, prefetch;
    const int32_t* live;
    const int32_t* labels;
    const int32_t* steps;
    const float* label_logits;
    float2* parts;                  // [gridDim.x][row_ld]
    int32_t* status;
    uint64_t budget_ns;
};

// Of 32 values a lane, column by column over the lanes: lane j gets column j's.
template <typename Op>
__device__ __forceinline__ float reduce_columns(float (&v)[32], Op op) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const bool upper = lane & d;
#pragma unroll
        for (int i = 0; i < d; ++i) {
            const float other = __shfl_xor_sync(~0u, upper ? v[i] : v[i + d], d);
            v[i] = op(upper ? v[i + d] : v[i], other);
        }
    }
    return v[0];
}

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kFewThreads, 1) head_few_kernel(const __grid_constant__ Few P) {
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t full_bar[kFewRing], empty_bar[kFewRing], tfull_bar[2], tempty_bar[2], drain_bar;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_sh;
    __shared__ float2 of_warp[kFewWarps][kFewRows];
    __shared__ __align__(16) float back_of[2][kFewRows];       // of a row's sums, and of the last of them
    volatile int* abort_flag = &abort_sh;
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                               ~static_cast<uintptr_t>(1023));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = static_cast<int>(cluster_ctarank()), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const bool leader = rank == 0;
    const uint64_t budget = P.budget_ns;
    auto give_up = [&]() {
        atomicOr(P.status, 1);
        *abort_flag = 1;
    };
    if (threadIdx.x == 0) {
        for (int s = 0; s < kFewRing; ++s) {
            mbar_init(&full_bar[s], 2);
            mbar_init(&empty_bar[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(&tfull_bar[a], 1);
            mbar_init(&tempty_bar[a], 2 * kFewWarps);
        }
        mbar_init(&drain_bar, 1);
        abort_sh = 0;
        fence_barrier_init();
        fence_proxy_async_smem();
    }
    if (warp == 0 && lane == 0) {
        tma_prefetch_desc(&P.w_k);
        tma_prefetch_desc(&P.h_n);
        // While the rows are being gathered: this pair's first tile into L2 (a hint; nothing depends
        // on what it finds).
        if (pair < P.prefetch)
            for (int k = 0; k < P.dim; k += kSlice) tma_prefetch_3d(&P.w_k, k, pair * kTile + rank * kHalf, 0);
    }
    if (warp == 1) {
        tmem_alloc_pair(&tmem_slot, 2 * kTile);
        tmem_relinquish_pair();
    }
    chain_wait();
    tc_fence_before();
    cluster_sync();
    tc_fence_after();
    const uint32_t tmem_base = tmem_slot;
    const int live = *after_wait(P.live);
    const int tiles = live > 0 ? P.vocab_tiles : 0, slices = (P.dim + kSlice - 1) / kSlice;

    if (warp == 0) {
        if (lane == 0) {
            uint32_t stage = 0, phase = 0;
            const uint32_t bytes = 2 * (kABytes + P.columns / 2 * kSlice * 2);
            bool ok = true;
            for (int t = pair; t < tiles && ok; t += pairs)
                for (int k0 = 0; k0 < slices; k0 += kFewGroup) {
                    ok = mbar_wait_cluster_bounded(&empty_bar[stage], phase ^ 1u, budget, abort_flag);
                    if (!ok) break;
                    const int nsub = min(kFewGroup, slices - k0);
                    const uint32_t fb = mapa_shared(smem_u32(&full_bar[stage]), 0);
                    if (leader) mbar_arrive_expect_tx(&full_bar[stage], nsub * bytes);
                    for (int j = 0; j < nsub; ++j) {
                        uint8_t* const sa = smem + (stage * kFewGroup + j) * kFewSliceBytes;
                        tma_load_3d_pair(sa, &P.w_k, (k0 + j) * kSlice, t * kTile + rank * kHalf, 0, fb);
                        tma_load_3d_pair(sa + kABytes, &P.h_n, (k0 + j) * kSlice, rank * (P.columns / 2), 0, fb);
                    }
                    if (!leader) mbar_arrive_cluster_relaxed(fb);
                    if (++stage == kFewRing) stage = 0, phase ^= 1u;
                }
            if (!ok) give_up();
        }
    } else if (warp == 1) {
        if (lane == 0 && leader) {
            uint32_t stage = 0, phase = 0;
            int turn = 0;
            bool ok = true;
            const uint32_t idesc = idesc_16bit_f32(kTile, P.columns, false);
            for (int t = pair; t < tiles && ok; t += pairs, ++turn) {
                const uint32_t acc = turn & 1;
                ok = mbar_wait_cluster_bounded(&tempty_bar[acc], ((turn >> 1) & 1u) ^ 1u, budget, abort_flag);
                if (!ok) break;
                tc_fence_after();
                uint32_t d = tmem_base + acc * kTile;
                int in_sum = 0;
                for (int k0 = 0; k0 < slices; k0 += kFewGroup) {
                    ok = mbar_wait_cluster_bounded(&full_bar[stage], phase, budget, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    for (int j = 0; j < min(kFewGroup, slices - k0); ++j) {
                        if (in_sum == P.each) in_sum = 0, d += P.columns;
                        mma_slice<false, false>(d, smem_u32(smem + (stage * kFewGroup + j) * kFewSliceBytes), idesc,
                                                in_sum++ == 0);
                    }
                    tc_commit_pair_multicast(&empty_bar[stage], 0x3);
                    if (++stage == kFewRing) stage = 0, phase ^= 1u;
                }
                if (ok) tc_commit_pair_multicast(&tfull_bar[acc], 0x3);
            }
            if (!ok) give_up();
            tc_commit_pair_multicast(&drain_bar, 0x1);      // no TMEM is freed while MMAs may be in flight
            if (!mbar_wait_cluster_bounded(&drain_bar, 0, budget, nullptr)) give_up();
        }
    } else {
        const int quarter = warp & 3, chunks = P.columns / 32;
        const uint32_t tempty[2] = {mapa_shared(smem_u32(&tempty_bar[0]), 0), mapa_shared(smem_u32(&tempty_bar[1]), 0)};
        if (threadIdx.x - 64 < kFewRows) {
            const int row = threadIdx.x - 64, steps = row < live ? P.steps[row] : 0;
            back_of[0][row] = 1.f + kLostPerStep * min((kSlice / 16) * P.each, steps);
            back_of[1][row] = 1.f + kLostPerStep * min((kSlice / 16) * (slices - (slices - 1) / P.each * P.each), steps);
        }
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kFewWarps) : "memory");
        float m[kFewRows / 32], s[kFewRows / 32], of_label[kFewRows / 32];
        int label[kFewRows / 32];
#pragma unroll
        for (int c = 0; c < kFewRows / 32; ++c) {
            m[c] = -INFINITY, s[c] = 0.f;
            label[c] = c < chunks && 32 * c + lane < live ? P.labels[32 * c + lane] : -1;
            of_label[c] = label[c] >= 0 ? P.label_logits[32 * c + lane] : 0.f;
        }
        int turn = 0;
        for (int t = pair; t < tiles; t += pairs, ++turn) {
            const uint32_t acc = turn & 1;
            int ok = 1;
            if (lane == 0) ok = mbar_wait_cluster_bounded(&tfull_bar[acc], (turn >> 1) & 1u, budget, abort_flag) ? 1 : 0;
            if (!__shfl_sync(~0u, ok, 0)) {
                if (lane == 0) give_up();
                break;
            }
            tc_fence_after();
            const int first = t * kTile + rank * kHalf + quarter * 32;      // this warp's entries of the table
#pragma unroll
            for (int c = 0; c < kFewRows / 32; ++c) {
                if (c >= chunks) break;
                uint32_t rv[32], from = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16) + acc * kTile + 32 * c;
                tmem_ld_issue(from, rv);
                tmem_ld_wait(rv);
                float v[32], w[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = first + lane < P.vocab ? 0.f : -INFINITY;
                for (int k = 0; k < slices; k += P.each) {
                    if (k > 0) {
                        tmem_ld_issue(from += P.columns, rv);
                        tmem_ld_wait(rv);
                    }
                    const float4* const back = reinterpret_cast<const float4*>(back_of[k + P.each < slices ? 0 : 1] + 32 * c);
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const float4 b = back[j / 4];
                        v[j] = fmaf(__uint_as_float(rv[j]), b.x, v[j]);
                        v[j + 1] = fmaf(__uint_as_float(rv[j + 1]), b.y, v[j + 1]);
                        v[j + 2] = fmaf(__uint_as_float(rv[j + 2]), b.z, v[j + 2]);
                        v[j + 3] = fmaf(__uint_as_float(rv[j + 3]), b.w, v[j + 3]);
                    }
                }
                const int at = label[c] - first;
                for (unsigned mine = __ballot_sync(~0u, at >= 0 && at < 32); mine != 0; mine &= mine - 1) {
                    const int row = __ffs(mine) - 1, entry = __shfl_sync(~0u, at, row);
                    const float value = __shfl_sync(~0u, of_label[c], row);
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (j == row && lane == entry) v[j] = value;
                }
#pragma unroll
                for (int j = 0; j < 32; ++j) w[j] = v[j];
                const float top = reduce_columns(w, [](float a, float b) { return fmaxf(a, b); });
                const float next = fmaxf(m[c], top), base = next == -INFINITY ? 0.f : next;
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = exp2_fast((v[j] - __shfl_sync(~0u, base, j)) * kLog2);
                const float sum = reduce_columns(v, [](float a, float b) { return a + b; });
                s[c] = s[c] * exp2_fast((m[c] - base) * kLog2) + sum;
                m[c] = next;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(tempty[acc]);
        }
#pragma unroll
        for (int c = 0; c < kFewRows / 32; ++c) of_warp[warp - 2][32 * c + lane] = make_float2(m[c], s[c]);
        asm volatile("bar.sync 1, %0;" ::"n"(32 * kFewWarps) : "memory");
        const int row = threadIdx.x - 64;
        if (row < P.columns) {
            float2 a = of_warp[0][row];
#pragma unroll
            for (int i = 1; i < kFewWarps; ++i) a = joined(a, of_warp[i][row]);
            P.parts[static_cast<int64_t>(blockIdx.x) * P.row_ld + row] = a;
        }
    }
    tc_fence_before();
    cluster_sync();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, 2 * kTile);
    }
}

// ------------------------------------------------------------------ rows that count
constexpr int kScanThreads = 1024;
constexpr int32_t kLeftOut = -1, kWrong = -2;       // rows that are not among the live ones

struct Scan {
    const void* labels;
    int32_t labels_i64;
    int32_t rows, vocab;
    const float* weight;            // or null for ones
    const float* dloss;             // the gradient alone: or null for ones
    const float2* stats;            // the gradient alone, else null
    float* loss;                    // forward: of the rows that are left out
    float2* out_stats;              // forward, or null
    int32_t* place;                 // [rows] compact row, kLeftOut or kWrong
    int32_t* row;                   // [row_ld] row of a compact one
    int32_t* live;
    int32_t* c_labels;
    float* c_weights;
    float2* c_stats;
    uint32_t* counters;             // zeroed
    int64_t ncounters;
};

// A block numbers the live rows in their order, THREADS * ROWS rows at a time; their number.
// WRITE: to the arrays of S, with the zeroed counters and the rows that fill the last tile.
// src, labels: shared arrays of the live rows' numbers and labels, or null.
template <int THREADS, int ROWS>
__device__ __forceinline__ int scan_rows(const Scan& S, bool write, int* src, int* labels) {
    constexpr int kWarps = THREADS / 32;
    static_assert(ROWS <= kWarps && kWarps <= 32, "a warp adds up the counts of THREADS rows");
    __shared__ int before[ROWS * kWarps];   // live rows of a warp's 32, then those before them in the same THREADS
    __shared__ int of_row[ROWS];            // live rows of each THREADS
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (write)
        for (int64_t i = tid; i < S.ncounters; i += THREADS) S.counters[i] = 0;
    int so_far = 0;
    for (int64_t base = 0; base < S.rows; base += THREADS * ROWS) {
        int64_t label[ROWS];
        float w[ROWS], up[ROWS];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int64_t n = base + k * THREADS + tid;
            label[k] = -1;
            w[k] = up[k] = 1.f;
            if (n >= S.rows) continue;
            label[k] = S.labels_i64 ? static_cast<const int64_t*>(S.labels)[n] : static_cast<const int32_t*>(S.labels)[n];
            if (S.weight != nullptr) w[k] = S.weight[n];
            if (S.dloss != nullptr) up[k] = S.dloss[n];
        }
        unsigned votes[ROWS];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            const int64_t n = base + k * THREADS + tid;
            const bool counts = label[k] >= 0 && w[k] != 0.f && up[k] != 0.f, on = counts && label[k] < S.vocab;
            if (write && !on && n < S.rows) {
                S.place[n] = counts ? kWrong : kLeftOut;
                if (S.loss != nullptr) S.loss[n] = counts ? __uint_as_float(0x7fffffffu) : 0.f;
                if (S.out_stats != nullptr) S.out_stats[n] = make_float2(0.f, 0.f);
            }
            votes[k] = __ballot_sync(~0u, on);
            if (lane == 0) before[k * kWarps + warp] = __popc(votes[k]);
        }
        __syncthreads();
        if (warp < ROWS) {                  // the counts of one THREADS
            const int own = lane < kWarps ? before[warp * kWarps + lane] : 0;
            int upto = own;
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const int v = __shfl_up_sync(~0u, upto, d);
                if (lane >= d) upto += v;
            }
            if (lane < kWarps) before[warp * kWarps + lane] = upto - own;
            if (lane == 31) of_row[warp] = upto;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            if (votes[k] >> lane & 1) {
                const int64_t n = base + k * THREADS + tid;
                const int at = so_far + before[k * kWarps + warp] + __popc(votes[k] & ((1u << lane) - 1));
                if (src != nullptr) src[at] = static_cast<int>(n), labels[at] = static_cast<int>(label[k]);
                if (write) {
                    S.place[n] = at;
                    S.row[at] = static_cast<int32_t>(n);
                    S.c_labels[at] = static_cast<int32_t>(label[k]);
                    S.c_weights[at] = w[k] * up[k];
                    if (S.stats != nullptr) S.c_stats[at] = S.stats[n];
                }
            }
            so_far += of_row[k];
        }
        __syncthreads();
    }
    const int live = so_far;
    if (write) {
        // The rest of the last tile: rows of zeros, whose dl is 0.
        const int padded = (live + kTile - 1) / kTile * kTile;
        for (int at = live + tid; at < padded; at += THREADS) {
            S.c_labels[at] = -1;
            S.c_weights[at] = 0.f;
            S.c_stats[at] = make_float2(0.f, 1.f);
        }
        if (tid == 0) *S.live = live;
    }
    return live;
}
__global__ void __launch_bounds__(kScanThreads) head_scan_kernel(const __grid_constant__ Scan S) {
    chain_pass_wait();
    scan_rows<kScanThreads, 8>(S, true, nullptr, nullptr);
}

// A matrix of `cols` columns as bf16 planes whose sum it is, rows of ld with zeros behind.
struct Pack {
    const void* from;
    int64_t from_ld;
    const int32_t* row;             // source rows, or null for all in order
    const int32_t* live;            // their number, or null: `rows`
    int32_t rows, cols, ld, planes;
    int64_t plane;                  // entries of a plane
    bf16* to;
    const int32_t* labels;          // of hidden rows: with the table, for the labels' logits; else null
    const void* table;
    int64_t table_ld;
    int32_t table_bf16, table_vec;
    float* label_logits;
    int32_t* steps;                 // of hidden rows: see Gemm; else null
};

// A warp takes a row, eight entries a lane at a time; VEC: they start on 16-byte addresses.
template <typename T, bool VEC>
__device__ __forceinline__ void load_eight(const T* p, int left, float (&v)[8]) {
    if (VEC && left >= 8) {
        load_vec<T, 8>(p, v);
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float x[1] = {0.f};
        if (j < left) load_vec<T, 1>(p + j, x);
        v[j] = x[0];
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void pack_row(const Pack& K, int64_t at, bool on, int64_t source, int64_t label) {
    const int lane = threadIdx.x & 31;
    const T* const from = static_cast<const T*>(K.from) + source * K.from_ld;
    constexpr int kAhead = 4;
    float dot = 0.f;
    int steps = 0;
    for (int c0 = 8 * lane; c0 - 8 * lane < K.ld; c0 += 256 * kAhead) {         // (all lanes equally often)
        float v[kAhead][8];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) load_eight<T, VEC>(from + c0 + 256 * i, on ? K.cols - c0 - 256 * i : 0, v[i]);
        if (K.steps != nullptr) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                bool some = false;
#pragma unroll
                for (int j = 0; j < 8; ++j) some |= v[i][j] != 0.f;
                const unsigned lanes = __ballot_sync(~0u, some);
                steps += __popc((lanes | lanes >> 1) & 0x55555555u);
            }
        }
        if (label >= 0) {
            // A label's logit, of all the largest and a sum of terms of one sign, in fp32: TMEM's sum of
            // 1280 terms would be 1e-5 off, and a small loss as much of itself.
            float w[kAhead][8];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int64_t e = label * K.table_ld + c0 + 256 * i;
                const int left = K.cols - c0 - 256 * i;
                if (K.table_bf16) {
                    if (K.table_vec) load_eight<bf16, true>(static_cast<const bf16*>(K.table) + e, left, w[i]);
                    else load_eight<bf16, false>(static_cast<const bf16*>(K.table) + e, left, w[i]);
                } else {
                    if (K.table_vec) load_eight<float, true>(static_cast<const float*>(K.table) + e, left, w[i]);
                    else load_eight<float, false>(static_cast<const float*>(K.table) + e, left, w[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) dot = fmaf(v[i][j], w[i][j], dot);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = c0 + 256 * i;
            if (c >= K.ld) continue;
            bf16* to = K.to + at * K.ld + c;
            for (int p = 0; p < K.planes; ++p, to += K.plane) {
                uint32_t u[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    u[j] = pack_bf16(v[i][2 * j], v[i][2 * j + 1]);
                    v[i][2 * j] -= __uint_as_float(u[j] << 16);
                    v[i][2 * j + 1] -= __uint_as_float(u[j] & 0xffff0000u);
                }
                *reinterpret_cast<uint4*>(to) = make_uint4(u[0], u[1], u[2], u[3]);
            }
        }
    }
    if (K.steps != nullptr && lane == 0) K.steps[at] = steps;
    if (label >= 0) {
        dot = warp_sum(dot);
        if (lane == 0) K.label_logits[at] = dot;
    }
}
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) head_pack_kernel(const __grid_constant__ Pack K) {
    const int64_t at = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    chain_pass_wait();
    int live = K.rows, end = K.rows;
    if (K.live != nullptr) {
        live = *after_wait(K.live);
        end = (live + kTile - 1) / kTile * kTile;
    }
    if (at >= end) return;
    const bool on = at < live;
    pack_row<T, VEC>(K, at, on, on ? (K.row != nullptr ? after_wait(K.row)[at] : at) : 0,
                     K.labels != nullptr && on ? after_wait(K.labels)[at] : -1);
}

// Both for up to kGatherRows rows: every block numbers them for itself (a launch and its
// latencies less: the loss of 24 rows 41 -> 37 us a call; loss and gradients of 300, 226 -> 222).
// MOST: one row a thread up to 256 (of 128 rows, 162 -> 152 us).
constexpr int kGatherRows = 1024;
template <typename T, bool VEC, int MOST>
__global__ void __launch_bounds__(256) head_gather_kernel(const __grid_constant__ Scan S, const __grid_constant__ Pack K) {
    __shared__ int src[MOST], labels[MOST];
    const int at = blockIdx.x * 8 + (threadIdx.x >> 5);
    chain_pass_wait();
    const int live = scan_rows<256, MOST / 256>(S, blockIdx.x == 0, src, labels);
    if (at >= (live + kTile - 1) / kTile * kTile) return;
    const bool on = at < live;
    pack_row<T, VEC>(K, at, on, on ? src[at] : 0, on ? labels[at] : -1);
}

// Losses and statistics of the live rows from their parts: a block takes 32 rows, its warps
// a share of the parts each.
constexpr int kJoinWarps = 32;
struct Join {
    const int32_t *live, *row;
    const float2* parts;
    int32_t nparts, row_ld;
    const float* label_logits;
    const float* c_weights;
    float* loss;
    float2* out_stats;              // or null
    float2* c_stats;
    const int32_t* status;
};
__global__ void __launch_bounds__(32 * kJoinWarps) head_join_kernel(const __grid_constant__ Join J) {
    __shared__ float2 of_warp[kJoinWarps][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x * 32 + lane;
    chain_wait();
    const int live = *after_wait(J.live);
    if (blockIdx.x * 32 >= live) return;
    float2 a = make_float2(-INFINITY, 0.f);
    const float2* const parts = after_wait(J.parts);
#pragma unroll 4
    for (int j = warp; j < J.nparts; j += kJoinWarps) a = joined(a, parts[static_cast<int64_t>(j) * J.row_ld + row]);
    of_warp[warp][lane] = a;
    __syncthreads();
    // lane j of a warp has warp j's part of its row; the warp joins them
    a = of_warp[lane][warp];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1)
        a = joined(a, make_float2(__shfl_xor_sync(~0u, a.x, d), __shfl_xor_sync(~0u, a.y, d)));
    const int mine = blockIdx.x * 32 + warp;
    if (lane != 0 || mine >= live) return;
    const int n = J.row[mine];
    const float loss = J.c_weights[mine] * (logf(a.y) + (a.x - J.label_logits[mine]));
    J.loss[n] = *J.status != 0 ? __uint_as_float(0x7fffffffu) : loss;
    if (J.out_stats != nullptr) J.out_stats[n] = a;
    J.c_stats[mine] = a;
}

// The hidden rows' gradient from the parts of dH, zeros for rows left out.
struct Spread {
    const int32_t* place;
    const float* acc;
    int32_t rows, dim, dim_ld, splits;
    int32_t share;                  // warps of a row's parts
    int32_t row_ld;
    int64_t part;                   // entries of a part
    void* to;
    int64_t to_ld;
    const int32_t* status;
};
// A warp takes a row, eight entries a lane at a time (VEC: they are stored as vectors).
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) head_spread_kernel(const __grid_constant__ Spread K) {
    const int64_t n = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    const int lane = threadIdx.x & 31;
    chain_wait();
    if (n >= K.rows) return;
    const int at = after_wait(K.place)[n];
    const bool lost = *K.status != 0 || at == kWrong;
    const float* const acc = after_wait(K.acc) + static_cast<int64_t>(max(at, 0)) * K.dim_ld;
    T* const to = static_cast<T*>(K.to) + n * K.to_ld;
    constexpr int kAhead = 2;
    for (int c0 = 8 * lane; c0 < K.dim; c0 += 256 * kAhead) {
        float v[kAhead][8] = {};
        if (at >= 0) {
#pragma unroll 4
            for (int s = 0; s < K.splits; ++s)
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    if (c0 + 256 * i >= K.dim) continue;
                    float x[8];
                    load_vec<float, 8>(acc + s * K.part + c0 + 256 * i, x);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[i][j] += x[j];
                }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = c0 + 256 * i;
            if (c >= K.dim) continue;
            if (lost) {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = __uint_as_float(0x7fffffffu);
            }
            if (VEC) {
                store_vec<T, 8>(to + c, v[i]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x[1] = {v[i][j]};
                    if (c + j < K.dim) store_vec<T, 1>(to + c + j, x);
                }
            }
        }
    }
}

// The same where few rows have several parts: `share` warps take a part each in turn, of 256
// columns of a row, and add their sums up in one order (24 rows of 1280 in 29 parts: loss and
// gradients 54 us less; 2048 rows of 1024 in two parts: 26 us where a warp a row takes 12).
constexpr int kSpreadWarps = 8;
constexpr int64_t kSpreadRows = 1024;
template <typename T>
__global__ void __launch_bounds__(32 * kSpreadWarps) head_spread_parts_kernel(const __grid_constant__ Spread K) {
    __shared__ __align__(16) float of_warp[kSpreadWarps][256];
    const int chunks = (K.dim + 255) / 256, share = K.share;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, first = warp - warp % share;
    const int64_t n = blockIdx.x / chunks * static_cast<int64_t>(kSpreadWarps / share) + warp / share;
    const int c0 = static_cast<int>(blockIdx.x % chunks) * 256, c = c0 + 8 * lane;
    chain_wait();
    const int at = n < K.rows ? after_wait(K.place)[n] : kLeftOut;
    float v[8] = {};
    if (at >= 0 && c < K.dim) {
        const float* const acc = after_wait(K.acc) + static_cast<int64_t>(at) * K.dim_ld + c;
#pragma unroll 4
        for (int s = warp - first; s < K.splits; s += share) {
            float x[8];
            load_vec<float, 8>(acc + s * K.part, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += x[j];
        }
    }
    store_vec<float, 8>(&of_warp[warp][8 * lane], v);
    __syncthreads();
    if (n >= K.rows) return;
    const bool lost = *K.status != 0 || at == kWrong;
    T* const to = static_cast<T*>(K.to) + n * K.to_ld + c0;
    for (int e = threadIdx.x - 32 * first; e < min(256, K.dim - c0); e += 32 * share) {
        float sum[1] = {0.f};
        for (int w = first; w < first + share; ++w) sum[0] += of_warp[w][e];
        if (lost) sum[0] = __uint_as_float(0x7fffffffu);
        store_vec<T, 1>(to + e, sum);
    }
}

// The same of TURNED products, whose parts of dH hold the dimension's entries as rows: a block
// takes eight of them for 32 hidden rows.
template <typename T>
__global__ void __launch_bounds__(256) head_spread_turned_kernel(const __grid_constant__ Spread K) {
    __shared__ float square[32][9];
    const int groups = (K.dim + 7) / 8, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n0 = static_cast<int>(blockIdx.x / groups) * 32, d0 = static_cast<int>(blockIdx.x % groups) * 8;
    chain_wait();
    const int32_t* const place = after_wait(K.place);
    const int at = n0 + lane < K.rows ? place[n0 + lane] : kLeftOut;
    float v = 0.f;
    if (at >= 0 && d0 + warp < K.dim) {
        const float* const acc = after_wait(K.acc) + static_cast<int64_t>(d0 + warp) * K.row_ld + at;
#pragma unroll 8
        for (int s = 0; s < K.splits; ++s) v += acc[s * K.part];
    }
    if (*K.status != 0 || at == kWrong) v = __uint_as_float(0x7fffffffu);
    square[lane][warp] = v;
    __syncthreads();
    const int n = n0 + threadIdx.x / 8, e = threadIdx.x % 8;
    if (n >= K.rows || d0 + e >= K.dim) return;
    const float x[1] = {square[threadIdx.x / 8][e]};
    store_vec<T, 1>(static_cast<T*>(K.to) + n * K.to_ld + d0 + e, x);
}

// ----------------------------------------------------------------------- host
constexpr int64_t kMaxRows = int64_t{1} << 22, kMaxDim = int64_t{1} << 16, kMaxVocab = int64_t{1} << 24;

PFN_cuTensorMapEncodeTiled_v12000 encoder() {
    static const PFN_cuTensorMapEncodeTiled_v12000 f = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult q{};
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &q) != cudaSuccess ||
            q != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            fn = nullptr;
        }
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn);
    }();
    return f;
}

// bf16 (or fp32) [planes][rows][cols], rows ld apart; boxes of box_cols x box_rows.
bool map_of(CUtensorMap* map, const void* base, int64_t cols, int64_t rows, int64_t planes, int64_t ld, uint32_t box_rows,
            uint32_t box_cols = kSlice, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B, bool fp32 = false) {
    const cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(planes)};
    const cuuint64_t bytes = fp32 ? 4 : 2;
    const cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * bytes, static_cast<cuuint64_t>(rows * ld) * bytes};
    const cuuint32_t box[3] = {box_cols, box_rows, 1}, one[3] = {1, 1, 1};
    return encoder()(map, fp32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, one,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Shared-memory opt-in and the pairs that can be resident, per device.
cudaError_t configure(int* pairs) {
    constexpr int kDevices = 64;
    static std::mutex mu;
    static int known[kDevices] = {};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= kDevices) return cudaErrorInvalidDevice;
    std::lock_guard<std::mutex> lock(mu);
    if (known[dev] == 0) {
        const int bytes = static_cast<int>(kSmem);
        for (auto kernel : {head_gemm_kernel<false>, head_gemm_kernel<true>, head_gemm_kernel<true, true>})
            if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e == cudaSuccess)
            e = cudaFuncSetAttribute(head_few_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kFewSmem));
        if (e != cudaSuccess) return e;
        int n = 0;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(2, 1, 1);
        cfg.blockDim = dim3(kThreads, 1, 1);
        cfg.dynamicSmemBytes = kSmem;
        if (cudaOccupancyMaxActiveClusters(&n, head_gemm_kernel<true>, &cfg) != cudaSuccess || n <= 0) {
            cudaGetLastError();
            n = std::max(1, sm_count() / 2);
        }
        known[dev] = n;
    }
    *pairs = known[dev];
    return cudaSuccess;
}

// Products of planes whose numbers add up to two at most, the smallest first, where TMEM's
// sums lose least (as they come, an error of 1.8e-5 for 4096 x 6 terms; so, a sixth of it).
Pairs pairs_of(int a, int b) {
    Pairs p = {0, 0, 0};
    for (int sum = 2; sum >= 0; --sum)
        for (int i = 0; i <= sum; ++i) {
            if (i >= a || sum - i >= b) continue;
            p.a |= static_cast<uint32_t>(i) << 4 * p.n;
            p.b |= static_cast<uint32_t>(sum - i) << 4 * p.n;
            ++p.n;
        }
    return p;
}

int check(const malt_head_t* h) {
    if (h == nullptr || h->rows < 0 || h->dim < 1 || h->vocab < 1) return MALT_ERR_INVALID_ARG;
    if (!float_type(h->hidden_dtype) || !float_type(h->table_dtype) || !index_type(h->labels_dtype))
        return MALT_ERR_UNSUPPORTED;
    if (h->rows > kMaxRows || h->dim > kMaxDim || h->vocab > kMaxVocab) return MALT_ERR_UNSUPPORTED;
    const HeadPlan p = head_plan(h->rows, h->dim, h->vocab);
    const int64_t items = static_cast<int64_t>(p.row_tiles) * p.vocab_tiles +
                          (static_cast<int64_t>(p.pieces) * p.row_tiles + p.vocab_tiles) * p.dim_tiles;
    if (items >= (int64_t{1} << 30)) return MALT_ERR_UNSUPPORTED;
    if (h->hidden_ld < h->dim || h->table_ld < h->dim) return MALT_ERR_INVALID_ARG;
    return MALT_OK;
}
int check_data(const malt_head_t* h) {
    if (h->table == nullptr || (h->rows > 0 && (h->hidden == nullptr || h->labels == nullptr))) return MALT_ERR_INVALID_ARG;
    if (!aligned_to(h->hidden, type_bytes(h->hidden_dtype)) || !aligned_to(h->table, type_bytes(h->table_dtype)) ||
        !aligned_to(h->labels, type_bytes(h->labels_dtype)) || !aligned_to(h->weight, 4))
        return MALT_ERR_MISALIGNED;
    return MALT_OK;
}

// Where a call's buffers lie in its workspace.
struct Layout {
    HeadPlan plan;
    int h_planes, w_planes, d_planes;
    bool pack_table;
    int64_t row_ld, dim_ld;
    int64_t place, row, live, labels, weights, stats, steps, label_logits, parts, counters, ncounters, hidden, table, dl, acc, scratch;
    int64_t bytes;
};
// The table is read where it lies if it is bf16 and TMA can address it.
bool direct_table(const malt_head_t* h) {
    return h->table_dtype == MALT_BF16 && aligned_to(h->table, 16) && h->table_ld % 8 == 0;
}
// Slices of one of the sums of a logit of few rows: as short as a part.
int few_each(const malt_head_t* h) {
    const int64_t columns = (h->rows + 31) / 32 * 32, slices = (h->dim + kSlice - 1) / kSlice;
    const int64_t sums = std::min<int64_t>(kTile / std::max<int64_t>(columns, 32), kFewSums);
    return static_cast<int>((slices + sums - 1) / sums);
}
bool few_rows(const malt_head_t* h, const Layout& L) {
    return h->rows <= kFewRows && L.h_planes == 1 && L.w_planes == 1 && few_each(h) <= kLogitPart;
}
Layout layout_of(const malt_head_t* h, bool forward, bool gradient) {
    Layout L = {};
    L.plan = head_plan(h->rows, h->dim, h->vocab);
    const HeadPlan& p = L.plan;
    const bool exact = h->hidden_dtype == MALT_F32 || h->table_dtype == MALT_F32;
    L.h_planes = h->hidden_dtype == MALT_F32 ? kPlanes : 1;
    L.w_planes = h->table_dtype == MALT_F32 ? kPlanes : 1;
    L.d_planes = exact ? kPlanes : h->rows <= kTurnedRows ? 2 : 1;
    L.pack_table = !direct_table(h);
    L.row_ld = static_cast<int64_t>(p.row_tiles) * kTile;
    L.dim_ld = (h->dim + 7) / 8 * 8;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t o = at;
        at += (bytes + 255) / 256 * 256;
        return o;
    };
    // counters: queues of both passes, a status word, and what the gradient's tiles wait for
    L.ncounters = 4;
    if (gradient)
        L.ncounters += static_cast<int64_t>(p.pieces) * p.row_tiles + p.vocab_tiles +
                       static_cast<int64_t>(p.splits) * p.row_tiles * p.dim_tiles + p.pieces;
    L.counters = take(4 * L.ncounters);
    L.live = take(4);
    L.place = take(4 * h->rows);
    L.row = take(4 * L.row_ld);
    L.labels = take(4 * L.row_ld);
    L.weights = take(4 * L.row_ld);
    L.stats = take(8 * L.row_ld);
    L.steps = take(4 * L.row_ld);
    L.hidden = take(2 * L.h_planes * L.row_ld * L.dim_ld);
    if (L.pack_table) L.table = take(2 * L.w_planes * h->vocab * L.dim_ld);
    if (exact || h->dim > kLogitPart * kSlice) L.scratch = take(4ll * 2 * kMostPairs * kHalf * kTile);
    L.label_logits = take(4 * L.row_ld);
    if (forward) {
        L.parts = take(8 * L.row_ld * std::max<int64_t>(2 * p.vocab_tiles, few_rows(h, L) ? 2 * kMostPairs : 0));
    }
    if (gradient) {
        L.dl = take(2 * static_cast<int64_t>(p.buffers) * L.d_planes * L.row_ld * p.piece_tiles * kTile);
        L.acc = take(4 * static_cast<int64_t>(p.splits) * L.row_ld * L.dim_ld);
    }
    L.bytes = at;
    return L;
}

struct Outputs {
    float* loss;                // forward
    float2* stats;
    const float2* in_stats;     // the gradient alone
    const float* dloss;
    void* dhidden;
    int64_t dhidden_ld;
    void* dtable;
    int64_t dtable_ld;
    int32_t dtable_dtype, accumulate;
};

using PackKernel = void (*)(Pack);
PackKernel pack_kernel(const Pack& K, int32_t dtype) {
    const bool vec = K.from_ld % 8 == 0 && aligned_to(K.from, 16);
    if (dtype == MALT_BF16) return vec ? head_pack_kernel<bf16, true> : head_pack_kernel<bf16, false>;
    return vec ? head_pack_kernel<float, true> : head_pack_kernel<float, false>;
}

using GatherKernel = void (*)(Scan, Pack);
template <int MOST>
GatherKernel gather_kernel(const Pack& K, int32_t dtype) {
    const bool vec = K.from_ld % 8 == 0 && aligned_to(K.from, 16);
    if (dtype == MALT_BF16) return vec ? head_gather_kernel<bf16, true, MOST> : head_gather_kernel<bf16, false, MOST>;
    return vec ? head_gather_kernel<float, true, MOST> : head_gather_kernel<float, false, MOST>;
}

cudaError_t launch_all(const malt_head_t* h, const Outputs& O, bool forward, bool gradient, char* ws, cudaStream_t s) {
    const Layout L = layout_of(h, forward, gradient);
    const HeadPlan& p = L.plan;
    int pairs = 0;
    cudaError_t e = configure(&pairs);
    if (e != cudaSuccess) return e;
    if (encoder() == nullptr) return cudaErrorNotSupported;
    auto at = [&](int64_t o) { return reinterpret_cast<void*>(ws + o); };
    uint32_t* const counters = static_cast<uint32_t*>(at(L.counters));
    int32_t* const status = reinterpret_cast<int32_t*>(counters + 2);
    const int32_t rows = static_cast<int32_t>(h->rows);

    Scan S = {};
    S.labels = h->labels;
    S.labels_i64 = h->labels_dtype == MALT_I64;
    S.rows = rows;
    S.vocab = static_cast<int32_t>(h->vocab);
    S.weight = h->weight;
    S.dloss = O.dloss;
    S.stats = O.in_stats;
    S.loss = O.loss;
    S.out_stats = O.stats;
    S.place = static_cast<int32_t*>(at(L.place));
    S.row = static_cast<int32_t*>(at(L.row));
    S.live = static_cast<int32_t*>(at(L.live));
    S.c_labels = static_cast<int32_t*>(at(L.labels));
    S.c_weights = static_cast<float*>(at(L.weights));
    S.c_stats = static_cast<float2*>(at(L.stats));
    S.counters = counters;
    S.ncounters = L.ncounters;
    Pack K = {};
    K.from = h->hidden;
    K.from_ld = h->hidden_ld;
    K.row = S.row;
    K.live = S.live;
    K.rows = rows;
    K.cols = static_cast<int32_t>(h->dim);
    K.ld = static_cast<int32_t>(L.dim_ld);
    K.planes = L.h_planes;
    K.plane = L.row_ld * L.dim_ld;
    K.to = static_cast<bf16*>(at(L.hidden));
    K.labels = S.c_labels;
    K.table = h->table;
    K.table_ld = h->table_ld;
    K.table_bf16 = h->table_dtype == MALT_BF16;
    K.table_vec = h->table_ld % 8 == 0 && aligned_to(h->table, 16);
    K.label_logits = static_cast<float*>(at(L.label_logits));
    K.steps = static_cast<int32_t*>(at(L.steps));
    if (rows <= kGatherRows) {
        const GatherKernel gather = rows <= 256 ? gather_kernel<256>(K, h->hidden_dtype)
                                                : gather_kernel<kGatherRows>(K, h->hidden_dtype);
        e = launch_chained(gather, static_cast<unsigned>(L.row_ld / 8), 256, 0, s, S, K);
    } else {
        e = launch_chained(head_scan_kernel, 1, kScanThreads, 0, s, S);
        if (e == cudaSuccess)
            e = launch_chained(pack_kernel(K, h->hidden_dtype), static_cast<unsigned>(L.row_ld / 8), 256, 0, s, K);
    }
    if (e != cudaSuccess) return e;
    if (L.pack_table) {
        K.from = h->table;
        K.from_ld = h->table_ld;
        K.row = nullptr;
        K.live = nullptr;
        K.labels = nullptr;
        K.steps = nullptr;
        K.rows = static_cast<int32_t>(h->vocab);
        K.planes = L.w_planes;
        K.plane = h->vocab * L.dim_ld;
        K.to = static_cast<bf16*>(at(L.table));
        e = launch_chained(pack_kernel(K, h->table_dtype), static_cast<unsigned>((h->vocab + 7) / 8), 256, 0, s, K);
        if (e != cudaSuccess) return e;
    }

    Gemm G = {};
    const bool turned = h->rows <= kTurnedRows;
    G.columns = static_cast<int32_t>((h->rows + 63) / 64 * 64);
    const void* const w = L.pack_table ? at(L.table) : h->table;
    const int64_t w_ld = L.pack_table ? L.dim_ld : h->table_ld, w_cols = L.pack_table ? L.dim_ld : h->dim;
    bool ok = map_of(&G.h_k, at(L.hidden), L.dim_ld, L.row_ld, L.h_planes, L.dim_ld, kHalf) &&
              map_of(&G.w_k, w, w_cols, h->vocab, L.w_planes, w_ld, kHalf);
    if (ok && gradient) {
        const int64_t piece = static_cast<int64_t>(p.piece_tiles) * kTile, planes = p.buffers * L.d_planes;
        ok = map_of(&G.h_mn, at(L.hidden), L.dim_ld, L.row_ld, L.h_planes, L.dim_ld, kSlice) &&
             map_of(&G.w_mn, w, w_cols, h->vocab, L.w_planes, w_ld, kSlice) &&
             map_of(&G.d_k, at(L.dl), piece, L.row_ld, planes, piece, !turned ? kHalf : L.d_planes == 2 ? G.columns : G.columns / 2) &&
             map_of(&G.d_mn, at(L.dl), piece, L.row_ld, planes, piece, kSlice) &&
             map_of(&G.d_out, at(L.dl), piece, L.row_ld, planes, piece, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B) &&
             map_of(&G.acc_out, at(L.acc), turned ? L.row_ld : L.dim_ld, turned ? L.dim_ld : L.row_ld, p.splits,
                    turned ? L.row_ld : L.dim_ld, 32, 16, CU_TENSOR_MAP_SWIZZLE_64B, true);
    }
    if (!ok) return cudaErrorInvalidValue;
    G.plan = p;
    G.logits = pairs_of(L.h_planes, L.w_planes);
    G.abreast = L.d_planes == 2;
    G.hidden = pairs_of(G.abreast ? 1 : L.d_planes, L.w_planes);
    G.table = pairs_of(L.d_planes, L.h_planes);
    G.d_planes = L.d_planes;
    G.exact = L.d_planes == kPlanes;
    G.scratch = static_cast<float*>(at(L.scratch));
    G.dim = static_cast<int32_t>(h->dim);
    G.dim_ld = static_cast<int32_t>(L.dim_ld);
    G.vocab = static_cast<int32_t>(h->vocab);
    G.row_ld = static_cast<int32_t>(L.row_ld);
    G.live = S.live;
    G.labels = S.c_labels;
    G.weights = S.c_weights;
    G.steps = static_cast<const int32_t*>(at(L.steps));
    G.stats = S.c_stats;
    G.parts = static_cast<float2*>(at(L.parts));
    G.label_logits = static_cast<const float*>(at(L.label_logits));
    G.status = status;
    // 1 s, and what a tile's longest reduction takes at a tenth of a pair's rate
    const int64_t longest = 6 * std::max({h->dim, L.row_ld, static_cast<int64_t>(p.piece_tiles) * kTile});
    G.budget_ns = 1000000000ull + static_cast<uint64_t>(longest) * 66;
    const unsigned most = static_cast<unsigned>(std::min(pairs, kMostPairs));
    if (forward) {
        int32_t nparts = 2 * p.vocab_tiles;
        if (few_rows(h, L)) {
            Few F = {};
            F.w_k = G.w_k;
            F.columns = static_cast<int32_t>((h->rows + 31) / 32 * 32);
            F.each = few_each(h);
            if (!map_of(&F.h_n, at(L.hidden), L.dim_ld, L.row_ld, 1, L.dim_ld, F.columns / 2)) return cudaErrorInvalidValue;
            F.dim = G.dim;
            F.vocab = G.vocab;
            F.vocab_tiles = p.vocab_tiles;
            F.row_ld = G.row_ld;
            // (a table that is packed is not there yet)
            F.prefetch = L.pack_table ? 0 : static_cast<int32_t>(std::min<int64_t>(p.vocab_tiles, kPrefetchBytes / (kTile * 2 * L.dim_ld)));
            F.live = S.live;
            F.labels = S.c_labels;
            F.steps = G.steps;
            F.label_logits = G.label_logits;
            F.parts = G.parts;
            F.status = status;
            F.budget_ns = G.budget_ns;
            const unsigned grid = std::min<unsigned>(most, p.vocab_tiles);
            nparts = static_cast<int32_t>(2 * grid);
            e = launch_chained(head_few_kernel, 2 * grid, kFewThreads, kFewSmem, s, F);
        } else {
            G.queue = counters;
            const int64_t items = static_cast<int64_t>(p.row_tiles) * p.vocab_tiles;
            e = launch_chained(head_gemm_kernel<false>, 2 * static_cast<unsigned>(std::min<int64_t>(most, items)), kThreads,
                               kSmem, s, G);
        }
        if (e != cudaSuccess) return e;
        Join J = {};
        J.live = S.live;
        J.row = S.row;
        J.parts = G.parts;
        J.nparts = nparts;
        J.row_ld = G.row_ld;
        J.label_logits = G.label_logits;
        J.c_weights = S.c_weights;
        J.loss = O.loss;
        J.out_stats = O.stats;
        J.c_stats = S.c_stats;
        J.status = status;
        e = launch_chained(head_join_kernel, static_cast<unsigned>(L.row_ld / 32), 32 * kJoinWarps, 0, s, J);
        if (e != cudaSuccess) return e;
    }
    if (!gradient) return cudaSuccess;
    G.backward = 1;
    G.dtable = O.dtable;
    G.dtable_ld = O.dtable_ld;
    G.dtable_bf16 = O.dtable_dtype == MALT_BF16;
    G.accumulate = O.accumulate;
    // Boxes need rows on 16 bytes and of whole 16 bytes (they write what a row's last unit has behind it
    // too), and add in fp32 only.
    const int64_t unit = 16 / type_bytes(O.dtable_dtype);
    G.dtable_boxes = aligned_to(O.dtable, 16) && O.dtable_ld % unit == 0 && h->dim % unit == 0 &&
                     !(G.dtable_bf16 && O.accumulate);
    if (G.dtable_boxes &&
        !map_of(&G.t_out, O.dtable, h->dim, h->vocab, 1, O.dtable_ld, 32, G.dtable_bf16 ? 32 : 16, CU_TENSOR_MAP_SWIZZLE_64B,
                !G.dtable_bf16))
        return cudaErrorInvalidValue;
    G.queue = counters + 1;
    G.row_done = counters + 4;
    G.col_done = G.row_done + static_cast<int64_t>(p.pieces) * p.row_tiles;
    G.hidden_done = G.col_done + p.vocab_tiles;
    G.piece_done = G.hidden_done + static_cast<int64_t>(p.splits) * p.row_tiles * p.dim_tiles;
    if (turned && !map_of(&G.h_k, at(L.hidden), L.dim_ld, L.row_ld, L.h_planes, L.dim_ld, G.columns / 2))
        return cudaErrorInvalidValue;
    const unsigned grid = std::min<unsigned>(most, head_items(p, p.row_tiles));
    e = launch_chained(turned ? head_gemm_kernel<true, true> : head_gemm_kernel<true>, 2 * grid, kThreads, kSmem, s, G);
    if (e != cudaSuccess || rows == 0) return e;
    Spread D = {};
    D.place = S.place;
    D.acc = static_cast<const float*>(at(L.acc));
    D.rows = rows;
    D.dim = G.dim;
    D.dim_ld = G.dim_ld;
    D.row_ld = G.row_ld;
    D.splits = p.splits;
    D.part = L.row_ld * L.dim_ld;
    D.to = O.dhidden;
    D.to_ld = O.dhidden_ld;
    D.status = status;
    const bool vec = h->dim % 8 == 0 && D.to_ld % 8 == 0 && aligned_to(D.to, 16);
    void (*spread)(Spread);
    if (turned) {
        spread = h->hidden_dtype == MALT_BF16 ? head_spread_turned_kernel<bf16> : head_spread_turned_kernel<float>;
        return launch_chained(spread, static_cast<unsigned>((h->rows + 31) / 32 * ((h->dim + 7) / 8)), 256, 0, s, D);
    }
    if (p.splits > 1 && h->rows <= kSpreadRows) {
        spread = h->hidden_dtype == MALT_BF16 ? head_spread_parts_kernel<bf16> : head_spread_parts_kernel<float>;
        for (D.share = 2; D.share < p.splits && D.share < kSpreadWarps;) D.share *= 2;
        const int64_t each = kSpreadWarps / D.share;        // rows of a block
        return launch_chained(spread, static_cast<unsigned>((h->rows + each - 1) / each * ((h->dim + 255) / 256)),
                              32 * kSpreadWarps, 0, s, D);
    }
    if (h->hidden_dtype == MALT_BF16) spread = vec ? head_spread_kernel<bf16, true> : head_spread_kernel<bf16, false>;
    else spread = vec ? head_spread_kernel<float, true> : head_spread_kernel<float, false>;
    return launch_chained(spread, static_cast<unsigned>((h->rows + 7) / 8), 256, 0, s, D);
}

int run(const malt_head_t* h, const Outputs& O, bool forward, bool gradient, void* workspace, size_t bytes, void* stream,
        const char* name) {
    int rc = check(h);
    if (rc == MALT_OK) rc = check_data(h);
    if (rc != MALT_OK) return rc;
    if (h->rows > 0) {
        if (forward && O.loss == nullptr) return MALT_ERR_INVALID_ARG;
        if (!forward && O.in_stats == nullptr) return MALT_ERR_INVALID_ARG;
        if (gradient && O.dhidden == nullptr) return MALT_ERR_INVALID_ARG;
    }
    if (!aligned_to(O.loss, 4) || !aligned_to(O.stats, 8) || !aligned_to(O.in_stats, 8) || !aligned_to(O.dloss, 4))
        return MALT_ERR_MISALIGNED;
    if (gradient) {
        if (O.dtable == nullptr || O.dtable_ld < h->dim || O.dhidden_ld < h->dim) return MALT_ERR_INVALID_ARG;
        if (!float_type(O.dtable_dtype)) return MALT_ERR_UNSUPPORTED;
        if (!aligned_to(O.dtable, type_bytes(O.dtable_dtype)) || !aligned_to(O.dhidden, type_bytes(h->hidden_dtype)))
            return MALT_ERR_MISALIGNED;
    }
    const int64_t need = layout_of(h, forward, gradient).bytes;
    if (workspace == nullptr || bytes < static_cast<size_t>(need)) return MALT_ERR_INVALID_ARG;
    if (!aligned_to(workspace, 256)) return MALT_ERR_MISALIGNED;
    if (h->rows == 0 && !gradient) return MALT_OK;
    if (h->rows == 0 && O.accumulate) return MALT_OK;
    // (inputs are read while outputs are written)
    const int hidden_bytes = type_bytes(h->hidden_dtype);
    const Extent out[] = {extent_of(O.loss, 4 * h->rows), extent_of(O.stats, 8 * h->rows),
                          extent_of(O.dhidden, h->rows, h->dim, O.dhidden_ld, hidden_bytes),
                          extent_of(O.dtable, h->vocab, h->dim, O.dtable_ld, type_bytes(O.dtable_dtype)),
                          extent_of(workspace, need)};
    const Extent in[] = {extent_of(h->hidden, h->rows, h->dim, h->hidden_ld, hidden_bytes),
                         extent_of(h->table, h->vocab, h->dim, h->table_ld, type_bytes(h->table_dtype)),
                         extent_of(h->labels, type_bytes(h->labels_dtype) * h->rows), extent_of(h->weight, 4 * h->rows),
                         extent_of(O.in_stats, 8 * h->rows), extent_of(O.dloss, 4 * h->rows)};
    for (const Extent& o : out) {
        for (const Extent& i : in)
            if (overlap(o, i)) return MALT_ERR_INVALID_ARG;
        for (const Extent* other = out; other != &o; ++other)
            if (overlap(o, *other)) return MALT_ERR_INVALID_ARG;
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (h->rows == 0)
        return cuda_status(cudaMemset2DAsync(O.dtable, O.dtable_ld * type_bytes(O.dtable_dtype), 0,
                                             h->dim * type_bytes(O.dtable_dtype), h->vocab, s), name);
    nvtxRangePushA(name);
    const cudaError_t e = launch_all(h, O, forward, gradient, static_cast<char*>(workspace), s);
    nvtxRangePop();
    return cuda_status(e, name);
}

}  // namespace
}  // namespace malt

extern "C" {

size_t malt_head_workspace_bytes(const malt_head_t* h, int32_t forward, int32_t gradient) {
    if (malt::check(h) != MALT_OK) return 0;
    return static_cast<size_t>(malt::layout_of(h, forward != 0, gradient != 0).bytes);
}

int malt_head_forward(const malt_head_t* h, float* loss, float* stats, void* workspace, size_t workspace_bytes,
                      void* stream) {
    malt::Outputs O = {};
    O.loss = loss;
    O.stats = reinterpret_cast<float2*>(stats);
    return malt::run(h, O, true, false, workspace, workspace_bytes, stream, "malt_head_forward");
}

int malt_head_backward(const malt_head_t* h, const float* stats, const float* dloss, void* dhidden, int64_t dhidden_ld,
                       void* dtable, int64_t dtable_ld, int32_t dtable_dtype, int32_t accumulate, void* workspace,
                       size_t workspace_bytes, void* stream) {
    malt::Outputs O = {};
    O.in_stats = reinterpret_cast<const float2*>(stats);
    O.dloss = dloss;
    O.dhidden = dhidden, O.dhidden_ld = dhidden_ld;
    O.dtable = dtable, O.dtable_ld = dtable_ld, O.dtable_dtype = dtable_dtype, O.accumulate = accumulate != 0;
    return malt::run(h, O, false, true, workspace, workspace_bytes, stream, "malt_head_backward");
}

int malt_head_forward_backward(const malt_head_t* h, float* loss, float* stats, void* dhidden, int64_t dhidden_ld,
                               void* dtable, int64_t dtable_ld, int32_t dtable_dtype, int32_t accumulate,
                               void* workspace, size_t workspace_bytes, void* stream) {
    malt::Outputs O = {};
    O.loss = loss;
    O.stats = reinterpret_cast<float2*>(stats);
    O.dhidden = dhidden, O.dhidden_ld = dhidden_ld;
    O.dtable = dtable, O.dtable_ld = dtable_ld, O.dtable_dtype = dtable_dtype, O.accumulate = accumulate != 0;
    return malt::run(h, O, true, true, workspace, workspace_bytes, stream, "malt_head_forward_backward");
}

}  // extern "C"
