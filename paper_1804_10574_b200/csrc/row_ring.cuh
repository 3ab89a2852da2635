// Rows on their way through shared memory: a block's first thread copies the rows that the block will work on, several ahead,
// by bulk copies (TMA without a tensor map) into a ring of stages.  The threads read their values from there as often as they
// need them; after the first barrier of the next row's reductions, when all are done with a row, its stage takes another.
// Memory stays busy through the reductions, without registers for what is on the way or for what is needed again.
//
// A bulk copy moves whole 16-byte units.  Tensors start on 16-byte boundaries; a row that does not is copied from the boundary
// before it to the one behind it, never past the tensor's own whole units: the last row's last few values may have to be read
// from memory.
#pragma once
#include "f32x2.cuh"
#include "pair_mma.cuh"

namespace ddg {

namespace {

constexpr int kRingMostStages = 8;

struct RingShape {
    int row_bytes;    // of a row
    int slot_bytes;   // a row's place in a stage, on 16-byte boundaries
    int stages;
    size_t floor16;   // a tensor's bytes in whole 16-byte units
    unsigned polls;   // of a bounded wait
};

// Where row `row` starts in its slot, and how many of its bytes are there.
struct RingRow { int phase, valid; };
__device__ __forceinline__ RingRow ring_row(const RingShape &g, int row) {
    const size_t at = (size_t)row * g.row_bytes;
    return RingRow{(int)(at & 15), (int)min((size_t)g.row_bytes, g.floor16 > at ? g.floor16 - at : (size_t)0)};
}

template <int TENSORS> struct RowRing {
    const RingShape &g;
    uint32_t base;      // shared memory of the stages
    uint64_t *full;
    Waiter wt;
    uint32_t stage, parity, issued;

    __device__ __forceinline__ RowRing(const RingShape &shape, uint32_t smem, uint64_t *full_, int *abort_flag)
        : g(shape), base(smem), full(full_), wt{abort_flag, abort_flag, shape.polls}, stage(0), parity(0), issued(0) {}

    __device__ __forceinline__ void init() {  // by one thread, before a barrier of the block
        for (int i = 0; i < g.stages; ++i) mbar_init(smem_u32(&full[i]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *wt.abort_flag = 0;
    }
    // By the copying thread: the next row into the stage that is free.  A tensor that is not there (nullptr) is left out.  Nothing
    // is copied any more once a wait ran out.
    __device__ __forceinline__ void copy(int row, const void *const (&src)[TENSORS]) {
        if (*wt.abort_flag) return;
        const size_t at = (size_t)row * g.row_bytes, from = at & ~(size_t)15, to = min((at + g.row_bytes + 15) & ~(size_t)15, g.floor16);
        const uint32_t s = issued % (uint32_t)g.stages, bytes = to > from ? (uint32_t)(to - from) : 0u, bar = smem_u32(&full[s]);
        int n = 0;
#pragma unroll
        for (int k = 0; k < TENSORS; ++k) n += src[k] != nullptr;
        mbar_expect_tx(bar, bytes * n);
        if (bytes) {
#pragma unroll
            for (int k = 0; k < TENSORS; ++k)
                if (src[k]) bulk_copy_g2s(base + (s * TENSORS + k) * g.slot_bytes, (const uint8_t *)src[k] + from, bytes, bar);
        }
        ++issued;
    }
    // The copying thread, at its end: what it issued has landed, whatever became of the readers.
    __device__ __forceinline__ void drain() {
        for (uint32_t i = issued > (uint32_t)g.stages ? issued - g.stages : 0; i < issued; ++i) mbar_drain(smem_u32(&full[i % g.stages]), (i / g.stages) & 1u);
    }
    // false when the wait ran out (what stands in the stage is not the row)
    __device__ __forceinline__ bool wait() { return mbar_wait(smem_u32(&full[stage]), parity, wt, 82); }
    __device__ __forceinline__ uint32_t slot(int tensor) const { return base + (stage * TENSORS + tensor) * g.slot_bytes; }
    __device__ __forceinline__ void next() { if (++stage == (uint32_t)g.stages) { stage = 0; parity ^= 1u; } }
};

// A thread's share of a row: ITER vectors of VEC values, vector i at columns (i threads + t) VEC on, worked in groups of pairs: a
// vector, or (VEC = 1) two values.  Columns past the row are zeros.
template <int VEC> constexpr int kGroup = VEC > 1 ? VEC / 2 : 1;  // pairs

// Group i of a row in a slot.  Value c stands at phase + c * sizeof(T); vectors: phase 0, and all of the row is there.
template <typename T, int VEC> __device__ __forceinline__ void slot_load(uint32_t slot, const RingRow &at, const T *row, int C, int i, F2 (&v)[kGroup<VEC>]) {
    if constexpr (VEC > 1) {
        const int c = (i * blockDim.x + threadIdx.x) * VEC;
        uint32_t w[4] = {0u, 0u, 0u, 0u};
        if (c < C) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(slot + c * (uint32_t)sizeof(T)));
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) {
            if constexpr (sizeof(T) == 2) v[j] = bf16_pair(w[j]);
            else v[j] = f2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
        }
    } else {
        float e[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int c = (2 * i + j) * blockDim.x + threadIdx.x;
            if (c >= C) {
                e[j] = 0.f;
            } else if (c * (int)sizeof(T) >= at.valid) {
                e[j] = to_f(row[c]);
            } else if constexpr (sizeof(T) == 2) {
                uint16_t w;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(slot + at.phase + c * 2u));
                e[j] = __uint_as_float((uint32_t)w << 16);
            } else {
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(e[j]) : "r"(slot + at.phase + c * 4u));
            }
        }
        v[0] = f2(e[0], e[1]);
    }
}
// A thread's share of what all rows have in common, as it lies in memory.
template <typename T, int VEC, int ITER> struct Share {
    static constexpr int N = VEC * ITER;
    static_assert(N % 2 == 0 && (VEC == 1 || VEC * sizeof(T) == 16), "whole units or single values");
    alignas(16) T e[N];
    __device__ __forceinline__ void load(const T *row, int C) {
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * blockDim.x + threadIdx.x) * VEC;
            if constexpr (VEC > 1) *reinterpret_cast<uint4 *>(e + i * VEC) = c < C ? *reinterpret_cast<const uint4 *>(row + c) : make_uint4(0u, 0u, 0u, 0u);
            else e[i] = c < C ? row[c] : from_f<T>(0.f);
        }
    }
    __device__ __forceinline__ F2 pair(int k) const {  // values 2k and 2k + 1
        if constexpr (sizeof(T) == 2 && VEC > 1) return bf16_pair(reinterpret_cast<const uint32_t *>(e)[k]);
        else return f2(to_f(e[2 * k]), to_f(e[2 * k + 1]));
    }
};
// Group i to a row in memory, in the element type.
template <typename T, int VEC> __device__ __forceinline__ void group_store(T *row, int C, int i, const F2 (&v)[kGroup<VEC>]) {
    if constexpr (VEC > 1) {
        const int c = (i * blockDim.x + threadIdx.x) * VEC;
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 2) w[j] = to_bf16_pair(v[j]);
            else w[j] = __float_as_uint(j % 2 ? parts(v[j / 2]).y : parts(v[j / 2]).x);
        }
        if (c < C) *reinterpret_cast<uint4 *>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
        const int c = 2 * i * blockDim.x + threadIdx.x, d = c + blockDim.x;
        const float2 p = parts(v[0]);
        if (c < C) row[c] = from_f<T>(p.x);
        if (d < C) row[d] = from_f<T>(p.y);
    }
}
template <typename T, int VEC, int ITER> __device__ __forceinline__ void share_store(T *row, int C, const F2 (&v)[VEC * ITER / 2]) {
    constexpr int G = kGroup<VEC>;
#pragma unroll
    for (int i = 0; i < VEC * ITER / 2 / G; ++i) {
        F2 g[G];
#pragma unroll
        for (int j = 0; j < G; ++j) g[j] = v[i * G + j];
        group_store<T, VEC>(row, C, i, g);
    }
}
// The same as fp32; the row starts on a 16-byte boundary (VEC > 1).
template <int VEC, int ITER> __device__ __forceinline__ void share_store_f32(float *row, int C, const F2 (&v)[VEC * ITER / 2]) {
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * blockDim.x + threadIdx.x) * VEC;
        if (c >= C) continue;
        if constexpr (VEC > 1) {
#pragma unroll
            for (int j = 0; j < VEC; j += 4) {
                const float2 a = parts(v[(i * VEC + j) / 2]), b = parts(v[(i * VEC + j) / 2 + 1]);
                *reinterpret_cast<float4 *>(row + c + j) = make_float4(a.x, a.y, b.x, b.y);
            }
        } else {
            row[c] = i % 2 ? parts(v[i / 2]).y : parts(v[i / 2]).x;
        }
    }
}

// Sums (or, as bits, maxima) over a row's threads, which are the block: one barrier, buffers of two rounds in turn (red: six
// times 32 floats, zeros at first, on a 16-byte boundary; what is summed and what is a maximum keep to their own rows).
template <int N> __device__ __forceinline__ void ring_sum(float (&v)[N], float (*red)[32], uint32_t &round) {
    static_assert(N <= 3, "the buffers' size");
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = warp_sum(v[k]);
    float (*to)[32] = red + (round & 1u) * 3;
    ++round;
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) to[k][warp] = v[k];
    }
    __syncthreads();
    // the warps' sums in index order, four at a time (those of warps that are not there are zeros)
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = 0.f;
    for (int w = 0; w < warps; w += 4) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float4 q = *reinterpret_cast<const float4 *>(&to[k][w]);
            v[k] += (q.x + q.y) + (q.z + q.w);
        }
    }
}
// A sum and a maximum (of bits) in one round.
__device__ __forceinline__ void ring_sum_max(float &sum, uint32_t &top, float (*red)[32], uint32_t &round) {
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    sum = warp_sum(sum);
    top = __reduce_max_sync(0xffffffffu, top);
    float (*to)[32] = red + (round & 1u) * 3;
    ++round;
    if (lane == 0) { to[0][warp] = sum; to[1][warp] = __uint_as_float(top); }
    __syncthreads();
    sum = 0.f;
    for (int w = 0; w < warps; w += 4) {
        const float4 q = *reinterpret_cast<const float4 *>(&to[0][w]);
        sum += (q.x + q.y) + (q.z + q.w);
        const uint4 m = *reinterpret_cast<const uint4 *>(&to[1][w]);
        top = max(max(top, max(m.x, m.y)), max(m.z, m.w));
    }
}
__device__ __forceinline__ uint32_t ring_max(uint32_t v, float (*red)[32], uint32_t &round) {
    const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    v = __reduce_max_sync(0xffffffffu, v);
    float *to = red[(round & 1u) * 3 + 1];
    ++round;
    if (lane == 0) to[warp] = __uint_as_float(v);
    __syncthreads();
    for (int w = 0; w < warps; w += 4) {
        const uint4 m = *reinterpret_cast<const uint4 *>(to + w);
        v = max(max(v, max(m.x, m.y)), max(m.z, m.w));
    }
    return v;
}

// ---- host side -------------------------------------------------------------------------------------------------------
// Threads of a row (whole warps) that have `iter` vectors each.
inline int ring_threads(int nvec, int iter) { return ((nvec + iter - 1) / iter + 31) / 32 * 32; }
constexpr size_t kRingSmem = 216 * 1024;
// Blocks of an SM for rows of `threads` threads, and the shared memory of each; `extra` bytes of it are not the ring's.  Two
// stages at least, else 0 blocks.
struct RingPlan { int threads, per_sm; size_t smem; };
inline RingShape ring_shape(int rows, int row_bytes, int tensors, size_t smem, unsigned polls);
inline RingPlan ring_plan(int C, int row_bytes, int vec, int iter, int tensors, size_t extra) {
    RingPlan p{};
    const int threads = std::max(64, ring_threads((C + vec - 1) / vec, iter));
    if (threads > 512) return p;
    p.per_sm = std::min(8, std::max(1, 512 / threads));
    while (p.per_sm > 1 && ring_shape(1, row_bytes, tensors, kRingSmem / p.per_sm / 16 * 16 - extra, 0).stages < 2) --p.per_sm;
    p.smem = kRingSmem / p.per_sm / 16 * 16;
    if (p.smem > extra && ring_shape(1, row_bytes, tensors, p.smem - extra, 0).stages >= 2) p.threads = threads;
    return p;
}
template <typename K> bool ring_ready(K kernel, int &ready_dev) {
    int dev = 0;
    cudaGetDevice(&dev);
    if (ready_dev != dev) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kRingSmem) != cudaSuccess) return false;
        ready_dev = dev;
    }
    return true;
}
inline RingShape ring_shape(int rows, int row_bytes, int tensors, size_t smem, unsigned polls) {
    RingShape g;
    g.row_bytes = row_bytes;
    g.slot_bytes = row_bytes % 16 == 0 ? row_bytes : (row_bytes + 31) / 16 * 16;
    g.stages = (int)std::min<size_t>(kRingMostStages, smem / ((size_t)tensors * g.slot_bytes));
    g.floor16 = (size_t)rows * row_bytes / 16 * 16;
    g.polls = polls;
    return g;
}

}  // namespace

}  // namespace ddg
