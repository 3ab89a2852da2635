// Rows on their way through shared memory: a block copies the rows that it will work on, several ahead, by bulk copies (TMA
// without a tensor map) into a ring of stages.  The threads read their values from there as often as they need them; after the
// first barrier of the next row's reductions, when all are done with a row, its stage takes another.
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

// Where row `row` starts in its slot.
__device__ __forceinline__ int ring_phase(const RingShape &g, int row) { return (int)((size_t)row * g.row_bytes & 15); }

template <int TENSORS> struct RowRing {
    const RingShape &g;
    uint32_t base;      // shared memory of the stages
    uint64_t *full;
    Waiter wt;
    int *lost_at;       // shared memory: the first row whose wait ran out (rows come in ascending order)
    uint32_t stage, parity;  // of the row that is read next
    uint32_t head, issued;   // stage that is filled next; rows that this thread had copied
    const uint8_t *src[TENSORS];  // nullptr: a tensor that is not there
    static constexpr bool kMany = TENSORS > 2;
    const uint8_t **list;         // many tensors: the same in shared memory, for the warps that copy
    int tensors;
    bool lost;

    __device__ __forceinline__ RowRing(const RingShape &shape, uint32_t smem, uint64_t *full_, int (&flags)[2], const uint8_t *(&list_)[TENSORS], const void *const (&all)[TENSORS])
        : g(shape), base(smem), full(full_), wt{&flags[0], &flags[0], shape.polls}, lost_at(&flags[1]), stage(0), parity(0), head(0), issued(0), list(list_), tensors(0), lost(false) {
#pragma unroll
        for (int k = 0; k < TENSORS; ++k) {
            src[k] = (const uint8_t *)all[k];
            tensors += all[k] != nullptr;
        }
    }

    __device__ __forceinline__ void init() {  // by one thread, before a barrier of the block
        for (int i = 0; i < g.stages; ++i) mbar_init(smem_u32(&full[i]), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *wt.abort_flag = 0;
        *lost_at = 0x7fffffff;
        if constexpr (kMany) {
#pragma unroll
            for (int k = 0; k < TENSORS; ++k) list[k] = src[k];
        }
    }
    // By all threads: a row into the stage that is free, while row `now` is worked on (-1: none yet), after a barrier behind the
    // wait for that.  The first lane of each warp issues a share of the copies: each takes its warp a few hundred cycles.  Once a
    // wait for this row or one before ran out nothing is copied any more; the barrier has made that the same for all warps, so
    // that a stage gets all of its copies or none, and the first thread knows what is on the way.
    __device__ __forceinline__ void copy(int row, int now) {
        const int warps = blockDim.x >> 5, warp = threadIdx.x >> 5;
        if ((threadIdx.x & 31) == 0 && warp < TENSORS && !lost_by(now)) {
            const size_t at = (size_t)row * g.row_bytes, from = at & ~(size_t)15, to = min((at + g.row_bytes + 15) & ~(size_t)15, g.floor16);
            const uint32_t bytes = to > from ? (uint32_t)(to - from) : 0u, bar = smem_u32(&full[head]);
            // (what lands before the barrier expects it is counted all the same: its phase ends with this arrival)
            if (warp == 0) mbar_expect_tx(bar, bytes * tensors);
            // (8192 x 5120 backward: 112 us with the loop, 120 with a test per tensor; packing 8192 x 4096: 25 and 21)
            if constexpr (kMany) {
#pragma unroll 1
                for (int k = warp; k < TENSORS; k += warps)
                    if (list[k] && bytes) bulk_copy_g2s(base + (head * TENSORS + k) * g.slot_bytes, list[k] + from, bytes, bar);
            } else {
#pragma unroll
                for (int k = 0; k < TENSORS; ++k)
                    if (k % min(warps, TENSORS) == warp && src[k] && bytes) bulk_copy_g2s(base + (head * TENSORS + k) * g.slot_bytes, src[k] + from, bytes, bar);
            }
            ++issued;
        }
        if (++head == (uint32_t)g.stages) head = 0;
    }
    // The first thread, at its end: what was issued has landed, whatever became of the readers.
    __device__ __forceinline__ void drain() {
        for (uint32_t i = issued > (uint32_t)g.stages ? issued - g.stages : 0; i < issued; ++i) mbar_drain(smem_u32(&full[i % g.stages]), (i / g.stages) & 1u);
    }
    // By all threads: false when a wait of the thread ran out, this one or one before (what stands in the stage may not be the
    // row).  T: type of the tensors' values, VEC = 1 where rows keep to no boundary.
    template <typename T, int VEC> __device__ __forceinline__ bool wait(int row) {
        if (!lost && !mbar_wait(smem_u32(&full[stage]), parity, wt, 82)) {
            lost = true;
            atomicMin(lost_at, row);
        }
        if (VEC == 1 && (size_t)(row + 1) * g.row_bytes > g.floor16) {  // the tensor's last values, which no copy brought
            const size_t at = (size_t)row * g.row_bytes;
            const int there = g.floor16 > at ? (int)(g.floor16 - at) / (int)sizeof(T) : 0, all = g.row_bytes / (int)sizeof(T);
#pragma unroll
            for (int k = 0; k < TENSORS; ++k)
                if (src[k])
                    for (int c = there + threadIdx.x; c < all; c += blockDim.x) {
                        const uint32_t to = slot(k) + (uint32_t)(at & 15) + c * (uint32_t)sizeof(T);
                        const uint8_t *from = src[k] + at + c * sizeof(T);
                        if constexpr (sizeof(T) == 2) asm volatile("st.shared.u16 [%0], %1;" ::"r"(to), "h"(*reinterpret_cast<const uint16_t *>(from)) : "memory");
                        else asm volatile("st.shared.b32 [%0], %1;" ::"r"(to), "r"(*reinterpret_cast<const uint32_t *>(from)) : "memory");
                    }
            __syncthreads();
        }
        return !lost;
    }
    // Whether any thread's wait for this row or one before ran out.  Behind a barrier that follows the wait for the row all threads
    // get the same answer: what a faster one's wait for the next row may add is a later row.
    __device__ __forceinline__ bool lost_by(int row) const { return *(volatile int *)lost_at <= row; }
    __device__ __forceinline__ uint32_t slot(int tensor) const { return base + (stage * TENSORS + tensor) * g.slot_bytes; }
    __device__ __forceinline__ void next() { if (++stage == (uint32_t)g.stages) { stage = 0; parity ^= 1u; } }
};

// A thread's share of a row: ITER vectors of VEC values, vector i at columns (i threads + t) VEC on, worked in groups of pairs: a
// vector, or (VEC = 1) two values.  Columns past the row are zeros.
template <int VEC> constexpr int kGroup = VEC > 1 ? VEC / 2 : 1;  // pairs

// Group i of a row in a slot.  Value c stands at phase + c * sizeof(T) (vectors: phase 0).
// FULL: no thread's columns lie past the row.
template <typename T, int VEC, bool FULL = false> __device__ __forceinline__ void slot_load(uint32_t slot, int phase, int C, int threads, int i, F2 (&v)[kGroup<VEC>]) {
    if constexpr (VEC > 1) {
        const int c = (i * threads + threadIdx.x) * VEC;
        uint32_t w[4] = {0u, 0u, 0u, 0u};
        const uint32_t from = slot + c * (uint32_t)sizeof(T);
        if constexpr (VEC * sizeof(T) == 16) {
            if (FULL || c < C) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(from));
        } else {
            if (FULL || c < C) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(from));
        }
#pragma unroll
        for (int j = 0; j < VEC / 2; ++j) {
            if constexpr (sizeof(T) == 2) v[j] = bf16_pair(w[j]);
            else v[j] = f2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
        }
    } else {
        float e[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t c = (2 * i + j) * threads + threadIdx.x, from = slot + phase + c * (uint32_t)sizeof(T);
            if (c < (uint32_t)C) {
                if constexpr (sizeof(T) == 2) {
                    uint16_t w;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(from));
                    e[j] = __uint_as_float((uint32_t)w << 16);
                } else {
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(e[j]) : "r"(from));
                }
            }
        }
        v[0] = f2(e[0], e[1]);
    }
}
// A thread's share of what all rows have in common, as it lies in memory.
template <typename T, int VEC, int ITER> struct Share {
    static constexpr int N = VEC * ITER;
    static_assert(N % 2 == 0 && (VEC == 1 || VEC * sizeof(T) == 8 || VEC * sizeof(T) == 16), "vectors of 8 or 16 bytes, or single values");
    typedef Pack<T, VEC> Vec;
    alignas(16) T e[N];
    __device__ __forceinline__ void load(const T *row, int C, int threads) {
#pragma unroll
        for (int i = 0; i < ITER; ++i) {
            const int c = (i * threads + threadIdx.x) * VEC;
            if constexpr (VEC > 1) {
                Vec p;
#pragma unroll
                for (int j = 0; j < VEC; ++j) p.v[j] = from_f<T>(0.f);
                if (c < C) p = *reinterpret_cast<const Vec *>(row + c);
                *reinterpret_cast<Vec *>(e + i * VEC) = p;
            } else {
                e[i] = c < C ? row[c] : from_f<T>(0.f);
            }
        }
    }
    __device__ __forceinline__ F2 pair(int k) const {  // values 2k and 2k + 1
        if constexpr (sizeof(T) == 2 && VEC > 1) return bf16_pair(reinterpret_cast<const uint32_t *>(e)[k]);
        else return f2(to_f(e[2 * k]), to_f(e[2 * k + 1]));
    }
};
// Group i to a row in memory, in the element type.
template <typename T, int VEC, bool FULL = false> __device__ __forceinline__ void group_store(T *row, int C, int threads, int i, const F2 (&v)[kGroup<VEC>]) {
    if constexpr (VEC > 1) {
        const int c = (i * threads + threadIdx.x) * VEC;
        constexpr int W = VEC * sizeof(T) / 4;
        uint32_t w[W];
#pragma unroll
        for (int j = 0; j < W; ++j) {
            if constexpr (sizeof(T) == 2) w[j] = to_bf16_pair(v[j]);
            else w[j] = __float_as_uint(j % 2 ? parts(v[j / 2]).y : parts(v[j / 2]).x);
        }
        if (FULL || c < C) {
            if constexpr (W == 4) *reinterpret_cast<uint4 *>(row + c) = make_uint4(w[0], w[1], w[2], w[3]);
            else *reinterpret_cast<uint2 *>(row + c) = make_uint2(w[0], w[1]);
        }
    } else {
        const int c = 2 * i * threads + threadIdx.x, d = c + threads;
        const float2 p = parts(v[0]);
        if (c < C) row[c] = from_f<T>(p.x);
        if (d < C) row[d] = from_f<T>(p.y);
    }
}
template <typename T, int VEC, int ITER, bool FULL = false> __device__ __forceinline__ void share_store(T *row, int C, int threads, const F2 (&v)[VEC * ITER / 2]) {
    constexpr int G = kGroup<VEC>;
#pragma unroll
    for (int i = 0; i < VEC * ITER / 2 / G; ++i) {
        F2 g[G];
#pragma unroll
        for (int j = 0; j < G; ++j) g[j] = v[i * G + j];
        group_store<T, VEC, FULL>(row, C, threads, i, g);
    }
}
// The same as fp32; the row starts on a 16-byte boundary (VEC > 1).
template <int VEC, int ITER> __device__ __forceinline__ void share_store_f32(float *row, int C, int threads, const F2 (&v)[VEC * ITER / 2]) {
#pragma unroll
    for (int i = 0; i < ITER; ++i) {
        const int c = (i * threads + threadIdx.x) * VEC;
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

// Sums (or, as bits, maxima) over the threads of `warps` warps, the block's first ones: one barrier of the block, buffers of two rounds in turn (red: six
// times 32 floats, zeros at first, on a 16-byte boundary; what is summed and what is a maximum keep to their own rows).
template <int N> __device__ __forceinline__ void ring_sum(float (&v)[N], int warps, float (*red)[32], uint32_t &round) {
    static_assert(N <= 3, "the buffers' size");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
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
    F2 s[N];
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = f2(0.f);
    for (int w = 0; w < warps; w += 4) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const float4 q = *reinterpret_cast<const float4 *>(&to[k][w]);
            s[k] = (s[k] + f2(q.x, q.y)) + f2(q.z, q.w);
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = sum2(s[k]);
}
// A sum and a maximum (of bits) in one round.
__device__ __forceinline__ void ring_sum_max(float &sum, uint32_t &top, int warps, float (*red)[32], uint32_t &round) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    sum = warp_sum(sum);
    top = __reduce_max_sync(0xffffffffu, top);
    float (*to)[32] = red + (round & 1u) * 3;
    ++round;
    if (lane == 0) { to[0][warp] = sum; to[1][warp] = __uint_as_float(top); }
    __syncthreads();
    F2 s = f2(0.f);
    for (int w = 0; w < warps; w += 4) {
        const float4 q = *reinterpret_cast<const float4 *>(&to[0][w]);
        s = (s + f2(q.x, q.y)) + f2(q.z, q.w);  // as ring_sum does
        const uint4 m = *reinterpret_cast<const uint4 *>(&to[1][w]);
        top = max(max(top, max(m.x, m.y)), max(m.z, m.w));
    }
    sum = sum2(s);
}
__device__ __forceinline__ uint32_t ring_max(uint32_t v, int warps, float (*red)[32], uint32_t &round) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
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
// Dynamic shared memory of a block, of per_sm that an SM holds: what it has (228 KB) less 1 KB of the system's and 1 KB of
// variables for each.
inline size_t ring_smem_of(int per_sm) { return (size_t)(226 * 1024 / per_sm - 2048) / 16 * 16; }
// Blocks of an SM for rows of `threads` threads, and the shared memory of each; `extra` bytes of it are not the ring's.  Two
// stages at least, else 0 blocks.
struct RingPlan { int threads, per_sm; size_t smem; int iter; };
inline RingShape ring_shape(int rows, int row_bytes, int tensors, size_t smem, unsigned polls);
// `registers` of a thread limit the blocks too.
inline RingPlan ring_plan(int C, int row_bytes, int vec, int iter, int tensors, size_t extra, int registers = 128) {
    RingPlan p{};
    const int threads = std::max(64, ring_threads((C + vec - 1) / vec, iter));
    if (threads > 512) return p;
    p.iter = iter;
    p.per_sm = std::min(8, 65536 / (registers * threads));
    while (p.per_sm > 1 && ring_shape(1, row_bytes, tensors, ring_smem_of(p.per_sm) - extra, 0).stages < 2) --p.per_sm;
    p.smem = ring_smem_of(p.per_sm);
    if (p.smem > extra && ring_shape(1, row_bytes, tensors, p.smem - extra, 0).stages >= 2) p.threads = threads;
    return p;
}
template <typename K> bool ring_ready(K kernel, int &ready_dev) {
    int dev = 0;
    cudaGetDevice(&dev);
    if (ready_dev != dev) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ring_smem_of(1)) != cudaSuccess) return false;
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
