// Products by CTA pairs (cta_group::2): two CTAs of a cluster work on one tile of 256 rows, each loads half of A and half of B.
// Wrappers of the instructions, and the ways a warp's 32 rows of results leave.
#pragma once
#include "cluster.cuh"
#include "tc_common.cuh"

namespace ddg {

namespace {

constexpr int kTile = 256;        // rows of a tile of the CTA pair, columns of an accumulator
constexpr int kHalf = 128;        // rows of A, and of B per accumulator, that one CTA of the pair loads
constexpr int kKBox = 64;         // K values of a box: 128 bytes of bf16, one swizzle row
constexpr int kOutBuf = 32 * kKBox * 2;  // an epilogue warp's 32 rows of 64 bf16 values on their way out

// Hands an accumulator back.  What it orders are the tcgen05 loads before the fence, not memory: a releasing arrival would
// wait for the stores of the tile before (gradient of the logits, 4096 x 512 x 16384: 94 us with it, 89 us without).
__device__ __forceinline__ void mbar_arrive_remote(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// one half of a stage: lands in this CTA's shared memory, counts on the barrier of the pair's first CTA
__device__ __forceinline__ void tma_load_pair(uint32_t dst, const CUtensorMap *map, uint32_t cluster_bar, int c0, int c1) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
        ::"r"(dst), "l"(map), "r"(cluster_bar), "r"(c0), "r"(c1)
        : "memory");
}
__device__ __forceinline__ void mma_pair(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// the same with 8-bit integers and 32-bit integer sums: 32 K values, which are as many bytes
__device__ __forceinline__ void mma_pair_i8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
    return ok != 0;
}
// arrives on the barrier at this offset in both CTAs when the MMAs issued so far are done
__device__ __forceinline__ void commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(bar), "h"((uint16_t)3) : "memory");
}
// Waits for work that is known to be in flight, which ends by itself: the limit is there for broken hardware alone.
__device__ __forceinline__ void mbar_drain(uint32_t bar, uint32_t parity) {
    for (unsigned i = 0; i < kSpinLimit; ++i) {
        if (mbar_try(bar, parity)) return;
        if (i > 4096) __nanosleep(64);
    }
}
constexpr uint32_t kGaveUp = 1u << 31;

__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float bf16_round(float v) { return __bfloat162float(__float2bfloat16_rn(v)); }

// 64 columns of the warp's 32 rows as bf16 to (x, y) of a matrix, through shared memory: whole 128-byte lines leave by
// TMA, and rows and columns past the matrix are clipped.  (Gradient of the logits, 4096 x 512 x 16384: 62 us; with stores
// of 64 bytes a thread, straight from registers, 89 us.)
__device__ __forceinline__ void store_box(const CUtensorMap *map, uint32_t buf, int lane, int x, int y, const float *v) {
    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");  // the box before has been read
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 8; ++j)  // the 128-byte swizzle of the map
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(buf + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(pack2(v[8 * j], v[8 * j + 1])),
                     "r"(pack2(v[8 * j + 2], v[8 * j + 3])), "r"(pack2(v[8 * j + 4], v[8 * j + 5])), "r"(pack2(v[8 * j + 6], v[8 * j + 7]))
                     : "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) {
        asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(buf), "r"(x), "r"(y) : "memory");
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
    }
}

// The same as fp32: 32 columns to a box of 128-byte lines, twice.
__device__ __forceinline__ void store_box_f32(const CUtensorMap *map, uint32_t buf, int lane, int x, int y, const float *v) {
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float *f = v + 32 * half + 4 * j;
            asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(buf + lane * 128 + ((j ^ (lane & 7)) << 4)), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]) : "memory");
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) {
            asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(map), "r"(buf), "r"(x + 32 * half), "r"(y) : "memory");
            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
        }
    }
}

// The same for matrices that a tensor map cannot write (rows off 16-byte boundaries, fp32): rows row0 .. of a [rows][n]
// matrix, columns col .. col + 63 as far as there are; the lanes write neighbouring values of a row.  (7244 x 3955 x 223,
// forward and backward: 230 us; with a row per lane, two bytes at a time, here and in the copies, 499 us.)
template <bool BF16>
__device__ __forceinline__ void store_rows(void *out, uint32_t buf, int lane, int row0, int rows, int col, int n, const float *v) {
    const int last = min(32, rows - row0);
#pragma unroll
    for (int half = 0; half < (BF16 ? 1 : 2); ++half) {  // 128 bytes of a row at a time
        __syncwarp();  // what stood there has been read
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float *f = v + (BF16 ? 8 * j : 32 * half + 4 * j);
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(buf + lane * 128 + ((j ^ (lane & 7)) << 4)), "r"(BF16 ? pack2(f[0], f[1]) : __float_as_uint(f[0])),
                         "r"(BF16 ? pack2(f[2], f[3]) : __float_as_uint(f[1])), "r"(BF16 ? pack2(f[BF16 ? 4 : 0], f[BF16 ? 5 : 0]) : __float_as_uint(f[2])),
                         "r"(BF16 ? pack2(f[BF16 ? 6 : 0], f[BF16 ? 7 : 0]) : __float_as_uint(f[3])) : "memory");
        }
        __syncwarp();
        const int c = col + 32 * half + lane;
#pragma unroll 8
        for (int r = 0; r < last; ++r) {
            const size_t at = (size_t)(row0 + r) * n + c;
            if (BF16) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {  // columns lane and lane + 32
                    const int e = lane + 32 * k;
                    uint16_t w;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(w) : "r"(buf + r * 128 + (((e >> 3) ^ (r & 7)) << 4) + (e & 7) * 2));
                    if (c + 32 * k < n) reinterpret_cast<uint16_t *>(out)[at + 32 * k] = w;
                }
            } else {
                float w;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(w) : "r"(buf + r * 128 + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4));
                if (c < n) reinterpret_cast<float *>(out)[at] = w;
            }
        }
    }
}

// ---- host side ---------------------------------------------------------------------------------------------------
// A row-major matrix of `type` in boxes of 128 bytes by box_rows; ld: elements from a row to the next.
inline bool box_map(CUtensorMapDataType type, int elem_bytes, const void *ptr, int rows, int cols, size_t ld, int box_rows, CUtensorMap *out) {
    PFN_cuTensorMapEncodeTiled_v12000 enc = tc_encode_fn();
    if (!enc) return false;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)ld * elem_bytes};
    cuuint32_t box[2] = {(cuuint32_t)(128 / elem_bytes), (cuuint32_t)box_rows};
    cuuint32_t estr[2] = {1, 1};
    return enc(out, type, 2, const_cast<void *>(ptr), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

}  // namespace ddg
