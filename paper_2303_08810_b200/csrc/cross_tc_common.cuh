// Cross attention on the 5th-generation tensor cores: what the forward and backward kernels share.
#pragma once

#include "cross_common.cuh"
#include "tma_map.h"

namespace bra {
namespace cross_tc {

using namespace ptx;

constexpr uint32_t POLL_LIMIT = 4000000u;

// Which of the 128 keys from key0 on are seen, 32 a word, the same in all lanes of a warp.
struct Seen { uint32_t w[4]; };
__device__ __forceinline__ uint32_t below(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }
// the mask's bytes of a lane (one of each word), read a block ahead of their use
__device__ __forceinline__ uint32_t mask_bytes(const uint8_t* mask, int key0, int end, int lane) {
    uint32_t v = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int j = key0 + 32 * w + lane;
        if (j < end && __ldg(mask + j)) v |= 1u << w;
    }
    return v;
}
__device__ __forceinline__ Seen seen_of(const uint8_t* mask, uint32_t bytes, int key0, int end) {
    Seen s;
#pragma unroll
    for (int w = 0; w < 4; ++w) s.w[w] = mask ? __ballot_sync(0xffffffffu, (bytes >> w) & 1) : below(end - key0 - 32 * w);
    return s;
}

// one attempt first: the loop around further ones costs a hundred cycles even where it is not needed
__device__ __forceinline__ void wait_for(uint64_t* bar, uint32_t parity, bool& ok) {
    if (!mbar_try_wait(bar, parity)) ok = mbar_wait(bar, parity, POLL_LIMIT) && ok;
}

// 32 channels (as 16 pairs) of a warp's 32 rows, thread = row, to global memory by way of 2 KB of shared memory: four lanes a row, so that
// a store instruction writes eight rows of 64 bytes instead of 32 of 16 (forward of 16 x 1024 x 1024, 12 heads of 64: 98 -> 95 us; the gradients'
// kernels have no registers left for it: 504 -> 529 us at 2 x 4096 x 4096, 16 heads of 64).
// to: the row's first channel; null: not stored.
constexpr int ROWS32 = 2048;
struct RowPointers { __nv_bfloat16* at[4]; };
__device__ __forceinline__ RowPointers rows_of_warp(__nv_bfloat16* mine, int lane) {
    RowPointers p;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        p.at[k] = reinterpret_cast<__nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), 8 * k + (lane >> 2)));
    return p;
}
__device__ __forceinline__ void store_rows32(uint32_t stage, const uint32_t (&v)[16], const RowPointers& to, int channel, int lane) {
    __syncwarp();
#pragma unroll
    for (int c = 0; c < 4; ++c)
        sts_f32x4(stage + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4), __uint_as_float(v[4 * c]), __uint_as_float(v[4 * c + 1]),
                  __uint_as_float(v[4 * c + 2]), __uint_as_float(v[4 * c + 3]));
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = 8 * k + (lane >> 2), c = lane & 3;
        const float4 t = lds_f32x4(stage + r * 64 + ((c ^ ((r >> 1) & 3)) << 4));
        if (to.at[k]) *reinterpret_cast<float4*>(to.at[k] + channel + 8 * c) = t;
    }
}

// Work for fewer CTAs than SMs: every walk of `blocks` blocks is cut in parts, as many as make one part an SM at most.  Joining the parts
// costs about what three blocks do (8 pairs of tiles, 8 heads of 32, forward, whole / cut, us: 2 blocks 7.7 / 9.5, 4 blocks 11.0 / 10.4,
// 8 blocks 17.4 / 11.1).
struct TcSplit { int splits, part; };
inline TcSplit tc_split(long long tiles, int blocks) {
    long long splits = tiles > 0 ? kSMs / tiles : 1;
    if (splits > blocks) splits = blocks;
    if (splits < 1) splits = 1;
    TcSplit s;
    s.part = (int)((blocks + splits - 1) / splits);
    if (blocks - s.part < 3) s.part = blocks;
    s.splits = (blocks + s.part - 1) / s.part;
    return s;
}

// [B, tokens, heads, D] with `stride` elements from token to token; box: BOX channels x heads x tokens of one image
inline bool rows_map(CUtensorMap* m, const void* base, int D, int heads, long long tokens, int B, long long stride, int box_ch, int box_heads, int box_tokens) {
    EncodeTiledFn enc = tma_encoder();
    if (!enc) return false;
    const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)tokens, (cuuint64_t)B};
    const cuuint64_t strides[3] = {(cuuint64_t)D * 2, (cuuint64_t)stride * 2, (cuuint64_t)(stride * tokens) * 2};
    const cuuint32_t box[4] = {(cuuint32_t)box_ch, (cuuint32_t)box_heads, (cuuint32_t)box_tokens, 1};
    const cuuint32_t es[4] = {1, 1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
               box_ch == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace cross_tc
}  // namespace bra
