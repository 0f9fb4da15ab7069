// Cross attention: what the forward and backward kernels share.
//
// Query heads that share a key head are rows of one problem: row r of (image, key head) is query token r / group, head
// r % group of the head's group.  So keys and values are read once for all heads of a group, and one query token of many heads
// (a step of generation) fills a tile of rows as many tokens of one head do.
#pragma once

#include "bra_internal.h"
#include "fast_div.h"
#include "mma_common.cuh"
#include "sm100_ptx.cuh"

namespace bra {

constexpr int CROSS_COUNTERS = 2048;                // parts of split sums that are done, one counter per output tile
static_assert(kSMs <= CROSS_COUNTERS, "walks are split where output tiles are fewer than SMs");
constexpr int CROSS_MASKED_KEYS = 1 << 19;          // most keys of an image with a key mask: their bits are held in shared memory

struct CrossDims {
    int B, Nq, Nk, heads, kv, group, D;
    int rows;                                       // Nq * group
    int esize;
    long long q_stride, k_stride, v_stride, o_stride;
    float scale;
};

struct CrossArgs {
    const void *Q, *K, *V, *O, *dO;
    void *Oo, *dQ, *dK, *dV;
    float* lse;
    const int32_t* key_len;
    const uint8_t* key_mask;
    float2* stats;                                  // of the rows: log2 of the softmax denominator, delta (layout: the kernels' own)
    float* part;                                    // fp32 sums of split work
    int32_t* done;
    int32_t* status;                                // error words (bra_device_status)
    int Nq, Nk, heads, kv, group, rows;
    long long q_stride, k_stride, v_stride, o_stride;
    float scale, scale_log2, scale_log2_lo;         // scale; scale log2 e, and what its rounding left
    int tiles, splits, split_len;                   // output tiles of a pair; parts of the summed axis and their length
    FastDiv tiles_div, splits_div, kv_div, group_div;
};

// Scratch: error words, counters, rows' statistics, partial sums.
struct CrossWs { size_t status, done, stats, part, total; };
CrossWs cross_ws(const CrossDims& d);

// How an axis that is summed over is cut where there are too few output tiles for the GPU.
struct CrossSplit { int tiles, splits, len; };
CrossSplit cross_split(long long pairs, long long rows, int tile_rows, int summed, int step, int per_sm);

CrossArgs cross_args(const CrossDims& d, char* ws);
inline void cross_cut(CrossArgs& a, const CrossSplit& s) {
    a.tiles = s.tiles; a.splits = s.splits; a.split_len = s.len;
    a.tiles_div = fast_div(s.tiles); a.splits_div = fast_div(s.splits);
}

// Launchers (bf16: _mma and _tc; fp32: _tf32).  part_floats: what the scratch of their split sums holds.
cudaError_t launch_cross_attend_mma(const CrossDims& d, CrossArgs a, cudaStream_t st);
bool cross_attend_tc_pays(const CrossDims& d);
cudaError_t launch_cross_attend_tc(const CrossDims& d, CrossArgs a, cudaStream_t st);
cudaError_t launch_cross_backward_mma(const CrossDims& d, CrossArgs a, cudaStream_t st);
bool cross_backward_tc_pays(const CrossDims& d);
size_t cross_backward_tc_stats(const CrossDims& d);         // bytes of its rows' statistics
size_t cross_backward_tc_part(const CrossDims& d);
size_t cross_attend_tc_part(const CrossDims& d);
cudaError_t launch_cross_backward_tc(const CrossDims& d, CrossArgs a, cudaStream_t st);
cudaError_t launch_cross_attend_tf32(const CrossDims& d, CrossArgs a, cudaStream_t st);
cudaError_t launch_cross_backward_tf32(const CrossDims& d, CrossArgs a, cudaStream_t st);
size_t cross_attend_mma_part(const CrossDims& d);
size_t cross_backward_mma_part(const CrossDims& d);
size_t cross_attend_tf32_part(const CrossDims& d);
size_t cross_backward_tf32_part(const CrossDims& d);

#ifdef __CUDACC__
// This CTA's place: blockIdx.x = (pair * splits + split) * tiles + tile
struct CrossPlace {
    int tile, split, b, kvh;
    long long pair;
    __device__ __forceinline__ explicit CrossPlace(const CrossArgs& a) {
        const uint32_t i = blockIdx.x;
        const uint32_t ps = fdiv(i, a.tiles_div);
        tile = (int)(i - ps * a.tiles);
        const uint32_t p = fdiv(ps, a.splits_div);
        split = (int)(ps - p * a.splits);
        pair = p;
        b = (int)fdiv(p, a.kv_div);
        kvh = (int)(p - (uint32_t)b * a.kv);
    }
};

// Row r of a pair in tensors laid out like Q (token stride given), and in lse / delta.
__device__ __forceinline__ long long cross_row(const CrossArgs& a, const CrossPlace& at, int r, long long stride, int D) {
    const int token = (int)fdiv((uint32_t)r, a.group_div), g = r - token * a.group;
    return ((long long)at.b * a.Nq + token) * stride + (long long)(at.kvh * a.group + g) * D;
}
__device__ __forceinline__ long long cross_stat(const CrossArgs& a, const CrossPlace& at, int r) {
    const int token = (int)fdiv((uint32_t)r, a.group_div), g = r - token * a.group;
    return ((long long)at.b * a.heads + at.kvh * a.group + g) * a.Nq + token;
}

// The keys lo .. hi - 1 of an image, of which `bits` (shared memory; null: all) says which are seen.
struct KeyRange {
    int lo, hi;
    const uint32_t* bits;
    // of the 32 keys from lo + 32 t on
    __device__ __forceinline__ uint32_t word(int t) const {
        const int n = hi - lo - 32 * t;
        uint32_t w = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
        if (bits && w) w &= bits[t];
        return w;
    }
};
__device__ __forceinline__ int cross_key_end(const CrossArgs& a, int b) {
    return a.key_len ? min(max(__ldg(a.key_len + b), 0), a.Nk) : a.Nk;
}
// Keys [lo, end) of image b cut to those that exist; the mask's bits go to `words` (call by all threads; a barrier has to follow
// before they are read).
__device__ __forceinline__ KeyRange cross_keys(const CrossArgs& a, int b, int lo, int end, uint32_t* words) {
    KeyRange r;
    r.lo = lo;
    r.hi = max(lo, min(end, cross_key_end(a, b)));
    r.bits = nullptr;
    if (a.key_mask) {
        const uint8_t* m = a.key_mask + (long long)b * a.Nk;
        const int lane = threadIdx.x & 31;
        for (int t = threadIdx.x >> 5; 32 * t < r.hi - lo; t += blockDim.x >> 5) {
            const int j = lo + 32 * t + lane;
            const uint32_t w = __ballot_sync(0xffffffffu, j < r.hi && m[j] != 0);
            if (lane == 0) words[t] = w;
        }
        r.bits = words;
    }
    return r;
}

// True in all threads of the CTA that is the last of `parts` to come by counter i, whose count it puts back to zero.  What the
// others wrote before is visible then.
__device__ __forceinline__ bool cross_last(int32_t* counter, int parts, int* flag) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        const int before = atomicAdd(counter, 1);
        *flag = before == parts - 1;
        if (before == parts - 1) *counter = 0;
    }
    __syncthreads();
    __threadfence();
    return *flag != 0;
}

// The parts of split rows: `rows` rows of D sums, then the reference maximum (raw score) and the sum of a row, `pitch` floats apart, a
// part `part` floats behind the one before.  Adds them in order and writes the rows.  weight: shared memory, rows x splits floats and
// rows more.  done(row, value index / 4, values) stores four channels, lse(row, log2 of the sum, whether there is one).
template <int D, typename Done, typename Lse>
__device__ __forceinline__ void cross_join(const float* parts, long long part, int pitch, int rows, int splits, float c, float* weight, Done&& done, Lse&& lse) {
    float* inv = weight + rows * splits;
    for (int r = threadIdx.x; r < rows; r += blockDim.x) {
        const float* row = parts + r * pitch + D;
        float top = -INFINITY, sum = 0.f;
        for (int s = 0; s < splits; ++s) {
            const float2 v = __ldcg(reinterpret_cast<const float2*>(row + s * part));
            weight[r * splits + s] = v.x;
            top = fmaxf(top, v.x);
        }
        const float ref = top == -INFINITY ? 0.f : top * c;
        for (int s = 0; s < splits; ++s) {
            const float f = exp2f(fmaf(weight[r * splits + s], c, -ref));
            weight[r * splits + s] = f;
            sum = fmaf(f, __ldcg(row + s * part + 1), sum);
        }
        inv[r] = sum == 0.f ? 0.f : 1.f / sum;
        lse(r, ref, sum);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * (D / 4); i += blockDim.x) {
        const int r = i / (D / 4), ch = i % (D / 4);
        const float* at = parts + r * pitch + 4 * ch;
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int s = 0; s < splits; ++s) {
            const float4 v = __ldcg(reinterpret_cast<const float4*>(at + s * part));
            const float f = weight[r * splits + s];
            t.x = fmaf(f, v.x, t.x); t.y = fmaf(f, v.y, t.y); t.z = fmaf(f, v.z, t.z); t.w = fmaf(f, v.w, t.w);
        }
        const float k = inv[r];
        done(r, ch, make_float4(t.x * k, t.y * k, t.z * k, t.w * k));
    }
}

// ---------------------------------------------------------------- rows of D bf16 channels in shared memory
// Chunks of 16 bytes, exclusive-or'ed with the row so that the eight rows of an ldmatrix matrix lie in different banks.
template <int D>
__device__ __forceinline__ uint32_t chunk_at(int row, int chunk) {
    constexpr int CH = D / 8;                       // chunks of a row
    const int x = CH >= 8 ? (row & 7) : CH == 4 ? ((row >> 1) & 3) : ((row >> 2) & 1);
    return (uint32_t)(row * (D * 2) + ((chunk ^ x) << 4));
}
// A fragment (16 rows from row0, channels 16 k ...) of rows in shared memory
template <int D>
__device__ __forceinline__ void a_frag(uint32_t base, int row0, int k, int lane, uint32_t* r) {
    ldmatrix_x4(base + chunk_at<D>(row0 + (lane & 15), 2 * k + (lane >> 4)), r);
}
// B fragments for a contraction over channels: rows n0 .. n0+15 as columns; r[0], r[1]: n0..n0+7, r[2], r[3]: the next eight
template <int D>
__device__ __forceinline__ void b_frag(uint32_t base, int n0, int k, int lane, uint32_t* r) {
    ldmatrix_x4(base + chunk_at<D>(n0 + (lane & 7) + ((lane >> 4) << 3), 2 * k + ((lane >> 3) & 1)), r);
}
// B fragments for a contraction over rows k0 .. k0+15, channels 16 c ...: r[0], r[1]: first eight channels, r[2], r[3]: the next
template <int D>
__device__ __forceinline__ void bt_frag(uint32_t base, int k0, int c, int lane, uint32_t* r) {
    ldmatrix_x4_trans(base + chunk_at<D>(k0 + (lane & 15), 2 * c + (lane >> 4)), r);
}

// The lanes of a quad hold, for four blocks of eight channels, a pair of channels each; afterwards lane t4 has all of block t4.
__device__ __forceinline__ uint4 quad_chunk(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, int t4) {
    uint32_t w[4] = {w0, w1, w2, w3};
    const bool b0 = t4 & 1, b1 = t4 & 2;
    uint32_t s0 = b0 ? w[0] : w[1], s1 = b0 ? w[2] : w[3];
    s0 = __shfl_xor_sync(0xffffffffu, s0, 1);
    s1 = __shfl_xor_sync(0xffffffffu, s1, 1);
    if (b0) { w[0] = s0; w[2] = s1; } else { w[1] = s0; w[3] = s1; }
    s0 = b1 ? w[0] : w[2]; s1 = b1 ? w[1] : w[3];
    s0 = __shfl_xor_sync(0xffffffffu, s0, 2);
    s1 = __shfl_xor_sync(0xffffffffu, s1, 2);
    if (b1) { w[0] = s0; w[1] = s1; } else { w[2] = s0; w[3] = s1; }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// Rows g4 and g4 + 8 of a 16 x D accumulator tile, times f0 and f1, as bf16 to row pointers p0, p1 (null: not stored).
template <int D>
__device__ __forceinline__ void store_tile_rows(const float (&acc)[D / 8][4], float f0, float f1, __nv_bfloat16* p0, __nv_bfloat16* p1, int t4) {
    if constexpr (D >= 32) {
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            uint32_t w[2][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[0][i] = pack2_bf16(acc[4 * c + i][0] * f0, acc[4 * c + i][1] * f0);
                w[1][i] = pack2_bf16(acc[4 * c + i][2] * f1, acc[4 * c + i][3] * f1);
            }
            const uint4 v0 = quad_chunk(w[0][0], w[0][1], w[0][2], w[0][3], t4), v1 = quad_chunk(w[1][0], w[1][1], w[1][2], w[1][3], t4);
            if (p0) *reinterpret_cast<uint4*>(p0 + 32 * c + 8 * t4) = v0;
            if (p1) *reinterpret_cast<uint4*>(p1 + 32 * c + 8 * t4) = v1;
        }
    } else {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            if (p0) *reinterpret_cast<uint32_t*>(p0 + 8 * i + 2 * t4) = pack2_bf16(acc[i][0] * f0, acc[i][1] * f0);
            if (p1) *reinterpret_cast<uint32_t*>(p1 + 8 * i + 2 * t4) = pack2_bf16(acc[i][2] * f1, acc[i][3] * f1);
        }
    }
}
#endif  // __CUDACC__

}  // namespace bra
