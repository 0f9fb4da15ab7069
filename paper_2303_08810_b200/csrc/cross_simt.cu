// Cross attention and its gradients in fp32 on CUDA cores (tensor cores round their operands).  The same walks as the tensor-core
// kernels: one pass over the keys with the running maximum and sum of the softmax; for the gradients one kernel that keeps query
// rows and walks the keys (dQ), one that keeps keys and walks the query rows (dK, dV).
//
// A CTA of 128 threads: 16 groups of rows x 8 groups of columns.  A thread holds the scores of RI rows x BN / 8 walked rows and
// then the sums of RI rows x D / 8 channels, both from 16-byte shared-memory loads whose rows are four floats longer than they
// need to be, so that the eight walked rows of a warp lie in different banks.  Bound by the FMA pipe and shared-memory loads.
#include "cross_common.cuh"

#include <math.h>

namespace bra {
namespace {

constexpr int THREADS = 128;

template <int D, int BN_, int RI>
struct Shape {
    static constexpr int BN = BN_, BM = 16 * RI, LD = D + 4, LP = BN + 4;
    static constexpr int VW = D >= 32 ? 4 : D / 8;          // neighbouring channels of a thread
    static constexpr int NJ = D / (8 * VW);
    static constexpr int COLS = BN / 8;
};

// `rows` rows of D floats into shared memory, rows that `where` does not place as zeros
template <int D, int LD, typename F>
__device__ __forceinline__ void load_rows(float* to, int rows, F&& where) {
    for (int u = threadIdx.x; u < rows * (D / 4); u += THREADS) {
        const int row = u / (D / 4), ch = u % (D / 4) * 4;
        const float* p = where(row);
        *reinterpret_cast<float4*>(to + row * LD + ch) = p ? __ldg(reinterpret_cast<const float4*>(p + ch)) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
}

// s[i][j] = x[row i] . y[column j]
template <typename S, int D, int RI>
__device__ __forceinline__ void dots(float (&s)[RI][S::COLS], const float* x, const float* y, int ty, int tx) {
#pragma unroll
    for (int i = 0; i < RI; ++i)
#pragma unroll
        for (int j = 0; j < S::COLS; ++j) s[i][j] = 0.f;
#pragma unroll 2
    for (int k = 0; k < D; k += 4) {
        float4 xv[RI];
#pragma unroll
        for (int i = 0; i < RI; ++i) xv[i] = *reinterpret_cast<const float4*>(x + (ty * RI + i) * S::LD + k);
#pragma unroll
        for (int j = 0; j < S::COLS; ++j) {
            const float4 yv = *reinterpret_cast<const float4*>(y + (tx + 8 * j) * S::LD + k);
#pragma unroll
            for (int i = 0; i < RI; ++i) {
                s[i][j] = fmaf(xv[i].x, yv.x, s[i][j]);
                s[i][j] = fmaf(xv[i].y, yv.y, s[i][j]);
                s[i][j] = fmaf(xv[i].z, yv.z, s[i][j]);
                s[i][j] = fmaf(xv[i].w, yv.w, s[i][j]);
            }
        }
    }
}
// acc[i][channels of the thread] += sum over the walked rows of p[row i][n] y[n]
template <typename S, int D, int RI>
__device__ __forceinline__ void weigh(float (&acc)[RI][D / 8], const float* p, const float* y, int ty, int tx) {
#pragma unroll 2
    for (int n = 0; n < S::BN; n += 4) {
        float4 pv[RI];
#pragma unroll
        for (int i = 0; i < RI; ++i) pv[i] = *reinterpret_cast<const float4*>(p + (ty * RI + i) * S::LP + n);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float* row = y + (n + e) * S::LD + tx * S::VW;
#pragma unroll
            for (int j = 0; j < S::NJ; ++j) {
                float v[S::VW];
                if constexpr (S::VW == 4) {
                    const float4 t = *reinterpret_cast<const float4*>(row + 32 * j);
                    v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
                } else {
                    const float2 t = *reinterpret_cast<const float2*>(row);
                    v[0] = t.x; v[1] = t.y;
                }
#pragma unroll
                for (int i = 0; i < RI; ++i) {
                    const float w = e == 0 ? pv[i].x : e == 1 ? pv[i].y : e == 2 ? pv[i].z : pv[i].w;
#pragma unroll
                    for (int q = 0; q < S::VW; ++q) acc[i][j * S::VW + q] = fmaf(w, v[q], acc[i][j * S::VW + q]);
                }
            }
        }
    }
}
template <typename S, int RI>
__device__ __forceinline__ void keep_cols(float* p, const float (&s)[RI][S::COLS], int ty, int tx) {
#pragma unroll
    for (int i = 0; i < RI; ++i)
#pragma unroll
        for (int j = 0; j < S::COLS; ++j) p[(ty * RI + i) * S::LP + tx + 8 * j] = s[i][j];
}
template <typename S, int D>
__device__ __forceinline__ void put_row(float* to, const float* acc, float f, int tx) {
#pragma unroll
    for (int j = 0; j < S::NJ; ++j)
#pragma unroll
        for (int q = 0; q < S::VW; ++q) to[j * 8 * S::VW + tx * S::VW + q] = acc[j * S::VW + q] * f;
}
__device__ __forceinline__ float max8(float v) {
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float sum8(float v) {
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// ---------------------------------------------------------------- forward
template <int D, int RI>
__global__ void __launch_bounds__(THREADS) cross_attend_simt_kernel(const CrossArgs a) {
    using S = Shape<D, D == 128 ? 32 : 64, RI>;
    constexpr int BN = S::BN, BM = S::BM;
    extern __shared__ __align__(16) float sh[];
    __shared__ int flag;
    float *xq = sh, *yk = xq + BM * S::LD, *yv = yk + BN * S::LD, *ps = yv + BN * S::LD;
    const CrossPlace at(a);
    const int ty = threadIdx.x >> 3, tx = threadIdx.x & 7;
    const KeyRange keys = cross_keys(a, at.b, at.split * a.split_len, min(a.Nk, (at.split + 1) * a.split_len),
                                     reinterpret_cast<uint32_t*>(ps + BM * S::LP));
    const float* Q = static_cast<const float*>(a.Q);
    const float* K = static_cast<const float*>(a.K) + (long long)at.b * a.Nk * a.k_stride + (long long)at.kvh * D;
    const float* V = static_cast<const float*>(a.V) + (long long)at.b * a.Nk * a.v_stride + (long long)at.kvh * D;
    load_rows<D, S::LD>(xq, BM, [&](int row) {
        const int r = at.tile * BM + row;
        return r < a.rows ? Q + cross_row(a, at, r, a.q_stride, D) : nullptr;
    });
    float o[RI][D / 8] = {}, m[RI], l[RI];
#pragma unroll
    for (int i = 0; i < RI; ++i) { m[i] = -INFINITY; l[i] = 0.f; }
    const float c = a.scale_log2;
    const int tiles = (keys.hi - keys.lo + BN - 1) / BN;
    for (int tile = 0; tile < tiles; ++tile) {
        __syncthreads();
        uint32_t seen[BN / 32];
#pragma unroll
        for (int w = 0; w < BN / 32; ++w) seen[w] = keys.word(tile * (BN / 32) + w);
        auto has = [&](int row) { return (seen[BN == 32 ? 0 : row >> 5] >> (row & 31)) & 1; };
        load_rows<D, S::LD>(yk, BN, [&](int row) { return has(row) ? K + (keys.lo + tile * BN + row) * a.k_stride : nullptr; });
        load_rows<D, S::LD>(yv, BN, [&](int row) { return has(row) ? V + (keys.lo + tile * BN + row) * a.v_stride : nullptr; });
        __syncthreads();
        float s[RI][S::COLS];
        dots<S, D, RI>(s, xq, yk, ty, tx);
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            float top = m[i];
#pragma unroll
            for (int j = 0; j < S::COLS; ++j) {
                if (!has(tx + 8 * j)) s[i][j] = -INFINITY;
                top = fmaxf(top, s[i][j]);
            }
            top = max8(top);
            const float ref = top == -INFINITY ? 0.f : top * c;
            const float keep = exp2f(fmaf(m[i], c, -ref));
            m[i] = top;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < S::COLS; ++j) {
                s[i][j] = exp2f(fmaf(s[i][j], c, -ref));
                sum += s[i][j];
            }
            l[i] = l[i] * keep + sum;
#pragma unroll
            for (int j = 0; j < D / 8; ++j) o[i][j] *= keep;
        }
        keep_cols<S, RI>(ps, s, ty, tx);
        __syncwarp();                                       // a row's scores are all of one warp
        weigh<S, D, RI>(o, ps, yv, ty, tx);
    }
#pragma unroll
    for (int i = 0; i < RI; ++i) {
        l[i] = sum8(l[i]);
        const int r = at.tile * BM + ty * RI + i;
        if (r >= a.rows) continue;
        if (a.splits == 1) {
            put_row<S, D>(static_cast<float*>(a.Oo) + cross_row(a, at, r, a.o_stride, D), o[i], l[i] == 0.f ? 0.f : 1.f / l[i], tx);
            if (a.lse && tx == 0)
                a.lse[cross_stat(a, at, r)] = l[i] == 0.f ? -INFINITY : (m[i] * c + log2f(l[i])) * 0.69314718055994531f;
        } else {
            float* part = a.part + ((at.pair * a.tiles + at.tile) * a.splits + at.split) * (long long)(BM * S::LD) + (ty * RI + i) * S::LD;
            put_row<S, D>(part, o[i], 1.f, tx);
            if (tx == 0) { part[D] = m[i]; part[D + 1] = l[i]; }
        }
    }
    if (a.splits == 1 || !cross_last(a.done + at.pair * a.tiles + at.tile, a.splits, &flag)) return;
    const long long one = BM * S::LD;
    cross_join<D>(a.part + (at.pair * a.tiles + at.tile) * a.splits * one, one, S::LD, min(BM, a.rows - at.tile * BM), a.splits, c, sh,
                  [&](int row, int ch, float4 v) {
                      *reinterpret_cast<float4*>(static_cast<float*>(a.Oo) + cross_row(a, at, at.tile * BM + row, a.o_stride, D) + 4 * ch) = v;
                  },
                  [&](int row, float ref, float sum) {
                      if (a.lse) a.lse[cross_stat(a, at, at.tile * BM + row)] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
                  });
}

// ---------------------------------------------------------------- gradients
template <int D, bool DKV>
__global__ void __launch_bounds__(THREADS) cross_grad_simt_kernel(const CrossArgs a) {
    constexpr int RI = 4;
    using S = Shape<D, D >= 64 ? 32 : 64, RI>;
    constexpr int BN = S::BN, BM = S::BM;
    extern __shared__ __align__(16) float sh[];
    __shared__ int flag;
    float *x1 = sh, *x2 = x1 + BM * S::LD, *y1 = x2 + BM * S::LD, *y2 = y1 + BN * S::LD, *ps = y2 + BN * S::LD, *ds = ps + BM * S::LP;
    const CrossPlace at(a);
    const int ty = threadIdx.x >> 3, tx = threadIdx.x & 7;
    const int key_lo = DKV ? at.tile * BM : at.split * a.split_len;
    const KeyRange keys = cross_keys(a, at.b, key_lo, min(a.Nk, DKV ? key_lo + BM : key_lo + a.split_len),
                                     reinterpret_cast<uint32_t*>(ds + BM * S::LP));
    __syncthreads();
    const int walk_lo = DKV ? at.split * a.split_len : keys.lo;
    const int walk_hi = DKV ? min(a.rows, walk_lo + a.split_len) : keys.hi;
    const float *Q = static_cast<const float*>(a.Q), *dO = static_cast<const float*>(a.dO);
    const float* K = static_cast<const float*>(a.K) + (long long)at.b * a.Nk * a.k_stride + (long long)at.kvh * D;
    const float* V = static_cast<const float*>(a.V) + (long long)at.b * a.Nk * a.v_stride + (long long)at.kvh * D;
    const int padded = (a.rows + 63) / 64 * 64;
    float2* stats = a.stats + at.pair * padded;
    auto sees = [&](int row) { return (keys.word(row >> 5) >> (row & 31)) & 1; };       // row: from key_lo on

    load_rows<D, S::LD>(x1, BM, [&](int row) -> const float* {
        const int r = at.tile * BM + row;
        if (DKV) return sees(row) ? K + r * a.k_stride : nullptr;
        return r < a.rows ? Q + cross_row(a, at, r, a.q_stride, D) : nullptr;
    });
    load_rows<D, S::LD>(x2, BM, [&](int row) -> const float* {
        const int r = at.tile * BM + row;
        if (DKV) return sees(row) ? V + r * a.v_stride : nullptr;
        return r < a.rows ? dO + cross_row(a, at, r, a.o_stride, D) : nullptr;
    });
    float lse2[RI], delta[RI];
    if (!DKV) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            const int row = ty * RI + i, r = at.tile * BM + row;
            lse2[i] = INFINITY;
            delta[i] = 0.f;
            if (r < a.rows) {
                const float* o = static_cast<const float*>(a.O) + cross_row(a, at, r, a.o_stride, D);
                for (int ch = tx; ch < D; ch += 8) delta[i] = fmaf(__ldg(o + ch), x2[row * S::LD + ch], delta[i]);
                const float e = __ldg(a.lse + cross_stat(a, at, r));
                lse2[i] = e == -INFINITY ? INFINITY : e * 1.4426950408889634f;
            }
            delta[i] = sum8(delta[i]);
            if (at.split == 0 && tx == 0) stats[r] = make_float2(lse2[i], r < a.rows ? delta[i] : 0.f);
        }
    }
    float acc[RI][D / 8] = {}, accv[DKV ? RI : 1][D / 8] = {};
    const float c = a.scale_log2;
    int tiles = walk_hi > walk_lo ? (walk_hi - walk_lo + BN - 1) / BN : 0;
    if (DKV && keys.hi <= keys.lo) tiles = 0;
    for (int tile = 0; tile < tiles; ++tile) {
        __syncthreads();
        load_rows<D, S::LD>(y1, BN, [&](int row) -> const float* {
            const int j = walk_lo + tile * BN + row;
            if (DKV) return j < walk_hi ? Q + cross_row(a, at, j, a.q_stride, D) : nullptr;
            return sees(tile * BN + row) ? K + j * a.k_stride : nullptr;
        });
        load_rows<D, S::LD>(y2, BN, [&](int row) -> const float* {
            const int j = walk_lo + tile * BN + row;
            if (DKV) return j < walk_hi ? dO + cross_row(a, at, j, a.o_stride, D) : nullptr;
            return sees(tile * BN + row) ? V + j * a.v_stride : nullptr;
        });
        float2 st[DKV ? S::COLS : 1];
        if (DKV) {
#pragma unroll
            for (int j = 0; j < S::COLS; ++j) st[DKV ? j : 0] = __ldcg(stats + walk_lo + tile * BN + tx + 8 * j);
        }
        __syncthreads();
        float s[RI][S::COLS], dp[RI][S::COLS];
        dots<S, D, RI>(s, x1, y1, ty, tx);
        dots<S, D, RI>(dp, x2, y2, ty, tx);
#pragma unroll
        for (int j = 0; j < S::COLS; ++j) {
            const bool seen = DKV || sees(tile * BN + tx + 8 * j);
#pragma unroll
            for (int i = 0; i < RI; ++i) {
                const float p = seen ? exp2f(fmaf(s[i][j], c, DKV ? -st[DKV ? j : 0].x : -lse2[i])) : 0.f;
                s[i][j] = p;
                dp[i][j] = p * (dp[i][j] - (DKV ? st[DKV ? j : 0].y : delta[i]));
            }
        }
        keep_cols<S, RI>(ds, dp, ty, tx);
        if (DKV) keep_cols<S, RI>(ps, s, ty, tx);
        __syncwarp();
        weigh<S, D, RI>(acc, ds, y1, ty, tx);
        if constexpr (DKV) weigh<S, D, RI>(accv, ps, y2, ty, tx);
    }
    if (a.splits > 1) {
        const long long one = (long long)(DKV ? 2 : 1) * BM * D;
        float* mine = a.part + ((at.pair * a.tiles + at.tile) * a.splits + at.split) * one;
#pragma unroll
        for (int i = 0; i < RI; ++i) {
            put_row<S, D>(mine + (ty * RI + i) * D, acc[i], 1.f, tx);
            if constexpr (DKV) put_row<S, D>(mine + (BM + ty * RI + i) * D, accv[i], 1.f, tx);
        }
        if (!cross_last(a.done + at.pair * a.tiles + at.tile, a.splits, &flag)) return;
        const float* all = a.part + (at.pair * a.tiles + at.tile) * a.splits * one;
#pragma unroll
        for (int i = 0; i < RI; ++i)
#pragma unroll
            for (int e = 0; e < D / 8; ++e) {
                const int ch = e / S::VW * 8 * S::VW + tx * S::VW + e % S::VW;
                float t = 0.f, u = 0.f;
                for (int sp = 0; sp < a.splits; ++sp) {
                    t += __ldcg(all + sp * one + (ty * RI + i) * D + ch);
                    if (DKV) u += __ldcg(all + sp * one + (BM + ty * RI + i) * D + ch);
                }
                acc[i][e] = t;
                if constexpr (DKV) accv[i][e] = u;
            }
    }
#pragma unroll
    for (int i = 0; i < RI; ++i) {
        const int row = ty * RI + i, r = at.tile * BM + row;
        if constexpr (DKV) {
            if (r >= a.Nk) continue;
            if (!sees(row)) {               // hidden: its sums are of scores it does not have
#pragma unroll
                for (int e = 0; e < D / 8; ++e) acc[i][e] = accv[i][e] = 0.f;
            }
            const long long j = (long long)at.b * a.Nk + r;
            put_row<S, D>(static_cast<float*>(a.dK) + j * a.k_stride + (long long)at.kvh * D, acc[i], a.scale, tx);
            put_row<S, D>(static_cast<float*>(a.dV) + j * a.v_stride + (long long)at.kvh * D, accv[i], 1.f, tx);
        } else {
            if (r >= a.rows) continue;
            put_row<S, D>(static_cast<float*>(a.dQ) + cross_row(a, at, r, a.q_stride, D), acc[i], a.scale, tx);
        }
    }
}

// ---------------------------------------------------------------- host
bool few_rows(const CrossDims& d) { return d.rows <= 16; }

CrossSplit forward_split(const CrossDims& d) {
    return cross_split((long long)d.B * d.kv, d.rows, few_rows(d) ? 16 : 64, d.Nk, d.D == 128 ? 32 : 64, 2);
}
CrossSplit grad_split(const CrossDims& d, bool dkv) {
    return cross_split((long long)d.B * d.kv, dkv ? d.Nk : d.rows, 64, dkv ? d.rows : d.Nk, d.D >= 64 ? 32 : 64, 2);
}

template <typename Kernel>
cudaError_t launch(Kernel kernel, PerDeviceMax& attr, const CrossArgs& a, long long pairs, size_t smem, cudaStream_t st) {
    const cudaError_t e = attr.ensure((int)smem, [&] {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    });
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)(pairs * a.splits * a.tiles), THREADS, smem, st>>>(a);
    count_launch();
    return cudaGetLastError();
}
size_t mask_bytes(const CrossArgs& a, int keys) { return a.key_mask ? ((size_t)keys + 31) / 32 * 4 : 0; }

template <int D, int RI>
cudaError_t forward(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    using S = Shape<D, D == 128 ? 32 : 64, RI>;
    static PerDeviceMax attr;
    cross_cut(a, forward_split(d));
    size_t smem = sizeof(float) * (S::BM * S::LD + 2 * S::BN * S::LD + S::BM * S::LP) + mask_bytes(a, a.split_len);
    const size_t join = a.splits > 1 ? sizeof(float) * S::BM * (a.splits + 1) : 0;
    smem = smem > join ? smem : join;
    return launch(cross_attend_simt_kernel<D, RI>, attr, a, (long long)d.B * d.kv, smem, st);
}
template <int D, bool DKV>
cudaError_t grad(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    using S = Shape<D, D >= 64 ? 32 : 64, 4>;
    static PerDeviceMax attr;
    cross_cut(a, grad_split(d, DKV));
    const size_t smem = sizeof(float) * (2 * S::BM * S::LD + 2 * S::BN * S::LD + 2 * S::BM * S::LP) + mask_bytes(a, DKV ? S::BM : a.split_len);
    return launch(cross_grad_simt_kernel<D, DKV>, attr, a, (long long)d.B * d.kv, smem, st);
}
template <int D>
cudaError_t both(const CrossDims& d, const CrossArgs& a, cudaStream_t st) {
    const cudaError_t e = grad<D, false>(d, a, st);
    return e != cudaSuccess ? e : grad<D, true>(d, a, st);
}

}  // namespace

size_t cross_attend_simt_part(const CrossDims& d) {
    const CrossSplit s = forward_split(d);
    return s.splits > 1 ? (size_t)s.splits * s.tiles * d.B * d.kv * (few_rows(d) ? 16 : 64) * (d.D + 4) : 0;
}
size_t cross_backward_simt_part(const CrossDims& d) {
    size_t most = 0;
    for (int dkv = 0; dkv < 2; ++dkv) {
        const CrossSplit s = grad_split(d, dkv);
        const size_t n = s.splits > 1 ? (size_t)s.splits * s.tiles * d.B * d.kv * (1 + dkv) * 64 * d.D : 0;
        most = n > most ? n : most;
    }
    return most;
}

cudaError_t launch_cross_attend_simt(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    const bool few = few_rows(d);
    switch (d.D) {
        case 16: return few ? forward<16, 1>(d, a, st) : forward<16, 4>(d, a, st);
        case 32: return few ? forward<32, 1>(d, a, st) : forward<32, 4>(d, a, st);
        case 64: return few ? forward<64, 1>(d, a, st) : forward<64, 4>(d, a, st);
        default: return few ? forward<128, 1>(d, a, st) : forward<128, 4>(d, a, st);
    }
}
cudaError_t launch_cross_backward_simt(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    switch (d.D) {
        case 16: return both<16>(d, a, st);
        case 32: return both<32>(d, a, st);
        case 64: return both<64>(d, a, st);
        default: return both<128>(d, a, st);
    }
}

}  // namespace bra
