// Cross attention and its gradients in fp32 on CUDA cores (tensor cores round their operands).  The same walks as the tensor-core
// kernels: one pass over the keys with the running maximum and sum of the softmax; for the gradients one kernel that keeps query
// rows and walks the keys (dQ), one that keeps keys and walks the query rows (dK, dV).
//
// A kept row lives in registers: 16 channels a lane, D / 16 lanes a row (every D / 16th 16-byte chunk each, so that the lanes of a row
// read neighbouring chunks).  Walked rows cross shared memory in tiles, two in flight, and are read as broadcasts: a 16-byte load feeds
// four FMAs (packed in pairs), with no transposed or padded copies and no exchange but the sum over the lanes of a row.
// Measured (B200, 16 x 784 x 196, 4 heads of 32, forward and gradients): tiles of 4 x 8 scores a thread with both sides in shared
// memory 300 us, bound by shared-memory loads.
//
// Groups of walked rows are worked on together, so that their dot products overlap; a group's contribution to O is summed by itself
// and added to the rescaled O in one FMA, which shortens the chain of roundings by the size of the group.
#include "cross_common.cuh"

#include <math.h>

namespace bra {
namespace {

constexpr int THREADS = 128;

template <int D>
struct Shape {
    static constexpr int LANES = D / 16;                    // of a row
    static constexpr int CH = D / LANES;                    // channels of a lane
    static constexpr int CHUNKS = CH / 4;
    static constexpr int ROWS = THREADS / LANES;            // kept rows of a CTA
    static constexpr int BN = D == 128 ? 32 : 64;           // walked rows of a tile
    static constexpr int TILE = BN * D;                     // floats
};

// a lane's channels
template <int CH> struct Slice { float2 v[CH / 2]; };

template <int D>
__device__ __forceinline__ void fetch(Slice<Shape<D>::CH>& s, const float* row, int part) {
    using S = Shape<D>;
#pragma unroll
    for (int i = 0; i < S::CHUNKS; ++i) {
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row) t = __ldg(reinterpret_cast<const float4*>(row) + i * S::LANES + part);
        s.v[2 * i] = make_float2(t.x, t.y);
        s.v[2 * i + 1] = make_float2(t.z, t.w);
    }
}
template <int D>
__device__ __forceinline__ void put(float* row, const Slice<Shape<D>::CH>& s, float f, int part) {
    using S = Shape<D>;
#pragma unroll
    for (int i = 0; i < S::CHUNKS; ++i)
        reinterpret_cast<float4*>(row)[i * S::LANES + part] =
            make_float4(s.v[2 * i].x * f, s.v[2 * i].y * f, s.v[2 * i + 1].x * f, s.v[2 * i + 1].y * f);
}
// dot[g] = kept row . walked rows at + g * D; the same in all lanes of the row
template <int D, int G>
__device__ __forceinline__ void dots(float (&dot)[G], const Slice<Shape<D>::CH>& x, uint32_t at, int part) {
    using S = Shape<D>;
    float2 acc[G] = {};
#pragma unroll
    for (int i = 0; i < S::CHUNKS; ++i)
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const float4 t = ptx::lds_f32x4(at + (uint32_t)(g * D + (i * S::LANES + part) * 4) * 4);
            acc[g] = __ffma2_rn(x.v[2 * i], make_float2(t.x, t.y), acc[g]);
            acc[g] = __ffma2_rn(x.v[2 * i + 1], make_float2(t.z, t.w), acc[g]);
        }
#pragma unroll
    for (int g = 0; g < G; ++g) {
        dot[g] = acc[g].x + acc[g].y;
#pragma unroll
        for (int o = 1; o < S::LANES; o <<= 1) dot[g] += __shfl_xor_sync(0xffffffffu, dot[g], o);
    }
}
// acc = keep * acc + sum over g of w[g] * walked row g
template <int D, int G, bool KEEP>
__device__ __forceinline__ void weigh(Slice<Shape<D>::CH>& acc, const float (&w)[G], float keep, uint32_t at, int part) {
    using S = Shape<D>;
#pragma unroll
    for (int i = 0; i < S::CHUNKS; ++i) {
        float2 a = make_float2(0.f, 0.f), b = a;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const float4 t = ptx::lds_f32x4(at + (uint32_t)(g * D + (i * S::LANES + part) * 4) * 4);
            const float2 f = make_float2(w[g], w[g]);
            a = g ? __ffma2_rn(f, make_float2(t.x, t.y), a) : __fmul2_rn(f, make_float2(t.x, t.y));
            b = g ? __ffma2_rn(f, make_float2(t.z, t.w), b) : __fmul2_rn(f, make_float2(t.z, t.w));
        }
        const float2 k = make_float2(keep, keep);
        acc.v[2 * i] = KEEP ? __ffma2_rn(acc.v[2 * i], k, a) : __fadd2_rn(acc.v[2 * i], a);
        acc.v[2 * i + 1] = KEEP ? __ffma2_rn(acc.v[2 * i + 1], k, b) : __fadd2_rn(acc.v[2 * i + 1], b);
    }
}
// a tile of two walked tensors on its way to shared memory; where(row) places a row in both or says that it is zeros
template <int D, typename F>
__device__ __forceinline__ void copy_tile(uint32_t to, const float* p1, const float* p2, F&& where) {
    using S = Shape<D>;
#pragma unroll 4
    for (int u = threadIdx.x; u < S::BN * (D / 4); u += THREADS) {
        const int row = u / (D / 4), ch = u % (D / 4);
        long long o1, o2;
        const bool in = where(row, o1, o2);
        ptx::cp_async_16(to + u * 16, p1 + (in ? o1 : 0) + ch * 4, in ? 16 : 0);
        ptx::cp_async_16(to + S::TILE * 4 + u * 16, p2 + (in ? o2 : 0) + ch * 4, in ? 16 : 0);
    }
}

// ---------------------------------------------------------------- forward
template <int D>
__global__ void __launch_bounds__(THREADS) cross_attend_simt_kernel(const CrossArgs a) {
    using S = Shape<D>;
    constexpr int G = 8;
    extern __shared__ __align__(16) float sh[];             // two stages of K, V; the mask's bits
    __shared__ int flag;
    const CrossPlace at(a);
    const int slot = threadIdx.x / S::LANES, part = threadIdx.x % S::LANES;
    const KeyRange keys = cross_keys(a, at.b, at.split * a.split_len, min(a.Nk, (at.split + 1) * a.split_len),
                                     reinterpret_cast<uint32_t*>(sh + 4 * S::TILE));
    if (a.key_mask) __syncthreads();
    const float* K = static_cast<const float*>(a.K) + (long long)at.b * a.Nk * a.k_stride + (long long)at.kvh * D;
    const float* V = static_cast<const float*>(a.V) + (long long)at.b * a.Nk * a.v_stride + (long long)at.kvh * D;
    const int r = at.tile * S::ROWS + slot;
    const bool live = r < a.rows;
    const uint32_t base = ptx::smem_u32(sh);
    const int tiles = (keys.hi - keys.lo + S::BN - 1) / S::BN;
    auto copy = [&](int tile, int stage) {
        copy_tile<D>(base + stage * (S::TILE * 8), K, V, [&](int row, long long& o1, long long& o2) {
            const long long j = keys.lo + tile * S::BN + row;
            o1 = j * a.k_stride;
            o2 = j * a.v_stride;
            return (keys.word(tile * (S::BN / 32) + (row >> 5)) >> (row & 31)) & 1;
        });
        ptx::cp_async_commit();
    };
    if (tiles) copy(0, 0);
    Slice<S::CH> q, o = {};
    fetch<D>(q, live ? static_cast<const float*>(a.Q) + cross_row(a, at, r, a.q_stride, D) : nullptr, part);
    float m = -INFINITY, l = 0.f;
    const float c = a.scale_log2;
    for (int tile = 0; tile < tiles; ++tile) {
        if (tile + 1 < tiles) {
            copy(tile + 1, (tile + 1) & 1);
            ptx::cp_async_wait<1>();
        } else {
            ptx::cp_async_wait<0>();
        }
        __syncthreads();
        const uint32_t k = base + (tile & 1) * (8 * S::TILE), v = k + 4 * S::TILE;
#pragma unroll 1
        for (int n = 0; n < S::BN; n += G) {
            const uint32_t seen = keys.word(tile * (S::BN / 32) + (n >> 5)) >> (n & 31);
            if (!(seen & ((1u << G) - 1))) continue;
            float s[G];
            dots<D, G>(s, q, k + n * D * 4, part);
            float top = m;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                if (!((seen >> g) & 1)) s[g] = -INFINITY;
                top = fmaxf(top, s[g]);
            }
            const float ref = top == -INFINITY ? 0.f : top * c;
            const float keep = exp2f(fmaf(m, c, -ref));
            m = top;
            float sum = 0.f;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                s[g] = exp2f(fmaf(s[g], c, -ref));
                sum += s[g];
            }
            l = fmaf(l, keep, sum);
            weigh<D, G, true>(o, s, keep, v + n * D * 4, part);
        }
        __syncthreads();
    }
    if (live) {
        if (a.splits == 1) {
            put<D>(static_cast<float*>(a.Oo) + cross_row(a, at, r, a.o_stride, D), o, l == 0.f ? 0.f : 1.f / l, part);
            if (a.lse && part == 0) a.lse[cross_stat(a, at, r)] = l == 0.f ? -INFINITY : (m * c + log2f(l)) * 0.69314718055994531f;
        } else {
            float* to = a.part + ((at.pair * a.tiles + at.tile) * a.splits + at.split) * (long long)(S::ROWS * (D + 4)) + slot * (D + 4);
            put<D>(to, o, 1.f, part);
            if (part == 0) { to[D] = m; to[D + 1] = l; }
        }
    }
    if (a.splits == 1 || !cross_last(a.done + at.pair * a.tiles + at.tile, a.splits, &flag)) return;
    const long long one = S::ROWS * (D + 4);
    cross_join<D>(a.part + (at.pair * a.tiles + at.tile) * a.splits * one, one, D + 4, min(S::ROWS, a.rows - at.tile * S::ROWS), a.splits, c, sh,
                  [&](int row, int ch, float4 v) {
                      *reinterpret_cast<float4*>(static_cast<float*>(a.Oo) + cross_row(a, at, at.tile * S::ROWS + row, a.o_stride, D) + 4 * ch) = v;
                  },
                  [&](int row, float ref, float sum) {
                      if (a.lse) a.lse[cross_stat(a, at, at.tile * S::ROWS + row)] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
                  });
}

// ---------------------------------------------------------------- gradients
template <int D, bool DKV>
__global__ void __launch_bounds__(THREADS) cross_grad_simt_kernel(const CrossArgs a) {
    using S = Shape<D>;
    constexpr int G = 4;
    extern __shared__ __align__(16) float sh[];             // two stages of Y1, Y2 and (dK, dV) their statistics; the mask's bits
    constexpr int STAGE = 2 * S::TILE + (DKV ? 2 * S::BN : 0);
    __shared__ int flag;
    const CrossPlace at(a);
    const int slot = threadIdx.x / S::LANES, part = threadIdx.x % S::LANES;
    const int key_lo = DKV ? at.tile * S::ROWS : at.split * a.split_len;
    const KeyRange keys = cross_keys(a, at.b, key_lo, min(a.Nk, DKV ? key_lo + S::ROWS : key_lo + a.split_len),
                                     reinterpret_cast<uint32_t*>(sh + 2 * STAGE));
    if (a.key_mask) __syncthreads();
    const int walk_lo = DKV ? at.split * a.split_len : keys.lo;
    const int walk_hi = DKV ? min(a.rows, walk_lo + a.split_len) : keys.hi;
    const float *Q = static_cast<const float*>(a.Q), *dO = static_cast<const float*>(a.dO);
    const float* K = static_cast<const float*>(a.K) + (long long)at.b * a.Nk * a.k_stride + (long long)at.kvh * D;
    const float* V = static_cast<const float*>(a.V) + (long long)at.b * a.Nk * a.v_stride + (long long)at.kvh * D;
    const int padded = (a.rows + 63) / 64 * 64;
    float2* stats = a.stats + at.pair * padded;
    const uint32_t base = ptx::smem_u32(sh);
    int tiles = walk_hi > walk_lo ? (walk_hi - walk_lo + S::BN - 1) / S::BN : 0;
    if (DKV && keys.hi <= keys.lo) tiles = 0;               // nothing to walk for hidden keys
    auto copy = [&](int tile, int stage) {
        copy_tile<D>(base + stage * (STAGE * 4), DKV ? Q : K, DKV ? dO : V, [&](int row, long long& o1, long long& o2) -> bool {
            const int j = walk_lo + tile * S::BN + row;
            if (DKV) {
                if (j >= walk_hi) return false;
                o1 = cross_row(a, at, j, a.q_stride, D);
                o2 = cross_row(a, at, j, a.o_stride, D);
                return true;
            }
            o1 = j * a.k_stride;
            o2 = j * a.v_stride;
            return (keys.word(tile * (S::BN / 32) + (row >> 5)) >> (row & 31)) & 1;
        });
        // (a tile that is cut by the end of a part reads the statistics of rows of the next, whose Q and dO are zeros here)
        if (DKV && threadIdx.x < S::BN / 2)
            ptx::cp_async_16(base + (stage * STAGE + 2 * S::TILE) * 4 + threadIdx.x * 16, stats + walk_lo + tile * S::BN + threadIdx.x * 2, 16);
        ptx::cp_async_commit();
    };
    if (tiles) copy(0, 0);

    const int r = at.tile * S::ROWS + slot;
    const bool in = DKV ? (keys.word(slot >> 5) >> (slot & 31)) & 1 : r < a.rows;       // seen, or there
    Slice<S::CH> x1, x2, acc = {}, accv = {};
    fetch<D>(x1, !in ? nullptr : DKV ? K + r * a.k_stride : Q + cross_row(a, at, r, a.q_stride, D), part);
    fetch<D>(x2, !in ? nullptr : DKV ? V + r * a.v_stride : dO + cross_row(a, at, r, a.o_stride, D), part);
    float lse2 = INFINITY, delta = 0.f;
    if (!DKV) {
        Slice<S::CH> o;
        fetch<D>(o, in ? static_cast<const float*>(a.O) + cross_row(a, at, r, a.o_stride, D) : nullptr, part);
        float2 d = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < S::CH / 2; ++i) d = __ffma2_rn(o.v[i], x2.v[i], d);
        delta = d.x + d.y;
#pragma unroll
        for (int x = 1; x < S::LANES; x <<= 1) delta += __shfl_xor_sync(0xffffffffu, delta, x);
        if (in) {
            const float e = __ldg(a.lse + cross_stat(a, at, r));
            if (e != -INFINITY) lse2 = e * 1.4426950408889634f;                          // else no key is seen: every p is 2^-inf
        }
        if (at.split == 0 && part == 0 && r < padded) stats[r] = make_float2(lse2, in ? delta : 0.f);
    }
    const float c = a.scale_log2;
    for (int tile = 0; tile < tiles; ++tile) {
        if (tile + 1 < tiles) {
            copy(tile + 1, (tile + 1) & 1);
            ptx::cp_async_wait<1>();
        } else {
            ptx::cp_async_wait<0>();
        }
        __syncthreads();
        const uint32_t y1 = base + (tile & 1) * (STAGE * 4), y2 = y1 + 4 * S::TILE, st = y2 + 4 * S::TILE;
#pragma unroll 1
        for (int n = 0; n < S::BN; n += G) {
            const uint32_t seen = DKV ? 0xfu : keys.word(tile * (S::BN / 32) + (n >> 5)) >> (n & 31);
            if (!(seen & ((1u << G) - 1))) continue;
            float s[G], dp[G];
            dots<D, G>(s, x1, y1 + n * D * 4, part);
            dots<D, G>(dp, x2, y2 + n * D * 4, part);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float2 ld = DKV ? ptx::lds_f32x2(st + 8 * (n + g)) : make_float2(lse2, delta);
                s[g] = (seen >> g) & 1 ? exp2f(fmaf(s[g], c, -ld.x)) : 0.f;
                dp[g] = s[g] * (dp[g] - ld.y);
            }
            weigh<D, G, false>(acc, dp, 1.f, y1 + n * D * 4, part);
            if constexpr (DKV) weigh<D, G, false>(accv, s, 1.f, y2 + n * D * 4, part);
        }
        __syncthreads();
    }
    if (a.splits > 1) {
        const long long one = (long long)(DKV ? 2 : 1) * S::ROWS * D;
        float* mine = a.part + ((at.pair * a.tiles + at.tile) * a.splits + at.split) * one;
        put<D>(mine + slot * D, acc, 1.f, part);
        if constexpr (DKV) put<D>(mine + (S::ROWS + slot) * D, accv, 1.f, part);
        if (!cross_last(a.done + at.pair * a.tiles + at.tile, a.splits, &flag)) return;
        const float* all = a.part + (at.pair * a.tiles + at.tile) * a.splits * one;
        acc = {};
        accv = {};
        for (int sp = 0; sp < a.splits; ++sp)
#pragma unroll
            for (int i = 0; i < S::CHUNKS; ++i) {
                const float4 t = __ldcg(reinterpret_cast<const float4*>(all + sp * one + slot * D) + i * S::LANES + part);
                acc.v[2 * i] = __fadd2_rn(acc.v[2 * i], make_float2(t.x, t.y));
                acc.v[2 * i + 1] = __fadd2_rn(acc.v[2 * i + 1], make_float2(t.z, t.w));
                if constexpr (DKV) {
                    const float4 u = __ldcg(reinterpret_cast<const float4*>(all + sp * one + (S::ROWS + slot) * D) + i * S::LANES + part);
                    accv.v[2 * i] = __fadd2_rn(accv.v[2 * i], make_float2(u.x, u.y));
                    accv.v[2 * i + 1] = __fadd2_rn(accv.v[2 * i + 1], make_float2(u.z, u.w));
                }
            }
    }
    if constexpr (DKV) {
        if (r >= a.Nk) return;
        if (!in) { acc = {}; accv = {}; }                   // hidden: its sums are of scores it does not have
        const long long j = (long long)at.b * a.Nk + r;
        put<D>(static_cast<float*>(a.dK) + j * a.k_stride + (long long)at.kvh * D, acc, a.scale, part);
        put<D>(static_cast<float*>(a.dV) + j * a.v_stride + (long long)at.kvh * D, accv, 1.f, part);
    } else if (in) {
        put<D>(static_cast<float*>(a.dQ) + cross_row(a, at, r, a.q_stride, D), acc, a.scale, part);
    }
}

// ---------------------------------------------------------------- host
int kept(const CrossDims& d) { return THREADS * 16 / d.D; }
int step(const CrossDims& d) { return d.D == 128 ? 32 : 64; }

CrossSplit forward_split(const CrossDims& d) { return cross_split((long long)d.B * d.kv, d.rows, kept(d), d.Nk, step(d), 3); }
CrossSplit grad_split(const CrossDims& d, bool dkv) {
    return cross_split((long long)d.B * d.kv, dkv ? d.Nk : d.rows, kept(d), dkv ? d.rows : d.Nk, step(d), 3);
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

template <int D>
cudaError_t forward(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    using S = Shape<D>;
    static PerDeviceMax attr;
    cross_cut(a, forward_split(d));
    size_t smem = sizeof(float) * 4 * S::TILE + mask_bytes(a, a.split_len);
    const size_t join = a.splits > 1 ? sizeof(float) * S::ROWS * (a.splits + 1) : 0;
    smem = smem > join ? smem : join;
    return launch(cross_attend_simt_kernel<D>, attr, a, (long long)d.B * d.kv, smem, st);
}
template <int D, bool DKV>
cudaError_t grad(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    using S = Shape<D>;
    static PerDeviceMax attr;
    cross_cut(a, grad_split(d, DKV));
    const size_t smem = sizeof(float) * 2 * (2 * S::TILE + (DKV ? 2 * S::BN : 0)) + mask_bytes(a, DKV ? S::ROWS : a.split_len);
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
    return s.splits > 1 ? (size_t)s.splits * s.tiles * d.B * d.kv * kept(d) * (d.D + 4) : 0;
}
size_t cross_backward_simt_part(const CrossDims& d) {
    size_t most = 0;
    for (int dkv = 0; dkv < 2; ++dkv) {
        const CrossSplit s = grad_split(d, dkv);
        const size_t n = s.splits > 1 ? (size_t)s.splits * s.tiles * d.B * d.kv * (1 + dkv) * kept(d) * d.D : 0;
        most = n > most ? n : most;
    }
    return most;
}

cudaError_t launch_cross_attend_simt(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    switch (d.D) {
        case 16: return forward<16>(d, a, st);
        case 32: return forward<32>(d, a, st);
        case 64: return forward<64>(d, a, st);
        default: return forward<128>(d, a, st);
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
