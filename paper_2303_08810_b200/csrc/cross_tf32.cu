// Cross attention and its gradients in fp32 on the warp-level tensor cores.  Every operand is the sum of two tf32 numbers, x = hi + lo
// with |lo| <= 2^-11 |x|, and a product is hi hi + hi lo + lo hi, accumulated in fp32: what is dropped is at most 2^-22 (lo lo) and
// what lo loses below its own last bit 2^-22, each a quarter of a step of fp32's own products (2^-24) times four - below the rounding of
// a dot product's sum.  Softmax statistics and all sums are fp32.
//
// The walks are those of the bf16 kernels: one pass over the keys with the running maximum and sum of the softmax (64 rows a CTA, 16 a
// warp; at most 16 rows: every warp has them all and a quarter of each tile's keys); for the gradients one kernel that keeps 64 query
// rows and walks the keys (dQ), one that keeps 64 keys and walks the query rows (dK, dV).  Tiles of the walked side cross shared memory,
// two in flight, as they are; operands are split where they are loaded.
//
// A contraction may run in any order and an output's columns may be any channels, so a lane takes neighbouring channels: of 32 channels,
// 8 t .. 8 t + 7 where it contracts over them (k steps take two of them each), 4 g .. 4 g + 3 where they are columns; scores 2 t and 2 t + 1 of an
// accumulator are the rows t and t + 4 of the next product's k step.  So every operand comes from 16-byte loads, P and dS need no exchange,
// and rows 16 bytes longer than they need be lie in different banks.
//
// Exponents: s c - ref with c = scale log2 e as the sum of two floats and ref the rounded reference itself, so that neither c's rounding nor
// a reference that moves shows (scores of +-10 would put 10^-6 into P).
// What bounds it: issue (0.38 - 0.46 instructions a cycle and scheduler at two to three warps, tensor pipe 41 - 58 %): operands are split by every
// warp that reads them.  Measured (B200), us, forward + gradients, this / on CUDA cores with kept rows in registers and walked ones as
// broadcasts: 16 x 784 x 196, 4 heads of 32 48 + 131 / 248, 4 x 1024 x 1024, 4 heads of 64 137 + 363 / 1252.
#include "cross_common.cuh"

#include <math.h>

namespace bra {
namespace {

constexpr int THREADS = 128, KEPT = 64;
// Walked rows of a tile, and the step by which walks are cut: a part's length is a multiple of it, so only the end of the rows (or keys)
// cuts a tile.
constexpr int walk_tile(int D) { return D == 128 ? 32 : 64; }

template <int D>
struct Shape {
    static constexpr int GW = D < 32 ? D : 32, NG = D / GW;     // channels of a group, groups
    static constexpr int LC = GW / 4;                           // neighbouring channels of a lane, contracted over
    static constexpr int NB = GW / 8;                           // column blocks of a group, columns of a lane
    static constexpr int BN = walk_tile(D);
    static constexpr int LD = (D + 4) * 4;                      // bytes of a row in shared memory
    static constexpr int TILE = BN * LD;
};

struct Split { uint32_t hi, lo; };
__device__ __forceinline__ Split split(float x) {
    Split s;
    s.hi = (__float_as_uint(x) + 0x1000u) & 0xffffe000u;        // to the nearest; infinities and NaN stay what they are or become NaN
    s.lo = __float_as_uint(x - __uint_as_float(s.hi));
    return s;
}
__device__ __forceinline__ void mma_tf32(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
struct Frag { Split a[4]; };
// d += sum over k of a[k] * (b0[k], b1[k]).  The tensor core's own additions cut off what does not fit, always towards zero, so a
// chain of them drifts (75 into one O: 6e-6).  So a few products go to an accumulator of their own, the small ones first, and only its
// rounded sum is added to d.
template <int K>
__device__ __forceinline__ void mma_split(float* d, const Frag (&a)[K], const Split (&b0)[K], const Split (&b1)[K]) {
    float t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
        mma_tf32(t, a[k].a[0].lo, a[k].a[1].lo, a[k].a[2].lo, a[k].a[3].lo, b0[k].hi, b1[k].hi);
        mma_tf32(t, a[k].a[0].hi, a[k].a[1].hi, a[k].a[2].hi, a[k].a[3].hi, b0[k].lo, b1[k].lo);
    }
#pragma unroll
    for (int k = 0; k < K; ++k) mma_tf32(t, a[k].a[0].hi, a[k].a[1].hi, a[k].a[2].hi, a[k].a[3].hi, b0[k].hi, b1[k].hi);
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] += t[i];
}

// the LC neighbouring channels of a lane in group g of rows r and r + 8 (null: zeros)
template <int D>
__device__ __forceinline__ void fetch(float (&x)[Shape<D>::NG][2][Shape<D>::LC], const float* r0, const float* r1, int t4) {
    using S = Shape<D>;
#pragma unroll
    for (int g = 0; g < S::NG; ++g)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float* r = i ? r1 : r0;
#pragma unroll
            for (int q = 0; q < S::LC; q += 4) {
                float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
                if (r) v = __ldg(reinterpret_cast<const float4*>(r + g * S::GW + t4 * S::LC + q));
                x[g][i][q] = v.x; x[g][i][q + 1] = v.y; x[g][i][q + 2] = v.z; x[g][i][q + 3] = v.w;
            }
        }
}
// s[n] += kept rows . walked rows row0 + 8 n ..., n < N
template <int D, int N>
__device__ __forceinline__ void scores(float (&s)[N][4], const float (&x)[Shape<D>::NG][2][Shape<D>::LC], uint32_t tile, int row0, int g4, int t4) {
    using S = Shape<D>;
#pragma unroll
    for (int g = 0; g < S::NG; ++g) {
        Frag a[S::LC / 2];
#pragma unroll
        for (int k = 0; k < S::LC / 2; ++k) {
            a[k].a[0] = split(x[g][0][2 * k]);
            a[k].a[1] = split(x[g][1][2 * k]);
            a[k].a[2] = split(x[g][0][2 * k + 1]);
            a[k].a[3] = split(x[g][1][2 * k + 1]);
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const uint32_t at = tile + (row0 + 8 * n + g4) * S::LD + (g * S::GW + t4 * S::LC) * 4;
            float y[S::LC];
#pragma unroll
            for (int q = 0; q < S::LC; q += 4) {
                const float4 v = ptx::lds_f32x4(at + 4 * q);
                y[q] = v.x; y[q + 1] = v.y; y[q + 2] = v.z; y[q + 3] = v.w;
            }
            Split b0[S::LC / 2], b1[S::LC / 2];
#pragma unroll
            for (int k = 0; k < S::LC / 2; ++k) {
                b0[k] = split(y[2 * k]);
                b1[k] = split(y[2 * k + 1]);
            }
            mma_split(s[n], a, b0, b1);
        }
    }
}
// acc[group][column block] += p (its columns are the walked rows row0 + 8 n ...) times walked rows
template <int D, int N>
__device__ __forceinline__ void gather(float (&acc)[Shape<D>::NG][Shape<D>::NB][4], const float (&p)[N][4], uint32_t tile, int row0, int g4, int t4) {
    using S = Shape<D>;
    constexpr int TWO = N % 2 ? 1 : 2;                          // blocks of eight walked rows at once
#pragma unroll
    for (int n = 0; n < N; n += TWO) {
        Frag a[TWO];
#pragma unroll
        for (int h = 0; h < TWO; ++h) {
            a[h].a[0] = split(p[n + h][0]);
            a[h].a[1] = split(p[n + h][2]);
            a[h].a[2] = split(p[n + h][1]);
            a[h].a[3] = split(p[n + h][3]);
        }
#pragma unroll
        for (int g = 0; g < S::NG; ++g) {
            float y0[TWO][4], y1[TWO][4];
#pragma unroll
            for (int h = 0; h < TWO; ++h) {
                const uint32_t at = tile + (row0 + 8 * (n + h) + 2 * t4) * S::LD + (g * S::GW + g4 * S::NB) * 4;
                if constexpr (S::NB == 4) {
                    const float4 u = ptx::lds_f32x4(at), v = ptx::lds_f32x4(at + S::LD);
                    y0[h][0] = u.x; y0[h][1] = u.y; y0[h][2] = u.z; y0[h][3] = u.w;
                    y1[h][0] = v.x; y1[h][1] = v.y; y1[h][2] = v.z; y1[h][3] = v.w;
                } else {
                    const float2 u = ptx::lds_f32x2(at), v = ptx::lds_f32x2(at + S::LD);
                    y0[h][0] = u.x; y0[h][1] = u.y;
                    y1[h][0] = v.x; y1[h][1] = v.y;
                }
            }
#pragma unroll
            for (int j = 0; j < S::NB; ++j) {
                Split b0[TWO], b1[TWO];
#pragma unroll
                for (int h = 0; h < TWO; ++h) {
                    b0[h] = split(y0[h][j]);
                    b1[h] = split(y1[h][j]);
                }
                mma_split(acc[g][j], a, b0, b1);
            }
        }
    }
}
// rows g4 (i = 0) or g4 + 8 (1) of the accumulators, times f: a lane has LC neighbouring channels of every group
template <int D>
__device__ __forceinline__ void put(float* row, const float (&acc)[Shape<D>::NG][Shape<D>::NB][4], int i, float f, int t4) {
    using S = Shape<D>;
#pragma unroll
    for (int g = 0; g < S::NG; ++g) {
        float v[S::LC];
#pragma unroll
        for (int j = 0; j < S::NB; ++j) {
            v[j] = acc[g][j][2 * i] * f;
            v[S::NB + j] = acc[g][j][2 * i + 1] * f;
        }
#pragma unroll
        for (int q = 0; q < S::LC; q += 4)
            *reinterpret_cast<float4*>(row + g * S::GW + t4 * S::LC + q) = make_float4(v[q], v[q + 1], v[q + 2], v[q + 3]);
    }
}
template <int D>
__device__ __forceinline__ void take(float (&acc)[Shape<D>::NG][Shape<D>::NB][4], const float* row, int i, int t4) {
    using S = Shape<D>;
#pragma unroll
    for (int g = 0; g < S::NG; ++g) {
        float v[S::LC];
#pragma unroll
        for (int q = 0; q < S::LC; q += 4) {
            const float4 u = __ldcg(reinterpret_cast<const float4*>(row + g * S::GW + t4 * S::LC + q));
            v[q] = u.x; v[q + 1] = u.y; v[q + 2] = u.z; v[q + 3] = u.w;
        }
#pragma unroll
        for (int j = 0; j < S::NB; ++j) {
            acc[g][j][2 * i] += v[j];
            acc[g][j][2 * i + 1] += v[S::NB + j];
        }
    }
}
// a tile of two walked tensors on its way to shared memory; where(row) places a row in both or says that it is zeros
template <int D, typename F>
__device__ __forceinline__ void copy_tile(uint32_t to, const float* p1, const float* p2, F&& where) {
    using S = Shape<D>;
#pragma unroll 4
    for (int u = threadIdx.x; u < S::BN * (D / 4); u += THREADS) {
        const int row = u / (D / 4), ch = u % (D / 4);
        long long o1 = 0, o2 = 0;
        const bool in = where(row, o1, o2);
        ptx::cp_async_16(to + row * S::LD + ch * 16, p1 + (in ? o1 : 0) + ch * 4, in ? 16 : 0);
        ptx::cp_async_16(to + S::TILE + row * S::LD + ch * 16, p2 + (in ? o2 : 0) + ch * 4, in ? 16 : 0);
    }
}
// s (c + c_lo) - ref - ref_lo
__device__ __forceinline__ float exponent(float s, const float2& c, float ref, float ref_lo) {
    return fmaf(s, c.x, -ref) + fmaf(s, c.y, -ref_lo);
}

// ---------------------------------------------------------------- forward
// KEYS: at most 16 rows, which every warp has; a warp takes a quarter of each tile's keys
template <int D, bool KEYS>
__global__ void __launch_bounds__(THREADS, 3) cross_attend_tf32_kernel(const CrossArgs a) {
    using S = Shape<D>;
    constexpr int ROWS = KEYS ? 16 : KEPT, N = S::BN / 8 / (KEYS ? 4 : 1);
    extern __shared__ __align__(16) char sh[];              // two stages of K, V; the mask's bits
    __shared__ int flag;
    const CrossPlace at(a);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g4 = lane >> 2, t4 = lane & 3;
    const KeyRange keys = cross_keys(a, at.b, at.split * a.split_len, min(a.Nk, (at.split + 1) * a.split_len),
                                     reinterpret_cast<uint32_t*>(sh + 4 * S::TILE));
    if (a.key_mask) __syncthreads();
    const float* K = static_cast<const float*>(a.K) + (long long)at.b * a.Nk * a.k_stride + (long long)at.kvh * D;
    const float* V = static_cast<const float*>(a.V) + (long long)at.b * a.Nk * a.v_stride + (long long)at.kvh * D;
    const uint32_t base = ptx::smem_u32(sh);
    const int tiles = (keys.hi - keys.lo + S::BN - 1) / S::BN;
    auto copy = [&](int tile, int stage) {
        copy_tile<D>(base + stage * (2 * S::TILE), K, V, [&](int row, long long& o1, long long& o2) -> bool {
            const long long j = keys.lo + tile * S::BN + row;
            o1 = j * a.k_stride;
            o2 = j * a.v_stride;
            return (keys.word(tile * (S::BN / 32) + (row >> 5)) >> (row & 31)) & 1;
        });
        ptx::cp_async_commit();
    };
    if (tiles) copy(0, 0);
    const int r0 = at.tile * ROWS + (KEYS ? 0 : warp * 16) + g4;
    const int r[2] = {r0, r0 + 8};
    float q[S::NG][2][S::LC], o[S::NG][S::NB][4] = {};
    {
        const float* p[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) p[i] = r[i] < a.rows ? static_cast<const float*>(a.Q) + cross_row(a, at, r[i], a.q_stride, D) : nullptr;
        fetch<D>(q, p[0], p[1], t4);
    }
    const float2 c = make_float2(a.scale_log2, a.scale_log2_lo);
    float m[2] = {-INFINITY, -INFINITY}, ref[2] = {0.f, 0.f}, l[2] = {0.f, 0.f};      // largest score, the reference made of it, sum
    for (int tile = 0; tile < tiles; ++tile) {
        if (tile + 1 < tiles) {
            copy(tile + 1, (tile + 1) & 1);
            ptx::cp_async_wait<1>();
        } else {
            ptx::cp_async_wait<0>();
        }
        __syncthreads();
        const uint32_t ks = base + (tile & 1) * (2 * S::TILE), vs = ks + S::TILE;
        const int row0 = KEYS ? warp * (S::BN / 4) : 0;
        float s[N][4] = {};
        scores<D, N>(s, q, ks, row0, g4, t4);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int j = row0 + 8 * n + 2 * t4;
            const uint32_t two = keys.word(tile * (S::BN / 32) + (j >> 5)) >> (j & 31);
            if (!(two & 1)) s[n][0] = s[n][2] = -INFINITY;
            if (!(two & 2)) s[n][1] = s[n][3] = -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float top = m[i];
#pragma unroll
            for (int n = 0; n < N; ++n) top = fmaxf(top, fmaxf(s[n][2 * i], s[n][2 * i + 1]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            if (top > m[i]) {
                const float now = top * c.x, keep = m[i] == -INFINITY ? 0.f : exp2f(ref[i] - now);
                m[i] = top;
                ref[i] = now;
                l[i] *= keep;
#pragma unroll
                for (int g = 0; g < S::NG; ++g)
#pragma unroll
                    for (int j = 0; j < S::NB; ++j) { o[g][j][2 * i] *= keep; o[g][j][2 * i + 1] *= keep; }
            }
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                s[n][2 * i] = s[n][2 * i] == -INFINITY ? 0.f : exp2f(exponent(s[n][2 * i], c, ref[i], 0.f));
                s[n][2 * i + 1] = s[n][2 * i + 1] == -INFINITY ? 0.f : exp2f(exponent(s[n][2 * i + 1], c, ref[i], 0.f));
                sum += s[n][2 * i] + s[n][2 * i + 1];
            }
            l[i] += sum;
        }
        gather<D, N>(o, s, vs, row0, g4, t4);
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    }
    // a row that has seen no key: reference -inf, for the joins
#pragma unroll
    for (int i = 0; i < 2; ++i) if (m[i] == -INFINITY) ref[i] = -INFINITY;

    if (KEYS) {
        // the four warps' sums to shared memory, as parts of a split; joined here, or left as one part
        float* parts = reinterpret_cast<float*>(sh);                // [warp][16][D + 4]
        constexpr int PITCH = D + 4, ONE = 16 * PITCH;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float* to = parts + warp * ONE + (g4 + 8 * i) * PITCH;
            put<D>(to, o, i, 1.f, t4);
            if (t4 == 0) { to[D] = ref[i]; to[D + 1] = l[i]; }
        }
        __syncthreads();
        float* part = a.splits == 1 ? nullptr : a.part + ((at.pair * a.tiles + at.tile) * a.splits + at.split) * (long long)ONE;
        for (int row = warp; row < min(16, a.rows); row += 4) {
            float top = -INFINITY, f[4], sum = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) top = fmaxf(top, parts[w * ONE + row * PITCH + D]);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                f[w] = top == -INFINITY ? 0.f : exp2f(parts[w * ONE + row * PITCH + D] - top);
                sum += f[w] * parts[w * ONE + row * PITCH + D + 1];
            }
            const float inv = part ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
            float* out = part ? part + row * PITCH : static_cast<float*>(a.Oo) + cross_row(a, at, row, a.o_stride, D);
            for (int ch = lane; ch < D; ch += 32) {
                float v = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) v = fmaf(f[w], parts[w * ONE + row * PITCH + ch], v);
                out[ch] = v * inv;
            }
            if (lane == 0) {
                if (part) { out[D] = top; out[D + 1] = sum; }
                else if (a.lse) a.lse[cross_stat(a, at, row)] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
            }
        }
        if (!part) return;
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (r[i] >= a.rows) continue;
            if (a.splits == 1) {
                put<D>(static_cast<float*>(a.Oo) + cross_row(a, at, r[i], a.o_stride, D), o, i, l[i] == 0.f ? 0.f : 1.f / l[i], t4);
                if (a.lse && t4 == 0) a.lse[cross_stat(a, at, r[i])] = l[i] == 0.f ? -INFINITY : (ref[i] + log2f(l[i])) * 0.69314718055994531f;
            } else {
                float* to = a.part + ((at.pair * a.tiles + at.tile) * a.splits + at.split) * (long long)(ROWS * (D + 4)) + (r[i] - at.tile * ROWS) * (D + 4);
                put<D>(to, o, i, 1.f, t4);
                if (t4 == 0) { to[D] = ref[i]; to[D + 1] = l[i]; }
            }
        }
        if (a.splits == 1) return;
    }
    if (!cross_last(a.done + at.pair * a.tiles + at.tile, a.splits, &flag)) return;
    const long long one = ROWS * (D + 4);
    cross_join<D>(a.part + (at.pair * a.tiles + at.tile) * a.splits * one, one, D + 4, min(ROWS, a.rows - at.tile * ROWS), a.splits, 1.f,
                  reinterpret_cast<float*>(sh),
                  [&](int row, int ch, float4 v) {
                      *reinterpret_cast<float4*>(static_cast<float*>(a.Oo) + cross_row(a, at, at.tile * ROWS + row, a.o_stride, D) + 4 * ch) = v;
                  },
                  [&](int row, float top, float sum) {
                      if (a.lse) a.lse[cross_stat(a, at, at.tile * ROWS + row)] = sum == 0.f ? -INFINITY : (top + log2f(sum)) * 0.69314718055994531f;
                  });
}

// ---------------------------------------------------------------- gradients
template <int D, bool DKV>
__global__ void __launch_bounds__(THREADS, D == 128 ? 1 : 2) cross_grad_tf32_kernel(const CrossArgs a) {
    using S = Shape<D>;
    constexpr int N = 4;                                    // blocks of eight walked rows at a time
    extern __shared__ __align__(16) char sh[];              // two stages of Y1, Y2 and (dK, dV) their statistics; the mask's bits
    constexpr int STAGE = 2 * S::TILE + (DKV ? 8 * S::BN : 0);
    __shared__ int flag;
    const CrossPlace at(a);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g4 = lane >> 2, t4 = lane & 3;
    const int key_lo = DKV ? at.tile * KEPT : at.split * a.split_len;
    const KeyRange keys = cross_keys(a, at.b, key_lo, min(a.Nk, DKV ? key_lo + KEPT : key_lo + a.split_len), reinterpret_cast<uint32_t*>(sh + 2 * STAGE));
    if (a.key_mask) __syncthreads();
    const int walk_lo = DKV ? at.split * a.split_len : keys.lo;
    const int walk_hi = DKV ? min(a.rows, walk_lo + a.split_len) : keys.hi;
    const float *Q = static_cast<const float*>(a.Q), *dO = static_cast<const float*>(a.dO);
    const float* K = static_cast<const float*>(a.K) + (long long)at.b * a.Nk * a.k_stride + (long long)at.kvh * D;
    const float* V = static_cast<const float*>(a.V) + (long long)at.b * a.Nk * a.v_stride + (long long)at.kvh * D;
    static_assert(KEPT % S::BN == 0, "the statistics of a walk's last tile");
    const int padded = (a.rows + KEPT - 1) / KEPT * KEPT;
    float2* stats = a.stats + at.pair * padded;             // log of the softmax denominator, delta
    const uint32_t base = ptx::smem_u32(sh);
    int tiles = walk_hi > walk_lo ? (walk_hi - walk_lo + S::BN - 1) / S::BN : 0;
    if (DKV && keys.hi <= keys.lo) tiles = 0;               // nothing to walk for hidden keys
    auto copy = [&](int tile, int stage) {
        copy_tile<D>(base + stage * STAGE, DKV ? Q : K, DKV ? dO : V, [&](int row, long long& o1, long long& o2) -> bool {
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
        // statistics exist up to the padded number of rows (a multiple of BN); rows that do not exist have (inf, 0), so their P and dS are
        // zero whatever their scores
        if (DKV && threadIdx.x < S::BN / 2)
            ptx::cp_async_16(base + stage * STAGE + 2 * S::TILE + threadIdx.x * 16, stats + walk_lo + tile * S::BN + threadIdx.x * 2, 16);
        ptx::cp_async_commit();
    };
    if (tiles) copy(0, 0);

    const int x0 = warp * 16 + g4;
    bool in[2];                                             // kept rows that are there (dQ) or seen (dK, dV)
    float x1[S::NG][2][S::LC], x2[S::NG][2][S::LC];
    float acc[S::NG][S::NB][4] = {}, accv[DKV ? S::NG : 1][S::NB][4] = {};
    float lse[2] = {INFINITY, INFINITY}, delta[2] = {0.f, 0.f};
    {
        const float *p1[2], *p2[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = x0 + 8 * i, r = at.tile * KEPT + row;
            in[i] = DKV ? (keys.word(row >> 5) >> (row & 31)) & 1 : r < a.rows;
            p1[i] = !in[i] ? nullptr : DKV ? K + r * a.k_stride : Q + cross_row(a, at, r, a.q_stride, D);
            p2[i] = !in[i] ? nullptr : DKV ? V + r * a.v_stride : dO + cross_row(a, at, r, a.o_stride, D);
        }
        fetch<D>(x1, p1[0], p1[1], t4);
        fetch<D>(x2, p2[0], p2[1], t4);
    }
    if (!DKV) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = at.tile * KEPT + x0 + 8 * i;
            if (in[i]) {
                const float* o = static_cast<const float*>(a.O) + cross_row(a, at, r, a.o_stride, D);
#pragma unroll
                for (int g = 0; g < S::NG; ++g)
#pragma unroll
                    for (int k = 0; k < S::LC; ++k) delta[i] = fmaf(__ldg(o + g * S::GW + t4 * S::LC + k), x2[g][i][k], delta[i]);
                const float e = __ldg(a.lse + cross_stat(a, at, r));
                if (e != -INFINITY) lse[i] = e;             // else no key is seen: every p is 2^-inf
            }
            delta[i] += __shfl_xor_sync(0xffffffffu, delta[i], 1);
            delta[i] += __shfl_xor_sync(0xffffffffu, delta[i], 2);
            if (at.split == 0 && t4 == 0) stats[r] = make_float2(lse[i], in[i] ? delta[i] : 0.f);
        }
    }
    const float2 c = make_float2(a.scale_log2, a.scale_log2_lo);
    // lse in base 2, as the sum of two floats
    constexpr float E_HI = 1.44269502162933349609375f, E_LO = 1.925963033500011079e-8f;
    auto base2 = [](float v, float& lo) {
        const float hi = v * E_HI;
        lo = v == INFINITY ? 0.f : fmaf(v, E_HI, -hi) + v * E_LO;
        return hi;
    };
    const bool mine = __any_sync(0xffffffffu, in[0] || in[1]);      // a warp without kept rows only copies
    float ref[2], ref_lo[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) ref[i] = base2(lse[i], ref_lo[i]);
    for (int tile = 0; tile < tiles; ++tile) {
        if (tile + 1 < tiles) {
            copy(tile + 1, (tile + 1) & 1);
            ptx::cp_async_wait<1>();
        } else {
            ptx::cp_async_wait<0>();
        }
        __syncthreads();
        const uint32_t y1 = base + (tile & 1) * STAGE, y2 = y1 + S::TILE, st = y2 + S::TILE;
#pragma unroll 1
        for (int row0 = 0; row0 < S::BN; row0 += 8 * N) {
            const uint32_t seen = !mine || walk_lo + tile * S::BN + row0 >= walk_hi ? 0u : DKV ? 0xffffffffu : keys.word(tile * (S::BN / 32) + (row0 >> 5));
            if (!seen) continue;
            float s[N][4] = {}, dp[N][4] = {};
            scores<D, N>(s, x1, y1, row0, g4, t4);
            scores<D, N>(dp, x2, y2, row0, g4, t4);
#pragma unroll
            for (int n = 0; n < N; ++n) {
                if constexpr (DKV) {
                    const float4 v = ptx::lds_f32x4(st + (row0 + 8 * n + 2 * t4) * 8);            // (lse, delta) of two walked rows
                    float lo0, lo1;
                    const float hi0 = base2(v.x, lo0), hi1 = base2(v.z, lo1);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        s[n][2 * i] = exp2f(exponent(s[n][2 * i], c, hi0, lo0));
                        s[n][2 * i + 1] = exp2f(exponent(s[n][2 * i + 1], c, hi1, lo1));
                        dp[n][2 * i] = s[n][2 * i] * (dp[n][2 * i] - v.y);
                        dp[n][2 * i + 1] = s[n][2 * i + 1] * (dp[n][2 * i + 1] - v.w);
                    }
                } else {
                    const uint32_t two = seen >> (8 * n + 2 * t4);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float p0 = two & 1 ? exp2f(exponent(s[n][2 * i], c, ref[i], ref_lo[i])) : 0.f;
                        const float p1 = two & 2 ? exp2f(exponent(s[n][2 * i + 1], c, ref[i], ref_lo[i])) : 0.f;
                        dp[n][2 * i] = p0 * (dp[n][2 * i] - delta[i]);
                        dp[n][2 * i + 1] = p1 * (dp[n][2 * i + 1] - delta[i]);
                    }
                }
            }
            gather<D, N>(acc, dp, y1, row0, g4, t4);
            if constexpr (DKV) gather<D, N>(accv, s, y2, row0, g4, t4);
        }
        __syncthreads();
    }
    if (a.splits > 1) {
        const long long one = (long long)(DKV ? 2 : 1) * KEPT * D;
        float* mine = a.part + ((at.pair * a.tiles + at.tile) * a.splits + at.split) * one;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            put<D>(mine + (x0 + 8 * i) * D, acc, i, 1.f, t4);
            if constexpr (DKV) put<D>(mine + (KEPT + x0 + 8 * i) * D, accv, i, 1.f, t4);
        }
        if (!cross_last(a.done + at.pair * a.tiles + at.tile, a.splits, &flag)) return;
        const float* all = a.part + (at.pair * a.tiles + at.tile) * a.splits * one;
#pragma unroll
        for (int g = 0; g < S::NG; ++g)
#pragma unroll
            for (int j = 0; j < S::NB; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    acc[g][j][k] = 0.f;
                    if constexpr (DKV) accv[g][j][k] = 0.f;
                }
        for (int sp = 0; sp < a.splits; ++sp)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                take<D>(acc, all + sp * one + (x0 + 8 * i) * D, i, t4);
                if constexpr (DKV) take<D>(accv, all + sp * one + (KEPT + x0 + 8 * i) * D, i, t4);
            }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = at.tile * KEPT + x0 + 8 * i;
        if constexpr (DKV) {
            if (r >= a.Nk) continue;
            const long long j = (long long)at.b * a.Nk + r;
            float *dk = static_cast<float*>(a.dK) + j * a.k_stride + (long long)at.kvh * D, *dv = static_cast<float*>(a.dV) + j * a.v_stride + (long long)at.kvh * D;
            if (!in[i]) {                   // hidden: its sums are of scores it does not have
#pragma unroll
                for (int g = 0; g < S::NG; ++g)
#pragma unroll
                    for (int n = 0; n < S::NB; ++n) acc[g][n][2 * i] = acc[g][n][2 * i + 1] = accv[g][n][2 * i] = accv[g][n][2 * i + 1] = 0.f;
            }
            put<D>(dk, acc, i, a.scale, t4);
            put<D>(dv, accv, i, 1.f, t4);
        } else if (in[i]) {
            put<D>(static_cast<float*>(a.dQ) + cross_row(a, at, r, a.q_stride, D), acc, i, a.scale, t4);
        }
    }
}

// ---------------------------------------------------------------- host
bool few_rows(const CrossDims& d) { return d.rows <= 16; }

CrossSplit forward_split(const CrossDims& d) { return cross_split((long long)d.B * d.kv, d.rows, few_rows(d) ? 16 : KEPT, d.Nk, walk_tile(d.D), 3); }
CrossSplit grad_split(const CrossDims& d, bool dkv) {
    return cross_split((long long)d.B * d.kv, dkv ? d.Nk : d.rows, KEPT, dkv ? d.rows : d.Nk, walk_tile(d.D), 2);
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

template <int D, bool KEYS>
cudaError_t forward(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    using S = Shape<D>;
    static PerDeviceMax attr;
    cross_cut(a, forward_split(d));
    size_t smem = 4 * S::TILE + mask_bytes(a, a.split_len);
    const size_t join = a.splits > 1 ? sizeof(float) * (KEYS ? 16 : KEPT) * (a.splits + 1) : 0, warps = KEYS ? sizeof(float) * 4 * 16 * (D + 4) : 0;
    smem = smem > join ? smem : join;
    smem = smem > warps ? smem : warps;
    return launch(cross_attend_tf32_kernel<D, KEYS>, attr, a, (long long)d.B * d.kv, smem, st);
}
template <int D, bool DKV>
cudaError_t grad(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    using S = Shape<D>;
    static PerDeviceMax attr;
    cross_cut(a, grad_split(d, DKV));
    const size_t smem = 2 * (2 * S::TILE + (DKV ? 8 * S::BN : 0)) + mask_bytes(a, DKV ? KEPT : a.split_len);
    return launch(cross_grad_tf32_kernel<D, DKV>, attr, a, (long long)d.B * d.kv, smem, st);
}
template <int D>
cudaError_t forward(const CrossDims& d, const CrossArgs& a, cudaStream_t st) {
    return few_rows(d) ? forward<D, true>(d, a, st) : forward<D, false>(d, a, st);
}
template <int D>
cudaError_t both(const CrossDims& d, const CrossArgs& a, cudaStream_t st) {
    const cudaError_t e = grad<D, false>(d, a, st);
    return e != cudaSuccess ? e : grad<D, true>(d, a, st);
}

}  // namespace

size_t cross_attend_tf32_part(const CrossDims& d) {
    const CrossSplit s = forward_split(d);
    return s.splits > 1 ? (size_t)s.splits * s.tiles * d.B * d.kv * (few_rows(d) ? 16 : KEPT) * (d.D + 4) : 0;
}
size_t cross_backward_tf32_part(const CrossDims& d) {
    size_t most = 0;
    for (int dkv = 0; dkv < 2; ++dkv) {
        const CrossSplit s = grad_split(d, dkv);
        const size_t n = s.splits > 1 ? (size_t)s.splits * s.tiles * d.B * d.kv * (1 + dkv) * KEPT * d.D : 0;
        most = n > most ? n : most;
    }
    return most;
}

cudaError_t launch_cross_attend_tf32(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    switch (d.D) {
        case 16: return forward<16>(d, a, st);
        case 32: return forward<32>(d, a, st);
        case 64: return forward<64>(d, a, st);
        default: return forward<128>(d, a, st);
    }
}
cudaError_t launch_cross_backward_tf32(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    switch (d.D) {
        case 16: return both<16>(d, a, st);
        case 32: return both<32>(d, a, st);
        case 64: return both<64>(d, a, st);
        default: return both<128>(d, a, st);
    }
}

}  // namespace bra
