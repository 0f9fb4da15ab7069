// Rotary positions of projected Q and K, both in one launch.
//
// A pair of channels (u, v) of a token turns by the angle coordinate * freq, the same for every head of Q and K.  The angle is
// formed in 64 bits: at coordinate 10^6 a 32-bit product is off by 0.03 turns of a radian, and B200's 64-bit rate makes it
// cheap.  It is brought to half a turn there and only then goes to 32 bits (sincospi, no slow path).
//
// What bounds it: HBM, every channel read and written once.  A CTA takes a few tokens: it first puts the (cos, sin) of every pair
// of them in shared memory - one evaluation per (token, pair), shared by all heads - and then streams the rows of all heads of Q
// and K through 16-byte loads, four in flight per thread.
#include "bra_internal.h"
#include "fast_div.h"

#include <math.h>

namespace bra {
namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_AHEAD = 4;           // units in flight per thread
constexpr int ROPE_MAX_TOKENS = 64;     // of a CTA

struct RopeArgs {
    const void *Q, *K;
    void *Qo, *Ko;
    const int32_t* positions;
    const double* freq;
    long long tokens, q_stride, k_stride;
    int N, heads, all_heads, D, rot, n, axes, width, first;
    int per_cta;                        // tokens of a CTA
    float magnitude, sine;              // sine: -1 for the inverse
    bool q_in_place, k_in_place;
    FastDiv units_div, row_div;         // units of a head, of a token's heads
    int units, row_units;
};

template <typename T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T v[V]; };

// What one unit covers.  Interleaved: max(VEC, 2) neighbouring channels, each pair turned or (behind rot) copied.  Half: VEC pairs,
// that is VEC channels and the VEC that lie n / 2 further on; behind the rotated channels, VEC copied ones.
template <typename T, int VEC, bool HALF>
struct Unit {
    static constexpr int W = HALF ? VEC : (VEC < 2 ? 2 : VEC);
    Pack<T, VEC> a[W / VEC], b;
    const T* src;
    T* dst;
    int c;                              // first channel
    int at;                             // (cos, sin) of the first pair; -1: channels that are copied
    bool live;

    __device__ __forceinline__ void load(const RopeArgs& g, long long token0, int i, int end) {
        live = i < end;
        if (!live) return;
        const int t = (int)fdiv((uint32_t)i, g.row_div), hu = i - t * g.row_units;
        const int h = (int)fdiv((uint32_t)hu, g.units_div), u = hu - h * g.units;
        const bool of_q = h < g.heads;
        const long long off = (token0 + t) * (of_q ? g.q_stride : g.k_stride) + (long long)(of_q ? h : h - g.heads) * g.D;
        src = static_cast<const T*>(of_q ? g.Q : g.K) + off;
        dst = static_cast<T*>(of_q ? g.Qo : g.Ko) + off;
        const bool in_place = of_q ? g.q_in_place : g.k_in_place;
        if (HALF) {
            const int pair = u * VEC;
            if (2 * pair < g.rot) {
                const int half = g.n >> 1, block = pair >= half ? 1 : 0;      // at most two blocks
                c = pair + block * half;
                at = t * (g.rot >> 1) + pair;
                a[0] = *reinterpret_cast<const Pack<T, VEC>*>(src + c);
                b = *reinterpret_cast<const Pack<T, VEC>*>(src + c + half);
            } else {
                c = g.rot + pair - (g.rot >> 1);
                at = -1;
                if (in_place) { live = false; return; }
                a[0] = *reinterpret_cast<const Pack<T, VEC>*>(src + c);
            }
        } else {
            c = u * W;
            at = c < g.rot ? t * (g.rot >> 1) + (c >> 1) : -1;
            if (at < 0 && in_place) { live = false; return; }
#pragma unroll
            for (int k = 0; k < W / VEC; ++k)
                if (VEC > 1 || c + k < g.D) a[k] = *reinterpret_cast<const Pack<T, VEC>*>(src + c + k * VEC);
        }
    }
    __device__ __forceinline__ void finish(const RopeArgs& g, const float2* turn) {
        if (!live) return;
        if (HALF) {
            if (at >= 0) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float2 cs = turn[at + e];
                    const float u = to_f(a[0].v[e]), v = to_f(b.v[e]);
                    a[0].v[e] = from_f<T>(u * cs.x - v * cs.y);
                    b.v[e] = from_f<T>(u * cs.y + v * cs.x);
                }
                *reinterpret_cast<Pack<T, VEC>*>(dst + c + (g.n >> 1)) = b;
            }
            *reinterpret_cast<Pack<T, VEC>*>(dst + c) = a[0];
        } else {
            if (at >= 0) {
#pragma unroll
                for (int e = 0; e < W; e += 2) {
                    if (c + e >= g.rot) break;                               // the rest of a partly rotated unit
                    const float2 cs = turn[at + e / 2];
                    T& x = a[e / VEC].v[e % VEC];
                    T& y = a[(e + 1) / VEC].v[(e + 1) % VEC];
                    const float u = to_f(x), v = to_f(y);
                    x = from_f<T>(u * cs.x - v * cs.y);
                    y = from_f<T>(u * cs.y + v * cs.x);
                }
            }
#pragma unroll
            for (int k = 0; k < W / VEC; ++k)
                if (VEC > 1 || c + k < g.D) *reinterpret_cast<Pack<T, VEC>*>(dst + c + k * VEC) = a[k];
        }
    }
};

template <typename T, int VEC, bool HALF>
__global__ void __launch_bounds__(ROPE_THREADS) rope_kernel(const RopeArgs g) {
    extern __shared__ float2 turn[];                     // [tokens of the CTA][rot / 2]
    const long long token0 = (long long)blockIdx.x * g.per_cta;
    const int here = (int)min((long long)g.per_cta, g.tokens - token0);
    const int pairs = g.rot >> 1, half = g.n >> 1;

    for (int i = threadIdx.x; i < here * pairs; i += ROPE_THREADS) {
        const int t = i / pairs, p = i - t * pairs;
        const int axis = p >= half ? 1 : 0;
        const long long token = token0 + t;
        int place;
        if (g.positions) {
            place = __ldg(g.positions + token * g.axes + axis);
        } else {
            const int in_image = (int)(token % g.N);
            place = g.axes == 1 ? g.first + in_image : axis ? in_image % g.width : in_image / g.width;
        }
        // turns = angle / 2 pi; the whole ones are dropped in 64 bits
        double turns = (double)place * __ldg(g.freq + (p - axis * half)) * 0.15915494309189533577;
        turns -= rint(turns);
        float s, c;
        sincospif(2.f * (float)turns, &s, &c);
        turn[i] = make_float2(c * g.magnitude, s * g.magnitude * g.sine);
    }
    __syncthreads();

    const int end = here * g.row_units;
    for (int i = threadIdx.x; i < end; i += ROPE_THREADS * ROPE_AHEAD) {
        Unit<T, VEC, HALF> unit[ROPE_AHEAD];
#pragma unroll
        for (int k = 0; k < ROPE_AHEAD; ++k) unit[k].load(g, token0, i + k * ROPE_THREADS, end);
#pragma unroll
        for (int k = 0; k < ROPE_AHEAD; ++k) unit[k].finish(g, turn);
    }
}

template <typename T, int VEC>
cudaError_t launch(const RopeArgs& a, bool half, unsigned ctas, size_t smem, cudaStream_t st) {
    if (half) rope_kernel<T, VEC, true><<<ctas, ROPE_THREADS, smem, st>>>(a);
    else      rope_kernel<T, VEC, false><<<ctas, ROPE_THREADS, smem, st>>>(a);
    count_launch();
    return cudaGetLastError();
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace
}  // namespace bra

using namespace bra;

extern "C" {

bra_status bra_rope_frequencies(int32_t rot_dim, int32_t axes, double base, int32_t scaling, double factor,
                                double original_length, double low, double high, double* freq) {
    if (!freq) return BRA_ERR_NULL;
    if ((axes != 1 && axes != 2) || rot_dim <= 0 || rot_dim % (2 * axes) || !(base > 0)) return BRA_ERR_SHAPE;
    if (scaling < BRA_ROPE_PLAIN || scaling > BRA_ROPE_PARTS) return BRA_ERR_UNSUPPORTED;
    if (scaling != BRA_ROPE_PLAIN && !(factor > 0)) return BRA_ERR_SHAPE;
    const int n = rot_dim / axes;
    if (scaling == BRA_ROPE_BASE && n <= 2) return BRA_ERR_SHAPE;
    if (scaling == BRA_ROPE_PARTS && (!(original_length > 0) || !(high > low))) return BRA_ERR_SHAPE;
    if (scaling == BRA_ROPE_BASE) base *= pow(factor, (double)n / (n - 2));
    const double two_pi = 6.283185307179586476925;
    for (int i = 0; i < n / 2; ++i) {
        double f = pow(base, -2.0 * i / n);
        if (scaling == BRA_ROPE_LINEAR) f /= factor;
        if (scaling == BRA_ROPE_PARTS) {
            double keep = (original_length * f / two_pi - low) / (high - low);
            keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
            f *= keep + (1 - keep) / factor;
        }
        freq[i] = f;
    }
    return BRA_OK;
}

bra_status bra_rope(const bra_rope_problem* p, const void* Q, const void* K, const int32_t* positions,
                    const double* freq, int32_t inverse, void* Qo, void* Ko, void* stream) {
    reset_launch_count();
    if (!p) return BRA_ERR_NULL;
    if (p->B <= 0 || p->N <= 0 || p->heads <= 0 || p->kv_heads < 0 || p->head_dim <= 0) return BRA_ERR_SHAPE;
    if ((p->axes != 1 && p->axes != 2) || p->rot_dim <= 0 || p->rot_dim % (2 * p->axes) || p->rot_dim > p->head_dim)
        return BRA_ERR_SHAPE;
    if (p->dtype != BRA_F32 && p->dtype != BRA_BF16) return BRA_ERR_DTYPE;
    if (p->layout != BRA_ROPE_INTERLEAVED && p->layout != BRA_ROPE_HALF) return BRA_ERR_UNSUPPORTED;
    const long long q_row = (long long)p->heads * p->head_dim, k_row = (long long)p->kv_heads * p->head_dim;
    if (q_row + k_row > (1 << 24)) return BRA_ERR_SHAPE;
    const long long qs = p->q_stride ? p->q_stride : q_row, ks = p->k_stride ? p->k_stride : k_row;
    if (qs < q_row || (p->kv_heads && ks < k_row)) return BRA_ERR_SHAPE;
    const long long tokens = (long long)p->B * p->N;
    if (qs >= (1ll << 40) / tokens || ks >= (1ll << 40) / tokens) return BRA_ERR_SHAPE;
    if (!positions && p->axes == 2 && p->width <= 0) return BRA_ERR_SHAPE;
    if (!positions && p->axes == 1 && (p->first < 0 || (long long)p->first + p->N > 0x7fffffffll)) return BRA_ERR_SHAPE;
    if (!Q || !Qo || !freq) return BRA_ERR_NULL;
    if ((p->kv_heads != 0) != (K != nullptr) || (K != nullptr) != (Ko != nullptr)) return BRA_ERR_NULL;
    if (!aligned16(Q) || !aligned16(K) || !aligned16(Qo) || !aligned16(Ko) || (reinterpret_cast<uintptr_t>(freq) & 7) ||
        (reinterpret_cast<uintptr_t>(positions) & 3))
        return BRA_ERR_ALIGN;

    RopeArgs a;
    a.Q = Q; a.K = K; a.Qo = Qo; a.Ko = Ko; a.positions = positions; a.freq = freq;
    a.tokens = tokens; a.q_stride = qs; a.k_stride = ks;
    a.N = p->N; a.heads = p->heads; a.all_heads = p->heads + p->kv_heads; a.D = p->head_dim;
    a.rot = p->rot_dim; a.n = p->rot_dim / p->axes; a.axes = p->axes; a.width = p->width; a.first = p->first;
    a.magnitude = p->magnitude > 0.f ? p->magnitude : 1.f;
    a.sine = inverse ? -1.f : 1.f;
    a.q_in_place = Q == Qo; a.k_in_place = K == Ko;

    // the widest unit that rows, heads and (half layout) the halves of a block allow
    const bool half = p->layout == BRA_ROPE_HALF;
    int vec = p->dtype == BRA_BF16 ? 8 : 4;
    auto fits = [&](int v) {
        return qs % v == 0 && (!p->kv_heads || ks % v == 0) && a.D % v == 0 && (!half || (a.n / 2) % v == 0);
    };
    while (vec > 1 && !fits(vec)) vec >>= 1;
    const int wide = half ? vec : (vec < 2 ? 2 : vec);
    a.units = half ? a.rot / 2 / vec + (a.D - a.rot) / vec : (a.D + wide - 1) / wide;
    a.row_units = a.units * a.all_heads;
    a.units_div = fast_div(a.units);
    a.row_div = fast_div(a.row_units);
    // Tokens of a CTA: four units a thread, as long as that leaves two CTAs for every SM; the table within 48 KB.
    long long per = (ROPE_THREADS * ROPE_AHEAD + a.row_units - 1) / a.row_units;
    per = per < tokens / (2 * kSMs) ? per : tokens / (2 * kSMs);
    const long long room = 48 * 1024 / (8ll * (a.rot / 2));
    if (room < 1) return BRA_ERR_UNSUPPORTED;           // more than 6144 pairs a head
    per = per < room ? per : room;
    per = per < ROPE_MAX_TOKENS ? per : ROPE_MAX_TOKENS;
    a.per_cta = per < 1 ? 1 : (int)per;
    const long long ctas = (tokens + a.per_cta - 1) / a.per_cta;
    if (ctas > 0x7fffffffll) return BRA_ERR_SHAPE;
    const size_t smem = sizeof(float2) * (size_t)a.per_cta * (a.rot / 2);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (p->dtype == BRA_BF16)
        e = vec == 8 ? launch<__nv_bfloat16, 8>(a, half, (unsigned)ctas, smem, st)
          : vec == 4 ? launch<__nv_bfloat16, 4>(a, half, (unsigned)ctas, smem, st)
          : vec == 2 ? launch<__nv_bfloat16, 2>(a, half, (unsigned)ctas, smem, st)
                     : launch<__nv_bfloat16, 1>(a, half, (unsigned)ctas, smem, st);
    else
        e = vec == 4 ? launch<float, 4>(a, half, (unsigned)ctas, smem, st)
          : vec == 2 ? launch<float, 2>(a, half, (unsigned)ctas, smem, st)
                     : launch<float, 1>(a, half, (unsigned)ctas, smem, st);
    return e == cudaSuccess ? BRA_OK : BRA_ERR_CUDA;
}

}  // extern "C"
