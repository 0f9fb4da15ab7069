// Rotary positions of projected Q and K, both in one launch.
//
// A pair of channels (u, v) of a token turns by the angle coordinate * freq, the same for every head of Q and K.  The angle is
// formed in 64 bits (at coordinate 10^6 a 32-bit product is off by 0.03 radians), and only what is left of it without whole turns
// goes to 32 bits and a float: half a step of an angle below half a turn is 9.4 10^-8 radians, of the order of the fp32 outputs' own rounding
// (their error against 64 bits 3.9 10^-8; of a plain form with angles in 64 bits 3.0 10^-8).
//
// What bounds it: HBM, every channel read and written once.  A thread has 16 bytes of a head (half layout: and the 16 that belong to
// them) of one token, makes the (cos, sin) of its pairs once, in registers, and walks the heads of Q and K with them - of all images,
// where the positions are those that the problem implies.  No shared memory, no barrier.  The walk is split where there are too few
// tokens for the GPU.  In fp32 a thread has four loads in flight; in bf16, whose 16 bytes are twice as many channels, registers for
// more threads are worth more than for more loads of each: one in flight at 40 (neighbours) or 48 registers (halves), against four at 64 and
// 108, 64 x 56 x 56 tokens, 2 + 2 heads of 32, us: 21.8 / 25.1 and 21.8 / 32.0; 16 x 1024, 12 + 12 heads of 64 26.8 / 32.4 and 23.9 / 36.9;
// in fp32 one in flight takes 36.7 / 34.5 there, 65537 tokens, 12 + 4 heads of 128 189 / 162.
// (Measured, B200, 64 x 56 x 56 tokens, 2 + 2 heads of 32, bf16, both ways / 65537 tokens, 12 + 4 heads of 128, fp32: tables in
// shared memory, a CTA per 64 or 2 tokens 98 / 213 us, CTAs that walk chunks of tokens 86 / 300 us.)
#include "bra_internal.h"
#include "fast_div.h"

#include <math.h>

namespace bra {
namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_ROUND = 4;           // units that make a thread's angles worth their while
template <typename T> constexpr int ROPE_AHEAD = sizeof(T) == 2 ? 1 : 4;        // units in flight per thread
// CTAs of an SM that registers have to allow
template <typename T, int VEC, bool HALF> constexpr int ROPE_CTAS = sizeof(T) == 2 && VEC >= 4 ? (HALF ? 5 : 6) : 1;

struct RopeArgs {
    const void *Q, *K;
    void *Qo, *Ko;
    const int32_t* positions;
    const double* freq;
    long long lanes;                    // threads that are needed: tokens with a position of their own, times units
    long long q_stride, k_stride;
    int N, heads, all_heads, D, rot, n, axes, width, first;
    int walk, part;                     // heads (of all images, where positions are implied) of a token, and of one part of them
    float magnitude, sine;              // sine: -1 for the inverse
    bool q_in_place, k_in_place;
    int units;                          // of a head
    FastDiv units_div, heads_div, width_div;
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
    static constexpr int PAIRS = HALF ? VEC : W / 2;
    Pack<T, VEC> a[W / VEC], b;
    T* dst;                             // null: nothing to do
    // turned: pairs of the unit that turn; whole: all its channels exist
    __device__ __forceinline__ void load(const T* src, T* to, int turned, bool whole, int half) {
        dst = to;
        if (HALF) {
            a[0] = *reinterpret_cast<const Pack<T, VEC>*>(src);
            if (turned) b = *reinterpret_cast<const Pack<T, VEC>*>(src + half);
        } else {
#pragma unroll
            for (int k = 0; k < W / VEC; ++k)
                if (VEC > 1 || k == 0 || whole) a[k] = *reinterpret_cast<const Pack<T, VEC>*>(src + k * VEC);
        }
    }
    __device__ __forceinline__ void finish(const float2 (&cs)[PAIRS], int turned, bool whole, int half) {
        if (HALF) {
            if (turned) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float u = to_f(a[0].v[e]), v = to_f(b.v[e]);
                    a[0].v[e] = from_f<T>(u * cs[e].x - v * cs[e].y);
                    b.v[e] = from_f<T>(u * cs[e].y + v * cs[e].x);
                }
                *reinterpret_cast<Pack<T, VEC>*>(dst + half) = b;
            }
            *reinterpret_cast<Pack<T, VEC>*>(dst) = a[0];
        } else {
#pragma unroll
            for (int e = 0; e < PAIRS; ++e)
                if (e < turned) {                                            // not the rest of a partly rotated unit
                    T& x = a[2 * e / VEC].v[2 * e % VEC];
                    T& y = a[(2 * e + 1) / VEC].v[(2 * e + 1) % VEC];
                    const float u = to_f(x), v = to_f(y);
                    x = from_f<T>(u * cs[e].x - v * cs[e].y);
                    y = from_f<T>(u * cs[e].y + v * cs[e].x);
                }
#pragma unroll
            for (int k = 0; k < W / VEC; ++k)
                if (VEC > 1 || k == 0 || whole) *reinterpret_cast<Pack<T, VEC>*>(dst + k * VEC) = a[k];
        }
    }
};

template <typename T, int VEC, bool HALF>
__global__ void __launch_bounds__(ROPE_THREADS, ROPE_CTAS<T, VEC, HALF>) rope_kernel(const RopeArgs g) {
    using U = Unit<T, VEC, HALF>;
    constexpr int AHEAD = ROPE_AHEAD<T>;
    const long long lane = (long long)blockIdx.x * ROPE_THREADS + threadIdx.x;
    if (lane >= g.lanes) return;
    const long long token = g.lanes <= 0x7fffffffll ? (long long)fdiv((uint32_t)lane, g.units_div) : lane / g.units;
    const int u = (int)(lane - token * g.units), half = g.n >> 1, pairs = g.rot >> 1;

    // the unit's first channel and pair, how many of its pairs turn
    int c, pair, turned;
    bool whole = true;
    if (HALF) {
        pair = u * VEC;
        turned = pair < pairs ? VEC : 0;
        c = turned ? pair + (pair >= half ? half : 0) : g.rot + pair - pairs;                 // at most two blocks
    } else {
        c = u * U::W;
        pair = c >> 1;
        turned = min(max(pairs - pair, 0), U::PAIRS);
        whole = c + U::W <= g.D;
    }
    float2 cs[U::PAIRS];
    if (turned) {
        const int axis = pair >= half ? 1 : 0;          // of the unit's first pair; an interleaved unit may reach into the next block
        int place[2];
        if (g.positions) {
            place[0] = __ldg(g.positions + token * g.axes);
            place[1] = g.axes == 2 ? __ldg(g.positions + token * 2 + 1) : 0;
        } else {
            const int row = g.axes == 2 ? (int)fdiv((uint32_t)token, g.width_div) : 0;
            place[0] = g.axes == 2 ? row : g.first + (int)token;
            place[1] = (int)token - row * g.width;
        }
#pragma unroll
        for (int e = 0; e < U::PAIRS; ++e) {
            if (e < turned) {
                const int ax = HALF ? axis : (pair + e >= half ? 1 : 0);
                // Turns per position as a fraction of 2^64: coordinate * that, modulo 2^64, is the angle without its whole turns, exactly.
                // (An infinite or NaN frequency leaves t NaN, which no integer can say.)
                double t = __ldg(g.freq + (pair + e - ax * half)) * 0.15915494309189533577;
                t -= floor(t);
                const unsigned long long step = t < 1.0 ? __double2ull_rn(t * 18446744073709551616.0) : 0ull;
                const unsigned long long angle = (unsigned long long)(long long)(ax ? place[1] : place[0]) * step;
                float sn, cn;
                sincospif((float)(int)(angle >> 32) * 4.656612873077392578125e-10f, &sn, &cn);      // 2^-31 half turns, in [-1, 1)
                const float nan = __int_as_float(0x7fffffff);
                cs[e] = t == t ? make_float2(cn * g.magnitude, sn * g.magnitude * g.sine) : make_float2(nan, nan);
            }
        }
    }

    int j = blockIdx.y * g.part;
    const int end = min(j + g.part, g.walk);
    int b = (int)fdiv((uint32_t)j, g.heads_div), h = j - b * g.all_heads;
    for (; j < end; j += AHEAD) {
        U unit[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            unit[k].dst = nullptr;
            if (j + k < end) {
                const bool of_q = h < g.heads;
                if (turned || !(of_q ? g.q_in_place : g.k_in_place)) {
                    const long long off = ((long long)b * g.N + token) * (of_q ? g.q_stride : g.k_stride) + (of_q ? h : h - g.heads) * g.D + c;
                    unit[k].load(static_cast<const T*>(of_q ? g.Q : g.K) + off, static_cast<T*>(of_q ? g.Qo : g.Ko) + off, turned, whole, half);
                }
                if (++h == g.all_heads) { h = 0; ++b; }
            }
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (unit[k].dst) unit[k].finish(cs, turned, whole, half);
    }
}

template <typename T, int VEC>
cudaError_t launch(const RopeArgs& a, bool half, dim3 ctas, cudaStream_t st) {
    if (half) rope_kernel<T, VEC, true><<<ctas, ROPE_THREADS, 0, st>>>(a);
    else      rope_kernel<T, VEC, false><<<ctas, ROPE_THREADS, 0, st>>>(a);
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
    a.q_stride = qs; a.k_stride = ks;
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
    a.units_div = fast_div(a.units);
    a.heads_div = fast_div(a.all_heads);
    a.width_div = fast_div(p->width > 0 ? p->width : 1);
    // Implied positions are the same in every image, and so are the angles.  Where tokens times units are fewer than the threads the
    // GPU holds twice, the walk over heads and images is split - down to one unit a thread, where even so there are too few to half fill it,
    // else in whole rounds (in single units / rounds, us: 16 x 1 token, 12 + 12 heads of 64 2.6 / 3.9, 4 x 999, 6 + 2 heads of 64, fp32 7.0 / 5.0,
    // 64 x 28 x 28, 4 + 4 heads of 32 15.5 / 14.2).
    const long long own = positions ? tokens : p->N;
    a.lanes = own * a.units;
    const long long walk = positions ? a.all_heads : (long long)p->B * a.all_heads;
    if (walk > (1 << 30)) return BRA_ERR_SHAPE;
    a.walk = (int)walk;
    const long long held = 2048ll * kSMs, want = (2 * held + a.lanes - 1) / a.lanes;
    long long part = (walk + want - 1) / want;
    if (a.lanes * walk >= held / 2) part = (part + ROPE_ROUND - 1) / ROPE_ROUND * ROPE_ROUND;
    const long long least = (walk + 65534) / 65535;
    part = part > least ? part : least;
    a.part = (int)part;
    const long long parts = (walk + part - 1) / part;
    const long long blocks = (a.lanes + ROPE_THREADS - 1) / ROPE_THREADS;
    if (blocks > 0x7fffffffll) return BRA_ERR_SHAPE;
    const dim3 ctas((unsigned)blocks, (unsigned)parts);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (p->dtype == BRA_BF16)
        e = vec == 8 ? launch<__nv_bfloat16, 8>(a, half, ctas, st)
          : vec == 4 ? launch<__nv_bfloat16, 4>(a, half, ctas, st)
          : vec == 2 ? launch<__nv_bfloat16, 2>(a, half, ctas, st)
                     : launch<__nv_bfloat16, 1>(a, half, ctas, st);
    else
        e = vec == 4 ? launch<float, 4>(a, half, ctas, st)
          : vec == 2 ? launch<float, 2>(a, half, ctas, st)
                     : launch<float, 1>(a, half, ctas, st);
    return e == cudaSuccess ? BRA_OK : BRA_ERR_CUDA;
}

}  // extern "C"
