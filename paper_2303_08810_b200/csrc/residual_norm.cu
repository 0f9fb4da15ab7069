// The norms on both sides of a block's end, fused with its gate and residual scale:
//   y' = post(y) * post_w + post_b,   h = alpha * x + gate * y',   n = pre(h) * w + b
// and the gradients of all of it.
//
// What bounds it: HBM.  A row is read once into registers - eight channels a thread - and normalised there: the variance is a second
// sum over the registers (of squared distances from the mean, so a large mean costs no precision), not a second read.  Rows of up to
// 256 channels belong to 1 to 32 lanes of a warp, several rows a warp; longer ones to a CTA of as many warps as they need, whose
// sums cross through shared memory, one barrier each.  The next row's loads are issued before this one's sums.
//
// The backward pass makes h again from x and y (both are read anyway for the norms' and the gate's gradients, and a rounded h would
// put its rounding into the fp32 gradients of the weights).  With hat the normalised row, r its factor and g = dn * w:
//   dH = dh + r (g - hat mean(g hat) [- mean(g)]),  dx = alpha dH,  dy' = gate dH,  and the same step again through post.
// Sums over tokens (weights, biases, gate) stay with the thread that owns the channel while its CTA walks a contiguous run of rows;
// each (CTA, image) it meets leaves one row of partial sums, and a second kernel adds those in order: no atomics, the same bits
// every time.  Run c of the rows meets image b at most once, and walking runs and images together raises c or b by at least one from
// one meeting to the next, so c + b numbers the meetings.
#include "bra_internal.h"

namespace bra {
namespace {

constexpr int NORM_E = 8;                   // channels of a thread
constexpr int NORM_MAX_C = 8192;

struct NormArgs {
    const void *x, *y, *dh, *dn;
    void *h, *n, *dx, *dy;
    const float *gate, *post_w, *post_b, *w, *b;
    float* part;                            // partial sums of the backward pass
    long long rows;
    int N;                                  // rows of an image
    int C;
    int group;                              // threads of a row
    int run;                                // rows of a CTA
    int gate_image, affine_image;           // [B, C] rather than [C]
    int pre, post;
    float eps, alpha;
    int sums;                               // which sums are wanted, SUM_* bits
    long long slots;
};

enum { SUM_W = 0, SUM_B = 1, SUM_GATE = 2, SUM_POST_W = 3, SUM_POST_B = 4, SUMS = 5 };

// ---------------------------------------------------------------- a thread's eight channels of a row
// VECD: neighbours (rows start on 16 bytes, C a multiple of eight).  Else channel j of thread t is t + j * group: neighbours over
// the threads.
template <typename T, bool VECD> struct Raw;
template <> struct Raw<__nv_bfloat16, true> { uint4 v; };
template <> struct Raw<float, true> { float4 v[2]; };
template <typename T> struct Raw<T, false> { T v[NORM_E]; };

template <bool VECD>
struct Cols {
    int t, group, C;
    __device__ __forceinline__ int at(int j) const { return VECD ? t * NORM_E + j : t + j * group; }
    __device__ __forceinline__ bool has(int j) const { return at(j) < C; }    // VECD: the same for every j
};

__device__ __forceinline__ void fetch(Raw<__nv_bfloat16, true>& r, const __nv_bfloat16* row, const Cols<true>& c) {
    r.v = make_uint4(0, 0, 0, 0);
    if (c.has(0)) r.v = __ldg(reinterpret_cast<const uint4*>(row + c.at(0)));
}
__device__ __forceinline__ void fetch(Raw<float, true>& r, const float* row, const Cols<true>& c) {
    r.v[0] = r.v[1] = make_float4(0, 0, 0, 0);
    if (c.has(0)) {
        r.v[0] = __ldg(reinterpret_cast<const float4*>(row + c.at(0)));
        r.v[1] = __ldg(reinterpret_cast<const float4*>(row + c.at(0)) + 1);
    }
}
template <typename T>
__device__ __forceinline__ void fetch(Raw<T, false>& r, const T* row, const Cols<false>& c) {
#pragma unroll
    for (int j = 0; j < NORM_E; ++j) r.v[j] = c.has(j) ? row[c.at(j)] : T(0.f);
}
__device__ __forceinline__ void widen(const Raw<__nv_bfloat16, true>& r, float* f) {
    const uint32_t w[4] = {r.v.x, r.v.y, r.v.z, r.v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen(const Raw<float, true>& r, float* f) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        f[4 * i] = r.v[i].x; f[4 * i + 1] = r.v[i].y; f[4 * i + 2] = r.v[i].z; f[4 * i + 3] = r.v[i].w;
    }
}
__device__ __forceinline__ void widen(const Raw<float, false>& r, float* f) {
#pragma unroll
    for (int j = 0; j < NORM_E; ++j) f[j] = r.v[j];
}
__device__ __forceinline__ void widen(const Raw<__nv_bfloat16, false>& r, float* f) {
#pragma unroll
    for (int j = 0; j < NORM_E; ++j) f[j] = __bfloat162float(r.v[j]);
}
template <typename T, bool VECD>
__device__ __forceinline__ void put(T* row, const float* f, const Cols<VECD>& c) {
    if constexpr (VECD) {
        if (c.has(0)) store_row<NORM_E>(row + c.at(0), f);
    } else {
#pragma unroll
        for (int j = 0; j < NORM_E; ++j)
            if (c.has(j)) {
                if constexpr (sizeof(T) == 2) row[c.at(j)] = __float2bfloat16_rn(f[j]);
                else row[c.at(j)] = f[j];
            }
    }
}
// a vector of C floats; `none` where it is not given
template <bool VECD>
__device__ __forceinline__ void weights(const float* p, float none, float* f, const Cols<VECD>& c) {
#pragma unroll
    for (int j = 0; j < NORM_E; ++j) f[j] = none;
    if (!p) return;
    if constexpr (VECD) {
        if (c.has(0)) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(p + c.at(0))), b = __ldg(reinterpret_cast<const float4*>(p + c.at(0)) + 1);
            f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < NORM_E; ++j) if (c.has(j)) f[j] = __ldg(p + c.at(j));
    }
}

__device__ __forceinline__ const float* row_of(const float* p, long long off) { return p ? p + off : nullptr; }

// ---------------------------------------------------------------- sums over a row
// WIDE: the row is the CTA's.  The buffers of two consecutive sums are different ones, so that one barrier a sum is enough.
template <bool WIDE>
struct RowSum {
    int group;
    float (*cross)[32][2];                  // [2][warps][values]
    int turn = 0;
    __device__ __forceinline__ float2 of(float a, float b) {
        const int width = WIDE ? 32 : group;
        for (int o = width >> 1; o; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        if (WIDE) {
            const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = group >> 5;
            if (lane == 0) { cross[turn][warp][0] = a; cross[turn][warp][1] = b; }
            __syncthreads();
            a = lane < warps ? cross[turn][lane][0] : 0.f;
            b = lane < warps ? cross[turn][lane][1] : 0.f;
            turn ^= 1;
#pragma unroll
            for (int o = 16; o; o >>= 1) {
                a += __shfl_xor_sync(0xffffffffu, a, o);
                b += __shfl_xor_sync(0xffffffffu, b, o);
            }
        }
        return make_float2(a, b);
    }
    __device__ __forceinline__ float of(float a) {
        const int width = WIDE ? 32 : group;
        for (int o = width >> 1; o; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
        if (WIDE) {
            const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = group >> 5;
            if (lane == 0) cross[turn][warp][0] = a;
            __syncthreads();
            a = lane < warps ? cross[turn][lane][0] : 0.f;
            turn ^= 1;
#pragma unroll
            for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
        }
        return a;
    }
};

// v becomes its normalised form; the factor is returned.  Channels that do not exist hold zeros and keep them.
template <bool WIDE, bool VECD>
__device__ __forceinline__ float normalise(int kind, float* v, const Cols<VECD>& c, float eps, RowSum<WIDE>& sum) {
    if (kind == BRA_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < NORM_E; ++j) s += v[j];
        const float mean = sum.of(s) / (float)c.C;
#pragma unroll
        for (int j = 0; j < NORM_E; ++j) v[j] = c.has(j) ? v[j] - mean : 0.f;
    }
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < NORM_E; ++j) s = fmaf(v[j], v[j], s);
    const float r = rsqrtf(sum.of(s) / (float)c.C + eps);
#pragma unroll
    for (int j = 0; j < NORM_E; ++j) v[j] *= r;
    return r;
}

// g becomes the gradient of the row whose normalised form hat had the gradient g
template <bool WIDE, bool VECD>
__device__ __forceinline__ void normalise_back(int kind, float* g, const float* hat, float r, const Cols<VECD>& c, RowSum<WIDE>& sum) {
    float a = 0.f, b = 0.f;
#pragma unroll
    for (int j = 0; j < NORM_E; ++j) { a = fmaf(g[j], hat[j], a); b += g[j]; }
    float2 m;
    if (kind == BRA_NORM_LAYER) m = sum.of(a, b);
    else m = make_float2(sum.of(a), 0.f);
    const float along = m.x / (float)c.C, mean = m.y / (float)c.C;
#pragma unroll
    for (int j = 0; j < NORM_E; ++j) g[j] = c.has(j) ? r * (g[j] - hat[j] * along - mean) : 0.f;
}

// ---------------------------------------------------------------- forward
// A CTA's groups take the rows of its run in turn.  All groups make the same number of rounds (idle ones on the last row,
// storing nothing), so that the shuffles and barriers of the sums are met by every thread.
// THREADS: the most a CTA has.  Above 512 a thread has 64 registers: weights are read where they are used, row by row.
template <typename T, bool VECD, bool WIDE, bool POST, int THREADS>
__global__ void __launch_bounds__(THREADS) norm_forward_kernel(const NormArgs a) {
    constexpr bool KEEP = THREADS <= 512;
    __shared__ float cross[2][32][2];
    const int groups = WIDE ? 1 : blockDim.x / a.group;
    const int mine = WIDE ? 0 : threadIdx.x / a.group;
    Cols<VECD> c{WIDE ? (int)threadIdx.x : (int)threadIdx.x % a.group, a.group, a.C};
    RowSum<WIDE> sum{a.group, cross};
    const long long first = (long long)blockIdx.x * a.run;
    const long long last = min(first + a.run, a.rows) - 1;
    const T *x = static_cast<const T*>(a.x), *y = static_cast<const T*>(a.y);

    Raw<T, VECD> rx, ry;
    {
        const long long row = min(first + mine, last);
        fetch(rx, x + row * a.C, c);
        if (y) fetch(ry, y + row * a.C, c);
    }
    const bool per_image = a.gate_image || a.affine_image;
    long long image_end = -1;                                 // last row whose image's weights are held
    float gate[NORM_E], pw[NORM_E], pb[NORM_E], w[NORM_E], b[NORM_E];
    const float *gate_p = a.gate, *w_p = a.w, *b_p = a.b;
    if (POST && KEEP) {
        weights<VECD>(a.post_w, 1.f, pw, c);
        weights<VECD>(a.post_b, 0.f, pb, c);
    }
    for (long long row0 = first; row0 <= last; row0 += groups) {
        const long long row = min(row0 + mine, last);
        const bool live = row0 + mine <= last;
        if (row > image_end) {
            const long long image = per_image ? row / a.N : 0;
            gate_p = row_of(a.gate, a.gate_image ? image * a.C : 0);
            w_p = row_of(a.w, a.affine_image ? image * a.C : 0);
            b_p = row_of(a.b, a.affine_image ? image * a.C : 0);
            if (KEEP) {
                weights<VECD>(gate_p, 1.f, gate, c);
                weights<VECD>(w_p, 1.f, w, c);
                weights<VECD>(b_p, 0.f, b, c);
            }
            image_end = per_image ? (image + 1) * a.N - 1 : last;
        }
        float v[NORM_E], u[NORM_E];
        widen(rx, v);
        if (y) widen(ry, u);
        if (row0 + groups <= last) {
            const long long next = min(row0 + groups + mine, last);
            fetch(rx, x + next * a.C, c);
            if (y) fetch(ry, y + next * a.C, c);
        }
        if (y) {
            if (POST) {
                normalise<WIDE>(a.post, u, c, a.eps, sum);
                if (!KEEP) { weights<VECD>(a.post_w, 1.f, pw, c); weights<VECD>(a.post_b, 0.f, pb, c); }
#pragma unroll
                for (int j = 0; j < NORM_E; ++j) u[j] = fmaf(u[j], pw[j], pb[j]);
            }
            if (!KEEP) weights<VECD>(gate_p, 1.f, gate, c);
#pragma unroll
            for (int j = 0; j < NORM_E; ++j) v[j] = c.has(j) ? fmaf(gate[j], u[j], a.alpha * v[j]) : 0.f;
        } else {
#pragma unroll
            for (int j = 0; j < NORM_E; ++j) v[j] *= a.alpha;
        }
        if (a.h && live) put<T, VECD>(static_cast<T*>(a.h) + row * a.C, v, c);
        if (a.pre != BRA_NORM_NONE) {
            normalise<WIDE>(a.pre, v, c, a.eps, sum);
            if (!KEEP) { weights<VECD>(w_p, 1.f, w, c); weights<VECD>(b_p, 0.f, b, c); }
#pragma unroll
            for (int j = 0; j < NORM_E; ++j) v[j] = fmaf(v[j], w[j], b[j]);
            if (live) put<T, VECD>(static_cast<T*>(a.n) + row * a.C, v, c);
        }
    }
}

// ---------------------------------------------------------------- backward
// KEEP: the sums over tokens stay in registers, and so do the weights.  Else (long rows, whose CTAs would have no registers left)
// the sums are in shared memory, each word its thread's own, and the weights are read again for every row.
template <typename T, bool VECD, bool WIDE, bool POST, int THREADS>
__global__ void __launch_bounds__(THREADS) norm_backward_kernel(const NormArgs a) {
    constexpr bool KEEP = THREADS == 128, AHEAD = THREADS <= 512;
    __shared__ float cross[2][32][2];
    extern __shared__ float sums_sh[];      // !KEEP: [SUMS][E][threads]; KEEP and several groups: [E][threads], to join the groups
    const int groups = WIDE ? 1 : blockDim.x / a.group;
    const int mine = WIDE ? 0 : threadIdx.x / a.group;
    Cols<VECD> c{WIDE ? (int)threadIdx.x : (int)threadIdx.x % a.group, a.group, a.C};
    RowSum<WIDE> sum{a.group, cross};
    const T *x = static_cast<const T*>(a.x), *y = static_cast<const T*>(a.y);
    const T *dh = static_cast<const T*>(a.dh), *dn = static_cast<const T*>(a.dn);
    const long long first = (long long)blockIdx.x * a.run;
    const long long last = min(first + a.run, a.rows) - 1;

    float acc[KEEP ? SUMS : 1][NORM_E] = {};
    auto shared_sum = [&](int s, int j) -> float& { return sums_sh[(s * NORM_E + j) * blockDim.x + threadIdx.x]; };
    auto add = [&](int s, int j, float v) {
        if constexpr (KEEP) acc[s][j] += v;
        else shared_sum(s, j) += v;
    };
    auto clear = [&](int s) {
#pragma unroll
        for (int j = 0; j < NORM_E; ++j) {
            if constexpr (KEEP) acc[s][j] = 0.f;
            else shared_sum(s, j) = 0.f;
        }
    };
    // this CTA's sum s, over its groups, into slot `slot`
    auto leave = [&](int s, long long slot) {
        float* to = a.part + ((size_t)s * a.slots + slot) * a.C;
        if (!WIDE && KEEP) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < NORM_E; ++j) sums_sh[j * blockDim.x + threadIdx.x] = acc[KEEP ? s : 0][j];
            __syncthreads();
            if (mine == 0) {
#pragma unroll
                for (int j = 0; j < NORM_E; ++j) {
                    float t = 0.f;
                    for (int g = 0; g < groups; ++g) t += sums_sh[j * blockDim.x + g * a.group + threadIdx.x];
                    if (c.has(j)) to[c.at(j)] = t;
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < NORM_E; ++j)
                if (c.has(j)) {
                    if constexpr (KEEP) to[c.at(j)] = acc[s][j];
                    else to[c.at(j)] = shared_sum(s, j);
                }
        }
        clear(s);
    };
    auto wants = [&](int s) { return (a.sums >> s) & 1; };
    auto of_image = [&](int s) { return s == SUM_GATE ? a.gate_image : s <= SUM_B ? a.affine_image : 0; };
    if constexpr (!KEEP) {
#pragma unroll
        for (int s = 0; s < SUMS; ++s) clear(s);
    }

    float gate[NORM_E], pw[NORM_E], pb[NORM_E], w[NORM_E];
    const bool per_image = a.gate_image || a.affine_image;
    long long begin = first;
    while (begin <= last) {                                   // the rows of one image
        const long long image = per_image ? begin / a.N : 0;
        const long long end = per_image ? min((image + 1) * a.N - 1, last) : last;
        const float* gate_p = row_of(a.gate, a.gate_image ? image * a.C : 0);
        const float* w_p = row_of(a.w, a.affine_image ? image * a.C : 0);
        if (KEEP) {
            weights<VECD>(gate_p, 1.f, gate, c);
            weights<VECD>(w_p, 1.f, w, c);
            if (POST) { weights<VECD>(a.post_w, 1.f, pw, c); weights<VECD>(a.post_b, 0.f, pb, c); }
        }
        Raw<T, VECD> rx, ry, rh, rn;
        auto get = [&](long long row) {
            fetch(rx, x + row * a.C, c);
            if (y) fetch(ry, y + row * a.C, c);
            if (dh) fetch(rh, dh + row * a.C, c);
            if (dn) fetch(rn, dn + row * a.C, c);
        };
        if (AHEAD) get(min(begin + mine, end));
        for (long long row0 = begin; row0 <= end; row0 += groups) {
            const long long row = min(row0 + mine, end);
            const bool live = row0 + mine <= end;
            float v[NORM_E], u[NORM_E], g[NORM_E], d[NORM_E];
            if (!AHEAD) get(row);
            widen(rx, v);
            if (y) widen(ry, u);
            if (dh) widen(rh, d);
            else {
#pragma unroll
                for (int j = 0; j < NORM_E; ++j) d[j] = 0.f;
            }
            if (dn) widen(rn, g);
            if (AHEAD && row0 + groups <= end) get(min(row0 + groups + mine, end));
            // !KEEP: the weights, as they are used
            auto post_weights = [&] { if (!KEEP && POST) { weights<VECD>(a.post_w, 1.f, pw, c); weights<VECD>(a.post_b, 0.f, pb, c); } };
            float ry_factor = 0.f;
            if (y) {
                if (POST) ry_factor = normalise<WIDE>(a.post, u, c, a.eps, sum);
                post_weights();
                if (!KEEP) weights<VECD>(gate_p, 1.f, gate, c);
#pragma unroll
                for (int j = 0; j < NORM_E; ++j)
                    v[j] = c.has(j) ? fmaf(gate[j], POST ? fmaf(u[j], pw[j], pb[j]) : u[j], a.alpha * v[j]) : 0.f;
            } else {
#pragma unroll
                for (int j = 0; j < NORM_E; ++j) v[j] *= a.alpha;
            }
            if (dn) {
                const float r = normalise<WIDE>(a.pre, v, c, a.eps, sum);
                if (!KEEP) weights<VECD>(w_p, 1.f, w, c);
#pragma unroll
                for (int j = 0; j < NORM_E; ++j) {
                    if (live) {
                        if (wants(SUM_W)) add(SUM_W, j, g[j] * v[j]);
                        if (wants(SUM_B)) add(SUM_B, j, g[j]);
                    }
                    g[j] *= w[j];
                }
                normalise_back<WIDE>(a.pre, g, v, r, c, sum);
#pragma unroll
                for (int j = 0; j < NORM_E; ++j) d[j] += g[j];
            }
            // d = dH
#pragma unroll
            for (int j = 0; j < NORM_E; ++j) v[j] = a.alpha * d[j];
            if (live) put<T, VECD>(static_cast<T*>(a.dx) + row * a.C, v, c);
            if (y) {
                post_weights();
                if (!KEEP) weights<VECD>(gate_p, 1.f, gate, c);
#pragma unroll
                for (int j = 0; j < NORM_E; ++j) {
                    if (live && wants(SUM_GATE)) add(SUM_GATE, j, d[j] * (POST ? fmaf(u[j], pw[j], pb[j]) : u[j]));
                    d[j] *= gate[j];
                    if (POST && live) {
                        if (wants(SUM_POST_W)) add(SUM_POST_W, j, d[j] * u[j]);
                        if (wants(SUM_POST_B)) add(SUM_POST_B, j, d[j]);
                    }
                }
                if (POST) {
#pragma unroll
                    for (int j = 0; j < NORM_E; ++j) d[j] = c.has(j) ? d[j] * pw[j] : 0.f;
                    normalise_back<WIDE>(a.post, d, u, ry_factor, c, sum);
                }
                if (live) put<T, VECD>(static_cast<T*>(a.dy) + row * a.C, d, c);
            }
        }
        if (per_image) {
#pragma unroll
            for (int s = 0; s < SUMS; ++s)
                if (wants(s) && of_image(s)) leave(s, (long long)blockIdx.x + image);
        }
        begin = end + 1;
    }
#pragma unroll
    for (int s = 0; s < SUMS; ++s)
        if (wants(s) && !of_image(s)) leave(s, blockIdx.x);
}

struct JoinArgs {
    const float* part;
    float* out[SUMS];
    long long slots, rows;
    int N, C, run, ctas, images;
    int image_sum[SUMS];                    // [B, C] rather than [C]
    int which[SUMS];
};

// Adds the partial sums in order: 32 channels a CTA, eight threads a channel, each every eighth slot.
__global__ void __launch_bounds__(256) norm_join_kernel(const JoinArgs a) {
    __shared__ float part[8][33];
    const int s = a.which[blockIdx.y];
    const int lane = threadIdx.x & 31, eighth = threadIdx.x >> 5;
    const int ch = blockIdx.x * 32 + lane;
    const int images = a.image_sum[s] ? a.images : 1;
    for (int image = blockIdx.z; image < images; image += gridDim.z) {
        long long c0 = 0, c1 = a.ctas - 1, slot = 0;
        if (a.image_sum[s]) {
            c0 = (long long)image * a.N / a.run;
            c1 = ((long long)(image + 1) * a.N - 1) / a.run;
            slot = image;
        }
        float t = 0.f;
        if (ch < a.C)
            for (long long c = c0 + eighth; c <= c1; c += 8) t += a.part[((size_t)s * a.slots + slot + c) * a.C + ch];
        part[eighth][lane] = t;
        __syncthreads();
        if (eighth == 0 && ch < a.C) {
#pragma unroll
            for (int k = 1; k < 8; ++k) t += part[k][lane];
            a.out[s][(size_t)(a.image_sum[s] ? image : 0) * a.C + ch] = t;
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------- host
struct Plan {
    int group, threads;
    bool wide;
    int run;                // rows of a CTA
    long long ctas;
};

Plan plan(long long rows, int C, bool backward) {
    Plan p;
    const int need = (C + NORM_E - 1) / NORM_E;
    p.wide = need > 32;
    if (p.wide) {
        p.group = (need + 31) / 32 * 32;
        p.threads = p.group;
    } else {
        p.group = 1;
        while (p.group < need) p.group <<= 1;
        p.threads = 128;
    }
    const int groups = p.wide ? 1 : p.threads / p.group;
    // about as many CTAs as the GPU holds at a time (registers: 128 to 160 a thread backwards, half of that forwards)
    long long most = (long long)kSMs * (p.threads <= 128 ? (backward ? 3 : 8) : p.threads <= 256 ? (backward ? 2 : 4) : backward ? 1 : 2);
    const long long rounds = (rows + groups - 1) / groups;
    if (most > rounds) most = rounds;
    const long long each = (rounds + most - 1) / most;
    p.run = (int)(each * groups);
    p.ctas = (rows + p.run - 1) / p.run;
    return p;
}

bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bra_status check(const bra_norm_problem* p) {
    if (!p) return BRA_ERR_NULL;
    if (p->B <= 0 || p->N <= 0 || p->C <= 0) return BRA_ERR_SHAPE;
    if ((long long)p->B * p->N >= (1ll << 40) / p->C) return BRA_ERR_SHAPE;
    if ((long long)p->B * p->N > 0x7fffffffll) return BRA_ERR_SHAPE;
    if (p->dtype != BRA_F32 && p->dtype != BRA_BF16) return BRA_ERR_DTYPE;
    if (p->pre < BRA_NORM_NONE || p->pre > BRA_NORM_LAYER || p->post < BRA_NORM_NONE || p->post > BRA_NORM_LAYER) return BRA_ERR_UNSUPPORTED;
    if (p->gate < BRA_GATE_NONE || p->gate > BRA_GATE_IMAGE) return BRA_ERR_UNSUPPORTED;
    if (p->C > NORM_MAX_C) return BRA_ERR_UNSUPPORTED;
    if (!(p->eps >= 0.f)) return BRA_ERR_SHAPE;
    return BRA_OK;
}

NormArgs args_of(const bra_norm_problem* p, const Plan& pl) {
    NormArgs a = {};
    a.rows = (long long)p->B * p->N;
    a.N = p->N; a.C = p->C; a.group = pl.group; a.run = pl.run;
    a.gate_image = p->gate == BRA_GATE_IMAGE; a.affine_image = p->per_image != 0;
    a.pre = p->pre; a.post = p->post; a.eps = p->eps; a.alpha = p->alpha;
    return a;
}

long long slots_of(const bra_norm_problem* p, const Plan& pl) {
    return pl.ctas + ((p->gate == BRA_GATE_IMAGE || p->per_image) ? p->B : 0);
}

template <typename T, bool VECD, bool WIDE, int THREADS>
cudaError_t forward_as(const NormArgs& a, const Plan& pl, cudaStream_t st) {
    if (a.post != BRA_NORM_NONE) norm_forward_kernel<T, VECD, WIDE, true, THREADS><<<(unsigned)pl.ctas, pl.threads, 0, st>>>(a);
    else                         norm_forward_kernel<T, VECD, WIDE, false, THREADS><<<(unsigned)pl.ctas, pl.threads, 0, st>>>(a);
    count_launch();
    return cudaGetLastError();
}
template <typename T, bool VECD>
cudaError_t forward(const NormArgs& a, const Plan& pl, cudaStream_t st) {
    if (!pl.wide) return forward_as<T, VECD, false, 128>(a, pl, st);
    if (pl.threads <= 128) return forward_as<T, VECD, true, 128>(a, pl, st);
    return pl.threads <= 512 ? forward_as<T, VECD, true, 512>(a, pl, st) : forward_as<T, VECD, true, 1024>(a, pl, st);
}

template <typename T, bool VECD, bool WIDE, bool POST, int THREADS>
cudaError_t backward_post(const NormArgs& a, const Plan& pl, cudaStream_t st) {
    constexpr bool KEEP = THREADS == 128;
    const size_t smem = sizeof(float) * NORM_E * pl.threads * (KEEP ? (WIDE ? 0 : 1) : SUMS);
    if (!KEEP) {
        static PerDeviceMax attr;
        const cudaError_t e = attr.ensure((int)smem, [&] {
            return cudaFuncSetAttribute(norm_backward_kernel<T, VECD, WIDE, POST, THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        });
        if (e != cudaSuccess) return e;
    }
    norm_backward_kernel<T, VECD, WIDE, POST, THREADS><<<(unsigned)pl.ctas, pl.threads, smem, st>>>(a);
    count_launch();
    return cudaGetLastError();
}
template <typename T, bool VECD, bool WIDE, int THREADS>
cudaError_t backward_as(const NormArgs& a, const Plan& pl, cudaStream_t st) {
    return a.post != BRA_NORM_NONE ? backward_post<T, VECD, WIDE, true, THREADS>(a, pl, st) : backward_post<T, VECD, WIDE, false, THREADS>(a, pl, st);
}
template <typename T, bool VECD>
cudaError_t backward(const NormArgs& a, const Plan& pl, cudaStream_t st) {
    if (!pl.wide) return backward_as<T, VECD, false, 128>(a, pl, st);
    if (pl.threads <= 128) return backward_as<T, VECD, true, 128>(a, pl, st);
    return pl.threads <= 512 ? backward_as<T, VECD, true, 512>(a, pl, st) : backward_as<T, VECD, true, 1024>(a, pl, st);
}

bool vectors(const bra_norm_problem* p) { return p->C % NORM_E == 0; }

}  // namespace
}  // namespace bra

using namespace bra;

extern "C" {

size_t bra_norm_workspace_bytes(const bra_norm_problem* p) {
    if (check(p) != BRA_OK) return 0;
    const Plan pl = plan((long long)p->B * p->N, p->C, true);
    return (sizeof(float) * SUMS * (size_t)slots_of(p, pl) * p->C + 255) & ~size_t(255);
}

bra_status bra_residual_norm(const bra_norm_problem* p, const void* x, const void* y, const float* gate,
                             const float* post_w, const float* post_b, const float* w, const float* b,
                             void* h, void* n, void* stream) {
    reset_launch_count();
    bra_status s = check(p);
    if (s != BRA_OK) return s;
    if (!x || (!h && !n)) return BRA_ERR_NULL;
    if ((p->pre != BRA_NORM_NONE) != (n != nullptr)) return BRA_ERR_NULL;
    if ((p->gate != BRA_GATE_NONE) != (gate != nullptr)) return BRA_ERR_NULL;
    if (!y && (p->gate != BRA_GATE_NONE || p->post != BRA_NORM_NONE)) return BRA_ERR_NULL;
    for (const void* q : {x, y, (const void*)h, (const void*)n, (const void*)gate, (const void*)post_w, (const void*)post_b, (const void*)w, (const void*)b})
        if (!aligned_to(q, 16)) return BRA_ERR_ALIGN;
    if (n == x || n == y || n == h) return BRA_ERR_UNSUPPORTED;
    const Plan pl = plan((long long)p->B * p->N, p->C, false);
    NormArgs a = args_of(p, pl);
    a.x = x; a.y = y; a.gate = gate; a.post_w = post_w; a.post_b = post_b; a.w = w; a.b = b; a.h = h; a.n = n;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (p->dtype == BRA_BF16) e = vectors(p) ? forward<__nv_bfloat16, true>(a, pl, st) : forward<__nv_bfloat16, false>(a, pl, st);
    else                      e = vectors(p) ? forward<float, true>(a, pl, st) : forward<float, false>(a, pl, st);
    return e == cudaSuccess ? BRA_OK : BRA_ERR_CUDA;
}

bra_status bra_residual_norm_backward(const bra_norm_problem* p, const void* x, const void* y, const float* gate,
                                      const float* post_w, const float* post_b, const float* w,
                                      const void* dh, const void* dn, void* dx, void* dy, float* d_gate,
                                      float* d_post_w, float* d_post_b, float* d_w, float* d_b,
                                      void* ws, size_t ws_bytes, void* stream) {
    reset_launch_count();
    bra_status s = check(p);
    if (s != BRA_OK) return s;
    if (!x || !dx || (!dh && !dn)) return BRA_ERR_NULL;
    if ((p->pre != BRA_NORM_NONE) != (dn != nullptr) || (y != nullptr) != (dy != nullptr)) return BRA_ERR_NULL;
    if ((p->gate != BRA_GATE_NONE) != (gate != nullptr)) return BRA_ERR_NULL;
    if (!y && (p->gate != BRA_GATE_NONE || p->post != BRA_NORM_NONE)) return BRA_ERR_NULL;
    if ((d_gate && p->gate == BRA_GATE_NONE) || ((d_post_w || d_post_b) && p->post == BRA_NORM_NONE) ||
        ((d_w || d_b) && p->pre == BRA_NORM_NONE))
        return BRA_ERR_UNSUPPORTED;
    for (const void* q : {x, y, dh, dn, (const void*)dx, (const void*)dy, (const void*)gate, (const void*)post_w, (const void*)post_b,
                          (const void*)w, (const void*)d_gate, (const void*)d_post_w, (const void*)d_post_b, (const void*)d_w, (const void*)d_b})
        if (!aligned_to(q, 16)) return BRA_ERR_ALIGN;
    if (dx == dy) return BRA_ERR_UNSUPPORTED;
    for (const void* q : {x, y, dh, dn})
        if (q && (q == dx || q == dy)) return BRA_ERR_UNSUPPORTED;      // rows are read ahead of the ones written
    if (!ws) return BRA_ERR_NULL;
    if (!aligned_to(ws, 256)) return BRA_ERR_ALIGN;
    if (ws_bytes < bra_norm_workspace_bytes(p)) return BRA_ERR_WORKSPACE;
    const Plan pl = plan((long long)p->B * p->N, p->C, true);
    NormArgs a = args_of(p, pl);
    a.x = x; a.y = y; a.gate = gate; a.post_w = post_w; a.post_b = post_b; a.w = w; a.dh = dh; a.dn = dn; a.dx = dx; a.dy = dy;
    a.part = static_cast<float*>(ws);
    a.slots = slots_of(p, pl);
    JoinArgs j = {};
    j.part = a.part; j.slots = a.slots; j.rows = a.rows; j.N = p->N; j.C = p->C; j.run = pl.run; j.ctas = (int)pl.ctas; j.images = p->B;
    float* outs[SUMS] = {d_w, d_b, d_gate, d_post_w, d_post_b};
    const int of_image[SUMS] = {a.affine_image, a.affine_image, a.gate_image, 0, 0};
    int wanted = 0, most_images = 1;
    for (int k = 0; k < SUMS; ++k) {
        j.out[k] = outs[k];
        j.image_sum[k] = of_image[k];
        if (!outs[k]) continue;
        a.sums |= 1 << k;
        j.which[wanted++] = k;
        if (of_image[k]) most_images = p->B;
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (p->dtype == BRA_BF16) e = vectors(p) ? backward<__nv_bfloat16, true>(a, pl, st) : backward<__nv_bfloat16, false>(a, pl, st);
    else                      e = vectors(p) ? backward<float, true>(a, pl, st) : backward<float, false>(a, pl, st);
    if (e != cudaSuccess) return BRA_ERR_CUDA;
    if (wanted) {
        const dim3 grid((p->C + 31) / 32, wanted, most_images < GRID_YZ ? most_images : GRID_YZ);
        norm_join_kernel<<<grid, 256, 0, st>>>(j);
        count_launch();
        if (cudaGetLastError() != cudaSuccess) return BRA_ERR_CUDA;
    }
    return BRA_OK;
}

}  // extern "C"
