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
#include "sm100_ptx.cuh"

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

// Eight channels of a thread as four pairs: packed fp32 arithmetic halves the instructions, which are what bounds short rows
// (498 a round of four 64-channel rows before, at 0.63 issued per cycle and scheduler).
struct Eight {
    float2 v[4];
    __device__ __forceinline__ void fill(float f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = make_float2(f, f);
    }
};
__device__ __forceinline__ float2 both(float f) { return make_float2(f, f); }
__device__ __forceinline__ float total(const Eight& a) {
    const float2 s = __fadd2_rn(__fadd2_rn(a.v[0], a.v[1]), __fadd2_rn(a.v[2], a.v[3]));
    return s.x + s.y;
}
__device__ __forceinline__ float dot(const Eight& a, const Eight& b) {
    float2 s = __fmul2_rn(a.v[0], b.v[0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) s = __ffma2_rn(a.v[i], b.v[i], s);
    return s.x + s.y;
}

// ---------------------------------------------------------------- a thread's eight channels of a row
// VECD: neighbours (rows start on 16 bytes, C a multiple of eight).  Else channel j of thread t is t + j * group: neighbours over
// the threads.
template <bool VECD>
struct Cols {
    int t, group, C;
    bool any;                               // VECD: whether these channels exist, all or none
    __device__ __forceinline__ Cols(int t_, int group_, int C_) : t(t_), group(group_), C(C_), any(t_ * NORM_E < C_) {}
    __device__ __forceinline__ int at(int j) const { return VECD ? t * NORM_E + j : t + j * group; }
    __device__ __forceinline__ bool has(int j) const { return VECD ? any : at(j) < C; }
    // f for channels that exist, 0 for the others
    __device__ __forceinline__ float2 only(float f, int i) const {
        return VECD ? both(any ? f : 0.f) : make_float2(has(2 * i) ? f : 0.f, has(2 * i + 1) ? f : 0.f);
    }
};

__device__ __forceinline__ void widen(const uint32_t (&w)[4], Eight& f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}

// How far rows are read ahead: through a ring in shared memory whose 16- or 4-byte slots are each one thread's own, so that neither
// registers nor barriers are spent on rows in flight; one slot more than rows in flight, so that none is written that was read in the
// same round.  Rows of bf16 that start on two bytes cannot be copied so (four at least) and go through registers, one row ahead.
// DEPTH: rows in flight, as many as shared memory has room for; 0: rows are read when it is their turn.
template <typename T, bool VECD, int TENSORS, int DEPTH>
struct Ahead {
    static constexpr bool RING = DEPTH > 0 && (VECD || sizeof(T) == 4);
    static constexpr int ROWS = RING || DEPTH == 0 ? DEPTH : 1;
    static constexpr int CHUNKS = VECD ? NORM_E * (int)sizeof(T) / 16 : NORM_E, CHUNK = VECD ? 16 : 4;
    static constexpr size_t bytes(int threads) { return RING ? (size_t)(DEPTH + 1) * TENSORS * NORM_E * sizeof(T) * threads : 0; }
    T raw[RING || DEPTH == 0 ? 1 : TENSORS][NORM_E];
    const T* row[TENSORS];                  // of the row that is fetched next, at this thread's first channel; null: no such tensor
    uint32_t base, pitch;                   // this thread's first slot, bytes between its chunks
    uint32_t get = 0, put = 0;              // offsets of the rows that are read and fetched next
    __device__ __forceinline__ void restart() { get = put; }         // nothing that was fetched is left to read
    __device__ __forceinline__ explicit Ahead(const void* smem) : base(ptx::smem_u32(smem) + threadIdx.x * CHUNK), pitch(blockDim.x * CHUNK) {}
    __device__ __forceinline__ uint32_t step(uint32_t at) const {
        at += TENSORS * CHUNKS * pitch;
        return at == (DEPTH + 1) * TENSORS * CHUNKS * pitch ? 0 : at;
    }
    // fetches a row of every tensor (live: it exists) and moves on by `stride` elements
    __device__ __forceinline__ void fetch(bool live, long long stride, const Cols<VECD>& c) {
#pragma unroll
        for (int k = 0; k < TENSORS; ++k) {
            if (!row[k]) continue;
            if (live) {
                if constexpr (RING) {
                    const uint32_t to = base + put + k * CHUNKS * pitch;
#pragma unroll
                    for (int j = 0; j < CHUNKS; ++j) {
                        if constexpr (VECD) ptx::cp_async_16(to + j * pitch, c.any ? row[k] + j * (16 / (int)sizeof(T)) : row[k] - c.at(0), c.any ? 16 : 0);
                        else ptx::cp_async_4(to + j * pitch, c.has(j) ? row[k] + j * c.group : row[k] - c.t, c.has(j) ? 4 : 0);
                    }
                } else if constexpr (DEPTH > 0) {
#pragma unroll
                    for (int j = 0; j < NORM_E; ++j) raw[k][j] = c.has(j) ? row[k][j * c.group] : T(0.f);
                }
            }
            row[k] += stride;
        }
        if (RING) {
            ptx::cp_async_commit();
            put = step(put);
        }
    }
    __device__ __forceinline__ void arrived() { if constexpr (RING) ptx::cp_async_wait<DEPTH - 1>(); }
    __device__ __forceinline__ void read(int tensor, Eight& f, const Cols<VECD>& c) const {
        if constexpr (DEPTH == 0) {
            float v[NORM_E] = {};
            if constexpr (VECD) {
                if (c.any) load_row<NORM_E>(row[tensor], v);
            } else {
#pragma unroll
                for (int j = 0; j < NORM_E; ++j) if (c.has(j)) v[j] = (float)row[tensor][j * c.group];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) f.v[i] = make_float2(v[2 * i], v[2 * i + 1]);
        } else if constexpr (RING) {
            const uint32_t from = base + get + tensor * CHUNKS * pitch;
            if constexpr (VECD && sizeof(T) == 2) {
                const float4 v = ptx::lds_f32x4(from);
                widen({__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w)}, f);
            } else if constexpr (VECD) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float4 v = ptx::lds_f32x4(from + k * pitch);
                    f.v[2 * k] = make_float2(v.x, v.y);
                    f.v[2 * k + 1] = make_float2(v.z, v.w);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) f.v[i] = make_float2(ptx::lds_f32(from + 2 * i * pitch), ptx::lds_f32(from + (2 * i + 1) * pitch));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) f.v[i] = make_float2(__bfloat162float(raw[tensor][2 * i]), __bfloat162float(raw[tensor][2 * i + 1]));
        }
    }
    __device__ __forceinline__ void next() { if (RING) get = step(get); }
};

// 4096 channels of fp32 backwards: 82 KB of sums and a ring of 131 KB; 8192: 164 KB of sums
__host__ __device__ constexpr int forward_depth(int threads) { return threads <= 512 ? 3 : 2; }
__host__ __device__ constexpr int backward_depth(int threads) { return threads <= 128 ? 3 : threads <= 512 ? 1 : 0; }

template <typename T, bool VECD>
__device__ __forceinline__ void put(T* row, const Eight& f, const Cols<VECD>& c) {
    if constexpr (VECD) {
        const float v[NORM_E] = {f.v[0].x, f.v[0].y, f.v[1].x, f.v[1].y, f.v[2].x, f.v[2].y, f.v[3].x, f.v[3].y};
        if (c.any) store_row<NORM_E>(row + c.at(0), v);
    } else {
#pragma unroll
        for (int j = 0; j < NORM_E; ++j) {
            const float v = j & 1 ? f.v[j / 2].y : f.v[j / 2].x;
            if (c.has(j)) {
                if constexpr (sizeof(T) == 2) row[c.at(j)] = __float2bfloat16_rn(v);
                else row[c.at(j)] = v;
            }
        }
    }
}
// a vector of C floats; `none` where it is not given
template <bool VECD>
__device__ __forceinline__ void weights(const float* p, float none, Eight& f, const Cols<VECD>& c) {
    f.fill(none);
    if (!p) return;
    if constexpr (VECD) {
        if (c.any) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(p + c.at(0))), b = __ldg(reinterpret_cast<const float4*>(p + c.at(0)) + 1);
            f.v[0] = make_float2(a.x, a.y); f.v[1] = make_float2(a.z, a.w); f.v[2] = make_float2(b.x, b.y); f.v[3] = make_float2(b.z, b.w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (c.has(2 * i)) f.v[i].x = __ldg(p + c.at(2 * i));
            if (c.has(2 * i + 1)) f.v[i].y = __ldg(p + c.at(2 * i + 1));
        }
    }
}

__device__ __forceinline__ const float* row_of(const float* p, long long off) { return p ? p + off : nullptr; }

// ---------------------------------------------------------------- sums over a row
// G: lanes of a row; 0: the row is the CTA's.  The buffers of two consecutive sums are different ones, so that one barrier a sum
// is enough.
template <int G>
struct RowSum {
    float2 (*cross)[32];                    // [2][warps]
    int turn = 0;
    __device__ __forceinline__ float2 of(float a, float b) {
#pragma unroll
        for (int o = (G ? G : 32) >> 1; o; o >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, o);
            b += __shfl_xor_sync(0xffffffffu, b, o);
        }
        if (G == 0) {
            const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
            if (lane == 0) cross[turn][warp] = make_float2(a, b);
            __syncthreads();
            if (warps <= 4) {
                float2 s = cross[turn][0];
                for (int w = 1; w < warps; ++w) s = __fadd2_rn(s, cross[turn][w]);
                a = s.x; b = s.y;
            } else {
                const float2 s = lane < warps ? cross[turn][lane] : make_float2(0.f, 0.f);
                a = s.x; b = s.y;
#pragma unroll
                for (int o = 16; o; o >>= 1) {
                    a += __shfl_xor_sync(0xffffffffu, a, o);
                    b += __shfl_xor_sync(0xffffffffu, b, o);
                }
            }
            turn ^= 1;
        }
        return make_float2(a, b);
    }
    __device__ __forceinline__ float of(float a) {
#pragma unroll
        for (int o = (G ? G : 32) >> 1; o; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
        if (G == 0) {
            const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
            if (lane == 0) cross[turn][warp].x = a;
            __syncthreads();
            if (warps <= 4) {
                a = cross[turn][0].x;
                for (int w = 1; w < warps; ++w) a += cross[turn][w].x;
            } else {
                a = lane < warps ? cross[turn][lane].x : 0.f;
#pragma unroll
                for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
            }
            turn ^= 1;
        }
        return a;
    }
};

// v becomes its normalised form; the factor is returned.  Channels that do not exist hold zeros and keep them.
template <int G, bool VECD>
__device__ __forceinline__ float normalise(int kind, Eight& v, const Cols<VECD>& c, float eps, float per_channel, RowSum<G>& sum) {
    if (kind == BRA_NORM_LAYER) {
        const float mean = sum.of(total(v)) * per_channel;
#pragma unroll
        for (int i = 0; i < 4; ++i) v.v[i] = __fadd2_rn(v.v[i], c.only(-mean, i));
    }
    const float r = rsqrtf(fmaf(sum.of(dot(v, v)), per_channel, eps));
#pragma unroll
    for (int i = 0; i < 4; ++i) v.v[i] = __fmul2_rn(v.v[i], both(r));
    return r;
}

// g becomes the gradient of the row whose normalised form hat had the gradient g: r (g - hat mean(g hat) [- mean(g)])
template <int G, bool VECD>
__device__ __forceinline__ void normalise_back(int kind, Eight& g, const Eight& hat, float r, const Cols<VECD>& c, float per_channel, RowSum<G>& sum) {
    float2 m = make_float2(0.f, 0.f);
    if (kind == BRA_NORM_LAYER) m = sum.of(dot(g, hat), total(g));
    else m.x = sum.of(dot(g, hat));
    const float along = -r * (m.x * per_channel), mean = -r * (m.y * per_channel);
#pragma unroll
    for (int i = 0; i < 4; ++i) g.v[i] = __ffma2_rn(g.v[i], both(r), __ffma2_rn(hat.v[i], both(along), c.only(mean, i)));
}

// ---------------------------------------------------------------- forward
// A CTA's groups take the rows of its run in turn.  All groups make the same number of rounds (those without a row compute on what
// the ring holds and store nothing), so that the shuffles and barriers of the sums are met by every thread.
// THREADS: the most a CTA has.  Above 512 a thread has 64 registers: weights are read where they are used, row by row.
template <typename T, bool VECD, int G, bool POST, int THREADS>
__global__ void __launch_bounds__(THREADS) norm_forward_kernel(const NormArgs a) {
    constexpr bool KEEP = THREADS <= 512;
    __shared__ float2 cross[2][32];
    extern __shared__ __align__(16) char ring[];
    const int groups = G ? THREADS / (G ? G : 1) : 1;
    const int mine = G ? threadIdx.x / (G ? G : 1) : 0;
    const Cols<VECD> c(G ? threadIdx.x % (G ? G : 1) : threadIdx.x, G ? G : blockDim.x, a.C);
    RowSum<G> sum{cross};
    const int first = (int)(blockIdx.x * (long long)a.run), end = (int)min((long long)first + a.run, a.rows);
    const float per_channel = 1.f / (float)a.C;
    const bool has_y = a.y != nullptr;
    const long long start = (long long)(first + mine) * a.C, stride = (long long)groups * a.C;

    Ahead<T, VECD, 2, forward_depth(THREADS)> in(ring);
    in.row[0] = static_cast<const T*>(a.x) + start + c.at(0);
    in.row[1] = has_y ? static_cast<const T*>(a.y) + start + c.at(0) : nullptr;
    T* h = a.h ? static_cast<T*>(a.h) + start : nullptr;
    T* n = a.n ? static_cast<T*>(a.n) + start : nullptr;
    int ask = first + mine;
#pragma unroll
    for (int k = 0; k < in.ROWS; ++k, ask += groups) in.fetch(ask < end, stride, c);
    const bool per_image = a.gate_image || a.affine_image;
    int image_end = first + mine;                             // rows before it have the weights that are held
    Eight gate, pw, pb, w, b;
    const float *gate_p = a.gate, *w_p = a.w, *b_p = a.b;
    if (POST && KEEP) {
        weights<VECD>(a.post_w, 1.f, pw, c);
        weights<VECD>(a.post_b, 0.f, pb, c);
    }
    for (int row0 = first; row0 < end; row0 += groups) {
        const int row = row0 + mine;
        const bool live = row < end;
        if (row >= image_end && live) {
            const int image = per_image ? row / a.N : 0;
            gate_p = row_of(a.gate, a.gate_image ? (long long)image * a.C : 0);
            w_p = row_of(a.w, a.affine_image ? (long long)image * a.C : 0);
            b_p = row_of(a.b, a.affine_image ? (long long)image * a.C : 0);
            if (KEEP) {
                weights<VECD>(gate_p, 1.f, gate, c);
                weights<VECD>(w_p, 1.f, w, c);
                weights<VECD>(b_p, 0.f, b, c);
            }
            image_end = per_image ? (int)min((long long)(image + 1) * a.N, (long long)end) : end;
        }
        Eight v, u;
        in.arrived();
        in.read(0, v, c);
        if (has_y) in.read(1, u, c);
        in.fetch(ask < end, stride, c);
        ask += groups;
        in.next();
#pragma unroll
        for (int i = 0; i < 4; ++i) v.v[i] = __fmul2_rn(v.v[i], both(a.alpha));
        if (has_y) {
            if (POST) {
                normalise<G>(a.post, u, c, a.eps, per_channel, sum);
                if (!KEEP) { weights<VECD>(a.post_w, 1.f, pw, c); weights<VECD>(a.post_b, 0.f, pb, c); }
#pragma unroll
                for (int i = 0; i < 4; ++i) u.v[i] = __ffma2_rn(u.v[i], pw.v[i], pb.v[i]);
            }
            if (!KEEP) weights<VECD>(gate_p, 1.f, gate, c);
#pragma unroll
            for (int i = 0; i < 4; ++i) v.v[i] = __ffma2_rn(gate.v[i], u.v[i], v.v[i]);
        }
        if (h) {
            if (live) put<T, VECD>(h, v, c);
            h += stride;
        }
        if (n) {
            normalise<G>(a.pre, v, c, a.eps, per_channel, sum);
            if (!KEEP) { weights<VECD>(w_p, 1.f, w, c); weights<VECD>(b_p, 0.f, b, c); }
#pragma unroll
            for (int i = 0; i < 4; ++i) v.v[i] = __ffma2_rn(v.v[i], w.v[i], b.v[i]);
            if (live) put<T, VECD>(n, v, c);
            n += stride;
        }
    }
}

// ---------------------------------------------------------------- backward
// THREADS 128: the sums over tokens stay in registers, and so do the weights.  More (long rows, whose CTAs would have no registers
// left): the sums are in shared memory, each word its thread's own, and the weights are read again for every row.
template <typename T, bool VECD, int G, bool POST, int THREADS>
__global__ void __launch_bounds__(THREADS) norm_backward_kernel(const NormArgs a) {
    constexpr bool KEEP = THREADS == 128;
    __shared__ float2 cross[2][32];
    // !KEEP: [SUMS][E][threads]; KEEP and several groups: [E][threads], to join the groups; then the ring of rows
    extern __shared__ __align__(16) float sums_sh[];
    const int groups = G ? THREADS / (G ? G : 1) : 1;
    const int mine = G ? threadIdx.x / (G ? G : 1) : 0;
    const Cols<VECD> c(G ? threadIdx.x % (G ? G : 1) : threadIdx.x, G ? G : blockDim.x, a.C);
    RowSum<G> sum{cross};
    Ahead<T, VECD, 4, backward_depth(THREADS)> in(sums_sh + NORM_E * blockDim.x * (KEEP ? (G ? 1 : 0) : SUMS));
    const bool has_y = a.y != nullptr, has_n = a.dn != nullptr;
    const int first = (int)(blockIdx.x * (long long)a.run), last = (int)min((long long)first + a.run, a.rows) - 1;
    const float per_channel = 1.f / (float)a.C;

    Eight acc[KEEP ? SUMS : 1];
    auto shared_sum = [&](int s, int i) -> float2& { return reinterpret_cast<float2*>(sums_sh)[(s * 4 + i) * blockDim.x + threadIdx.x]; };
    auto clear = [&](int s) {
        if constexpr (KEEP) acc[s].fill(0.f);
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i) shared_sum(s, i) = both(0.f);
        }
    };
    // sum s += a * b
    auto add = [&](int s, const Eight& p, const Eight& q) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (KEEP) acc[s].v[i] = __ffma2_rn(p.v[i], q.v[i], acc[s].v[i]);
            else shared_sum(s, i) = __ffma2_rn(p.v[i], q.v[i], shared_sum(s, i));
        }
    };
    auto add1 = [&](int s, const Eight& p) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (KEEP) acc[s].v[i] = __fadd2_rn(p.v[i], acc[s].v[i]);
            else shared_sum(s, i) = __fadd2_rn(p.v[i], shared_sum(s, i));
        }
    };
    // this CTA's sum s, over its groups, into slot `slot`
    auto leave = [&](int s, long long slot) {
        float* to = a.part + ((size_t)s * a.slots + slot) * a.C;
        Eight t;
        if constexpr (KEEP) t = acc[KEEP ? s : 0];
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i) t.v[i] = shared_sum(s, i);
        }
        if (G && KEEP) {
            float2* join = reinterpret_cast<float2*>(sums_sh);
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 4; ++i) join[i * THREADS + threadIdx.x] = t.v[i];
            __syncthreads();
            if (mine == 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    t.v[i] = both(0.f);
                    for (int g = 0; g < groups; ++g) t.v[i] = __fadd2_rn(t.v[i], join[i * THREADS + g * G + threadIdx.x]);
                }
            }
        }
        if (mine == 0) put<float, VECD>(to, t, c);
        clear(s);
    };
    auto wants = [&](int s) { return (a.sums >> s) & 1; };
    auto of_image = [&](int s) { return s == SUM_GATE ? a.gate_image : s <= SUM_B ? a.affine_image : 0; };
#pragma unroll
    for (int s = 0; s < SUMS; ++s) clear(s);

    Eight gate, pw, pb, w;
    const bool per_image = a.gate_image || a.affine_image;
    int begin = first;
    while (begin <= last) {                                   // the rows of one image
        const int image = per_image ? begin / a.N : 0;
        const int end = per_image ? (int)min((long long)(image + 1) * a.N - 1, (long long)last) : last;
        const float* gate_p = row_of(a.gate, a.gate_image ? (long long)image * a.C : 0);
        const float* w_p = row_of(a.w, a.affine_image ? (long long)image * a.C : 0);
        if (KEEP) {
            weights<VECD>(gate_p, 1.f, gate, c);
            weights<VECD>(w_p, 1.f, w, c);
            if (POST) { weights<VECD>(a.post_w, 1.f, pw, c); weights<VECD>(a.post_b, 0.f, pb, c); }
        }
        const long long start = (long long)(begin + mine) * a.C, stride = (long long)groups * a.C;
        auto from = [&](const void* p) { return p ? static_cast<const T*>(p) + start + c.at(0) : nullptr; };
        in.row[0] = from(a.x); in.row[1] = from(a.y); in.row[2] = from(a.dh); in.row[3] = from(a.dn);
        T* dx = static_cast<T*>(a.dx) + start;
        T* dy = has_y ? static_cast<T*>(a.dy) + start : nullptr;
        int ask = begin + mine;
        in.restart();
#pragma unroll
        for (int k = 0; k < in.ROWS; ++k, ask += groups) in.fetch(ask <= end, stride, c);
        for (int row0 = begin; row0 <= end; row0 += groups) {
            const bool live = row0 + mine <= end;
            Eight v, u, g, d;
            in.arrived();
            in.read(0, v, c);
            if (has_y) in.read(1, u, c);
            if (a.dh) in.read(2, d, c);
            else d.fill(0.f);
            if (has_n) in.read(3, g, c);
            in.fetch(ask <= end, stride, c);
            ask += groups;
            in.next();
            // !KEEP: the weights, as they are used
            auto post_weights = [&] { if (!KEEP && POST) { weights<VECD>(a.post_w, 1.f, pw, c); weights<VECD>(a.post_b, 0.f, pb, c); } };
            float u_factor = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) v.v[i] = __fmul2_rn(v.v[i], both(a.alpha));
            if (has_y) {
                if (POST) u_factor = normalise<G>(a.post, u, c, a.eps, per_channel, sum);
                post_weights();
                if (!KEEP) weights<VECD>(gate_p, 1.f, gate, c);
#pragma unroll
                for (int i = 0; i < 4; ++i) v.v[i] = __ffma2_rn(gate.v[i], POST ? __ffma2_rn(u.v[i], pw.v[i], pb.v[i]) : u.v[i], v.v[i]);
            }
            if (has_n) {
                const float r = normalise<G>(a.pre, v, c, a.eps, per_channel, sum);
                if (!KEEP) weights<VECD>(w_p, 1.f, w, c);
                if (live) {
                    add(SUM_W, g, v);
                    add1(SUM_B, g);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) g.v[i] = __fmul2_rn(g.v[i], w.v[i]);
                normalise_back<G>(a.pre, g, v, r, c, per_channel, sum);
#pragma unroll
                for (int i = 0; i < 4; ++i) d.v[i] = __fadd2_rn(d.v[i], g.v[i]);
            }
            // d = dH
#pragma unroll
            for (int i = 0; i < 4; ++i) v.v[i] = __fmul2_rn(d.v[i], both(a.alpha));
            if (live) put<T, VECD>(dx, v, c);
            dx += stride;
            if (has_y) {
                post_weights();
                if (!KEEP) weights<VECD>(gate_p, 1.f, gate, c);
                if (live) {
                    Eight yy = u;
                    if (POST) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) yy.v[i] = __ffma2_rn(u.v[i], pw.v[i], pb.v[i]);
                    }
                    add(SUM_GATE, d, yy);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) d.v[i] = __fmul2_rn(d.v[i], gate.v[i]);
                if (POST) {
                    if (live) {
                        add(SUM_POST_W, d, u);
                        add1(SUM_POST_B, d);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) d.v[i] = __fmul2_rn(d.v[i], pw.v[i]);
                    normalise_back<G>(a.post, d, u, u_factor, c, per_channel, sum);
                }
                if (live) put<T, VECD>(dy, d, c);
                dy += stride;
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

// Adds the partial sums in order: 32 channels a CTA, WARPS warps that take every WARPS-th slot, eight of them in flight.
template <int WARPS>
__global__ void __launch_bounds__(32 * WARPS) norm_join_kernel(const JoinArgs a) {
    __shared__ float part[WARPS][33];
    const int s = a.which[blockIdx.y];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int ch = blockIdx.x * 32 + lane;
    const int images = a.image_sum[s] ? a.images : 1;
    float* out = a.out[s];
    pdl_wait();
    for (int image = blockIdx.z; image < images; image += gridDim.z) {
        int c0 = 0, c1 = a.ctas;                              // CTAs that left a row of sums, and the first one's slot
        long long slot = 0;
        if (a.image_sum[s]) {
            c0 = (int)((long long)image * a.N / a.run);
            c1 = (int)(((long long)(image + 1) * a.N - 1) / a.run) + 1;
            slot = image + c0;
        }
        float t = 0.f;
        if (ch < a.C) {
            const float* from = a.part + ((size_t)s * a.slots + slot + warp) * a.C + ch;
            const long long step = (long long)WARPS * a.C;
            int left = c1 - c0 - warp;                        // every WARPS-th of them
            for (; left > 7 * WARPS; left -= 8 * WARPS, from += 8 * step) {
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = __ldcg(from + k * step);
#pragma unroll
                for (int k = 0; k < 8; ++k) t += v[k];
            }
#pragma unroll
            for (int k = 0; k < 7; ++k)
                if (left > k * WARPS) t += __ldcg(from + k * step);
        }
        part[warp][lane] = t;
        __syncthreads();
        if (warp == 0 && ch < a.C) {
#pragma unroll
            for (int k = 1; k < WARPS; ++k) t += part[k][lane];
            out[(size_t)(a.image_sum[s] ? image : 0) * a.C + ch] = t;
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

Plan plan(const bra_norm_problem* q, bool backward) {
    Plan p;
    const long long rows = (long long)q->B * q->N;
    const int C = q->C;
    const int need = (C + NORM_E - 1) / NORM_E;
    p.wide = need > 32;
    if (p.wide) {
        p.group = (need + 31) / 32 * 32;
        p.threads = p.group;
    } else {
        p.group = need <= 8 ? 8 : need <= 16 ? 16 : 32;
        p.threads = 128;
    }
    const int groups = p.wide ? 1 : p.threads / p.group;
    // as many CTAs as an SM holds at a time, by registers and the ring
    const bool f32 = q->dtype == BRA_F32;
    int per_sm;
    const bool post = q->post != BRA_NORM_NONE;
    if (p.threads <= 128) per_sm = (backward ? (f32 || post ? 3 : 4) : (f32 || post ? 5 : 6)) * 128 / p.threads;
    else per_sm = (backward || f32 ? 512 : 1024) / p.threads;
    if (per_sm < 1) per_sm = 1;
    long long most = (long long)kSMs * per_sm;
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

// Dynamic shared memory of every kernel is a constant times its threads, the most of which THREADS says: allowed once per device.
template <typename Kernel>
cudaError_t launch_rows(Kernel kernel, size_t smem, const NormArgs& a, const Plan& pl, cudaStream_t st) {
    if (smem > 46 * 1024) {                 // 48 KB less what the kernels have of their own
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    kernel<<<(unsigned)pl.ctas, pl.threads, smem, st>>>(a);
    count_launch();
    return cudaGetLastError();
}

template <typename T, bool VECD, int G, int THREADS>
cudaError_t forward_as(const NormArgs& a, const Plan& pl, cudaStream_t st) {
    const size_t smem = Ahead<T, VECD, 2, forward_depth(THREADS)>::bytes(pl.threads);
    return a.post != BRA_NORM_NONE ? launch_rows(norm_forward_kernel<T, VECD, G, true, THREADS>, smem, a, pl, st)
                                   : launch_rows(norm_forward_kernel<T, VECD, G, false, THREADS>, smem, a, pl, st);
}
template <typename T, bool VECD, int G, int THREADS>
cudaError_t backward_as(const NormArgs& a, const Plan& pl, cudaStream_t st) {
    constexpr bool KEEP = THREADS == 128;
    const size_t smem = sizeof(float) * NORM_E * pl.threads * (KEEP ? (G ? 1 : 0) : SUMS) + Ahead<T, VECD, 4, backward_depth(THREADS)>::bytes(pl.threads);
    return a.post != BRA_NORM_NONE ? launch_rows(norm_backward_kernel<T, VECD, G, true, THREADS>, smem, a, pl, st)
                                   : launch_rows(norm_backward_kernel<T, VECD, G, false, THREADS>, smem, a, pl, st);
}
template <typename T, bool VECD>
cudaError_t launch(bool backward, const NormArgs& a, const Plan& pl, cudaStream_t st) {
#define BRA_NORM_AS(G, THREADS) (backward ? backward_as<T, VECD, G, THREADS>(a, pl, st) : forward_as<T, VECD, G, THREADS>(a, pl, st))
    if (!pl.wide) return pl.group == 8 ? BRA_NORM_AS(8, 128) : pl.group == 16 ? BRA_NORM_AS(16, 128) : BRA_NORM_AS(32, 128);
    if (pl.threads <= 128) return BRA_NORM_AS(0, 128);
    return pl.threads <= 512 ? BRA_NORM_AS(0, 512) : BRA_NORM_AS(0, 1024);
#undef BRA_NORM_AS
}
cudaError_t launch(bool backward, const bra_norm_problem* p, const NormArgs& a, const Plan& pl, cudaStream_t st) {
    const bool vec = p->C % NORM_E == 0;
    if (p->dtype == BRA_BF16) return vec ? launch<__nv_bfloat16, true>(backward, a, pl, st) : launch<__nv_bfloat16, false>(backward, a, pl, st);
    return vec ? launch<float, true>(backward, a, pl, st) : launch<float, false>(backward, a, pl, st);
}

}  // namespace
}  // namespace bra

using namespace bra;

extern "C" {

size_t bra_norm_workspace_bytes(const bra_norm_problem* p) {
    if (check(p) != BRA_OK) return 0;
    const Plan pl = plan(p, true);
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
    const Plan pl = plan(p, false);
    NormArgs a = args_of(p, pl);
    a.x = x; a.y = y; a.gate = gate; a.post_w = post_w; a.post_b = post_b; a.w = w; a.b = b; a.h = h; a.n = n;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return launch(false, p, a, pl, st) == cudaSuccess ? BRA_OK : BRA_ERR_CUDA;
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
    const Plan pl = plan(p, true);
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
    if (launch(true, p, a, pl, st) != cudaSuccess) return BRA_ERR_CUDA;
    if (wanted) {
        const dim3 grid((p->C + 31) / 32, wanted, most_images < GRID_YZ ? most_images : GRID_YZ);
        // many rows of sums for each output: many warps
        const long long each = pl.ctas / most_images;
        const cudaError_t e = each > 64 ? launch_kernel(norm_join_kernel<32>, grid, dim3(1024), 0, st, true, j)
                                        : launch_kernel(norm_join_kernel<8>, grid, dim3(256), 0, st, true, j);
        if (e != cudaSuccess) return BRA_ERR_CUDA;
        count_launch();
    }
    return BRA_OK;
}

}  // extern "C"
