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
#include "norm_cols.h"
#include "sm100_ptx.cuh"

namespace bra {
namespace {

struct NormArgs {
    const void *x, *y, *dh, *dn;
    void *h, *n, *dx, *dy;
    const float *gate, *post_w, *post_b, *w, *b;
    float* part;                            // partial sums of the backward pass
    long long rows;
    int N;                                  // rows of an image
    int C;
    int run;                                // rows of a CTA
    int gate_image, affine_image;           // [B, C] rather than [C]
    int pre, post;
    float eps, alpha;
    int ring_slots, ring_pitch;             // of rows that are a CTA's
    int sums;                               // which sums are wanted, SUM_* bits
    int place[5];                           // where in shared memory each of them is
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
template <bool VECD, bool FULL, bool QUADS>
struct Cols : NormCols<VECD, FULL, QUADS> {
    using NormCols<VECD, FULL, QUADS>::NormCols;
    // f for channels that exist, 0 for the others
    __device__ __forceinline__ float2 only(float f, int i) const {
        return VECD ? both(this->half(i >> 1) ? f : 0.f) : make_float2(this->has(2 * i) ? f : 0.f, this->has(2 * i + 1) ? f : 0.f);
    }
};

__device__ __forceinline__ void widen(const uint32_t (&w)[4], Eight& f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}

// How far rows are read ahead: through a ring in shared memory whose 16- or 4-byte slots are each one thread's own, so that neither
// registers nor barriers are spent on rows in flight; one slot more than rows in flight, so that none is written that was read in the
// same round.  Rows of bf16 that start on two bytes cannot be copied so (four at least) and go through registers, one row ahead.
// DEPTH: rounds in flight.
template <typename T, bool VECD, int TENSORS, int DEPTH, int R>
struct Ahead {
    static constexpr bool RING = VECD || sizeof(T) == 4;
    static constexpr int ROWS = RING ? DEPTH : 1;
    static constexpr int CHUNKS = VECD ? NORM_E * (int)sizeof(T) / 16 : NORM_E, CHUNK = VECD ? 16 : 4;
    static constexpr size_t bytes(int threads) { return RING ? (size_t)(DEPTH + 1) * TENSORS * R * NORM_E * sizeof(T) * threads : 0; }
    T raw[RING ? 1 : TENSORS * R][NORM_E];
    const T* row[TENSORS];                  // of the row that is fetched next, at this thread's first channel; null: no such tensor
    uint32_t base, pitch;                   // this thread's first slot, bytes between its chunks
    uint32_t get = 0, put = 0;              // offsets of the rows that are read and fetched next
    __device__ __forceinline__ void restart() { get = put; }         // nothing that was fetched is left to read
    __device__ __forceinline__ explicit Ahead(const void* smem) : base(ptx::smem_u32(smem) + threadIdx.x * CHUNK), pitch(blockDim.x * CHUNK) {}
    __device__ __forceinline__ uint32_t step(uint32_t at) const {
        at += TENSORS * R * CHUNKS * pitch;
        return at == (DEPTH + 1) * TENSORS * R * CHUNKS * pitch ? 0 : at;
    }
    // fetches R rows of every tensor, `between` elements apart, of which those with a number below `end` exist (first: of the first one,
    // then every `groups`th), and moves on by R of them
    template <typename Channels>
    __device__ __forceinline__ void fetch(int first, int groups, int end, int between, const Channels& c) {
#pragma unroll
        for (int k = 0; k < TENSORS; ++k) {
            if (!row[k]) continue;
#pragma unroll
            for (int q = 0; q < R; ++q) {
                const T* from = row[k] + q * between;
                if (first + q * groups < end) {
                    if constexpr (RING) {
                        const uint32_t to = base + put + (k * R + q) * CHUNKS * pitch;
#pragma unroll
                        for (int j = 0; j < CHUNKS; ++j) {
                            if constexpr (VECD) ptx::cp_async_16(to + j * pitch, c.half(j) ? from + (c.at(4 * j) - c.at(0)) : from - c.at(0), c.half(j) ? 16 : 0);
                            else ptx::cp_async_4(to + j * pitch, c.has(j) ? from + j * c.group : from - c.t, c.has(j) ? 4 : 0);
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < NORM_E; ++j) raw[k * R + q][j] = c.has(j) ? from[j * c.group] : T(0.f);
                    }
                }
            }
            row[k] += (long long)R * between;
        }
        if (RING) {
            ptx::cp_async_commit();
            put = step(put);
        }
    }
    __device__ __forceinline__ void arrived() { if constexpr (RING) ptx::cp_async_wait<DEPTH - 1>(); }
    __device__ __forceinline__ void read(int tensor, int q, Eight& f) const {
        if constexpr (RING) {
            const uint32_t from = base + get + (tensor * R + q) * CHUNKS * pitch;
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
            for (int i = 0; i < 4; ++i) f.v[i] = make_float2(__bfloat162float(raw[tensor * R + q][2 * i]), __bfloat162float(raw[tensor * R + q][2 * i + 1]));
        }
    }
    __device__ __forceinline__ void next() { if (RING) get = step(get); }
};

// The same for rows that are a CTA's: R rows of a tensor are one stretch of memory, which one thread copies (bulk copies, a barrier a
// slot), whatever their alignment: a stretch is copied from the 16-byte boundary before it to the one behind it, so the row starts
// `skew` bytes into its slot.  The tensor's own end need not be such a boundary: rows that reach into the last 16 bytes are read where
// they are, and so are all rows where shared memory has no room for a slot, or if a wait should give up.
constexpr int NORM_SLOTS = 4;
template <typename T, bool VECD, int TENSORS, int R>
struct Stretch {
    const T* tensor[TENSORS];               // whole ones; null: no such tensor
    uint64_t* full;                         // [slots]
    uint32_t base;
    int slots, pitch, C;                    // pitch: bytes of a tensor's part of a slot
    long long last_byte;                    // bytes of a tensor that may be copied
    uint32_t count = 0, asked = 0;          // units read and asked for
    int row = 0, end = 0;                   // of the unit that is read next, and the last row of this stretch of rows, plus one
    bool direct = false;
    __device__ __forceinline__ Stretch(const NormArgs& a, uint32_t smem, uint64_t* bars)
        : full(bars), base(smem), slots(a.ring_slots), pitch(a.ring_pitch), C(a.C), last_byte(a.rows * a.C * (long long)sizeof(T) / 16 * 16) {
        if (threadIdx.x == 0) {
            for (int i = 0; i < NORM_SLOTS; ++i) ptx::mbar_init(full + i, 1);
            ptx::fence_mbar_init();
        }
        __syncthreads();
    }
    __device__ __forceinline__ long long byte_of(int r) const { return (long long)r * C * (int)sizeof(T); }
    __device__ __forceinline__ bool copied(int first) const {
        return slots > 0 && (byte_of(min(first + R, end)) + 15) / 16 * 16 <= last_byte;
    }
    __device__ __forceinline__ void ask(int first) {                   // one thread
        if (first >= end) return;
        const uint32_t s = asked % slots;
        ++asked;
        if (!copied(first)) { ptx::mbar_arrive(full + s); return; }
        const long long from = byte_of(first) / 16 * 16, to = (byte_of(min(first + R, end)) + 15) / 16 * 16;
        int n = 0;
#pragma unroll
        for (int k = 0; k < TENSORS; ++k) n += tensor[k] != nullptr;
        ptx::mbar_expect_tx(full + s, (uint32_t)(to - from) * n);
#pragma unroll
        for (int k = 0; k < TENSORS; ++k)
            if (tensor[k]) ptx::bulk_load(base + (s * TENSORS + k) * pitch, reinterpret_cast<const char*>(tensor[k]) + from, (uint32_t)(to - from), full + s);
    }
    // rows first .. end_ - 1, from now on
    __device__ __forceinline__ void start(int first, int end_) {
        row = first;
        end = end_;
        if (threadIdx.x == 0)
            for (int i = 0; i < slots; ++i) ask(first + i * R);
    }
    __device__ __forceinline__ void arrived() {
        direct = !copied(row);
        if (slots > 0) {
            if (!ptx::mbar_try_wait(full + count % slots, (count / slots) & 1)) direct = !ptx::mbar_wait(full + count % slots, (count / slots) & 1) || direct;
        }
    }
    template <typename Channels>
    __device__ __forceinline__ void read(int tensor_at, int q, Eight& f, const Channels& c) const {
        float v[NORM_E] = {};
        if (direct) {
            const T* from = tensor[tensor_at] + (long long)min(row + q, end - 1) * C;
            if constexpr (VECD) {
                if constexpr (sizeof(T) == 4) {
                    if (c.any) load_row<4>(from + c.at(0), v);
                    if (c.more) load_row<4>(from + c.at(4), v + 4);
                } else {
                    if (c.any) load_row<NORM_E>(from + c.at(0), v);
                }
            } else {
#pragma unroll
                for (int j = 0; j < NORM_E; ++j) if (c.has(j)) v[j] = (float)from[c.at(j)];
            }
        } else {
            const uint32_t at = base + ((count % slots) * TENSORS + tensor_at) * pitch + (uint32_t)(byte_of(row) & 15) + q * C * (int)sizeof(T) + c.at(0) * (int)sizeof(T);
            if constexpr (VECD && sizeof(T) == 2) {
                float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
                if (c.any) t = ptx::lds_f32x4(at);
                widen({__float_as_uint(t.x), __float_as_uint(t.y), __float_as_uint(t.z), __float_as_uint(t.w)}, f);
                return;
            } else if constexpr (VECD) {
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (c.half(k)) {
                        const float4 t = ptx::lds_f32x4(at + 16 * k * c.group);
                        v[4 * k] = t.x; v[4 * k + 1] = t.y; v[4 * k + 2] = t.z; v[4 * k + 3] = t.w;
                    }
            } else {
#pragma unroll
                for (int j = 0; j < NORM_E; ++j)
                    if (c.has(j)) {
                        if constexpr (sizeof(T) == 4) v[j] = ptx::lds_f32(at + j * c.group * 4);
                        else v[j] = __uint_as_float((uint32_t)ptx::lds_u16(at + j * c.group * 2) << 16);
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) f.v[i] = make_float2(v[2 * i], v[2 * i + 1]);
    }
    // behind a barrier that all threads met after their reads: the slot takes the unit `slots` further on
    __device__ __forceinline__ void next() {
        if (threadIdx.x == 0 && slots > 0) ask(row + slots * R);
        row += R;
        ++count;
    }
};

// Which of the two: stretches where a thread would copy its channels one by one, or has no registers to address them by.  Measured
// (B200, us, forward + backward, stretches / slots of threads): 8 x 1024 x 768 bf16 52 + 92 / 20 + 36, x 4096 59 + 155 / 46 + 107; 765 bf16 21 + 38 /
// 21 + 47, 5001 fp32 181 + 470 / 205 + 524, 5000 fp32 154 + 383 / 188 + 378.  Since then, by two CTAs an SM up to 640 threads and fewer checks of
// what exists: 5001 fp32 130 + 300, 5000 fp32 112 + 285, 4500 bf16 183 + 331 -> 116 + 242.
template <bool VECD, int G, int THREADS>
constexpr bool STRETCHES = G == 0 && (!VECD || THREADS > 512);
// rounds in flight of the slots of threads
__host__ __device__ constexpr int forward_depth(int threads, int rows) { return rows == 1 ? 3 : 2; }
// Two rows at once, but not with a post-norm of rows that do not come by 16 bytes, which have no registers for it.  With a post-norm, one / two
// rows, gradients, us: 64 x 3136 x 64 (two CTAs an SM in the place of three) 47.3 / 45.1, 64 x 784 x 128 27.0 / 25.3, 16 x 1024 x 768 (168 registers) 70 / 55.
__host__ __device__ constexpr int backward_rows(int threads, bool post, bool vec) { return threads <= 128 && (vec || !post) ? 2 : 1; }
__host__ __device__ constexpr int backward_depth(int threads, int rows) { return threads > 128 ? 1 : rows == 1 ? 3 : 2; }

template <typename T, bool VECD, bool FULL, bool QUADS>
__device__ __forceinline__ void put(T* row, const Eight& f, const Cols<VECD, FULL, QUADS>& c) {
    if constexpr (VECD) {
        const float v[NORM_E] = {f.v[0].x, f.v[0].y, f.v[1].x, f.v[1].y, f.v[2].x, f.v[2].y, f.v[3].x, f.v[3].y};
        if constexpr (QUADS) {
            if (c.any) store_row<4>(row + c.at(0), v);
            if (c.more) store_row<4>(row + c.at(4), v + 4);
        } else {
            if (c.any) store_row<NORM_E>(row + c.at(0), v);
        }
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
template <bool VECD, bool FULL, bool QUADS>
__device__ __forceinline__ void weights(const float* p, float none, Eight& f, const Cols<VECD, FULL, QUADS>& c) {
    f.fill(none);
    if (!p) return;
    if constexpr (VECD) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            if (c.half(k)) {
                const float4 v = __ldg(reinterpret_cast<const float4*>(p + c.at(4 * k)));
                f.v[2 * k] = make_float2(v.x, v.y);
                f.v[2 * k + 1] = make_float2(v.z, v.w);
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
// G: lanes of a row; 0: the row is the CTA's.  K sums at once: their exchanges overlap and share a barrier.  The buffers of two
// consecutive calls are different ones, so that one barrier a call is enough.
constexpr int SUMS_AT_ONCE = 4;
template <int G>
struct RowSum {
    float (*cross)[32][SUMS_AT_ONCE];       // [2][warps]
    int turn = 0;
    template <int K>
    __device__ __forceinline__ void of(float (&a)[K]) {
#pragma unroll
        for (int o = (G ? G : 32) >> 1; o; o >>= 1)
#pragma unroll
            for (int k = 0; k < K; ++k) a[k] += __shfl_xor_sync(0xffffffffu, a[k], o);
        if (G == 0) {
            const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
            if (lane == 0)
#pragma unroll
                for (int k = 0; k < K; ++k) cross[turn][warp][k] = a[k];
            __syncthreads();
            if (warps <= 4) {
#pragma unroll
                for (int k = 0; k < K; ++k) a[k] = cross[turn][0][k];
                for (int w = 1; w < warps; ++w)
#pragma unroll
                    for (int k = 0; k < K; ++k) a[k] += cross[turn][w][k];
            } else {
#pragma unroll
                for (int k = 0; k < K; ++k) a[k] = lane < warps ? cross[turn][lane][k] : 0.f;
#pragma unroll
                for (int o = 16; o; o >>= 1)
#pragma unroll
                    for (int k = 0; k < K; ++k) a[k] += __shfl_xor_sync(0xffffffffu, a[k], o);
            }
            turn ^= 1;
        }
    }
};

// R rows become their normalised forms; their factors go to r.  Channels that do not exist hold zeros and keep them.
template <int G, int R, typename Channels>
__device__ __forceinline__ void normalise(int kind, Eight (&v)[R], float (&r)[R], const Channels& c, float eps, float per_channel, RowSum<G>& sum) {
    float s[R];
    if (kind == BRA_NORM_LAYER) {
#pragma unroll
        for (int q = 0; q < R; ++q) s[q] = total(v[q]);
        sum.of(s);
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const float mean = s[q] * per_channel;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[q].v[i] = __fadd2_rn(v[q].v[i], c.only(-mean, i));
        }
    }
#pragma unroll
    for (int q = 0; q < R; ++q) s[q] = dot(v[q], v[q]);
    sum.of(s);
#pragma unroll
    for (int q = 0; q < R; ++q) {
        r[q] = rsqrtf(fmaf(s[q], per_channel, eps));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[q].v[i] = __fmul2_rn(v[q].v[i], both(r[q]));
    }
}

// g becomes the gradient of the rows whose normalised forms hat had the gradients g: r (g - hat mean(g hat) [- mean(g)])
template <int G, int R, typename Channels>
__device__ __forceinline__ void normalise_back(int kind, Eight (&g)[R], const Eight (&hat)[R], const float (&r)[R], const Channels& c, float per_channel,
                                               RowSum<G>& sum) {
    float m[2 * R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
        m[q] = dot(g[q], hat[q]);
        m[R + q] = kind == BRA_NORM_LAYER ? total(g[q]) : 0.f;
    }
    sum.of(m);
#pragma unroll
    for (int q = 0; q < R; ++q) {
        const float along = -r[q] * (m[q] * per_channel), mean = -r[q] * (m[R + q] * per_channel);
#pragma unroll
        for (int i = 0; i < 4; ++i) g[q].v[i] = __ffma2_rn(g[q].v[i], both(r[q]), __ffma2_rn(hat[q].v[i], both(along), c.only(mean, i)));
    }
}

// ---------------------------------------------------------------- forward
// A CTA's groups take the rows of its run in turn, R rows a round.  All groups make the same number of rounds (those without a row
// compute on what the ring holds and store nothing), so that the shuffles and barriers of the sums are met by every thread.
// THREADS: the most a CTA has.  Above 512 a thread has 64 registers (up to 640, 48, for two CTAs an SM): weights are read where they are used,
// row by row.
// R: two rows are two independent chains of exchanges and sums (one: 310 instructions a round of four 64-channel rows, 0.62 of them
// issued per cycle and scheduler).
__host__ __device__ constexpr int forward_rows(int threads) { return threads <= 128 ? 2 : 1; }
template <typename T, bool VECD, int G, bool POST, int THREADS, int R, bool FULL>
__global__ void __launch_bounds__(THREADS, THREADS == 384 || THREADS == 640 ? 2 : 0) norm_forward_kernel(const NormArgs a) {
    constexpr bool KEEP = THREADS <= 512, STRETCH = STRETCHES<VECD, G, THREADS>;
    __shared__ float cross[2][32][SUMS_AT_ONCE];
    extern __shared__ __align__(16) char ring[];
    constexpr int GROUPS = G ? THREADS / (G ? G : 1) : 1;
    const int mine = G ? threadIdx.x / (G ? G : 1) : 0;
    const Cols<VECD, FULL, VECD && sizeof(T) == 4> c(G ? threadIdx.x % (G ? G : 1) : threadIdx.x, G ? G : blockDim.x, a.C);
    RowSum<G> sum{cross};
    const int first = (int)(blockIdx.x * (long long)a.run), end = (int)min((long long)first + a.run, a.rows);
    const float per_channel = 1.f / (float)a.C;
    const bool has_y = a.y != nullptr;
    const long long start = (long long)(first + mine) * a.C;
    const int between = GROUPS * a.C;

    // rows of lanes go through slots of threads, rows of a CTA through slots of its own
    __shared__ uint64_t full[NORM_SLOTS];
    auto rows_in = [&] {
        if constexpr (!STRETCH) return Ahead<T, VECD, 2, forward_depth(THREADS, R), R>(ring);
        else return Stretch<T, VECD, 2, R>(a, ptx::smem_u32(ring), full);
    };
    auto in = rows_in();
    if constexpr (!STRETCH) {
        in.row[0] = static_cast<const T*>(a.x) + start + c.at(0);
        in.row[1] = has_y ? static_cast<const T*>(a.y) + start + c.at(0) : nullptr;
    } else {
        in.tensor[0] = static_cast<const T*>(a.x);
        in.tensor[1] = static_cast<const T*>(a.y);
        in.start(first, end);
    }
    T* h = a.h ? static_cast<T*>(a.h) + start : nullptr;
    T* n = a.n ? static_cast<T*>(a.n) + start : nullptr;
    int ask = first + mine;
    if constexpr (!STRETCH) {
#pragma unroll
        for (int k = 0; k < in.ROWS; ++k, ask += R * GROUPS) in.fetch(ask, GROUPS, end, between, c);
    }
    const bool per_image = a.gate_image || a.affine_image;
    // rows before it have the weights that are held; with weights of images a round ends with its image (R = 1 then)
    int image_end = first + mine;
    Eight gate, pw, pb, w, b;
    const float *gate_p = a.gate, *w_p = a.w, *b_p = a.b;
    if (POST && KEEP) {
        weights(a.post_w, 1.f, pw, c);
        weights(a.post_b, 0.f, pb, c);
    }
    for (int row = first + mine; row - mine < end; row += R * GROUPS) {
        if (row >= image_end && row < end) {
            const int image = per_image ? row / a.N : 0;
            gate_p = row_of(a.gate, a.gate_image ? (long long)image * a.C : 0);
            w_p = row_of(a.w, a.affine_image ? (long long)image * a.C : 0);
            b_p = row_of(a.b, a.affine_image ? (long long)image * a.C : 0);
            if (KEEP) {
                weights(gate_p, 1.f, gate, c);
                weights(w_p, 1.f, w, c);
                weights(b_p, 0.f, b, c);
            }
            image_end = per_image ? (int)min((long long)(image + 1) * a.N, (long long)end) : end;
        }
        Eight v[R], u[R];
        float r[R];
        in.arrived();
        if constexpr (!STRETCH) {
#pragma unroll
            for (int q = 0; q < R; ++q) {
                in.read(0, q, v[q]);
                if (has_y) in.read(1, q, u[q]);
            }
            in.fetch(ask, GROUPS, end, between, c);
            ask += R * GROUPS;
            in.next();
        } else {
#pragma unroll
            for (int q = 0; q < R; ++q) {
                in.read(0, q, v[q], c);
                if (has_y) in.read(1, q, u[q], c);
            }
            if (!POST && !n) __syncthreads();                  // else the sums' barriers say that all have read
        }
#pragma unroll
        for (int q = 0; q < R; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[q].v[i] = __fmul2_rn(v[q].v[i], both(a.alpha));
        if (has_y) {
            if (POST) {
                normalise<G>(a.post, u, r, c, a.eps, per_channel, sum);
                if (!KEEP) { weights(a.post_w, 1.f, pw, c); weights(a.post_b, 0.f, pb, c); }
#pragma unroll
                for (int q = 0; q < R; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) u[q].v[i] = __ffma2_rn(u[q].v[i], pw.v[i], pb.v[i]);
            }
            if (!KEEP) weights(gate_p, 1.f, gate, c);
#pragma unroll
            for (int q = 0; q < R; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[q].v[i] = __ffma2_rn(gate.v[i], u[q].v[i], v[q].v[i]);
        }
        if (h) {
#pragma unroll
            for (int q = 0; q < R; ++q)
                if (row + q * GROUPS < end) put(h + q * between, v[q], c);
            h += (long long)R * between;
        }
        if (n) {
            normalise<G>(a.pre, v, r, c, a.eps, per_channel, sum);
            if (!KEEP) { weights(w_p, 1.f, w, c); weights(b_p, 0.f, b, c); }
#pragma unroll
            for (int q = 0; q < R; ++q) {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[q].v[i] = __ffma2_rn(v[q].v[i], w.v[i], b.v[i]);
                if (row + q * GROUPS < end) put(n + q * between, v[q], c);
            }
            n += (long long)R * between;
        }
        if constexpr (STRETCH) in.next();
    }
}

// ---------------------------------------------------------------- backward
// THREADS 128: the sums over tokens stay in registers, and so do the weights.  More (long rows, whose CTAs would have no registers
// left): the sums that are wanted are in shared memory, each word its thread's own, and the weights are read again for every row.
// (All five sums added to, wanted or not, and CTAs of 128 registers a thread, 8 x 1024 x 1536, rms, bf16 49.7 us, now 39.9; x 2500, layer,
// fp32 222, now 148.)
template <typename T, bool VECD, int G, bool POST, int THREADS, int R, bool FULL>
__global__ void __launch_bounds__(THREADS, THREADS == 384 || (THREADS == 128 && POST && R == 2 && (G || sizeof(T) == 4)) ? 2 : THREADS == 128 && POST && R == 2 ? 3 : 0) norm_backward_kernel(const NormArgs a) {
    constexpr bool KEEP = THREADS == 128, STRETCH = STRETCHES<VECD, G, THREADS>;
    __shared__ float cross[2][32][SUMS_AT_ONCE];
    // !KEEP: [wanted sums][E][threads]; KEEP and several groups: [E][threads], to join the groups; then the ring of rows
    extern __shared__ __align__(16) float sums_sh[];
    constexpr int GROUPS = G ? THREADS / (G ? G : 1) : 1;
    const int mine = G ? threadIdx.x / (G ? G : 1) : 0;
    const Cols<VECD, FULL, VECD && sizeof(T) == 4> c(G ? threadIdx.x % (G ? G : 1) : threadIdx.x, G ? G : blockDim.x, a.C);
    RowSum<G> sum{cross};
    __shared__ uint64_t full[NORM_SLOTS];
    auto rows_in = [&] {
        float* ring = sums_sh + NORM_E * blockDim.x * (KEEP ? (G ? 1 : 0) : __popc(a.sums));
        if constexpr (!STRETCH) return Ahead<T, VECD, 4, backward_depth(THREADS, R), R>(ring);
        else return Stretch<T, VECD, 4, R>(a, ptx::smem_u32(ring), full);
    };
    auto in = rows_in();
    if constexpr (STRETCH) {
        in.tensor[0] = static_cast<const T*>(a.x); in.tensor[1] = static_cast<const T*>(a.y);
        in.tensor[2] = static_cast<const T*>(a.dh); in.tensor[3] = static_cast<const T*>(a.dn);
    }
    const bool has_y = a.y != nullptr, has_n = a.dn != nullptr;
    const int first = (int)(blockIdx.x * (long long)a.run), last = (int)min((long long)first + a.run, a.rows) - 1;
    const float per_channel = 1.f / (float)a.C;

    Eight acc[KEEP ? SUMS : 1];
    auto wants = [&](int s) { return (a.sums >> s) & 1; };
    auto shared_sum = [&](int s, int i) -> float2& { return reinterpret_cast<float2*>(sums_sh)[(a.place[s] * 4 + i) * blockDim.x + threadIdx.x]; };
    auto clear = [&](int s) {
        if constexpr (KEEP) acc[s].fill(0.f);
        else if (wants(s)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) shared_sum(s, i) = both(0.f);
        }
    };
    // sum s += a * b
    auto add = [&](int s, const Eight& p, const Eight& q) {
        if (!KEEP && !wants(s)) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (KEEP) acc[s].v[i] = __ffma2_rn(p.v[i], q.v[i], acc[s].v[i]);
            else shared_sum(s, i) = __ffma2_rn(p.v[i], q.v[i], shared_sum(s, i));
        }
    };
    auto add1 = [&](int s, const Eight& p) {
        if (!KEEP && !wants(s)) return;
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
                    for (int g = 0; g < GROUPS; ++g) t.v[i] = __fadd2_rn(t.v[i], join[i * THREADS + g * G + threadIdx.x]);
                }
            }
        }
        if (mine == 0) put(to, t, c);
        clear(s);
    };
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
            weights(gate_p, 1.f, gate, c);
            weights(w_p, 1.f, w, c);
            if (POST) { weights(a.post_w, 1.f, pw, c); weights(a.post_b, 0.f, pb, c); }
        }
        const long long start = (long long)(begin + mine) * a.C;
        const int between = GROUPS * a.C;
        auto from = [&](const void* p) { return p ? static_cast<const T*>(p) + start + c.at(0) : nullptr; };
        if constexpr (!STRETCH) { in.row[0] = from(a.x); in.row[1] = from(a.y); in.row[2] = from(a.dh); in.row[3] = from(a.dn); }
        T* dx = static_cast<T*>(a.dx) + start;
        T* dy = has_y ? static_cast<T*>(a.dy) + start : nullptr;
        int ask = begin + mine;
        if constexpr (!STRETCH) {
            in.restart();
#pragma unroll
            for (int k = 0; k < in.ROWS; ++k, ask += R * GROUPS) in.fetch(ask, GROUPS, end + 1, between, c);
        } else {
            in.start(begin, end + 1);
        }
        for (int row = begin + mine; row - mine <= end; row += R * GROUPS) {
            Eight v[R], u[R], g[R], d[R];
            float r[R], u_factor[R];
            in.arrived();
            if constexpr (!STRETCH) {
#pragma unroll
                for (int q = 0; q < R; ++q) {
                    in.read(0, q, v[q]);
                    if (has_y) in.read(1, q, u[q]);
                    if (a.dh) in.read(2, q, d[q]);
                    else d[q].fill(0.f);
                    if (has_n) in.read(3, q, g[q]);
                }
                in.fetch(ask, GROUPS, end + 1, between, c);
                ask += R * GROUPS;
                in.next();
            } else {
#pragma unroll
                for (int q = 0; q < R; ++q) {
                    in.read(0, q, v[q], c);
                    if (has_y) in.read(1, q, u[q], c);
                    if (a.dh) in.read(2, q, d[q], c);
                    else d[q].fill(0.f);
                    if (has_n) in.read(3, q, g[q], c);
                }
                if (!POST && !has_n) __syncthreads();          // else the sums' barriers say that all have read
            }
            // !KEEP: the weights, as they are used
            auto post_weights = [&] { if (!KEEP && POST) { weights(a.post_w, 1.f, pw, c); weights(a.post_b, 0.f, pb, c); } };
            auto yy = [&](int q, int i) { return POST ? __ffma2_rn(u[q].v[i], pw.v[i], pb.v[i]) : u[q].v[i]; };
#pragma unroll
            for (int q = 0; q < R; ++q)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[q].v[i] = __fmul2_rn(v[q].v[i], both(a.alpha));
            if (has_y) {
                if (POST) normalise<G>(a.post, u, u_factor, c, a.eps, per_channel, sum);
                post_weights();
                if (!KEEP) weights(gate_p, 1.f, gate, c);
#pragma unroll
                for (int q = 0; q < R; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[q].v[i] = __ffma2_rn(gate.v[i], yy(q, i), v[q].v[i]);
            }
            if (has_n) {
                normalise<G>(a.pre, v, r, c, a.eps, per_channel, sum);
                if (!KEEP) weights(w_p, 1.f, w, c);
#pragma unroll
                for (int q = 0; q < R; ++q) {
                    if (row + q * GROUPS <= end) {
                        add(SUM_W, g[q], v[q]);
                        add1(SUM_B, g[q]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) g[q].v[i] = __fmul2_rn(g[q].v[i], w.v[i]);
                }
                normalise_back<G>(a.pre, g, v, r, c, per_channel, sum);
#pragma unroll
                for (int q = 0; q < R; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[q].v[i] = __fadd2_rn(d[q].v[i], g[q].v[i]);
            }
            // d = dH
#pragma unroll
            for (int q = 0; q < R; ++q) {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[q].v[i] = __fmul2_rn(d[q].v[i], both(a.alpha));
                if (row + q * GROUPS <= end) put(dx + q * between, v[q], c);
            }
            dx += (long long)R * between;
            if (has_y) {
                post_weights();
                if (!KEEP) weights(gate_p, 1.f, gate, c);
#pragma unroll
                for (int q = 0; q < R; ++q) {
                    const bool live = row + q * GROUPS <= end;
                    if (live) {
                        Eight z;
#pragma unroll
                        for (int i = 0; i < 4; ++i) z.v[i] = yy(q, i);
                        add(SUM_GATE, d[q], z);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[q].v[i] = __fmul2_rn(d[q].v[i], gate.v[i]);
                    if (POST) {
                        if (live) {
                            add(SUM_POST_W, d[q], u[q]);
                            add1(SUM_POST_B, d[q]);
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) d[q].v[i] = __fmul2_rn(d[q].v[i], pw.v[i]);
                    }
                }
                if (POST) normalise_back<G>(a.post, d, u, u_factor, c, per_channel, sum);
#pragma unroll
                for (int q = 0; q < R; ++q)
                    if (row + q * GROUPS <= end) put(dy + q * between, d[q], c);
                dy += (long long)R * between;
            }
            if constexpr (STRETCH) in.next();
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
    long long slots;
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
    int per_sm;             // CTAs of an SM
    int rows;               // of a group in a round
    int run;                // rows of a CTA
    long long ctas;
};

Plan plan(const bra_norm_problem* q, bool backward) {
    Plan p;
    const long long rows = (long long)q->B * q->N;
    const int C = q->C;
    p.wide = norm_wide(C);
    p.group = norm_group(C);
    p.threads = p.wide ? p.group : 128;
    const int groups = p.wide ? 1 : p.threads / p.group;
    // as many CTAs as an SM holds at a time, by registers and the ring (the gradients' two rows of fp32, 98 KB for 128 threads: two, not three,
    // 16 x 1024 x 512 75 -> 60 us)
    const bool f32 = q->dtype == BRA_F32;
    int& per_sm = p.per_sm;
    const bool post = q->post != BRA_NORM_NONE;
    p.rows = backward ? backward_rows(p.threads, post, C % NORM_E == 0) : q->gate == BRA_GATE_IMAGE || q->per_image ? 1 : forward_rows(p.threads);
    if (p.threads <= 128) per_sm = (backward ? (p.rows == 2 && ((f32 && C % NORM_E == 0) || (post && !p.wide)) ? 2 : 3) : p.rows == 2 ? 4 : f32 || post ? 5 : 6) * 128 / p.threads;
    else if (p.threads > 512) per_sm = !backward && p.threads <= 640 ? 2 : 1;
    else if (!backward) per_sm = (post ? 768 : f32 ? 800 : 1024) / p.threads;       // 80 registers; three rounds of fp32; 64 registers
    else {
        // 80 registers up to 384 threads (six warps a scheduler), 128 above; the sums that there can be and two rows of four tensors in
        // shared memory
        const int sums = (q->pre != BRA_NORM_NONE ? 2 : 0) + (q->gate != BRA_GATE_NONE ? 1 : 0) + (post ? 2 : 0);
        const int by_smem = 224 * 1024 / (NORM_E * (4 * sums + 8 * (f32 ? 4 : 2))), by_regs = p.threads <= 384 ? 768 : 512;
        per_sm = (by_smem < by_regs ? by_smem : by_regs) / p.threads;
    }
    if (per_sm < 1) per_sm = 1;
    long long most = (long long)kSMs * per_sm;
    const long long at_once = (long long)groups * p.rows, rounds = (rows + at_once - 1) / at_once;
    if (most > rounds) most = rounds;
    const long long each = (rounds + most - 1) / most;
    p.run = (int)(each * at_once);
    p.ctas = (rows + p.run - 1) / p.run;
    return p;
}

bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
// whether two tensors of [B, N, C] have bytes in common (null: no such tensor)
bool overlap(const bra_norm_problem* p, const void* a, const void* b) {
    const uintptr_t u = reinterpret_cast<uintptr_t>(a), v = reinterpret_cast<uintptr_t>(b);
    const uintptr_t bytes = (uintptr_t)p->B * p->N * p->C * (p->dtype == BRA_BF16 ? 2 : 4);
    return u && v && (u < v ? v - u : u - v) < bytes;
}

bra_status check(const bra_norm_problem* p) {
    if (!p) return BRA_ERR_NULL;
    if (p->B <= 0 || p->N <= 0 || p->C <= 0) return BRA_ERR_SHAPE;
    if ((long long)p->B * p->N >= (1ll << 40) / p->C) return BRA_ERR_SHAPE;
    if ((long long)p->B * p->N > (1ll << 30)) return BRA_ERR_SHAPE;         // rows are counted in 32 bits, those asked for ahead too
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
    a.N = p->N; a.C = p->C; a.run = pl.run;
    a.gate_image = p->gate == BRA_GATE_IMAGE; a.affine_image = p->per_image != 0;
    a.pre = p->pre; a.post = p->post; a.eps = p->eps; a.alpha = p->alpha;
    return a;
}

long long slots_of(const bra_norm_problem* p, const Plan& pl) {
    return pl.ctas + ((p->gate == BRA_GATE_IMAGE || p->per_image) ? p->B : 0);
}

template <auto KERNEL>
cudaError_t launch_rows(size_t smem, const NormArgs& a, const Plan& pl, cudaStream_t st) {
    static PerDeviceMax attr;
    if (smem > 46 * 1024) {                 // 48 KB less what the kernels have of their own
        const cudaError_t e = attr.ensure((int)smem, [&] { return cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
        if (e != cudaSuccess) return e;
    }
    KERNEL<<<(unsigned)pl.ctas, pl.threads, smem, st>>>(a);
    count_launch();
    return cudaGetLastError();
}

// Slots of rows that are a CTA's: as many as fit beside what the CTA has besides them and the other CTAs of the SM, four at most.
size_t ring_of(NormArgs& a, const Plan& pl, int esize, int tensors, size_t besides) {
    a.ring_pitch = (int)(((size_t)pl.rows * a.C * esize + 15) / 16 * 16 + 16);
    const size_t slot = (size_t)a.ring_pitch * tensors, room = 220 * 1024 / pl.per_sm;
    const size_t n = room > besides ? (room - besides) / slot : 0;
    a.ring_slots = (int)(n < NORM_SLOTS ? n : NORM_SLOTS);
    return slot * a.ring_slots;
}

template <typename T, bool VECD, int G, int THREADS, bool FULL>
cudaError_t forward_as(NormArgs a, const Plan& pl, cudaStream_t st) {
    const bool post = a.post != BRA_NORM_NONE;
    constexpr int R = forward_rows(THREADS);
    size_t smem;
    if (STRETCHES<VECD, G, THREADS>) smem = ring_of(a, pl, sizeof(T), 2, 0);
    else smem = pl.rows == 1 ? Ahead<T, VECD, 2, forward_depth(THREADS, 1), 1>::bytes(pl.threads) : Ahead<T, VECD, 2, forward_depth(THREADS, R), R>::bytes(pl.threads);
    // the only rows of fewer than 256 threads in so large a kernel are those without a post-norm
    if constexpr (!VECD && THREADS > 384 && !FULL) return launch_rows<norm_forward_kernel<T, VECD, G, false, THREADS, R, FULL>>(smem, a, pl, st);
    else if (R == 1 || pl.rows == 1)
        return post ? launch_rows<norm_forward_kernel<T, VECD, G, true, THREADS, 1, FULL>>(smem, a, pl, st)
                    : launch_rows<norm_forward_kernel<T, VECD, G, false, THREADS, 1, FULL>>(smem, a, pl, st);
    else
        return post ? launch_rows<norm_forward_kernel<T, VECD, G, true, THREADS, R, FULL>>(smem, a, pl, st)
                    : launch_rows<norm_forward_kernel<T, VECD, G, false, THREADS, R, FULL>>(smem, a, pl, st);
}
template <typename T, bool VECD, int G, int THREADS, bool FULL>
cudaError_t backward_as(NormArgs a, const Plan& pl, cudaStream_t st) {
    constexpr bool KEEP = THREADS == 128;
    int wanted = 0;
    for (int s = 0; s < SUMS; ++s)
        if ((a.sums >> s) & 1) a.place[s] = wanted++;
    const size_t sums = sizeof(float) * NORM_E * pl.threads * (KEEP ? (G ? 1 : 0) : wanted);
    const bool post = a.post != BRA_NORM_NONE;
    constexpr int RP = backward_rows(THREADS, true, VECD), RN = backward_rows(THREADS, false, VECD);
    const size_t smem = sums + (STRETCHES<VECD, G, THREADS> ? ring_of(a, pl, sizeof(T), 4, sums) : post ? Ahead<T, VECD, 4, backward_depth(THREADS, RP), RP>::bytes(pl.threads)
                                                                                   : Ahead<T, VECD, 4, backward_depth(THREADS, RN), RN>::bytes(pl.threads));
    return post ? launch_rows<norm_backward_kernel<T, VECD, G, true, THREADS, RP, FULL>>(smem, a, pl, st)
                : launch_rows<norm_backward_kernel<T, VECD, G, false, THREADS, RN, FULL>>(smem, a, pl, st);
}
template <typename T, bool VECD>
cudaError_t launch(bool backward, const NormArgs& a, const Plan& pl, cudaStream_t st) {
#define BRA_NORM_AS(G, THREADS, FULL) (backward ? backward_as<T, VECD, G, THREADS, FULL>(a, pl, st) : forward_as<T, VECD, G, THREADS, FULL>(a, pl, st))
    if (!pl.wide) return pl.group == 8 ? BRA_NORM_AS(8, 128, false) : pl.group == 16 ? BRA_NORM_AS(16, 128, false) : BRA_NORM_AS(32, 128, false);
    const NormKernel k = norm_kernel(pl.group, backward, a.post != BRA_NORM_NONE);
    if (k.threads == 128) return BRA_NORM_AS(0, 128, false);
    if (k.threads == 384) return BRA_NORM_AS(0, 384, false);
    // where channels come by eight nothing depends on FULL
    if constexpr (!VECD)
        if (!k.full) return forward_as<T, VECD, 0, 512, false>(a, pl, st);
    return k.threads == 512 ? BRA_NORM_AS(0, 512, !VECD) : k.threads == 640 ? BRA_NORM_AS(0, 640, !VECD) : BRA_NORM_AS(0, 1024, !VECD);
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
    // rows are read ahead of the ones written; h may stand in x's or y's very place, where each row is read before it is written
    for (const void* q : {x, y})
        if (overlap(p, n, q) || (h != q && overlap(p, h, q))) return BRA_ERR_UNSUPPORTED;
    if (overlap(p, n, h)) return BRA_ERR_UNSUPPORTED;
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
    if (overlap(p, dx, dy)) return BRA_ERR_UNSUPPORTED;
    for (const void* q : {x, y, dh, dn})
        if (overlap(p, q, dx) || overlap(p, q, dy)) return BRA_ERR_UNSUPPORTED;      // rows are read ahead of the ones written
    if (!ws) return BRA_ERR_NULL;
    if (!aligned_to(ws, 256)) return BRA_ERR_ALIGN;
    if (ws_bytes < bra_norm_workspace_bytes(p)) return BRA_ERR_WORKSPACE;
    const Plan pl = plan(p, true);
    NormArgs a = args_of(p, pl);
    a.x = x; a.y = y; a.gate = gate; a.post_w = post_w; a.post_b = post_b; a.w = w; a.dh = dh; a.dn = dn; a.dx = dx; a.dy = dy;
    a.part = static_cast<float*>(ws);
    a.slots = slots_of(p, pl);
    JoinArgs j = {};
    j.part = a.part; j.slots = a.slots; j.N = p->N; j.C = p->C; j.run = pl.run; j.ctas = (int)pl.ctas; j.images = p->B;
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
