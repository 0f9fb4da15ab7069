// Cross attention of bf16 queries to an encoder's states, warp-level tensor cores:
//   O = softmax(scale Q K^T over visible keys) V, one pass over the keys with the running maximum and sum of the softmax.
//
// ROWS: a CTA of four warps takes 64 rows, 16 a warp; tiles of 64 keys and values cross shared memory, two in flight
//   (cp.async; hidden keys and values are filled with zeros and never read, so what stands in them reaches nothing).
// KEYS: at most 16 rows (a step of generation with few heads): every warp has the same rows and its own tiles of 32 keys,
//   two in flight, no barrier in the loop; the four warps' sums are joined at the end.  Bound by the bytes of K and V.
// Where output tiles are too few for the GPU the keys are split over CTAs; each leaves its unnormalised sums in scratch memory
// and the last one to finish (a counter says so) adds them in order.
//
// Softmax in base 2 with the scale folded in: p = 2^(s c - m c), one FMA and one ex2 a score; sums are of the unrounded p in
// fp32, P goes to bf16 for the second product (half a step, 2^-8, per term), accumulators are fp32.
#include "cross_common.cuh"

#include <math.h>

namespace bra {
namespace {

constexpr int THREADS = 128;

template <int D, bool KEYS>
struct Shape {
    static constexpr int BN = KEYS ? 32 : 64;               // keys of a tile
    static constexpr int TEAMS = KEYS ? 4 : 1;              // warps or the CTA
    static constexpr int TEAM_THREADS = THREADS / TEAMS;
    static constexpr int TILE = BN * D * 2;                 // bytes of a tile of K or V
    static constexpr int ROWS = KEYS ? 16 : 64;             // of a CTA
    static constexpr int JOIN = KEYS ? 4 * 16 * (D + 4) * 4 : 0;
    static constexpr int STAGES = 2 * 2 * TILE * TEAMS;
    static constexpr size_t smem = STAGES > JOIN ? STAGES : JOIN;
};

template <bool KEYS>
__device__ __forceinline__ void team_sync() {
    if (KEYS) __syncwarp();
    else __syncthreads();
}

template <int D, bool KEYS>
__global__ void __launch_bounds__(THREADS) cross_attend_kernel(const CrossArgs a) {
    using S = Shape<D, KEYS>;
    constexpr int BN = S::BN, NB = BN / 8, KD = D / 16;
    extern __shared__ __align__(128) char smem[];
    __shared__ int flag;
    const CrossPlace at(a);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g4 = lane >> 2, t4 = lane & 3;
    const KeyRange keys = cross_keys(a, at.b, at.split * a.split_len, min(a.Nk, (at.split + 1) * a.split_len),
                                     reinterpret_cast<uint32_t*>(smem + S::smem));
    if (a.key_mask) __syncthreads();

    const int row0 = at.tile * S::ROWS + (KEYS ? 0 : warp * 16);
    const int r[2] = {row0 + g4, row0 + g4 + 8};
    uint32_t q[KD][4];
    {
        const __nv_bfloat16* Q = static_cast<const __nv_bfloat16*>(a.Q);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bool in = r[i] < a.rows;
            const __nv_bfloat16* p = Q + (in ? cross_row(a, at, r[i], a.q_stride, D) : 0);
#pragma unroll
            for (int k = 0; k < KD; ++k) {
                q[k][i] = in ? __ldg(reinterpret_cast<const uint32_t*>(p + 16 * k + 2 * t4)) : 0u;
                q[k][2 + i] = in ? __ldg(reinterpret_cast<const uint32_t*>(p + 16 * k + 8 + 2 * t4)) : 0u;
            }
        }
    }

    const int team = KEYS ? warp : 0, member = KEYS ? lane : threadIdx.x;
    const uint32_t base = ptx::smem_u32(smem) + team * (4 * S::TILE);      // stage s: K at 2 s TILE, V behind it
    const __nv_bfloat16* K = static_cast<const __nv_bfloat16*>(a.K) + (long long)at.b * a.Nk * a.k_stride + (long long)at.kvh * D;
    const __nv_bfloat16* V = static_cast<const __nv_bfloat16*>(a.V) + (long long)at.b * a.Nk * a.v_stride + (long long)at.kvh * D;
    const int tiles = (keys.hi - keys.lo + BN - 1) / BN;

    auto copy = [&](int tile, int stage) {
        constexpr int CH = D / 8;
        uint32_t seen[BN / 32];
#pragma unroll
        for (int w = 0; w < BN / 32; ++w) seen[w] = keys.word(tile * (BN / 32) + w);
#pragma unroll
        for (int i = 0; i < BN * CH / S::TEAM_THREADS; ++i) {
            const int u = member + i * S::TEAM_THREADS, row = u / CH, ch = u % CH;
            const bool in = (seen[BN == 32 ? 0 : row >> 5] >> (row & 31)) & 1;
            const long long j = in ? keys.lo + tile * BN + row : 0;
            const uint32_t to = base + stage * (2 * S::TILE) + chunk_at<D>(row, ch);
            ptx::cp_async_16(to, K + j * a.k_stride + ch * 8, in ? 16 : 0);
            ptx::cp_async_16(to + S::TILE, V + j * a.v_stride + ch * 8, in ? 16 : 0);
        }
    };

    float o[D / 8][4] = {};
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
    const float c = a.scale_log2;
    int stage = 0;
    if (team < tiles) copy(team, 0);
    ptx::cp_async_commit();
    for (int tile = team; tile < tiles; tile += S::TEAMS, stage ^= 1) {
        if (tile + S::TEAMS < tiles) copy(tile + S::TEAMS, stage ^ 1);
        ptx::cp_async_commit();
        ptx::cp_async_wait<1>();
        team_sync<KEYS>();
        const uint32_t ks = base + stage * (2 * S::TILE), vs = ks + S::TILE;

        float s[NB][4] = {};
#pragma unroll
        for (int k = 0; k < KD; ++k)
#pragma unroll
            for (int n = 0; n < NB; n += 2) {
                uint32_t b[4];
                b_frag<D>(ks, 8 * n, k, lane, b);
                mma_bf16(s[n], q[k], b[0], b[1]);
                mma_bf16(s[n + 1], q[k], b[2], b[3]);
            }
        uint32_t seen[BN / 32];
        bool all = true;
#pragma unroll
        for (int w = 0; w < BN / 32; ++w) {
            seen[w] = keys.word(tile * (BN / 32) + w);
            all = all && seen[w] == 0xffffffffu;
        }
        if (!all) {
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const uint32_t two = seen[n / 4] >> ((n & 3) * 8 + 2 * t4);
                if (!(two & 1)) s[n][0] = s[n][2] = -INFINITY;
                if (!(two & 2)) s[n][1] = s[n][3] = -INFINITY;
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float top = m[i];
#pragma unroll
            for (int n = 0; n < NB; ++n) top = ptx::fmax3(top, s[n][2 * i], s[n][2 * i + 1]);
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            const float ref = top == -INFINITY ? 0.f : top * c;           // no key seen so far: every p is 2^-inf
            const float keep = ex2_approx(m[i] * c - ref);
            m[i] = top;
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                s[n][2 * i] = ex2_approx(fmaf(s[n][2 * i], c, -ref));
                s[n][2 * i + 1] = ex2_approx(fmaf(s[n][2 * i + 1], c, -ref));
                sum += s[n][2 * i] + s[n][2 * i + 1];
            }
            l[i] = l[i] * keep + sum;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) { o[n][2 * i] *= keep; o[n][2 * i + 1] *= keep; }
        }
#pragma unroll
        for (int k = 0; k < BN / 16; ++k) {
            const uint32_t p[4] = {pack2_bf16(s[2 * k][0], s[2 * k][1]), pack2_bf16(s[2 * k][2], s[2 * k][3]),
                                   pack2_bf16(s[2 * k + 1][0], s[2 * k + 1][1]), pack2_bf16(s[2 * k + 1][2], s[2 * k + 1][3])};
#pragma unroll
            for (int n = 0; n < KD; ++n) {
                uint32_t b[4];
                bt_frag<D>(vs, 16 * k, n, lane, b);
                mma_bf16(o[2 * n], p, b[0], b[1]);
                mma_bf16(o[2 * n + 1], p, b[2], b[3]);
            }
        }
        team_sync<KEYS>();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
        l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    }
    ptx::cp_async_wait<0>();

    if (KEYS) {
        // join of the four warps: 32 threads of a warp hold 16 rows; warp w then finishes rows 4 w .. 4 w + 3
        float* sh = reinterpret_cast<float*>(smem);                 // [warp][16][D + 4]: D sums, m, l
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float* to = sh + (warp * 16 + g4 + 8 * i) * (D + 4);
#pragma unroll
            for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(to + 8 * n + 2 * t4) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
            if (t4 == 0) { to[D] = m[i]; to[D + 1] = l[i]; }
        }
        __syncthreads();
        for (int k = 0; k < 4; ++k) {
            const int row = 4 * warp + k;
            if (row >= a.rows - row0) break;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < 4; ++w) top = fmaxf(top, sh[(w * 16 + row) * (D + 4) + D]);
            const float ref = top == -INFINITY ? 0.f : top * c;
            float f[4], sum = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                f[w] = ex2_approx(sh[(w * 16 + row) * (D + 4) + D] * c - ref);
                sum += f[w] * sh[(w * 16 + row) * (D + 4) + D + 1];
            }
            if (a.splits == 1) {
                const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;      // a NaN stays one
                __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.Oo) + cross_row(a, at, row0 + row, a.o_stride, D);
                for (int ch = lane; ch < D; ch += 32) {
                    float v = 0.f;
#pragma unroll
                    for (int w = 0; w < 4; ++w) v += f[w] * sh[(w * 16 + row) * (D + 4) + ch];
                    out[ch] = __float2bfloat16_rn(v * inv);
                }
                if (a.lse && lane == 0)
                    a.lse[cross_stat(a, at, row0 + row)] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
            } else {
                float* part = a.part + ((at.pair * a.tiles + at.tile) * a.splits + at.split) * (long long)(S::ROWS * (D + 4)) + row * (D + 4);
                for (int ch = lane; ch < D; ch += 32) {
                    float v = 0.f;
#pragma unroll
                    for (int w = 0; w < 4; ++w) v += f[w] * sh[(w * 16 + row) * (D + 4) + ch];
                    part[ch] = v;
                }
                if (lane == 0) { part[D] = top; part[D + 1] = sum; }
            }
        }
    } else if (a.splits == 1) {
        float inv[2];
        __nv_bfloat16* p[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            inv[i] = l[i] == 0.f ? 0.f : 1.f / l[i];
            const bool in = r[i] < a.rows;
            p[i] = in ? static_cast<__nv_bfloat16*>(a.Oo) + cross_row(a, at, r[i], a.o_stride, D) : nullptr;
            if (a.lse && in && t4 == 0)
                a.lse[cross_stat(a, at, r[i])] = l[i] == 0.f ? -INFINITY : (m[i] * c + log2f(l[i])) * 0.69314718055994531f;
        }
        store_tile_rows<D>(o, inv[0], inv[1], p[0], p[1], t4);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if (r[i] >= a.rows) continue;
            float* part = a.part + ((at.pair * a.tiles + at.tile) * a.splits + at.split) * (long long)(S::ROWS * (D + 4)) +
                          (r[i] - at.tile * S::ROWS) * (D + 4);
#pragma unroll
            for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(part + 8 * n + 2 * t4) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
            if (t4 == 0) { part[D] = m[i]; part[D + 1] = l[i]; }
        }
    }
    if (a.splits == 1) return;

    if (!cross_last(a.done + at.pair * a.tiles + at.tile, a.splits, &flag)) return;
    const long long one = S::ROWS * (D + 4);
    cross_join<D>(a.part + (at.pair * a.tiles + at.tile) * a.splits * one, one, D + 4, min(S::ROWS, a.rows - at.tile * S::ROWS), a.splits, c,
                  reinterpret_cast<float*>(smem),
                  [&](int row, int ch, float4 v) {
                      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.Oo) + cross_row(a, at, at.tile * S::ROWS + row, a.o_stride, D) + 4 * ch;
                      *reinterpret_cast<uint2*>(out) = make_uint2(pack2_bf16(v.x, v.y), pack2_bf16(v.z, v.w));
                  },
                  [&](int row, float ref, float sum) {
                      if (a.lse) a.lse[cross_stat(a, at, at.tile * S::ROWS + row)] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
                  });
}

bool few_rows(const CrossDims& d) { return d.rows <= 16; }

CrossSplit split_of(const CrossDims& d) {
    const bool keys = few_rows(d);
    return cross_split((long long)d.B * d.kv, d.rows, keys ? 16 : 64, d.Nk, keys ? 128 : 64, 3);
}

template <int D, bool KEYS>
cudaError_t launch(CrossArgs a, long long pairs, cudaStream_t st) {
    using S = Shape<D, KEYS>;
    size_t smem = S::smem + (a.key_mask ? ((size_t)a.split_len + 31) / 32 * 4 : 0);
    const size_t join = a.splits > 1 ? sizeof(float) * S::ROWS * (a.splits + 1) : 0;
    smem = smem > join ? smem : join;
    static PerDeviceMax attr;
    const cudaError_t e = attr.ensure((int)smem, [&] {
        return cudaFuncSetAttribute(cross_attend_kernel<D, KEYS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    });
    if (e != cudaSuccess) return e;
    cross_attend_kernel<D, KEYS><<<(unsigned)(pairs * a.splits * a.tiles), THREADS, smem, st>>>(a);
    count_launch();
    return cudaGetLastError();
}

}  // namespace

size_t cross_attend_mma_part(const CrossDims& d) {
    const CrossSplit s = split_of(d);
    return s.splits > 1 ? (size_t)s.splits * s.tiles * d.B * d.kv * (few_rows(d) ? 16 : 64) * (d.D + 4) : 0;
}

cudaError_t launch_cross_attend_mma(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    cross_cut(a, split_of(d));
    const long long pairs = (long long)d.B * d.kv;
    if (few_rows(d)) {
        switch (d.D) {
            case 16: return launch<16, true>(a, pairs, st);
            case 32: return launch<32, true>(a, pairs, st);
            case 64: return launch<64, true>(a, pairs, st);
            default: return launch<128, true>(a, pairs, st);
        }
    }
    switch (d.D) {
        case 16: return launch<16, false>(a, pairs, st);
        case 32: return launch<32, false>(a, pairs, st);
        case 64: return launch<64, false>(a, pairs, st);
        default: return launch<128, false>(a, pairs, st);
    }
}

}  // namespace bra
