// Gradients of cross attention, bf16, warp-level tensor cores.  With P = 2^(scale log2e Q K^T - lse2), dP = dO V^T,
// delta = rowsum(dO o O) and dS = P o (dP - delta):  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO.
//
// Two kernels of one form, so that every sum has one owner and a fixed order (no atomics on results): one keeps 64 query rows and
// walks the keys (dQ), the other keeps 64 keys and walks the query rows of all heads of its group (dK, dV).  The side that is
// kept (X1, X2) is Q, dO or K, V; the side that is walked (Y1, Y2) is the other, 64 rows at a time (32 at head dim 128), two tiles
// in flight.  S and dP are made in both kernels: seven products instead of the five that one kernel with atomics on dQ needs.
// The first kernel also leaves each row's (lse2, delta) in scratch memory for the second.
// Where there are too few tiles on the kept side for the GPU (a short text under a large map) the walk is split over CTAs: each
// leaves fp32 sums in scratch memory and the last one adds them in order.
//
// P and dS go to bf16 for the products that contract over them (half a step, 2^-8, per term); everything else is fp32.
#include "cross_common.cuh"

#include <math.h>

namespace bra {
namespace {

constexpr int THREADS = 128, KEPT = 64;
// Walked rows of a tile, and the step by which walks are cut: a part's length is a multiple of it, so only the end of the rows (or keys)
// cuts a tile.
constexpr int walk_tile(int D) { return D == 128 ? 32 : 64; }

template <int D, bool DKV>
struct Shape {
    static constexpr int BN = walk_tile(D);
    static constexpr int TILE = BN * D * 2;
    static constexpr bool X_SHARED = D == 128;              // X fragments are read from shared memory for every tile
    static constexpr int STATS = DKV ? BN * 8 : 0;          // (lse2, delta) of the walked rows
    static constexpr int STAGE = 2 * TILE + STATS;
    static constexpr int X = X_SHARED ? 2 * KEPT * D * 2 : 0;
    static constexpr size_t smem = 2 * STAGE + X;
    static constexpr int SUMS = DKV ? 2 : 1;
    static_assert(KEPT % BN == 0, "the statistics of a walk's last tile");
};

template <int D, bool DKV>
__global__ void __launch_bounds__(THREADS) cross_grad_kernel(const CrossArgs a) {
    using S = Shape<D, DKV>;
    constexpr int BN = S::BN, NB = BN / 8, KD = D / 16, CH = D / 8;
    extern __shared__ __align__(128) char smem[];
    __shared__ int flag;
    const CrossPlace at(a);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g4 = lane >> 2, t4 = lane & 3;
    uint32_t* words = reinterpret_cast<uint32_t*>(smem + S::smem);

    // keys: all those of this CTA's walk (dQ), or the kept ones (dK, dV)
    const int key_lo = DKV ? at.tile * KEPT : at.split * a.split_len;
    const KeyRange keys = cross_keys(a, at.b, key_lo, min(a.Nk, DKV ? key_lo + KEPT : key_lo + a.split_len), words);
    if (a.key_mask) __syncthreads();
    const int walk_lo = DKV ? at.split * a.split_len : keys.lo;
    const int walk_hi = DKV ? min(a.rows, walk_lo + a.split_len) : keys.hi;

    const __nv_bfloat16* Q = static_cast<const __nv_bfloat16*>(a.Q);
    const __nv_bfloat16* dO = static_cast<const __nv_bfloat16*>(a.dO);
    const __nv_bfloat16* K = static_cast<const __nv_bfloat16*>(a.K) + (long long)at.b * a.Nk * a.k_stride + (long long)at.kvh * D;
    const __nv_bfloat16* V = static_cast<const __nv_bfloat16*>(a.V) + (long long)at.b * a.Nk * a.v_stride + (long long)at.kvh * D;
    const int padded = (a.rows + KEPT - 1) / KEPT * KEPT;
    float2* stats = a.stats + at.pair * padded;

    const int x0 = at.tile * KEPT + warp * 16;
    const int r[2] = {x0 + g4, x0 + g4 + 8};
    // of the kept rows: do they exist (dQ), are they seen (dK, dV)
    bool in[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        in[i] = DKV ? (keys.word((r[i] - key_lo) >> 5) >> ((r[i] - key_lo) & 31)) & 1 : r[i] < a.rows;

    const uint32_t base = ptx::smem_u32(smem), xs = base + 2 * S::STAGE;
    uint32_t x1[S::X_SHARED ? 1 : KD][4], x2[S::X_SHARED ? 1 : KD][4];
    float lse2[2] = {INFINITY, INFINITY}, delta[2] = {0.f, 0.f};
    {
        const __nv_bfloat16 *p1[2], *p2[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            p1[i] = DKV ? K + (in[i] ? r[i] * a.k_stride : 0) : Q + (in[i] ? cross_row(a, at, r[i], a.q_stride, D) : 0);
            p2[i] = DKV ? V + (in[i] ? r[i] * a.v_stride : 0) : dO + (in[i] ? cross_row(a, at, r[i], a.o_stride, D) : 0);
        }
        if constexpr (!DKV) {
            // delta = dO . O of the row, a quad's lanes each a quarter of the channels
            const __nv_bfloat16* O = static_cast<const __nv_bfloat16*>(a.O);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (in[i]) {
                    const __nv_bfloat16* o = O + cross_row(a, at, r[i], a.o_stride, D);
#pragma unroll
                    for (int k = 0; k < D / 8; ++k) {
                        const uint32_t u = __ldg(reinterpret_cast<const uint32_t*>(o + 8 * k + 2 * t4));
                        const uint32_t v = __ldg(reinterpret_cast<const uint32_t*>(p2[i] + 8 * k + 2 * t4));
                        delta[i] = fmaf(__uint_as_float(u << 16), __uint_as_float(v << 16), delta[i]);
                        delta[i] = fmaf(__uint_as_float(u & 0xffff0000u), __uint_as_float(v & 0xffff0000u), delta[i]);
                    }
                    const float e = __ldg(a.lse + cross_stat(a, at, r[i]));
                    lse2[i] = e == -INFINITY ? INFINITY : e * 1.4426950408889634f;     // no key seen: every p is 2^-inf
                }
                delta[i] += __shfl_xor_sync(0xffffffffu, delta[i], 1);
                delta[i] += __shfl_xor_sync(0xffffffffu, delta[i], 2);
                if (at.split == 0 && t4 == 0) stats[r[i]] = make_float2(lse2[i], in[i] ? delta[i] : 0.f);
            }
        }
        if constexpr (S::X_SHARED) {
            for (int u = threadIdx.x; u < KEPT * CH; u += THREADS) {
                const int row = u / CH, ch = u % CH, rr = at.tile * KEPT + row;
                const bool have = DKV ? (keys.word(row >> 5) >> (row & 31)) & 1 : rr < a.rows;
                const __nv_bfloat16* s1 = DKV ? K + (have ? rr * a.k_stride : 0) : Q + (have ? cross_row(a, at, rr, a.q_stride, D) : 0);
                const __nv_bfloat16* s2 = DKV ? V + (have ? rr * a.v_stride : 0) : dO + (have ? cross_row(a, at, rr, a.o_stride, D) : 0);
                ptx::cp_async_16(xs + chunk_at<D>(row, ch), s1 + ch * 8, have ? 16 : 0);
                ptx::cp_async_16(xs + KEPT * D * 2 + chunk_at<D>(row, ch), s2 + ch * 8, have ? 16 : 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int k = 0; k < KD; ++k) {
                    x1[k][i] = in[i] ? __ldg(reinterpret_cast<const uint32_t*>(p1[i] + 16 * k + 2 * t4)) : 0u;
                    x1[k][2 + i] = in[i] ? __ldg(reinterpret_cast<const uint32_t*>(p1[i] + 16 * k + 8 + 2 * t4)) : 0u;
                    x2[k][i] = in[i] ? __ldg(reinterpret_cast<const uint32_t*>(p2[i] + 16 * k + 2 * t4)) : 0u;
                    x2[k][2 + i] = in[i] ? __ldg(reinterpret_cast<const uint32_t*>(p2[i] + 16 * k + 8 + 2 * t4)) : 0u;
                }
        }
    }

    // a CTA whose keys are all hidden has nothing to walk
    int tiles = walk_hi > walk_lo ? (walk_hi - walk_lo + BN - 1) / BN : 0;
    if (DKV && keys.hi <= keys.lo) tiles = 0;

    auto copy = [&](int tile, int stage) {
        const uint32_t to0 = base + stage * S::STAGE;
#pragma unroll
        for (int i = 0; i < BN * CH / THREADS; ++i) {
            const int u = threadIdx.x + i * THREADS, row = u / CH, ch = u % CH;
            const int j = walk_lo + tile * BN + row;
            const uint32_t to = to0 + chunk_at<D>(row, ch);
            if (DKV) {
                const bool have = j < walk_hi;
                const long long q_off = have ? cross_row(a, at, j, a.q_stride, D) : 0, o_off = have ? cross_row(a, at, j, a.o_stride, D) : 0;
                ptx::cp_async_16(to, Q + q_off + ch * 8, have ? 16 : 0);
                ptx::cp_async_16(to + S::TILE, dO + o_off + ch * 8, have ? 16 : 0);
            } else {
                const bool have = (keys.word(tile * (BN / 32) + (row >> 5)) >> (row & 31)) & 1;
                const long long jj = have ? j : 0;
                ptx::cp_async_16(to, K + jj * a.k_stride + ch * 8, have ? 16 : 0);
                ptx::cp_async_16(to + S::TILE, V + jj * a.v_stride + ch * 8, have ? 16 : 0);
            }
        }
        // statistics exist up to the padded number of rows (a multiple of BN); rows that do not exist have (inf, 0), so their P and dS are
        // zero whatever their scores
        if (DKV && threadIdx.x < BN / 2)
            ptx::cp_async_16(to0 + 2 * S::TILE + threadIdx.x * 16, stats + walk_lo + tile * BN + threadIdx.x * 2, 16);
    };

    float acc[D / 8][4] = {}, accv[DKV ? D / 8 : 1][4] = {};
    const float c = a.scale_log2;
    if (tiles > 0) copy(0, 0);
    ptx::cp_async_commit();
    for (int tile = 0; tile < tiles; ++tile) {
        const int stage = tile & 1;
        if (tile + 1 < tiles) copy(tile + 1, stage ^ 1);
        ptx::cp_async_commit();
        ptx::cp_async_wait<1>();
        __syncthreads();
        const uint32_t y1 = base + stage * S::STAGE, y2 = y1 + S::TILE;
        float s[NB][4] = {}, dp[NB][4] = {};
#pragma unroll
        for (int k = 0; k < KD; ++k) {
            uint32_t f1[4], f2[4];
            if constexpr (S::X_SHARED) {
                a_frag<D>(xs, warp * 16, k, lane, f1);
                a_frag<D>(xs + KEPT * D * 2, warp * 16, k, lane, f2);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) { f1[i] = x1[k][i]; f2[i] = x2[k][i]; }
            }
#pragma unroll
            for (int n = 0; n < NB; n += 2) {
                uint32_t b[4];
                b_frag<D>(y1, 8 * n, k, lane, b);
                mma_bf16(s[n], f1, b[0], b[1]);
                mma_bf16(s[n + 1], f1, b[2], b[3]);
                b_frag<D>(y2, 8 * n, k, lane, b);
                mma_bf16(dp[n], f2, b[0], b[1]);
                mma_bf16(dp[n + 1], f2, b[2], b[3]);
            }
        }
        // s becomes P, dp becomes dS
        if constexpr (DKV) {
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const float4 st = ptx::lds_f32x4(y1 + 2 * S::TILE + (8 * n + 2 * t4) * 8);   // (lse2, delta) of two walked rows
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    s[n][2 * i] = ex2_approx(fmaf(s[n][2 * i], c, -st.x));
                    s[n][2 * i + 1] = ex2_approx(fmaf(s[n][2 * i + 1], c, -st.z));
                    dp[n][2 * i] = s[n][2 * i] * (dp[n][2 * i] - st.y);
                    dp[n][2 * i + 1] = s[n][2 * i + 1] * (dp[n][2 * i + 1] - st.w);
                }
            }
        } else {
            uint32_t seen[BN / 32];
#pragma unroll
            for (int w = 0; w < BN / 32; ++w) seen[w] = keys.word(tile * (BN / 32) + w);
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const uint32_t two = seen[n / 4] >> ((n & 3) * 8 + 2 * t4);
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float p0 = two & 1 ? ex2_approx(fmaf(s[n][2 * i], c, -lse2[i])) : 0.f;
                    const float p1 = two & 2 ? ex2_approx(fmaf(s[n][2 * i + 1], c, -lse2[i])) : 0.f;
                    dp[n][2 * i] = p0 * (dp[n][2 * i] - delta[i]);
                    dp[n][2 * i + 1] = p1 * (dp[n][2 * i + 1] - delta[i]);
                }
            }
        }
#pragma unroll
        for (int k = 0; k < BN / 16; ++k) {
            const uint32_t ds[4] = {pack2_bf16(dp[2 * k][0], dp[2 * k][1]), pack2_bf16(dp[2 * k][2], dp[2 * k][3]),
                                    pack2_bf16(dp[2 * k + 1][0], dp[2 * k + 1][1]), pack2_bf16(dp[2 * k + 1][2], dp[2 * k + 1][3])};
            const uint32_t p[4] = {pack2_bf16(s[2 * k][0], s[2 * k][1]), pack2_bf16(s[2 * k][2], s[2 * k][3]),
                                   pack2_bf16(s[2 * k + 1][0], s[2 * k + 1][1]), pack2_bf16(s[2 * k + 1][2], s[2 * k + 1][3])};
#pragma unroll
            for (int n = 0; n < KD; ++n) {
                uint32_t b[4];
                bt_frag<D>(y1, 16 * k, n, lane, b);
                mma_bf16(acc[2 * n], ds, b[0], b[1]);
                mma_bf16(acc[2 * n + 1], ds, b[2], b[3]);
                if constexpr (DKV) {
                    bt_frag<D>(y2, 16 * k, n, lane, b);
                    mma_bf16(accv[2 * n], p, b[0], b[1]);
                    mma_bf16(accv[2 * n + 1], p, b[2], b[3]);
                }
            }
        }
        __syncthreads();
    }
    ptx::cp_async_wait<0>();

    if (a.splits > 1) {
        const long long one = (long long)S::SUMS * KEPT * D;
        float* mine = a.part + ((at.pair * a.tiles + at.tile) * a.splits + at.split) * one;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float* to = mine + (warp * 16 + g4 + 8 * i) * D + 2 * t4;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) {
                *reinterpret_cast<float2*>(to + 8 * n) = make_float2(acc[n][2 * i], acc[n][2 * i + 1]);
                if constexpr (DKV) *reinterpret_cast<float2*>(to + KEPT * D + 8 * n) = make_float2(accv[n][2 * i], accv[n][2 * i + 1]);
            }
        }
        if (!cross_last(a.done + at.pair * a.tiles + at.tile, a.splits, &flag)) return;
        const float* all = a.part + (at.pair * a.tiles + at.tile) * a.splits * one;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float* from = all + (warp * 16 + g4 + 8 * i) * D + 2 * t4;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) {
                float2 t = make_float2(0.f, 0.f), u = t;
                for (int sp = 0; sp < a.splits; ++sp) {
                    const float2 v = __ldcg(reinterpret_cast<const float2*>(from + sp * one + 8 * n));
                    t.x += v.x; t.y += v.y;
                    if constexpr (DKV) {
                        const float2 w = __ldcg(reinterpret_cast<const float2*>(from + sp * one + KEPT * D + 8 * n));
                        u.x += w.x; u.y += w.y;
                    }
                }
                acc[n][2 * i] = t.x; acc[n][2 * i + 1] = t.y;
                if constexpr (DKV) { accv[n][2 * i] = u.x; accv[n][2 * i + 1] = u.y; }
            }
        }
    }
    if constexpr (DKV) {
        __nv_bfloat16 *pk[2], *pv[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bool have = r[i] < a.Nk;
            const long long j = (long long)at.b * a.Nk + r[i];
            pk[i] = have ? static_cast<__nv_bfloat16*>(a.dK) + j * a.k_stride + (long long)at.kvh * D : nullptr;
            pv[i] = have ? static_cast<__nv_bfloat16*>(a.dV) + j * a.v_stride + (long long)at.kvh * D : nullptr;
            if (!in[i]) {                   // hidden: its sums are of scores it does not have
#pragma unroll
                for (int n = 0; n < D / 8; ++n) acc[n][2 * i] = acc[n][2 * i + 1] = accv[n][2 * i] = accv[n][2 * i + 1] = 0.f;
            }
        }
        store_tile_rows<D>(acc, a.scale, a.scale, pk[0], pk[1], t4);
        store_tile_rows<D>(accv, 1.f, 1.f, pv[0], pv[1], t4);
    } else {
        __nv_bfloat16* p[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            p[i] = in[i] ? static_cast<__nv_bfloat16*>(a.dQ) + cross_row(a, at, r[i], a.q_stride, D) : nullptr;
        store_tile_rows<D>(acc, a.scale, a.scale, p[0], p[1], t4);
    }
}

CrossSplit split_of(const CrossDims& d, bool dkv) {
    return cross_split((long long)d.B * d.kv, dkv ? d.Nk : d.rows, KEPT, dkv ? d.rows : d.Nk, walk_tile(d.D), 2);
}

template <int D, bool DKV>
cudaError_t launch(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    using S = Shape<D, DKV>;
    cross_cut(a, split_of(d, DKV));
    const size_t smem = S::smem + (a.key_mask ? ((size_t)(DKV ? KEPT : a.split_len) + 31) / 32 * 4 : 0);
    static PerDeviceMax attr;
    const cudaError_t e = attr.ensure((int)smem, [&] {
        return cudaFuncSetAttribute(cross_grad_kernel<D, DKV>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    });
    if (e != cudaSuccess) return e;
    cross_grad_kernel<D, DKV><<<(unsigned)((long long)d.B * d.kv * a.splits * a.tiles), THREADS, smem, st>>>(a);
    count_launch();
    return cudaGetLastError();
}
template <int D>
cudaError_t both(const CrossDims& d, const CrossArgs& a, cudaStream_t st) {
    const cudaError_t e = launch<D, false>(d, a, st);
    return e != cudaSuccess ? e : launch<D, true>(d, a, st);
}

}  // namespace

size_t cross_backward_mma_part(const CrossDims& d) {
    size_t most = 0;
    for (int dkv = 0; dkv < 2; ++dkv) {
        const CrossSplit s = split_of(d, dkv);
        const size_t n = s.splits > 1 ? (size_t)s.splits * s.tiles * d.B * d.kv * (1 + dkv) * KEPT * d.D : 0;
        most = n > most ? n : most;
    }
    return most;
}

cudaError_t launch_cross_backward_mma(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    switch (d.D) {
        case 16: return both<16>(d, a, st);
        case 32: return both<32>(d, a, st);
        case 64: return both<64>(d, a, st);
        default: return both<128>(d, a, st);
    }
}

}  // namespace bra
