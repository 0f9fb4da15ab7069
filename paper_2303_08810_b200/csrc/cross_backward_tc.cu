// Gradients of cross attention, bf16, on the 5th-generation tensor cores: many rows, many keys.  With P = 2^(scale log2e Q K^T - lse2),
// dP = dO V^T, delta = rowsum(dO o O), dS = P o (dP - delta):  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO.
//
// Two kernels of one form, each sum with one owner and a fixed order: one keeps a tile of 128 query rows (Q, dO) and walks blocks of 128
// keys (dQ), the other keeps 128 keys (K, V) and walks blocks of query rows of all heads of its group (dK, dV).  X1, X2 are the kept tiles,
// Y1, Y2 the walked ones:
//   S = X1 Y1^T, dP = X2 Y2^T (128 x 128, fp32 in tensor memory),  A1 += dS Y1,  (dK, dV) A2 += P Y2,  dS and P read from tensor memory.
// A one-kernel form with atomics on dQ would need five products instead of seven; its sums would depend on the order of arrival.
//
// One CTA per SM walks tiles; two warpgroups share the 128 lanes of a tile, 64 columns each: a thread turns 64 scores into P and 64 values of
// dP into dS, and needs nothing from its neighbours (lse and delta are known).  Warp 8 copies (bulk tensor copies through a ring), warps 9 and
// 10 issue the products, warp 11 zeroes hidden keys' rows.  S and dP of the next block are made as soon as this one's are in registers, where P
// and dS have tensor memory of their own; at head dim 128 the four accumulators of dK, dV fill it, P lies over S and dS over dP.
// Per block the products are 1100 (dQ) and 1670 (dK, dV) cycles of the tensor pipe at head dim 64, 1560 and 2080 at 128; the
// exponentials 1024 of the MUFU; what bounds it is the chain from S over P to dS at two warps a scheduler.
//
// Rounding: P and dS to bf16 for the products that contract over them (half a step, 2^-8, per term); everything else is fp32.
#include "cross_tc_common.cuh"

#include <math.h>

namespace bra {
namespace {

using namespace cross_tc;

constexpr int THREADS = 384;

template <int D, bool DKV>
struct Shape {
    static constexpr int BOX = D < 64 ? D : 64, BOXES = D / BOX, ROW = BOX * 2, PLANE = 128 * ROW, TILE = PLANE * BOXES;
    static constexpr int STAGES = D == 128 ? 2 : 4;
    static constexpr uint32_t SWIZZLE = D < 64 ? 4 : 2;
    static constexpr int STAGE = 2 * TILE;                          // Y1, Y2
    // kept tiles in flight: where there is room, the next one's copy runs beside this one's last blocks (short walks are mostly ends)
    static constexpr int XS = D <= 64 ? 2 : 1;
    static constexpr int OFF_Y = XS * 2 * TILE, OFF_STAT = OFF_Y + STAGES * STAGE, OFF_BAR = OFF_STAT + (DKV ? STAGES * 1024 : 0);
    static constexpr size_t smem = OFF_BAR + 256 + 1024;
    // tensor memory: S 0, dP 128, A1 256, A2 behind it, P and dS behind both or over S and dP
    static constexpr bool S_APART = !DKV || D <= 64, DS_APART = !DKV || D <= 64;
    static constexpr int TM_DP = 128, TM_A1 = 256, TM_A2 = 256 + D;
    static constexpr int TM_P = S_APART ? 384 : 0, TM_DS = DS_APART ? (D <= 64 ? 448 : 384) : TM_DP;
    static constexpr int P_HALF = S_APART ? 32 : 64, DS_HALF = DS_APART ? 32 : 64;      // from the first warpgroup's columns to the second's
};

struct TcArgs {
    CrossArgs a;
    const float* stats;     // [pair][row block][2][128]: -log2 of the softmax denominator, -delta
    int tokens;             // of a tile of rows: 128 / group
    int row_blocks;         // of a pair
    int tiles;              // kept tiles of a pair
    int splits, part;       // parts of a walk and their length in blocks
    int total;              // parts of all tiles of all pairs
    FastDiv tiles_div, splits_div;
};

// SPLIT: walks are cut in parts
template <int D, bool DKV, bool SPLIT>
__global__ void __launch_bounds__(THREADS, 1)
cross_grad_tc_kernel(const TcArgs g, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_do) {
    using S = Shape<D, DKV>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bar = reinterpret_cast<uint64_t*>(smem + S::OFF_BAR);
    uint64_t *x_full = bar, *x_empty = bar + 2, *s_ready = bar + 4, *dp_ready = bar + 5, *s_free = bar + 6, *dp_free = bar + 7, *p_ready = bar + 8,
             *ds_ready = bar + 9, *pv_done = bar + 10, *acc_done = bar + 11, *y_full = bar + 12, *y_clean = y_full + S::STAGES,
             *y_empty = y_clean + S::STAGES;
    uint32_t* slot = reinterpret_cast<uint32_t*>(y_empty + S::STAGES);
    const uint32_t base = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const CrossArgs& a = g.a;

    if (threadIdx.x == 0) {
        for (int i = 0; i < 12; ++i) mbar_init(bar + i, i == 2 || i == 3 ? 2 : i >= 6 && i <= 9 ? 256 : 1);
        for (int s = 0; s < S::STAGES; ++s) { mbar_init(y_full + s, 1); mbar_init(y_clean + s, 1); mbar_init(y_empty + s, 2); }
        fence_mbar_init();
    }
    // rows of a block that no copy writes (a group that does not divide 128) meet a P of zero: they must be finite
    if (DKV && g.tokens * a.group < 128) {
        for (int i = threadIdx.x; i < S::STAGES * S::STAGE / 16; i += THREADS) sts_f32x4(base + S::OFF_Y + i * 16, 0.f, 0.f, 0.f, 0.f);
        fence_proxy_async_smem();
    }
    if (warp == 9) tmem_alloc(slot, 512);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *slot;
    bool ok = true;
    pdl_wait();                             // the statistics of the kernel before
    pdl_launch_dependents();

    // every role walks the same tiles
    // x0: first token of the kept tile (a query's or a key); j0: first block of this part of its walk
    struct Tile { int p, b, kvh, x0, end, j0, blocks; };
    auto tile_of = [&](int t) {
        Tile x;
        const int tile = SPLIT ? (int)fdiv((uint32_t)t, g.splits_div) : t;
        x.j0 = SPLIT ? (t - tile * g.splits) * g.part : 0;
        x.p = (int)fdiv((uint32_t)tile, g.tiles_div);
        x.x0 = (tile - x.p * g.tiles) * (DKV ? 128 : g.tokens);
        x.b = (int)fdiv((uint32_t)x.p, a.kv_div);
        x.kvh = x.p - x.b * a.kv;
        x.end = cross_key_end(a, x.b);
        x.blocks = DKV ? (x.x0 < x.end ? g.row_blocks : 0) : (x.end + 127) >> 7;
        if (SPLIT) x.blocks = min(max(x.blocks - x.j0, 0), g.part);
        return x;
    };

    // registers: launched with 168 a thread, 384 x 168 = 64512 = 256 x 224 + 128 x 56
    if (warp < 8) {
        // ------------------------------------------------ P and dS
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int half = warp >> 2, row = threadIdx.x & 127;
        const uint32_t tl = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const float c = a.scale_log2;
        const float2 c2 = make_float2(c, c);
        const int in_token = DKV ? 0 : (int)fdiv((uint32_t)row, a.group_div), head = DKV ? 0 : row - in_token * a.group;
        uint32_t n = 0;                         // blocks so far
        for (int t = blockIdx.x; t < g.total && ok; t += gridDim.x) {
            const Tile x = tile_of(t);
            const uint8_t* mask = a.key_mask ? a.key_mask + (long long)x.b * a.Nk : nullptr;
            float nl = 0.f, nd = 0.f;           // -lse2, -delta of the thread's row (dQ)
            if (!DKV) {
                const float* st = g.stats + ((long long)x.p * g.row_blocks + x.x0 / g.tokens) * 256 + row;
                nl = __ldcg(st);
                nd = __ldcg(st + 128);
            }
            const float2 nl2 = make_float2(nl, nl), nd2 = make_float2(nd, nd);
            uint32_t bytes = !DKV && mask ? mask_bytes(mask, x.j0 * 128, x.end, lane) : 0u;
            for (int j = 0; j < x.blocks; ++j, ++n) {
                const int stage = n % S::STAGES;
                const uint32_t stat = base + S::OFF_STAT + stage * 1024 + half * 256;
                const int key0 = (x.j0 + j) * 128;
                const bool cut = !DKV && (mask || key0 + 128 > x.end);            // some keys may be hidden
                uint32_t see[2] = {0u, 0u};
                if (cut) {
                    const Seen seen = seen_of(mask, bytes, key0, x.end);
                    see[0] = seen.w[2 * half];
                    see[1] = seen.w[2 * half + 1];
                    if (mask) bytes = mask_bytes(mask, key0 + 128, x.end, lane);
                }
                if (DKV) wait_for(y_full + stage, (n / S::STAGES) & 1, ok);       // the rows' statistics
                wait_for(s_ready, n & 1, ok);
                tc_fence_after_sync();
                uint32_t p[64];
                tmem_ld_32x32b_x32(tl + half * 64, p);
                tmem_ld_32x32b_x32(tl + half * 64 + 32, p + 32);
                tmem_ld_wait();
                if (S::S_APART) {
                    tc_fence_before_sync();
                    mbar_arrive(s_free);
                }
                auto pair = [](const uint32_t* r) { return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1])); };
#pragma unroll
                for (int k = 0; k < 64; k += 4) {
                    float2 m0 = nl2, m1 = nl2;
                    if (DKV) {
                        const float4 v = lds_f32x4(stat + k * 4);
                        m0 = make_float2(v.x, v.y);
                        m1 = make_float2(v.z, v.w);
                    }
                    const float2 u = __ffma2_rn(pair(p + k), c2, m0), v = __ffma2_rn(pair(p + k + 2), c2, m1);
                    p[k] = __float_as_uint(ex2_approx(u.x));
                    p[k + 1] = __float_as_uint(ex2_approx(u.y));
                    p[k + 2] = __float_as_uint(ex2_approx(v.x));
                    p[k + 3] = __float_as_uint(ex2_approx(v.y));
                }
                if (DKV) {
                    if (S::S_APART && j > 0) {
                        wait_for(pv_done, (n - 1) & 1, ok);
                        tc_fence_after_sync();
                    }
#pragma unroll
                    for (int k = 0; k < 64; k += 32) {
                        uint32_t q[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) q[e] = pack2_bf16(__uint_as_float(p[k + 2 * e]), __uint_as_float(p[k + 2 * e + 1]));
                        tmem_st_32x32b_x16(tl + S::TM_P + half * S::P_HALF + k / 2, q);
                    }
                    tmem_st_wait();
                    tc_fence_before_sync();
                    mbar_arrive(p_ready);
                }
                wait_for(dp_ready, n & 1, ok);
                tc_fence_after_sync();
                uint32_t dp[64];
                tmem_ld_32x32b_x32(tl + S::TM_DP + half * 64, dp);
                tmem_ld_32x32b_x32(tl + S::TM_DP + half * 64 + 32, dp + 32);
                tmem_ld_wait();
                if (S::DS_APART) {
                    tc_fence_before_sync();
                    mbar_arrive(dp_free);
                }
#pragma unroll
                for (int k = 0; k < 64; k += 4) {
                    float2 m0 = nd2, m1 = nd2;
                    if (DKV) {
                        const float4 v = lds_f32x4(stat + 512 + k * 4);
                        m0 = make_float2(v.x, v.y);
                        m1 = make_float2(v.z, v.w);
                    }
                    const float2 u = __fmul2_rn(pair(p + k), __fadd2_rn(pair(dp + k), m0)), v = __fmul2_rn(pair(p + k + 2), __fadd2_rn(pair(dp + k + 2), m1));
                    dp[k] = __float_as_uint(u.x);
                    dp[k + 1] = __float_as_uint(u.y);
                    dp[k + 2] = __float_as_uint(v.x);
                    dp[k + 3] = __float_as_uint(v.y);
                }
                if (cut) {
#pragma unroll
                    for (int k = 0; k < 64; ++k)
                        if (!((see[k >> 5] >> (k & 31)) & 1)) dp[k] = 0u;
                }
                if (S::DS_APART && j > 0) {
                    wait_for(acc_done, (n - 1) & 1, ok);
                    tc_fence_after_sync();
                }
#pragma unroll
                for (int k = 0; k < 64; k += 32) {
                    uint32_t q[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) q[e] = pack2_bf16(__uint_as_float(dp[k + 2 * e]), __uint_as_float(dp[k + 2 * e + 1]));
                    tmem_st_32x32b_x16(tl + S::TM_DS + half * S::DS_HALF + k / 2, q);
                }
                tmem_st_wait();
                tc_fence_before_sync();
                mbar_arrive(ds_ready);
                if (!ok) break;
            }
            if (!ok) break;
            if (x.blocks) {
                wait_for(acc_done, (n - 1) & 1, ok);
                if (DKV) wait_for(pv_done, (n - 1) & 1, ok);
                tc_fence_after_sync();
            }
            if (SPLIT) {
                // fp32 sums of a part, for the kernel that adds them; one warpgroup dK, the other dV, or half of dQ's channels each
                constexpr int COLS = DKV ? D : D / 2;
                bool live = ok;
                if (DKV && live) live = x.x0 + row < x.end && (!mask || __ldg(mask + x.x0 + row) != 0);
                float* out = a.part + ((long long)t * (DKV ? 2 : 1) + (DKV ? half : 0)) * (128 * D) + row * D + (DKV ? 0 : half * COLS);
#pragma unroll
                for (int k = 0; k < COLS; k += 16) {
                    uint32_t o[16];
                    if (x.blocks) {
                        tmem_ld_32x32b_x16(tl + (DKV && half ? S::TM_A2 : S::TM_A1) + (DKV ? 0 : half * COLS) + k, o);
                        tmem_ld_wait();
                    }
#pragma unroll
                    for (int q = 0; q < 16; q += 4)
                        *reinterpret_cast<float4*>(out + k + q) =
                            live && x.blocks ? make_float4(__uint_as_float(o[q]), __uint_as_float(o[q + 1]), __uint_as_float(o[q + 2]), __uint_as_float(o[q + 3]))
                                             : make_float4(0.f, 0.f, 0.f, 0.f);
                }
            } else if (DKV) {
                // one warpgroup stores dK, the other dV; thread = key
                const int key = x.x0 + row;
                bool live = key < x.end;
                if (live && mask) live = __ldg(mask + key) != 0;
                const bool have = key < a.Nk && ok;
                const float f = half ? 1.f : a.scale;
                __nv_bfloat16* out = half ? static_cast<__nv_bfloat16*>(a.dV) + ((long long)x.b * a.Nk + key) * a.v_stride
                                          : static_cast<__nv_bfloat16*>(a.dK) + ((long long)x.b * a.Nk + key) * a.k_stride;
                out += (long long)x.kvh * D;
#pragma unroll
                for (int k = 0; k < D; k += 32) {
                    uint32_t o[32];
                    if (x.blocks) {
                        tmem_ld_32x32b_x32(tl + (half ? S::TM_A2 : S::TM_A1) + k, o);
                        tmem_ld_wait();
                    }
                    if (have) {
#pragma unroll
                        for (int q = 0; q < 32; q += 8) {
                            uint32_t v[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                v[e] = live && x.blocks ? pack2_bf16(__uint_as_float(o[q + 2 * e]) * f, __uint_as_float(o[q + 2 * e + 1]) * f) : 0u;
                            *reinterpret_cast<uint4*>(out + k + q) = make_uint4(v[0], v[1], v[2], v[3]);
                        }
                    }
                }
            } else {
                // half of the row's channels each
                const int token = x.x0 + in_token;
                const bool have = in_token < g.tokens && token < a.Nq && ok;
                __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.dQ) + ((long long)x.b * a.Nq + token) * a.q_stride +
                                     (long long)(x.kvh * a.group + head) * D + half * (D / 2);
#pragma unroll
                for (int k = 0; k < D / 2; k += 16) {
                    uint32_t o[16];
                    if (x.blocks) {
                        tmem_ld_32x32b_x16(tl + S::TM_A1 + half * (D / 2) + k, o);
                        tmem_ld_wait();
                    }
                    if (have) {
#pragma unroll
                        for (int q = 0; q < 16; q += 8) {
                            uint32_t v[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                v[e] = x.blocks ? pack2_bf16(__uint_as_float(o[q + 2 * e]) * a.scale, __uint_as_float(o[q + 2 * e + 1]) * a.scale) : 0u;
                            *reinterpret_cast<uint4*>(out + k + q) = make_uint4(v[0], v[1], v[2], v[3]);
                        }
                    }
                }
            }
            tc_fence_before_sync();
        }
    } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 8) {
        // ------------------------------------------------ copies
        if (lane == 0) {
            uint32_t n_x = 0, n = 0;
            const uint32_t rows_box = (uint32_t)(g.tokens * a.group * S::ROW), keys_box = S::PLANE;
            for (int t = blockIdx.x; t < g.total && ok; t += gridDim.x) {
                const Tile x = tile_of(t);
                if (!x.blocks) continue;
                const int xb = n_x % S::XS;
                if (n_x >= S::XS) ok = mbar_wait(x_empty + xb, (n_x / S::XS - 1) & 1, POLL_LIMIT) && ok;
                ++n_x;
                if (!ok) break;
                mbar_expect_tx(x_full + xb, 2 * S::BOXES * (DKV ? keys_box : rows_box));
#pragma unroll
                for (int k = 0; k < S::BOXES; ++k) {
                    const uint32_t to = base + xb * (2 * S::TILE) + k * S::PLANE;
                    tma_load_4d(to, DKV ? &map_k : &map_q, x_full + xb, k * S::BOX, DKV ? x.kvh : x.kvh * a.group, x.x0, x.b);
                    tma_load_4d(to + S::TILE, DKV ? &map_v : &map_do, x_full + xb, k * S::BOX, DKV ? x.kvh : x.kvh * a.group, x.x0, x.b);
                }
                for (int j = 0; j < x.blocks && ok; ++j, ++n) {
                    const int s = n % S::STAGES;
                    if (n >= S::STAGES) ok = mbar_wait(y_empty + s, (n / S::STAGES - 1) & 1, POLL_LIMIT) && ok;
                    if (!ok) break;
                    mbar_expect_tx(y_full + s, 2 * S::BOXES * (DKV ? rows_box : keys_box) + (DKV ? 1024 : 0));
                    const int y0 = (x.j0 + j) * (DKV ? g.tokens : 128);
#pragma unroll
                    for (int k = 0; k < S::BOXES; ++k) {
                        const uint32_t to = base + S::OFF_Y + s * S::STAGE + k * S::PLANE;
                        tma_load_4d(to, DKV ? &map_q : &map_k, y_full + s, k * S::BOX, DKV ? x.kvh * a.group : x.kvh, y0, x.b);
                        tma_load_4d(to + S::TILE, DKV ? &map_do : &map_v, y_full + s, k * S::BOX, DKV ? x.kvh * a.group : x.kvh, y0, x.b);
                    }
                    if (DKV) bulk_load(base + S::OFF_STAT + s * 1024, g.stats + ((long long)x.p * g.row_blocks + x.j0 + j) * 256, 1024, y_full + s);
                }
            }
        }
    } else if (warp < 11) {
        // ------------------------------------------------ products: warp 9 makes S and A2, warp 10 dP and A1
        // An issuing lane is held as long as its products run, and by every wait and commit besides: with one warp for all four
        // the tensor pipe stood still for the 1100 cycles of those (of 2800 a block at head dim 64).
        constexpr uint32_t IDESC_S = umma_idesc_bf16(128, 128, false, false), IDESC_A = umma_idesc_bf16(128, D, false, true);
        const int which = warp - 9;                 // 0: X1, Y1 make S; 1: X2, Y2 make dP
        uint64_t *made = which ? dp_ready : s_ready, *taken = which ? dp_free : s_free, *given = which ? ds_ready : p_ready;
        constexpr bool APART = S::S_APART;          // the same for both
        static_assert(S::S_APART == S::DS_APART, "S and dP");
        const uint64_t x_desc = umma_smem_desc(base + which * S::TILE, 16, 8 * S::ROW, S::SWIZZLE);
        const uint64_t y_desc = umma_smem_desc(base + S::OFF_Y + which * S::TILE, 16, 8 * S::ROW, S::SWIZZLE);
        // dS meets Y1, P meets Y2
        const uint64_t z_desc = umma_smem_desc(base + S::OFF_Y + (which ^ 1) * S::TILE, S::BOXES > 1 ? S::PLANE : 16, 8 * S::ROW, S::SWIZZLE);
        const uint32_t to = tmem + (which ? S::TM_A1 : S::TM_A2), from = tmem + (which ? S::TM_DS : S::TM_P);
        constexpr int HALF = APART ? 32 : 64;
        static_assert(S::P_HALF == HALF && S::DS_HALF == HALF, "halves of P and dS");
        const bool gathers = DKV || which;
        uint32_t n_x = 0, n = 0;                    // tiles with a walk, blocks so far
        uint32_t xb = 0;                            // this tile's buffer
        auto scores = [&](uint32_t i, bool last) {
            const uint32_t s = i % S::STAGES;
            wait_for(y_full + s, (i / S::STAGES) & 1, ok);
            if (!ok) return;
            tc_fence_after_sync();
            const uint64_t y = y_desc + s * (S::STAGE >> 4), xd = x_desc + xb * (2 * S::TILE >> 4);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                constexpr int PER = S::BOX / 16;
                const uint32_t at = (uint32_t)(k / PER * S::PLANE + k % PER * 32) >> 4;
                umma_ss(tmem + which * S::TM_DP, xd + at, y + at, IDESC_S, k);
            }
            umma_commit(made);
            if (last) umma_commit(x_empty + xb);
            if (!gathers) umma_commit(y_empty + s);
        };
        // One lane alone: lanes that only waited along could fall two phases behind a barrier, whose parity then says nothing.
        for (int t = blockIdx.x; lane == 0 && t < g.total && ok; t += gridDim.x) {
            const Tile x = tile_of(t);
            if (!x.blocks) continue;
            xb = n_x % S::XS;
            wait_for(x_full + xb, (n_x / S::XS) & 1, ok);
            ++n_x;
            if (ok) scores(n, x.blocks == 1);
            for (int j = 0; j < x.blocks && ok; ++j, ++n) {
                const bool more = j + 1 < x.blocks;
                const uint32_t s = n % S::STAGES;
                if (APART) {
                    wait_for(taken, n & 1, ok);
                    if (more && ok) scores(n + 1, j + 2 == x.blocks);
                }
                if (gathers) {
                    if (!DKV) wait_for(y_clean + s, (n / S::STAGES) & 1, ok);
                    wait_for(given, n & 1, ok);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint64_t z = z_desc + s * (S::STAGE >> 4);
#pragma unroll
                    for (int k = 0; k < 8; ++k)                     // 16 walked rows
                        umma_ts(to, from + (k >> 2) * HALF + (k & 3) * 8, z + k * (16 * S::ROW >> 4), IDESC_A, j > 0 || k > 0);
                    umma_commit(which ? acc_done : pv_done);
                    umma_commit(y_empty + s);
                }
                if (!APART && more && ok) scores(n + 1, j + 2 == x.blocks);
            }
        }
    } else if (!DKV) {
        // ------------------------------------------------ rows of hidden keys, before dS (zero there) meets them
        uint32_t n = 0;
        for (int t = blockIdx.x; t < g.total && ok; t += gridDim.x) {
            const Tile x = tile_of(t);
            const uint8_t* mask = a.key_mask ? a.key_mask + (long long)x.b * a.Nk : nullptr;
            for (int j = 0; j < x.blocks && ok; ++j, ++n) {
                const int s = n % S::STAGES;
                const int key0 = (x.j0 + j) * 128;
                const Seen seen = seen_of(mask, mask ? mask_bytes(mask, key0, x.end, lane) : 0u, key0, x.end);
                ok = mbar_wait(y_full + s, (n / S::STAGES) & 1, POLL_LIMIT) && ok;
                if ((seen.w[0] & seen.w[1] & seen.w[2] & seen.w[3]) != 0xffffffffu) {
                    constexpr int CHUNKS = S::ROW / 16;
                    for (int r = lane / CHUNKS; r < 128; r += 32 / CHUNKS)
                        if (!((seen.w[r >> 5] >> (r & 31)) & 1)) {
#pragma unroll
                            for (int k = 0; k < S::BOXES; ++k)
                                sts_f32x4(base + S::OFF_Y + s * S::STAGE + k * S::PLANE + r * S::ROW + lane % CHUNKS * 16, 0.f, 0.f, 0.f, 0.f);
                        }
                    fence_proxy_async_smem();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(y_clean + s);
            }
        }
    }
    }
    __syncwarp();
    if (!ok) record_error(a.status, BRA_ERR_TIMEOUT, (int)blockIdx.x);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == 9) tmem_dealloc(tmem, 512);
}

// (-lse2, -delta) of every row, by blocks of 128 as the kernels above walk them; rows that do not exist and rows that see no key:
// (-inf, 0), so that every P of theirs is zero.  D / 8 lanes a row, 16 bytes each of O and dO.
template <int D>
__global__ void __launch_bounds__(256) cross_stats_kernel(const TcArgs g, float* stats) {
    constexpr int LANES = D / 8;
    const CrossArgs& a = g.a;
    pdl_launch_dependents();
    const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) / LANES;
    const int part = threadIdx.x % LANES;
    const long long block = i >> 7;
    const int row = (int)(i & 127);
    const int p = (int)(block / g.row_blocks), j = (int)(block - (long long)p * g.row_blocks);
    const int b = (int)fdiv((uint32_t)p, a.kv_div), kvh = p - b * a.kv;
    const int in_token = (int)fdiv((uint32_t)row, a.group_div), h = kvh * a.group + row - in_token * a.group;
    const int token = j * g.tokens + in_token;
    const bool have = p < g.total && in_token < g.tokens && token < a.Nq;      // total: pairs here
    float delta = 0.f;
    if (have) {
        const long long off = ((long long)b * a.Nq + token) * a.o_stride + (long long)h * D + part * 8;
        float o[8], d[8];
        load_row<8>(static_cast<const __nv_bfloat16*>(a.O) + off, o);
        load_row<8>(static_cast<const __nv_bfloat16*>(a.dO) + off, d);
#pragma unroll
        for (int e = 0; e < 8; ++e) delta = fmaf(o[e], d[e], delta);
    }
#pragma unroll
    for (int x = LANES / 2; x; x >>= 1) delta += __shfl_xor_sync(0xffffffffu, delta, x);
    if (part == 0 && p < g.total) {
        float l = -INFINITY;
        if (have) {
            const float e = __ldg(a.lse + ((long long)b * a.heads + h) * a.Nq + token);
            if (e != -INFINITY) l = -e * 1.4426950408889634f;
        }
        stats[block * 256 + row] = l;
        stats[block * 256 + 128 + row] = l == -INFINITY ? 0.f : -delta;
    }
}

// Adds the parts of split walks in order: thread = four channels of a kept row.
template <int D, bool DKV>
__global__ void __launch_bounds__(256) cross_grad_join_kernel(const TcArgs g, int pairs) {
    const CrossArgs& a = g.a;
    pdl_wait();
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int ch = (int)(i % (D / 4)) * 4, row = (int)(i / (D / 4)) & 127;
    const long long rest = i / (D / 4) / 128;
    const int which = DKV ? (int)(rest & 1) : 0;
    const long long tile = DKV ? rest >> 1 : rest;
    if (tile >= (long long)pairs * g.tiles) return;
    const int p = (int)(tile / g.tiles), x0 = (int)(tile - (long long)p * g.tiles) * (DKV ? 128 : g.tokens);
    const int b = (int)fdiv((uint32_t)p, a.kv_div), kvh = p - b * a.kv;
    __nv_bfloat16* out;
    if (DKV) {
        if (x0 + row >= a.Nk) return;
        const long long key = (long long)b * a.Nk + x0 + row;
        out = (which ? static_cast<__nv_bfloat16*>(a.dV) + key * a.v_stride : static_cast<__nv_bfloat16*>(a.dK) + key * a.k_stride) + (long long)kvh * D;
    } else {
        const int in_token = (int)fdiv((uint32_t)row, a.group_div), token = x0 + in_token;
        if (in_token >= g.tokens || token >= a.Nq) return;
        out = static_cast<__nv_bfloat16*>(a.dQ) + ((long long)b * a.Nq + token) * a.q_stride + (long long)(kvh * a.group + row - in_token * a.group) * D;
    }
    const float* from = a.part + (tile * g.splits * (DKV ? 2 : 1) + which) * (128 * D) + row * D + ch;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int s = 0; s < g.splits; ++s) {
        const float4 v = __ldcg(reinterpret_cast<const float4*>(from + (long long)s * (DKV ? 2 : 1) * (128 * D)));
        t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
    }
    const float f = which ? 1.f : a.scale;
    *reinterpret_cast<uint2*>(out + ch) = make_uint2(pack2_bf16(t.x * f, t.y * f), pack2_bf16(t.z * f, t.w * f));
}

int row_blocks(const CrossDims& d) { return (d.Nq + 128 / d.group - 1) / (128 / d.group); }

// Fewer kept tiles than SMs: walks are split, one part for an SM at most.
TcSplit grad_split(const CrossDims& d, bool dkv) {
    return tc_split((long long)d.B * d.kv * (dkv ? (d.Nk + 127) / 128 : row_blocks(d)), dkv ? row_blocks(d) : (d.Nk + 127) / 128);
}

template <int D, bool DKV>
cudaError_t launch_grad(const CrossDims& d, TcArgs g, const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const CUtensorMap& o, cudaStream_t st) {
    const TcSplit sp = grad_split(d, DKV);
    const int pairs = d.B * d.kv;
    g.tiles = DKV ? (d.Nk + 127) / 128 : g.row_blocks;
    g.splits = sp.splits;
    g.part = sp.part;
    g.total = pairs * g.tiles * g.splits;
    g.tiles_div = fast_div(g.tiles);
    g.splits_div = fast_div(g.splits);
    static PerDeviceOnce attr;
    cudaError_t e = attr.run([&] {
        const cudaError_t f = cudaFuncSetAttribute(cross_grad_tc_kernel<D, DKV, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<D, DKV>::smem);
        return f != cudaSuccess ? f : cudaFuncSetAttribute(cross_grad_tc_kernel<D, DKV, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Shape<D, DKV>::smem);
    });
    if (e != cudaSuccess) return e;
    const dim3 ctas(g.total < kSMs ? g.total : kSMs), threads_of(THREADS);
    e = g.splits > 1 ? launch_kernel(cross_grad_tc_kernel<D, DKV, true>, ctas, threads_of, Shape<D, DKV>::smem, st, true, g, q, k, v, o)
                     : launch_kernel(cross_grad_tc_kernel<D, DKV, false>, ctas, threads_of, Shape<D, DKV>::smem, st, true, g, q, k, v, o);
    if (e != cudaSuccess) return e;
    count_launch();
    if (g.splits == 1) return cudaSuccess;
    const long long threads = (long long)pairs * g.tiles * (DKV ? 2 : 1) * 128 * (D / 4);
    e = launch_kernel(cross_grad_join_kernel<D, DKV>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, true, g, pairs);
    if (e == cudaSuccess) count_launch();
    return e;
}

template <int D>
cudaError_t launch(const CrossDims& d, const CrossArgs& a, cudaStream_t st) {
    TcArgs g;
    g.a = a;
    float* stats = reinterpret_cast<float*>(a.stats);
    g.stats = stats;
    g.tokens = 128 / d.group;
    g.row_blocks = row_blocks(d);
    const int pairs = d.B * d.kv;
    constexpr int BOX = D < 64 ? D : 64;
    CUtensorMap q, k, v, o;
    if (!rows_map(&q, a.Q, D, d.heads, d.Nq, d.B, d.q_stride, BOX, d.group, g.tokens) || !rows_map(&k, a.K, D, d.kv, d.Nk, d.B, d.k_stride, BOX, 1, 128) ||
        !rows_map(&v, a.V, D, d.kv, d.Nk, d.B, d.v_stride, BOX, 1, 128) || !rows_map(&o, a.dO, D, d.heads, d.Nq, d.B, d.o_stride, BOX, d.group, g.tokens))
        return cudaErrorInvalidValue;
    cudaError_t e;
    g.total = pairs;
    const long long lanes = (long long)pairs * g.row_blocks * 128 * (D / 8);
    cross_stats_kernel<D><<<(unsigned)((lanes + 255) / 256), 256, 0, st>>>(g, stats);
    count_launch();
    if ((e = cudaGetLastError()) != cudaSuccess) return e;
    if ((e = launch_grad<D, false>(d, g, q, k, v, o, st)) != cudaSuccess) return e;
    return launch_grad<D, true>(d, g, q, k, v, o, st);
}

}  // namespace

size_t cross_backward_tc_stats(const CrossDims& d) { return sizeof(float) * 256 * (size_t)d.B * d.kv * row_blocks(d); }

size_t cross_backward_tc_part(const CrossDims& d) {
    const TcSplit q = grad_split(d, false), k = grad_split(d, true);
    const size_t pairs = (size_t)d.B * d.kv, tile = 128 * (size_t)d.D;
    const size_t nq = q.splits > 1 ? pairs * row_blocks(d) * q.splits * tile : 0, nk = k.splits > 1 ? pairs * ((d.Nk + 127) / 128) * k.splits * 2 * tile : 0;
    return nq > nk ? nq : nk;
}

// Measured (B200, us, these kernels / the warp-level ones): 1 x 196 x 100, 8 heads of 32 12.7 / 13.2, 64 images 40 / 43; 16 x 100 x 100, 8 heads
// of 64 13 / 16; 4 x 64 x 512 14.4 / 19.5; 1 x 4096 x 77, 4 heads of 32 17 / 30; 4 x 1024 x 512, 4 heads of 128 36 / 88; 16 x 1024 x 1024, 12 heads of
// 64 260 / 621.  At most 64 keys, half of a block: heads of 32 64 x 196 x 60 39 / 30, 3 x 12680 x 26, 24 heads on 6 217 / 182, but of 64 2 x 4096 x 60
// 33 / 50, of 128 3 x 2294 x 30, 18 heads on 9 77 / 122.  At most 64 rows: half of a tile and more is empty.
bool cross_backward_tc_pays(const CrossDims& d) {
    if (d.D < 32 || d.group > 128 || d.esize != 2) return false;
    const long long pairs = (long long)d.B * d.kv;
    if (pairs * row_blocks(d) > (1 << 24) || pairs * ((d.Nk + 127) / 128) > (1 << 24)) return false;
    return d.rows > 64 && (d.D > 32 || d.Nk > 64);
}

cudaError_t launch_cross_backward_tc(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    switch (d.D) {
        case 32: return launch<32>(d, a, st);
        case 64: return launch<64>(d, a, st);
        default: return launch<128>(d, a, st);
    }
}

}  // namespace bra
