// Cross attention of bf16 queries to an encoder's states on the 5th-generation tensor cores: many rows, many keys.
//
// One CTA per SM walks pairs of tiles of 128 rows of an (image, key head); its warps:
//   warps 0-3, 4-7   softmax of the first and second tile, thread = row = lane of tensor memory
//   warp 8           bulk tensor copies: Q of both tiles, then blocks of 128 keys and values through a ring
//   warps 9, 10      tcgen05.mma of the first and second tile, one lane: S = Q K^T (128 x 128, fp32 in tensor memory),
//                    O += P V with P (bf16 pairs) read from tensor memory
//   warp 11          zeroes the values of hidden keys in shared memory
// What bounds it is the softmax: 128 x 128 exponentials are 1024 cycles of an SM's MUFU, the two products 750 (head dim 64) to 1040
// (128) of its tensor pipe.  So the softmax must not wait for products.  Up to head dim 64, P has columns of its own and S of the
// next block is made as soon as this one's is in registers; the wait for P V of the block before is over by the time P is written.
// At 128, O of two tiles fills tensor memory, P lies over S, and S of the next block follows P V of this one; there the two warps of
// a scheduler take turns at the exponentials, so that one has its products made meanwhile.  K and V of a block serve both tiles; the next pair's Q is copied under the last softmax.
// Rows are query tokens times the heads that share a key head (the box of a bulk copy is all of a token's heads), 128 / group
// tokens a tile; where the group does not divide 128 the last lanes of a tile are idle.
//
// Softmax in base 2 with a reference maximum that moves only when a row's scores outgrow it by 2^8: p may be up to 256, sums and O
// carry the same factor, and O is rescaled in tensor memory only then (no key so far: O is zero).  P is rounded to bf16 for the
// second product (half a step, 2^-8, per term); sums are of the unrounded p; accumulators are fp32.
//
// Hidden keys: their scores are replaced (not added to), their values zeroed before the product, so infinities and NaN in them
// reach nothing.
#include "cross_tc_common.cuh"

#include <math.h>

namespace bra {
namespace {

using namespace cross_tc;

constexpr int THREADS = 384;                    // three warpgroups: two of softmax, one whose first two warps copy and multiply

template <int D>
struct Shape {
    static constexpr int BOX = D < 64 ? D : 64;             // channels of a bulk copy: rows of 64 or 128 bytes
    static constexpr int BOXES = D / BOX;
    static constexpr int ROW = BOX * 2;                     // bytes
    static constexpr int PLANE = 128 * ROW;                 // a box of 128 rows
    static constexpr int TILE = PLANE * BOXES;
    static constexpr int STAGES = D == 128 ? 2 : 4;         // of K and of V each
    static constexpr uint32_t SWIZZLE = D < 64 ? 4 : 2;     // 64 or 128 bytes
    // tensor memory: S of the tiles at 0 and 128, O from 256 on; P behind O where there is room, else over S
    static constexpr bool APART = D <= 64;
    static constexpr int TM_O = 256, O_STEP = APART ? 64 : 128, TM_P = APART ? 384 : 0, P_STEP = APART ? 64 : 128;
    // pairs of Q tiles in flight: where there is room, the next one's copy runs beside this one's last blocks
    static constexpr int QS = D <= 64 ? 2 : 1;
    static constexpr int OFF_K = QS * 2 * TILE, OFF_V = OFF_K + STAGES * TILE, OFF_OUT = OFF_V + STAGES * TILE, OFF_BAR = OFF_OUT + 8 * ROWS32;
    static constexpr size_t smem = OFF_BAR + 384 + 1024;    // barriers; slack for the alignment the swizzle wants
};

struct TcArgs {
    CrossArgs a;
    int tokens;             // of a tile: 128 / group
    int pairs;              // tile pairs of an (image, key head)
    int splits, part;       // parts of the walk over the keys and their length in blocks
    int total;              // parts of all pairs
    FastDiv pairs_div, splits_div;
};

// SPLIT: walks are cut in parts
template <int D, bool SPLIT>
__global__ void __launch_bounds__(THREADS, 1)
cross_attend_tc_kernel(const TcArgs g, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                       const __grid_constant__ CUtensorMap map_v) {
    using S = Shape<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint64_t* bar = reinterpret_cast<uint64_t*>(smem + S::OFF_BAR);
    uint64_t *q_full = bar, *q_empty = bar + 2, *s_ready = bar + 4, *s_free = bar + 6, *p_ready = bar + 8, *pv_done = bar + 10,
             *k_full = bar + 12, *k_empty = k_full + S::STAGES, *v_full = k_empty + S::STAGES, *v_clean = v_full + S::STAGES,
             *v_empty = v_clean + S::STAGES, *turn = v_empty + S::STAGES;      // turn: of the four warps of each tile
    uint32_t* slot = reinterpret_cast<uint32_t*>(turn + 8);
    const uint32_t base = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const CrossArgs& a = g.a;

    if (threadIdx.x == 0) {
        for (int w = 0; w < 2; ++w) {
            mbar_init(q_full + w, 1); mbar_init(q_empty + w, 2);
            mbar_init(s_ready + w, 1); mbar_init(s_free + w, 128); mbar_init(p_ready + w, 128); mbar_init(pv_done + w, 1);
        }
        for (int s = 0; s < S::STAGES; ++s) {
            mbar_init(k_full + s, 1); mbar_init(k_empty + s, 2); mbar_init(v_full + s, 1); mbar_init(v_clean + s, 1); mbar_init(v_empty + s, 2);
        }
        for (int i = 0; i < 8; ++i) mbar_init(turn + i, 1);
        fence_mbar_init();
    }
    if (warp == 9) tmem_alloc(slot, 512);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = *slot;
    bool ok = true;

    // every role walks the same tiles
    struct Tile { int b, kvh, token0, end, j0, blocks, both; };
    auto tile_of = [&](int t) {
        Tile x;
        const int pair = SPLIT ? (int)fdiv((uint32_t)t, g.splits_div) : t, p = (int)fdiv((uint32_t)pair, g.pairs_div);
        x.j0 = SPLIT ? (t - pair * g.splits) * g.part : 0;
        x.token0 = (pair - p * g.pairs) * 2 * g.tokens;
        x.b = (int)fdiv((uint32_t)p, a.kv_div);
        x.kvh = p - x.b * a.kv;
        x.end = cross_key_end(a, x.b);
        x.blocks = (x.end + 127) >> 7;
        if (SPLIT) x.blocks = min(max(x.blocks - x.j0, 0), g.part);
        x.both = x.token0 + g.tokens < a.Nq;
        return x;
    };

    // registers: launched with 168 a thread, 384 x 168 = 64512 = 256 x 224 + 128 x 56
    if (warp < 8) {
        // ------------------------------------------------ softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int w = warp >> 2, row = threadIdx.x & 127;
        const uint32_t tl = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t ts = tl + w * 128, to = tl + S::TM_O + w * S::O_STEP, tp = tl + S::TM_P + w * S::P_STEP;
        const float c = a.scale_log2, jump = 8.f / c;
        const float2 c2 = make_float2(c, c);
        const int in_token = (int)fdiv((uint32_t)row, a.group_div), head = row - in_token * a.group;
        uint32_t n_s = 0, n_turn = 0;           // blocks so far; those of pairs with two tiles
        for (int t = blockIdx.x; t < g.total && ok; t += gridDim.x) {
            const Tile x = tile_of(t);
            if (w && !x.both) continue;
            const uint8_t* mask = a.key_mask ? a.key_mask + (long long)x.b * a.Nk : nullptr;
            const int token = x.token0 + w * g.tokens + in_token;
            const bool live = in_token < g.tokens && token < a.Nq;
            float m = -INFINITY, l = 0.f;
            uint32_t bytes = mask ? mask_bytes(mask, x.j0 * 128, x.end, lane) : 0u;
            for (int j = 0; j < x.blocks; ++j) {
                const int key0 = (x.j0 + j) * 128;
                const bool cut = mask || key0 + 128 > x.end;          // some keys may be hidden
                Seen seen;
                if (cut) {
                    seen = seen_of(mask, bytes, key0, x.end);
                    if (mask) bytes = mask_bytes(mask, key0 + 128, x.end, lane);
                }
                wait_for(s_ready + w, n_s & 1, ok);
                tc_fence_after_sync();
                uint32_t r[128];
#pragma unroll
                for (int k = 0; k < 4; ++k) tmem_ld_32x32b_x32(ts + 32 * k, r + 32 * k);
                tmem_ld_wait();
                if (S::APART) {
                    tc_fence_before_sync();
                    mbar_arrive(s_free + w);
                }
                if (cut) {
#pragma unroll
                    for (int k = 0; k < 128; ++k)
                        if (!((seen.w[k >> 5] >> (k & 31)) & 1)) r[k] = 0xff800000u;
                }
                float m0 = -INFINITY, m1 = -INFINITY, m2 = -INFINITY, m3 = -INFINITY;
#pragma unroll
                for (int k = 0; k < 128; k += 8) {
                    m0 = fmax3(m0, __uint_as_float(r[k]), __uint_as_float(r[k + 1]));
                    m1 = fmax3(m1, __uint_as_float(r[k + 2]), __uint_as_float(r[k + 3]));
                    m2 = fmax3(m2, __uint_as_float(r[k + 4]), __uint_as_float(r[k + 5]));
                    m3 = fmax3(m3, __uint_as_float(r[k + 6]), __uint_as_float(r[k + 7]));
                }
                const float top = fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
                // P V of the block before is done: O may be read and (where P is apart) P written.  With P over S, S says so.
                bool waited = !S::APART || j == 0;
                auto wait_pv = [&] {
                    if (!waited) {
                        wait_for(pv_done + w, (n_s - 1) & 1, ok);
                        tc_fence_after_sync();
                        waited = true;
                    }
                };
                if (j == 0) {
                    m = top;
                } else if (__any_sync(0xffffffffu, top - m > jump)) {
                    wait_pv();
                    // a row's reference does not depend on what its neighbours, idle lanes among them, hold
                    const float up = top - m > jump ? top : m;
                    const float f = up == m ? 1.f : ex2_approx((m - up) * c);
                    m = up;
                    l *= f;
#pragma unroll
                    for (int k = 0; k < D; k += 16) {
                        uint32_t o[16];
                        tmem_ld_32x32b_x16(to + k, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int q = 0; q < 16; ++q) o[q] = __float_as_uint(__uint_as_float(o[q]) * f);
                        tmem_st_32x32b_x16(to + k, o);
                    }
                }
                // Turns at the exponentials: 2 x 4133 x 4096, 37 heads of 128, 755 -> 690 us.  (With P apart, where nothing else waits
                // for products, the hand-over costs more than it gives: 468 -> 519 us at 64.)
                if (!S::APART && x.both) {
                    if (w || n_turn) wait_for(turn + warp, (w ? n_turn : n_turn - 1) & 1, ok);
                    ++n_turn;
                }
                const float ref = m == -INFINITY ? 0.f : m * c;
                const float2 minus = make_float2(-ref, -ref);
                float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
                for (int k = 0; k < 128; k += 32) {
                    uint32_t p[16];
#pragma unroll
                    for (int q = 0; q < 32; q += 4) {
                        float2 u = __ffma2_rn(make_float2(__uint_as_float(r[k + q]), __uint_as_float(r[k + q + 1])), c2, minus);
                        float2 v = __ffma2_rn(make_float2(__uint_as_float(r[k + q + 2]), __uint_as_float(r[k + q + 3])), c2, minus);
                        u = make_float2(ex2_approx(u.x), ex2_approx(u.y));
                        v = make_float2(ex2_approx(v.x), ex2_approx(v.y));
                        s0 = __fadd2_rn(s0, u);
                        s1 = __fadd2_rn(s1, v);
                        p[q / 2] = pack2_bf16(u.x, u.y);
                        p[q / 2 + 1] = pack2_bf16(v.x, v.y);
                    }
                    if (k == 0) wait_pv();
                    tmem_st_32x32b_x16(tp + k / 2, p);
                }
                if (!S::APART && x.both) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(turn + (warp ^ 4));
                }
                l += (s0.x + s0.y) + (s1.x + s1.y);
                tmem_st_wait();
                tc_fence_before_sync();
                mbar_arrive(p_ready + w);
                ++n_s;
                if (!ok) break;
            }
            const float inv = l == 0.f ? 0.f : 1.f / l;
            if (x.blocks) {
                ok = mbar_wait(pv_done + w, (n_s - 1) & 1, POLL_LIMIT) && ok;
                tc_fence_after_sync();
            }
            if (SPLIT) {
                // unnormalised sums of a part, its reference maximum and denominator, for the kernel that joins them
                float* out = a.part + ((long long)t * 2 + w) * (128 * (D + 4)) + row * (D + 4);
#pragma unroll
                for (int k = 0; k < D; k += 16) {
                    uint32_t o[16];
                    if (x.blocks) {
                        tmem_ld_32x32b_x16(to + k, o);
                        tmem_ld_wait();
                    }
#pragma unroll
                    for (int q = 0; q < 16; q += 4)
                        *reinterpret_cast<float4*>(out + k + q) =
                            x.blocks ? make_float4(__uint_as_float(o[q]), __uint_as_float(o[q + 1]), __uint_as_float(o[q + 2]), __uint_as_float(o[q + 3]))
                                     : make_float4(0.f, 0.f, 0.f, 0.f);
                }
                *reinterpret_cast<float2*>(out + D) = make_float2(m, l);
                tc_fence_before_sync();
                continue;
            }
            const int h = x.kvh * a.group + head;
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.Oo) + ((long long)x.b * a.Nq + token) * a.o_stride + (long long)h * D;
            const RowPointers rows = rows_of_warp(live && ok ? out : nullptr, lane);
#pragma unroll
            for (int k = 0; k < D; k += 32) {
                uint32_t o[32], v[16];
                if (x.blocks) {
                    tmem_ld_32x32b_x32(to + k, o);
                    tmem_ld_wait();
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = x.blocks ? pack2_bf16(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv) : 0u;
                store_rows32(base + S::OFF_OUT + warp * ROWS32, v, rows, k, lane);
            }
            tc_fence_before_sync();
            if (a.lse && live && ok)
                a.lse[((long long)x.b * a.heads + h) * a.Nq + token] = l == 0.f ? -INFINITY : (m * c + log2f(l)) * 0.69314718055994531f;
        }
    } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    if (warp == 8) {
        // ------------------------------------------------ copies
        if (lane == 0) {
            uint32_t n_q = 0, n = 0;                // tiles and blocks so far
            for (int t = blockIdx.x; t < g.total && ok; t += gridDim.x) {
                const Tile x = tile_of(t);
                if (!x.blocks) continue;
                const int qb = n_q % S::QS;
                if (n_q >= S::QS) ok = mbar_wait(q_empty + qb, (n_q / S::QS - 1) & 1, POLL_LIMIT) && ok;
                ++n_q;
                if (!ok) break;
                const uint32_t q_box = (uint32_t)(g.tokens * a.group * S::ROW);
                mbar_expect_tx(q_full + qb, q_box * S::BOXES * (1 + x.both));
                for (int w = 0; w <= x.both; ++w)
#pragma unroll
                    for (int k = 0; k < S::BOXES; ++k)
                        tma_load_4d(base + (2 * qb + w) * S::TILE + k * S::PLANE, &map_q, q_full + qb, k * S::BOX, x.kvh * a.group, x.token0 + w * g.tokens, x.b);
                for (int j = 0; j < x.blocks && ok; ++j, ++n) {
                    const int s = n % S::STAGES;
                    const uint32_t parity = (n / S::STAGES - 1) & 1;
                    if (n >= S::STAGES) ok = mbar_wait(k_empty + s, parity, POLL_LIMIT) && ok;
                    if (!ok) break;
                    mbar_expect_tx(k_full + s, S::TILE);
#pragma unroll
                    for (int k = 0; k < S::BOXES; ++k)
                        tma_load_4d(base + S::OFF_K + s * S::TILE + k * S::PLANE, &map_k, k_full + s, k * S::BOX, x.kvh, (x.j0 + j) * 128, x.b);
                    if (n >= S::STAGES) ok = mbar_wait(v_empty + s, parity, POLL_LIMIT) && ok;
                    if (!ok) break;
                    mbar_expect_tx(v_full + s, S::TILE);
#pragma unroll
                    for (int k = 0; k < S::BOXES; ++k)
                        tma_load_4d(base + S::OFF_V + s * S::TILE + k * S::PLANE, &map_v, v_full + s, k * S::BOX, x.kvh, (x.j0 + j) * 128, x.b);
                }
            }
        }
    } else if (warp < 11) {
        // ------------------------------------------------ products
        constexpr uint32_t IDESC_S = umma_idesc_bf16(128, 128, false, false), IDESC_O = umma_idesc_bf16(128, D, false, true);
        const int w = warp - 9;
        uint32_t n_q = 0, nb = 0, nk = 0, nv = 0;   // tiles with keys, this tile's blocks so far; ring positions of K and V
        // The second tile's warp follows the ring through pairs that have only one, without products: a wait two phases ahead of a
        // barrier would not be one.
        bool idle = false;
        const uint64_t q_desc = umma_smem_desc(base + w * S::TILE, 16, 8 * S::ROW, S::SWIZZLE);
        const uint64_t k_desc = umma_smem_desc(base + S::OFF_K, 16, 8 * S::ROW, S::SWIZZLE);
        const uint64_t v_desc = umma_smem_desc(base + S::OFF_V, S::BOXES > 1 ? S::PLANE : 16, 8 * S::ROW, S::SWIZZLE);
        uint32_t qb = 0;                            // this pair's buffer
        auto scores = [&] {
            const int stage = nk % S::STAGES;
            wait_for(k_full + stage, (nk / S::STAGES) & 1, ok);
            if (!ok) return;
            tc_fence_after_sync();
            if (!idle) {
                const uint64_t kd = k_desc + stage * (S::TILE >> 4), qd = q_desc + qb * (2 * S::TILE >> 4);
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    constexpr int PER = S::BOX / 16;
                    const uint32_t at = (uint32_t)(k / PER * S::PLANE + k % PER * 32) >> 4;
                    umma_ss(tmem + w * 128, qd + at, kd + at, IDESC_S, k);
                }
                umma_commit(s_ready + w);
            }
            ++nk;
        };
        // stages are given back by both warps
        auto after_scores = [&](const Tile& x, int j) {
            umma_commit(k_empty + (nk - 1) % S::STAGES);
            if (j + 1 == x.blocks) umma_commit(q_empty + qb);
        };
        // One lane alone: lanes that only waited along could fall two phases behind a barrier, whose parity then says nothing.
        for (int t = blockIdx.x; lane == 0 && t < g.total && ok; t += gridDim.x) {
            const Tile x = tile_of(t);
            if (!x.blocks) continue;
            idle = w && !x.both;
            qb = n_q % S::QS;
            wait_for(q_full + qb, (n_q / S::QS) & 1, ok);
            ++n_q;
            if (!ok) break;
            scores();
            if (!ok) break;
            after_scores(x, 0);
            for (int j = 0; j < x.blocks && ok; ++j, ++nv, nb += !idle) {
                const int sv = nv % S::STAGES;
                const bool more = j + 1 < x.blocks;
                if (S::APART && more) {                         // S of this block is in registers
                    if (!idle) wait_for(s_free + w, nb & 1, ok);
                    if (ok) scores();
                    if (!ok) break;
                    after_scores(x, j + 1);
                }
                wait_for(v_clean + sv, (nv / S::STAGES) & 1, ok);
                if (!idle) wait_for(p_ready + w, nb & 1, ok);
                if (!ok) break;
                tc_fence_after_sync();
                if (!idle) {
                    const uint64_t vd = v_desc + sv * (S::TILE >> 4);
#pragma unroll
                    for (int k = 0; k < 8; ++k)                 // 16 keys: 8 columns of P, 16 rows of V
                        umma_ts(tmem + S::TM_O + w * S::O_STEP, tmem + S::TM_P + w * S::P_STEP + k * 8, vd + k * (16 * S::ROW >> 4), IDESC_O, j > 0 || k > 0);
                }
                if (!idle) umma_commit(pv_done + w);
                umma_commit(v_empty + sv);
                if (!S::APART && more) {
                    scores();
                    if (!ok) break;
                    after_scores(x, j + 1);
                }
            }
            // with no next block nobody waits for it, but the phase counts
            if (S::APART && ok && !idle) ok = mbar_wait(s_free + w, (nb - 1) & 1, POLL_LIMIT) && ok;
        }
    } else {
        // ------------------------------------------------ values of hidden keys
        uint32_t nv = 0;
        for (int t = blockIdx.x; t < g.total && ok; t += gridDim.x) {
            const Tile x = tile_of(t);
            const uint8_t* mask = a.key_mask ? a.key_mask + (long long)x.b * a.Nk : nullptr;
            for (int j = 0; j < x.blocks && ok; ++j, ++nv) {
                const int sv = nv % S::STAGES;
                const int key0 = (x.j0 + j) * 128;
                const Seen seen = seen_of(mask, mask ? mask_bytes(mask, key0, x.end, lane) : 0u, key0, x.end);
                ok = mbar_wait(v_full + sv, (nv / S::STAGES) & 1, POLL_LIMIT) && ok;
                if ((seen.w[0] & seen.w[1] & seen.w[2] & seen.w[3]) != 0xffffffffu) {
                    constexpr int CHUNKS = S::ROW / 16;
                    for (int r = lane / CHUNKS; r < 128; r += 32 / CHUNKS)
                        if (!((seen.w[r >> 5] >> (r & 31)) & 1)) {
#pragma unroll
                            for (int k = 0; k < S::BOXES; ++k)
                                sts_f32x4(base + S::OFF_V + sv * S::TILE + k * S::PLANE + r * S::ROW + lane % CHUNKS * 16, 0.f, 0.f, 0.f, 0.f);
                        }
                    fence_proxy_async_smem();
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(v_clean + sv);
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

// Joins the parts of split walks: a CTA for 16 rows.
template <int D>
__global__ void __launch_bounds__(128) cross_attend_join_kernel(const TcArgs g) {
    extern __shared__ float weight[];
    const CrossArgs& a = g.a;
    pdl_wait();
    const int pair = blockIdx.x >> 4, w = (blockIdx.x >> 3) & 1, row0 = (blockIdx.x & 7) * 16;
    const int p = (int)fdiv((uint32_t)pair, g.pairs_div);
    const int b = (int)fdiv((uint32_t)p, a.kv_div), kvh = p - b * a.kv, token0 = (pair - p * g.pairs) * 2 * g.tokens + w * g.tokens;
    const int rows = min(16, min(g.tokens, a.Nq - token0) * a.group - row0);
    if (rows <= 0) return;
    const long long tile = 128 * (D + 4);
    auto place = [&](int r, int& token, int& h) {
        const int in_token = (int)fdiv((uint32_t)(row0 + r), a.group_div);
        token = token0 + in_token;
        h = kvh * a.group + row0 + r - in_token * a.group;
    };
    cross_join<D>(a.part + ((long long)pair * g.splits * 2 + w) * tile + row0 * (D + 4), 2 * tile, D + 4, rows, g.splits, a.scale_log2, weight,
                  [&](int r, int ch, float4 v) {
                      int token, h;
                      place(r, token, h);
                      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.Oo) + ((long long)b * a.Nq + token) * a.o_stride + (long long)h * D + 4 * ch;
                      *reinterpret_cast<uint2*>(out) = make_uint2(pack2_bf16(v.x, v.y), pack2_bf16(v.z, v.w));
                  },
                  [&](int r, float ref, float sum) {
                      int token, h;
                      place(r, token, h);
                      if (a.lse) a.lse[((long long)b * a.heads + h) * a.Nq + token] = sum == 0.f ? -INFINITY : (ref + log2f(sum)) * 0.69314718055994531f;
                  });
}

int tile_pairs(const CrossDims& d) { return (d.Nq + 2 * (128 / d.group) - 1) / (2 * (128 / d.group)); }
TcSplit attend_split(const CrossDims& d) { return tc_split((long long)tile_pairs(d) * d.B * d.kv, (d.Nk + 127) / 128); }

template <int D>
cudaError_t launch(const CrossDims& d, const CrossArgs& a, cudaStream_t st) {
    using S = Shape<D>;
    TcArgs g;
    g.a = a;
    g.tokens = 128 / d.group;
    const TcSplit sp = attend_split(d);
    g.pairs = tile_pairs(d);
    g.splits = sp.splits;
    g.part = sp.part;
    g.total = g.pairs * d.B * d.kv * g.splits;
    g.pairs_div = fast_div(g.pairs);
    g.splits_div = fast_div(g.splits);
    CUtensorMap q, k, v;
    if (!rows_map(&q, a.Q, D, d.heads, d.Nq, d.B, d.q_stride, S::BOX, d.group, g.tokens) ||
        !rows_map(&k, a.K, D, d.kv, d.Nk, d.B, d.k_stride, S::BOX, 1, 128) || !rows_map(&v, a.V, D, d.kv, d.Nk, d.B, d.v_stride, S::BOX, 1, 128))
        return cudaErrorInvalidValue;
    static PerDeviceOnce attr;
    const cudaError_t e = attr.run([&] {
        const cudaError_t f = cudaFuncSetAttribute(cross_attend_tc_kernel<D, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::smem);
        return f != cudaSuccess ? f : cudaFuncSetAttribute(cross_attend_tc_kernel<D, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::smem);
    });
    if (e != cudaSuccess) return e;
    const int ctas = g.total < kSMs ? g.total : kSMs;
    if (g.splits > 1) cross_attend_tc_kernel<D, true><<<ctas, THREADS, S::smem, st>>>(g, q, k, v);
    else              cross_attend_tc_kernel<D, false><<<ctas, THREADS, S::smem, st>>>(g, q, k, v);
    count_launch();
    cudaError_t f = cudaGetLastError();
    if (f != cudaSuccess || g.splits == 1) return f;
    f = launch_kernel(cross_attend_join_kernel<D>, dim3(g.pairs * d.B * d.kv * 16), dim3(128), sizeof(float) * 16 * (g.splits + 1), st, true, g);
    if (f == cudaSuccess) count_launch();
    return f;
}

}  // namespace

size_t cross_attend_tc_part(const CrossDims& d) {
    const TcSplit s = attend_split(d);
    return s.splits > 1 ? (size_t)tile_pairs(d) * d.B * d.kv * s.splits * 2 * 128 * (d.D + 4) : 0;
}

// Measured (B200, us, this kernel / the warp-level one).  One block of keys: 64 x 4096 x 20, 4 heads of 32 100 / 96; up to 64 pairs of tiles
// (8 x 196 x 128, 8 heads of 32) 6.1 / 4.8; 128 pairs 6.2 / 6.6; 4 x 1024 x 100, 8 heads of 64 8.2 / 10.2.  More blocks: 8 x 196 x 256 7.8 / 6.5,
// 16 x 196 x 256 8.7 / 9.6, 1 x 100 x 512, 8 heads of 64 9.0 / 16.3, 4 x 100 x 2048 16.3 / 31.5, 1 x 1024 x 2048, 4 heads of 128 24 / 57,
// 2 x 4133 x 4096, 37 heads of 32 465 / 744, of 64 480 / 1137, of 128 601 / 2055.  At most 64 rows: half of a tile and more is empty, and the
// warp-level kernel splits the keys over more CTAs (16 rows and less have a form of their own there).
bool cross_attend_tc_pays(const CrossDims& d) {
    if (d.D < 32 || d.group > 128 || d.esize != 2) return false;
    const long long pairs = (long long)tile_pairs(d) * d.B * d.kv;
    if (pairs > (1 << 26)) return false;
    return d.rows > 64 && (d.Nk > 128 || (d.Nk > 64 && pairs >= 128));
}

cudaError_t launch_cross_attend_tc(const CrossDims& d, CrossArgs a, cudaStream_t st) {
    switch (d.D) {
        case 32: return launch<32>(d, a, st);
        case 64: return launch<64>(d, a, st);
        default: return launch<128>(d, a, st);
    }
}

}  // namespace bra
