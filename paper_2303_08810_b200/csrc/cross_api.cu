// Cross attention at the C boundary: argument checks, scratch layout, how sums are split, which kernels run.
#include "cross_common.cuh"

#include <math.h>

namespace bra {

CrossSplit cross_split(long long pairs, long long rows, int tile_rows, int summed, int step, int per_sm) {
    CrossSplit s;
    s.tiles = (int)((rows + tile_rows - 1) / tile_rows);
    s.splits = 1;
    const int steps = (summed + step - 1) / step;
    const long long out = pairs * s.tiles;
    // fewer output tiles than SMs, and more than two steps of the walk for each part
    if (out < kSMs) {
        const long long want = (long long)kSMs * per_sm / out, most = steps / 2;
        s.splits = (int)(want < most ? want : most);
        if (s.splits < 1) s.splits = 1;
    }
    const int each = (steps + s.splits - 1) / s.splits;
    s.len = each * step;
    s.splits = (steps + each - 1) / each;
    return s;
}

namespace {

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }
bool aligned_to(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bra_status make_dims(const bra_cross_problem* p, CrossDims* out) {
    if (!p) return BRA_ERR_NULL;
    if (p->B <= 0 || p->Nq <= 0 || p->Nk <= 0 || p->heads <= 0 || p->kv_heads <= 0 || p->heads % p->kv_heads || p->head_dim <= 0)
        return BRA_ERR_SHAPE;
    if (p->dtype != BRA_F32 && p->dtype != BRA_BF16) return BRA_ERR_DTYPE;
    if (p->head_dim != 16 && p->head_dim != 32 && p->head_dim != 64 && p->head_dim != 128) return BRA_ERR_UNSUPPORTED;
    CrossDims d;
    d.B = p->B; d.Nq = p->Nq; d.Nk = p->Nk; d.heads = p->heads; d.kv = p->kv_heads; d.group = p->heads / p->kv_heads; d.D = p->head_dim;
    d.esize = p->dtype == BRA_BF16 ? 2 : 4;
    const int vec = 16 / d.esize;
    const long long q_row = (long long)d.heads * d.D, kv_row = (long long)d.kv * d.D;
    d.q_stride = p->q_stride ? p->q_stride : q_row;
    d.k_stride = p->k_stride ? p->k_stride : kv_row;
    d.v_stride = p->v_stride ? p->v_stride : kv_row;
    d.o_stride = q_row;
    if (d.q_stride < q_row || d.k_stride < kv_row || d.v_stride < kv_row) return BRA_ERR_SHAPE;
    if (d.q_stride % vec || d.k_stride % vec || d.v_stride % vec) return BRA_ERR_ALIGN;
    const long long rows = (long long)d.Nq * d.group, most = 1ll << 30;
    // rows and keys are counted in 32 bits, CTAs too; elements in 64
    if (rows > most || d.Nk > most) return BRA_ERR_SHAPE;
    d.rows = (int)rows;
    const long long pairs = (long long)d.B * d.kv;
    if (pairs > most / ((rows + 15) / 16) || pairs > most / ((d.Nk + 63) / 64)) return BRA_ERR_SHAPE;
    const long long limit = 1ll << 40;
    if (d.q_stride > limit / d.B / d.Nq || d.k_stride > limit / d.B / d.Nk || d.v_stride > limit / d.B / d.Nk) return BRA_ERR_SHAPE;
    d.scale = p->scale > 0.f ? p->scale : 1.0f / sqrtf((float)d.D);
    *out = d;
    return BRA_OK;
}

bra_status check_ws(const CrossDims& d, const void* ws, size_t ws_bytes) {
    if (!ws) return BRA_ERR_NULL;
    if (!aligned_to(ws, 256)) return BRA_ERR_ALIGN;
    return ws_bytes < cross_ws(d).total ? BRA_ERR_WORKSPACE : BRA_OK;
}

}  // namespace

CrossWs cross_ws(const CrossDims& d) {
    CrossWs L;
    size_t off = 0;
    L.status = off; off += 256;
    L.done = off;  off += align256(sizeof(int32_t) * CROSS_COUNTERS);
    const size_t padded = sizeof(float2) * (size_t)d.B * d.kv * ((d.rows + 63) / 64 * 64), tc = cross_backward_tc_pays(d) ? cross_backward_tc_stats(d) : 0;
    L.stats = off; off += align256(padded > tc ? padded : tc);
    const size_t f = d.esize != 2 ? cross_attend_tf32_part(d) : cross_attend_tc_pays(d) ? cross_attend_tc_part(d) : cross_attend_mma_part(d);
    const size_t b = d.esize != 2 ? cross_backward_tf32_part(d) : cross_backward_tc_pays(d) ? cross_backward_tc_part(d) : cross_backward_mma_part(d);
    L.part = off;  off += align256(sizeof(float) * (f > b ? f : b));
    L.total = off;
    return L;
}

CrossArgs cross_args(const CrossDims& d, char* ws) {
    const CrossWs L = cross_ws(d);
    CrossArgs a = {};
    a.Nq = d.Nq; a.Nk = d.Nk; a.heads = d.heads; a.kv = d.kv; a.group = d.group; a.rows = d.rows;
    a.q_stride = d.q_stride; a.k_stride = d.k_stride; a.v_stride = d.v_stride; a.o_stride = d.o_stride;
    const double scale_log2 = (double)d.scale * 1.4426950408889634074;
    a.scale = d.scale;
    a.scale_log2 = (float)scale_log2;
    a.scale_log2_lo = (float)(scale_log2 - (double)a.scale_log2);
    a.status = reinterpret_cast<int32_t*>(ws + L.status);
    a.done = reinterpret_cast<int32_t*>(ws + L.done);
    a.stats = reinterpret_cast<float2*>(ws + L.stats);
    a.part = reinterpret_cast<float*>(ws + L.part);
    a.kv_div = fast_div(d.kv);
    a.group_div = fast_div(d.group);
    return a;
}

}  // namespace bra

using namespace bra;

extern "C" {

size_t bra_cross_workspace_bytes(const bra_cross_problem* p) {
    CrossDims d;
    return make_dims(p, &d) == BRA_OK ? cross_ws(d).total : 0;
}

bra_status bra_cross_attend(const bra_cross_problem* p, const void* Q, const void* K, const void* V,
                            const int32_t* key_len, const uint8_t* key_mask, void* O, float* lse,
                            void* ws, size_t ws_bytes, void* stream) {
    reset_launch_count();
    CrossDims d;
    bra_status s = make_dims(p, &d);
    if (s != BRA_OK) return s;
    if (!Q || !K || !V || !O) return BRA_ERR_NULL;
    if (!aligned_to(Q, 16) || !aligned_to(K, 16) || !aligned_to(V, 16) || !aligned_to(O, 16) || !aligned_to(key_len, 4) || !aligned_to(lse, 4))
        return BRA_ERR_ALIGN;
    if (key_mask && d.Nk > CROSS_MASKED_KEYS) return BRA_ERR_UNSUPPORTED;
    if ((s = check_ws(d, ws, ws_bytes)) != BRA_OK) return s;
    CrossArgs a = cross_args(d, static_cast<char*>(ws));
    a.Q = Q; a.K = K; a.V = V; a.Oo = O; a.lse = lse; a.key_len = key_len; a.key_mask = key_mask;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = d.esize != 2 ? launch_cross_attend_tf32(d, a, st)
                          : cross_attend_tc_pays(d) ? launch_cross_attend_tc(d, a, st) : launch_cross_attend_mma(d, a, st);
    return e == cudaSuccess ? BRA_OK : BRA_ERR_CUDA;
}

bra_status bra_cross_backward(const bra_cross_problem* p, const void* Q, const void* K, const void* V,
                              const int32_t* key_len, const uint8_t* key_mask, const void* O, const float* lse,
                              const void* dO, void* dQ, void* dK, void* dV,
                              void* ws, size_t ws_bytes, void* stream) {
    reset_launch_count();
    CrossDims d;
    bra_status s = make_dims(p, &d);
    if (s != BRA_OK) return s;
    if (!Q || !K || !V || !O || !lse || !dO || !dQ || !dK || !dV) return BRA_ERR_NULL;
    for (const void* q : {Q, K, V, O, dO, (const void*)dQ, (const void*)dK, (const void*)dV})
        if (!aligned_to(q, 16)) return BRA_ERR_ALIGN;
    if (!aligned_to(key_len, 4) || !aligned_to(lse, 4)) return BRA_ERR_ALIGN;
    if (key_mask && d.Nk > CROSS_MASKED_KEYS) return BRA_ERR_UNSUPPORTED;
    if ((s = check_ws(d, ws, ws_bytes)) != BRA_OK) return s;
    CrossArgs a = cross_args(d, static_cast<char*>(ws));
    a.Q = Q; a.K = K; a.V = V; a.O = O; a.dO = dO; a.dQ = dQ; a.dK = dK; a.dV = dV;
    a.lse = const_cast<float*>(lse); a.key_len = key_len; a.key_mask = key_mask;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = d.esize != 2 ? launch_cross_backward_tf32(d, a, st)
                          : cross_backward_tc_pays(d) ? launch_cross_backward_tc(d, a, st) : launch_cross_backward_mma(d, a, st);
    return e == cudaSuccess ? BRA_OK : BRA_ERR_CUDA;
}

}  // extern "C"
