// Which channels of a row a thread of the norms' kernels has, and which of them exist; which of the kernels runs rows of a size.
// Host code too, so that every width can be gone over without a GPU.
#pragma once

#include "fast_div.h"

namespace bra {

constexpr int NORM_E = 8;                   // channels of a thread
constexpr int NORM_MAX_C = 8192;

// VECD: neighbours (rows start on 16 bytes, C a multiple of eight).  Else channel j of thread t is t + j * group: neighbours over
// the threads.  FULL: rows of 256 threads and more, so that only the last of the eight channels may not exist (C > 8 group - 256, and
// that is at least 7 group there).
// QUADS (fp32 rows that start on 16 bytes): four at 4 t, four at 4 group + 4 t, so that a warp's 16-byte accesses are neighbours and fill sectors
// (with eight neighbours a thread, 16 x 1024 x 512, rms, forward + gradients 35 + 60 us, now 23 + 40; 4 x 1024 x 4096 77 + 198, now 47 + 127).
template <bool VECD, bool FULL, bool QUADS>
struct NormCols {
    int t, group, C;
    bool any, more;                         // VECD: whether the first four channels exist and the other four, all or none
    BRA_HD NormCols(int t_, int group_, int C_)
        : t(t_), group(group_), C(C_), any(t_ * (QUADS ? 4 : NORM_E) < C_), more(QUADS ? (group_ + t_) * 4 < C_ : any) {}
    BRA_HD int at(int j) const { return QUADS ? (j >> 2) * group * 4 + t * 4 + (j & 3) : VECD ? t * NORM_E + j : t + j * group; }
    BRA_HD bool half(int k) const { return k ? more : any; }
    BRA_HD bool has(int j) const { return VECD ? half(j >> 2) : (FULL && j < NORM_E - 1) || at(j) < C; }
};

// Threads of a row of C channels: lanes of a warp up to 256 channels (several rows a warp), whole warps above.
inline bool norm_wide(int C) { return (C + NORM_E - 1) / NORM_E > 32; }
inline int norm_group(int C) {
    const int need = (C + NORM_E - 1) / NORM_E;
    return need > 32 ? (need + 31) / 32 * 32 : need <= 8 ? 8 : need <= 16 ? 16 : 32;
}

// The kernel for rows of `group` threads that are a CTA's: the most threads its CTAs have, and whether it is compiled for FULL rows.
// 384: registers of two CTAs; the forward pass without a post-norm has those in any case, so there 512 takes shorter rows too.
struct NormKernel { int threads; bool full; };
inline NormKernel norm_kernel(int group, bool backward, bool post) {
    const int threads = group <= 128 ? 128 : group <= 384 && (backward || post) ? 384 : group <= 512 ? 512 : group <= 640 ? 640 : 1024;
    return {threads, threads > 384 && group >= 256};
}

}  // namespace bra
