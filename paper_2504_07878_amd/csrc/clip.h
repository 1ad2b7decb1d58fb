// The length of many gradients together, and its clipping: what the host side (clip_api.hip) and the kernels (clip_kernels.hip) share.
#pragma once
#include "tr_internal.h"

namespace tr {

// A launch takes up to CLIP_LIST gradients (as many as 4 KB of arguments hold), handed over by value (nothing of a call lies in memory that has to outlive it), as tiles of CLIP_TILE bytes
// numbered through: eight loads of 16 bytes a thread in flight (norm of 494 million bf16 elements 188 us, with four 209, with sixteen the same).
constexpr int CLIP_LIST = 112, CLIP_TILE = 32768;
constexpr int CLIP_GROUPS = 2048;              // most workgroups of a launch, each of which leaves a sum
constexpr int CLIP_SUMS = 4096;                // places for sums in the workspace

struct ClipList {
    const void *in[CLIP_LIST];
    void *out[CLIP_LIST];
    long long count[CLIP_LIST];
    uint32_t tile[CLIP_LIST + 1];              // first tile of each; the last one's end
    unsigned char half[CLIP_LIST];             // bf16
    int n;
};
static_assert(sizeof(ClipList) < 4000, "kernel arguments");

inline int clip_groups(const ClipList &l) { return l.tile[l.n] < CLIP_GROUPS ? (int)l.tile[l.n] : CLIP_GROUPS; }

// Sums of squares of a list, clip_groups of them, from sums[0] on
void launch_clip_squares(hipStream_t s, const ClipList &l, double *sums);
// The first n sums: into sums[0], and their root into norm (either may be NULL)
void launch_clip_join(hipStream_t s, const double *sums, int n, double *to, float *norm);
// out = in * min(1, max_norm / norm), norm the root of the first n sums, which is left in `norm` (where it is not NULL)
void launch_clip_scale(hipStream_t s, const ClipList &l, const double *sums, int n, double max_norm, float *norm);

}  // namespace tr
