// The length of many gradients together, and its clipping: what the host side (clip_api.hip) and the kernels (clip_kernels.hip) share.
#pragma once
#include "tr_internal.h"

namespace tr {

// A launch takes up to CLIP_LIST gradients (as many as 4 KB of arguments hold), handed over by value (nothing of a call lies in memory that has to outlive it), as tiles of CLIP_TILE bytes
// numbered through: eight loads of 16 bytes a thread in flight (norm of 494 million bf16 elements, read through the caches, 188 us, with four 209, with sixteen the same).
constexpr int CLIP_LIST = 112, CLIP_TILE = 32768;
constexpr int CLIP_GROUPS = 2048;              // most workgroups of a launch, each of which leaves a sum
// What is read once, or not again before it has left the last-level cache, is read past the caches (norm of 494 million bf16 elements 158 instead of 187 us; after another buffer was written,
// whose lines the loads would throw out, 175 instead of 255). Bytes at the end of the gradients that the cache is left for between the two passes of clipping (clip of 272 MB
// 124 us, of 2 GB 987; with 128 MB 130 and 996, with 256 MB 128 and 987, without any 132 and 993; all read through the caches 130 and 1094):
constexpr uint64_t CLIP_KEEP = 192 << 20;
constexpr int CLIP_SUMS = 4096;                // places for sums in the workspace

struct ClipList {
    const void *in[CLIP_LIST];
    void *out[CLIP_LIST];
    long long count[CLIP_LIST];
    uint32_t tile[CLIP_LIST + 1];              // first tile of each; the last one's end
    unsigned char half[CLIP_LIST];             // bf16
    int n;
    uint32_t past;                             // tiles before this one are read past the caches; backwards those from this one on
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
