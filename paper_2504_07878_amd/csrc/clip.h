// The length of many gradients together, and its clipping: what the host side (clip_api.hip) and the kernels (clip_kernels.hip) share.
#pragma once
#include "tr_internal.h"

namespace tr {

// A launch takes up to CLIP_LIST gradients, handed over by value (nothing of a call lies in memory that has to outlive it), as tiles of CLIP_TILE elements numbered through.
constexpr int CLIP_LIST = 112, CLIP_TILE = 8192;
constexpr int CLIP_GROUPS = 2048;              // most workgroups of a launch, each with a place for its sum

struct ClipList {
    const void *in[CLIP_LIST];
    void *out[CLIP_LIST];
    long long count[CLIP_LIST];
    uint32_t tile[CLIP_LIST + 1];              // first tile of each; the last one's end
    unsigned char half[CLIP_LIST];             // bf16
    int n;
};
static_assert(sizeof(ClipList) < 4000, "kernel arguments");

struct ClipState {                             // in the workspace; arrived is zero before and after every launch
    uint32_t arrived;
    float scale;                               // of the last call
    double squares;                            // of the lists before
    char pad[240];
    double part[CLIP_GROUPS];
};

// Sum of squares of a list, added to those of the lists before (first: there are none). The last list leaves the norm, and the scale for max_norm.
void launch_clip_squares(hipStream_t s, const ClipList &l, ClipState *state, bool first, bool last, double max_norm, float *norm);
// out = in * scale
void launch_clip_scale(hipStream_t s, const ClipList &l, const ClipState *state);

}  // namespace tr
