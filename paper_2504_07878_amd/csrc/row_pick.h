// Tokens drawn from rows of logits, and a row's largest logits: what the host side (row_pick_api.hip) and the kernels (row_pick_kernels.hip) share.
//
// The order of a row: larger logit first, of equal ones the lower id. Every filter keeps a prefix of that order, so that what is kept is all above some logit and the first few ids of those
// equal to it. Masses are whole numbers, exp((z - max) / T) in units of 2^-unit: their sums are the same in any order of adding, so that prefixes and draws do not depend on the schedule.
#pragma once
#include "tr_internal.h"

namespace tr {

constexpr int PICK_MAX_ROWS = 1 << 20, PICK_MAX_VOCAB = 1 << 20, PICK_MAX_ENTRIES = 1024;

struct PickArgs {
    const void *logits;
    long long stride;                // elements from row to row
    int rows, vocab, dtype;          // DT_*
    int unit;                        // masses are in units of 2^-unit: vocab of them stay below 2^63
    // draws: a number a row, or the value for all
    const float *u, *temperatures, *top_ps, *min_ps;
    const int *top_ks;
    float temperature, top_p, min_p;
    int top_k;
    int32_t *token;
    float *logprob;
    // largest logits
    int entries;
    int32_t *ids;
    float *values;
};

void launch_sample(hipStream_t s, const PickArgs &a);
void launch_top(hipStream_t s, const PickArgs &a);

}  // namespace tr
