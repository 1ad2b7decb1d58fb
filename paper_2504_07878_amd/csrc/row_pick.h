// Tokens drawn from rows of logits, and a row's largest logits: what the host side (row_pick_api.hip) and the kernels (row_pick_kernels.hip) share.
//
// The order of a row: larger logit first, of equal ones the lower id. Every filter keeps a prefix of that order, so that what is kept is all above some logit and the first few ids of those
// equal to it. Masses are whole numbers, exp((z - max) / T) in units of 2^-unit: their sums are the same in any order of adding, so that prefixes and draws do not depend on the schedule.
#pragma once
#include "tr_internal.h"

namespace tr {

constexpr int PICK_MAX_ROWS = 1 << 20, PICK_MAX_VOCAB = 1 << 20, PICK_MAX_ENTRIES = 1024;

// A wavefront reads a part of a row, a workgroup eight of them. Rows of more than one workgroup meet in the workspace: every part leaves its sum and its largest tokens, from which one
// workgroup decides. Workspace and launches are for PICK_ROWS rows at a time.
constexpr int PICK_THREADS = 512, PICK_WAVES = PICK_THREADS / 64, PICK_PART = 1024, PICK_GROUP = PICK_PART * PICK_WAVES;
constexpr int PICK_ONE = PICK_GROUP;                      // most tokens of a row that is one workgroup's from the start
constexpr int PICK_ROWS = 1024;
constexpr int PICK_LISTED = 8192;                         // most tokens of a row that parts leave, and that the deciding workgroup holds
constexpr int PICK_PART_LISTED = 128;                     // of one part
constexpr size_t PICK_KEEP = 192 << 20;                   // bytes of logits that a last-level cache may still hold when they are read again
constexpr int PICK_STEPS = 256;                           // of a histogram of masses over the logits of a row (256 rows of 152064, some of them flat: 127 us, with 128 steps 131, with 512 133)

struct alignas(16) PickHead {
    union { double sum; unsigned long long mass; };   // of the part's weights, relative to its own largest; of what it keeps, in units
    uint32_t top;          // largest key
    uint32_t from;         // all the part's tokens of this key or a larger one are listed
    uint32_t count, pad;   // those
};

// A row whose filters end below what the parts have listed
struct alignas(16) PickSearch {
    uint32_t stage;        // PICK_*
    uint32_t top_key, least;   // largest key; the smallest that min_p keeps
    float from, scale;     // logits below `from` in steps of 1 / scale
    uint32_t found, pad;   // the stage that it turned out to be
    unsigned long long want;   // mass that it keeps
};
enum { PICK_STEP = 1,      // the step, then the place in it
       PICK_LEAST = 2,     // everything from `least` on
       PICK_WHOLE = 3 };   // one workgroup looks through the row

struct PickArgs {
    const void *logits;
    long long stride;                // elements from row to row
    int rows, vocab, dtype;          // DT_*
    int unit;                        // masses are in units of 2^-unit: vocab of them stay below 2^63
    int groups, listed;              // workgroups a row, tokens a part may leave
    int listed_lanes;                // lanes whose largest token is among them
    // Logits are read past the caches where nothing reads them again, or where they do not fit (the largest 64 of 1024 rows of 151936: 119 instead of 125 us, after they were written 122 instead
    // of 189; where rows may be searched 256 bf16 rows take 127 through the caches and 129 past them)
    bool past;
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
    // workspace (rows of more than one workgroup)
    PickHead *head;                  // [rows][parts]; NULL: rows of one workgroup
    uint2 *list;                     // [rows][parts][listed]: key, id
    PickSearch *search;              // [rows]
    unsigned long long *steps;       // [rows][groups][PICK_STEPS]
    uint32_t *queue;                 // [0] how many rows are searched, then which; NULL: none can be
};

inline int pick_groups(int vocab) { return (vocab + PICK_GROUP - 1) / PICK_GROUP; }
inline int pick_listed(int groups)
{
    const int most = PICK_LISTED / (groups * PICK_WAVES);
    return most < PICK_PART_LISTED ? most : PICK_PART_LISTED;
}

// PICK_ROWS rows at most where a.head is there
void launch_sample(hipStream_t s, const PickArgs &a);
void launch_top(hipStream_t s, const PickArgs &a);

}  // namespace tr
