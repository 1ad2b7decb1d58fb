// Host side of tr_sample and tr_top: checks, before anything is enqueued, and launches.
#include "../../include/tokroute.h"
#include "row_pick.h"

#include <algorithm>
#include <cmath>

using namespace tr;

namespace {

bool config_ok(const tr_pick_config *c)
{
    return c && c->max_rows >= 1 && c->max_rows <= PICK_MAX_ROWS && c->vocab >= 1 && c->vocab <= PICK_MAX_VOCAB && (c->dtype == TR_F32 || c->dtype == TR_BF16);
}

size_t up(size_t v) { return (v + 255) / 256 * 256; }

// Rows of one workgroup need none of it but for the smallest size there is.
struct Plan { size_t head, list, search, steps, queue, total; };
Plan plan_of(const tr_pick_config *c)
{
    Plan p{};
    const size_t rows = std::min(c->max_rows, PICK_ROWS), groups = pick_groups(c->vocab);
    p.total = 256;
    if (c->vocab > PICK_ONE) {
        p.list = up(rows * groups * PICK_WAVES * sizeof(PickHead));
        p.search = p.list + up(rows * PICK_LISTED * 8);
        p.steps = p.search + up(rows * sizeof(PickSearch));
        p.queue = p.steps + up(rows * groups * PICK_STEPS * 8);
        p.total = p.queue + up((rows + 1) * 4);
    }
    return p;
}

size_t workspace_of(const tr_pick_config *c) { return plan_of(c).total; }

// What both calls check; TR_OK, or an error before anything is enqueued.
int arguments(const tr_pick_config *c, const tr_pick_rows *in, void *ws, size_t ws_bytes, PickArgs &a)
{
    if (!c || !in || !ws) return TR_ERR_INVALID_ARG;
    if (!config_ok(c)) return TR_ERR_SHAPE;
    if (ws_bytes < workspace_of(c) || in->rows > c->max_rows) return TR_ERR_CAPACITY;
    if (in->rows < 0 || (reinterpret_cast<uintptr_t>(ws) & 255)) return TR_ERR_INVALID_ARG;
    if (in->rows && (!in->logits || reinterpret_cast<uintptr_t>(in->logits) % (c->dtype == TR_BF16 ? 2 : 4))) return TR_ERR_INVALID_ARG;
    if (in->stride < c->vocab) return TR_ERR_INVALID_ARG;
    a = PickArgs{};
    a.logits = in->logits; a.stride = in->stride; a.rows = in->rows; a.vocab = c->vocab; a.dtype = c->dtype == TR_BF16 ? DT_BF16 : DT_F32;
    int bits = 0;
    while ((1 << bits) < c->vocab) ++bits;
    a.unit = std::min(51, 62 - bits);
    if (c->vocab > PICK_ONE) {
        a.groups = pick_groups(c->vocab);
        const Plan p = plan_of(c);
        char *const b = (char *)ws;
        a.head = (PickHead *)(b + p.head); a.list = (uint2 *)(b + p.list); a.search = (PickSearch *)(b + p.search); a.steps = (unsigned long long *)(b + p.steps); a.queue = (uint32_t *)(b + p.queue);
    }
    return TR_OK;
}

// Room for the tokens that go with x lanes in 64 whose largest of 16 is among them: t = 64 log(64 / (64 - x)) of tokens in any order, give or take sqrt(t - x)
struct Room {
    int of[64] = {};
    Room() { for (int x = 1; x < 64; ++x) { const double t = 64 * std::log(64.0 / (64 - x)); of[x] = (int)std::ceil(t + 3.5 * std::sqrt(t - x)) + 1; } }
};

// Tokens that a part leaves: as many as there is room for, or, where all rows have a top-k, enough for it. What is known of a row ends where the first part ends, so that each has to leave its
// share: with tokens in any order a part has L or more of the row's largest top_k by Poisson's distribution of top_k / parts, and one row in a hundred may have such a part (which then is
// read again, 10 us more for it; one row in a million: 1 us more for every call at top-k 16 to 64).
void list_tokens(PickArgs &a, int top_k)
{
    if (!a.head) return;
    // (without top-k half of it: of 64 flat rows of 20000 top-p 0.9 and min-p 0.05 take 34 instead of 45 us, while the largest 1000 take 31 instead of 68 with all of it)
    const int most = top_k > 0 || a.top_ks ? pick_listed(a.groups) : std::min(pick_listed(a.groups), PICK_PART_LISTED / 2), parts = a.groups * PICK_WAVES;
    static const Room room;
    int lanes = 63;
    if (top_k > 0) {
        const double mean = (double)top_k / parts;
        int least = 0;
        for (double p = std::exp(-mean); least < 63 && (least <= mean || p * parts > 1e-2); p *= mean / least) ++least;
        lanes = std::min(lanes, least * 4 / 3);      // (a part takes more than 3/4 of them)
    }
    while (lanes > 1 && room.of[lanes] > most) --lanes;
    a.listed_lanes = lanes;
    a.listed = std::min(most, room.of[lanes]);
}

// PICK_ROWS rows at a time where they meet in the workspace
template <class Launch> int enqueue(const PickArgs &all, Launch launch)
{
    const size_t size = all.dtype == DT_BF16 ? 2 : 4;
    const int most = all.head ? PICK_ROWS : PICK_MAX_ROWS;
    for (int at = 0; at < all.rows; at += most) {
        PickArgs a = all;
        a.rows = std::min(most, all.rows - at);
        a.past = !a.queue || a.rows * (size_t)a.vocab * size > PICK_KEEP;
        a.logits = (const char *)all.logits + (size_t)at * all.stride * size;
        for (const float **p : {&a.u, &a.temperatures, &a.top_ps, &a.min_ps}) if (*p) *p += at;
        if (a.top_ks) a.top_ks += at;
        if (a.token) { a.token += at; a.logprob += at; }
        if (a.ids) { a.ids += (size_t)at * all.entries; a.values += (size_t)at * all.entries; }
        launch(a);
    }
    return hipGetLastError() == hipSuccess ? TR_OK : TR_ERR_HIP;
}

bool aligned(const void *p) { return !(reinterpret_cast<uintptr_t>(p) & 3); }

}  // namespace

extern "C" {

size_t tr_pick_workspace_bytes(const tr_pick_config *cfg) { return config_ok(cfg) ? workspace_of(cfg) : 0; }

int tr_sample(const tr_pick_config *cfg, void *workspace, size_t workspace_bytes, void *hip_stream, const tr_pick_rows *in, const tr_sample_how *how, int32_t *token, float *logprob)
{
    PickArgs a;
    if (const int e = arguments(cfg, in, workspace, workspace_bytes, a)) return e;
    if (!how) return TR_ERR_INVALID_ARG;
    if (!how->temperatures && !(how->temperature >= 0.f)) return TR_ERR_INVALID_ARG;
    if (!how->top_ks && how->top_k < 0) return TR_ERR_INVALID_ARG;
    if (!how->top_ps && !(how->top_p >= 0.f && how->top_p <= 1.f)) return TR_ERR_INVALID_ARG;
    if (!how->min_ps && !(how->min_p >= 0.f && how->min_p <= 1.f)) return TR_ERR_INVALID_ARG;
    if (!aligned(how->u) || !aligned(how->temperatures) || !aligned(how->top_ks) || !aligned(how->top_ps) || !aligned(how->min_ps) || !aligned(token) || !aligned(logprob)) return TR_ERR_INVALID_ARG;
    if (!a.rows) return TR_OK;
    if (!how->u || !token || !logprob) return TR_ERR_INVALID_ARG;
    a.u = how->u; a.temperatures = how->temperatures; a.top_ks = how->top_ks; a.top_ps = how->top_ps; a.min_ps = how->min_ps;
    a.temperature = how->temperature; a.top_k = how->top_k < a.vocab ? how->top_k : 0; a.top_p = how->top_p; a.min_p = how->min_p;
    a.token = token; a.logprob = logprob;
    // (top-k ends within what the parts list but for rows whose largest logits lie oddly; one workgroup searches these)
    if (!(a.top_ps || a.min_ps || a.top_p < 1.f || a.min_p > 0.f) || !(a.top_ks || a.top_k == 0)) a.queue = nullptr;
    list_tokens(a, !a.temperatures && !(a.temperature > 0.f) ? 1 : a.top_ks ? 0 : a.top_k);
    return enqueue(a, [&](const PickArgs &p) { launch_sample((hipStream_t)hip_stream, p); });
}

int tr_top(const tr_pick_config *cfg, void *workspace, size_t workspace_bytes, void *hip_stream, const tr_pick_rows *in, int32_t entries, int32_t *ids, float *values)
{
    PickArgs a;
    if (const int e = arguments(cfg, in, workspace, workspace_bytes, a)) return e;
    if (entries < 1) return TR_ERR_INVALID_ARG;
    if (entries > PICK_MAX_ENTRIES) return TR_ERR_CAPACITY;
    if (!aligned(ids) || !aligned(values)) return TR_ERR_INVALID_ARG;
    if (!a.rows) return TR_OK;
    if (!ids || !values) return TR_ERR_INVALID_ARG;
    a.entries = entries; a.ids = ids; a.values = values;
    a.queue = nullptr;
    list_tokens(a, entries);
    return enqueue(a, [&](const PickArgs &p) { launch_top((hipStream_t)hip_stream, p); });
}

}  // extern "C"
