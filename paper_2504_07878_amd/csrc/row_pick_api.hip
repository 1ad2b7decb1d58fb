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

size_t workspace_of(const tr_pick_config *) { return 256; }

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
    a.unit = std::min(52, 62 - bits);
    return TR_OK;
}

int enqueued() { return hipGetLastError() == hipSuccess ? TR_OK : TR_ERR_HIP; }
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
    a.temperature = how->temperature; a.top_k = how->top_k; a.top_p = how->top_p; a.min_p = how->min_p;
    a.token = token; a.logprob = logprob;
    launch_sample((hipStream_t)hip_stream, a);
    return enqueued();
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
    launch_top((hipStream_t)hip_stream, a);
    return enqueued();
}

}  // extern "C"
