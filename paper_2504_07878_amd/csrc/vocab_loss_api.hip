// Host side of the losses over the vocabulary: checks, workspace and the order of launches behind tr_cross_entropy, tr_distill and their gradients.
#include "../../include/tokroute.h"
#include "vocab_loss.h"

#include <algorithm>
#include <cmath>

using namespace tr;

namespace {

size_t up(size_t v, size_t to) { return (v + to - 1) / to * to; }

constexpr int MAX_ROWS = 1 << 20, MAX_DIM = 1 << 16, MAX_VOCAB = 1 << 24;

bool config_ok(const tr_loss_config *c)
{
    if (!c || c->max_rows < 1 || c->max_rows > MAX_ROWS || c->dim < 1 || c->dim > MAX_DIM || c->vocab < 1 || c->vocab > MAX_VOCAB) return false;
    if (c->max_entries < 1 || c->max_entries > LOSS_MAX_ENTRIES) return false;
    return (c->hidden_dtype == TR_F32 && (c->weight_dtype == TR_F32 || c->weight_dtype == TR_BF16)) || (c->hidden_dtype == TR_BF16 && c->weight_dtype == TR_BF16);
}

// Where everything lies in the workspace, for a configuration; the sizes of a call's own launches follow from its rows, never beyond these.
struct Plan {
    int n_pad, d_pad, piece, g_ld, splits;
    int packed;        // columns of a piece whose head is packed
    size_t head, idx, state, part, value, G, acc, hp, wp, row, total;
};

bool is_bf16(const tr_loss_config *c) { return c->hidden_dtype == TR_BF16; }                                    // all products run on bf16 matrix instructions
// those of the softmax and of the probabilities do, on rows in three planes: the gradients take exp(z - lse) of the very products that lse was summed from
bool in_planes(const tr_loss_config *c) { return c->hidden_dtype == TR_F32 && c->weight_dtype == TR_BF16; }

// G stays at 512 MB or less, but a piece has 2048 columns at least (8192 rows x 151936 x 896, three quarters of the rows counting, all products of the gradients, pieces of
// 256 / 512 / 1024 MB: 5.60 / 5.45 / 5.42 ms); where the head is packed, that stays at 128 MB or less.
Plan plan_of(const tr_loss_config *c)
{
    Plan p{};
    const bool half = is_bf16(c);
    const int block = half ? BF16_BLOCK : F32_BLOCK;
    const size_t g_size = half ? 2 : 4, whole = up(c->vocab, BF16_BLOCK), steps = up(c->dim, 64);
    p.n_pad = (int)up(c->max_rows, BF16_BLOCK);
    p.d_pad = (int)steps;
    p.piece = (int)std::min(whole, std::max<size_t>(2048, (512u << 20) / g_size / p.n_pad / BF16_BLOCK * BF16_BLOCK));
    p.packed = (int)std::min(whole, std::max<size_t>(2048, (128u << 20) / 2 / steps / BF16_BLOCK * BF16_BLOCK));
    p.g_ld = p.piece + 128;
    const int mb = (int)(up(p.d_pad, block) / block), few = std::max(1, p.piece / 256);
    p.splits = half ? std::min(few, std::max(1, 32 / mb) * 8) : std::max(1, std::min(1024 / (mb * (p.n_pad / F32_BLOCK)), few));
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t was = at; at += up(bytes, 256); return was; };
    p.head = take(sizeof(LossHead));
    p.idx = take((size_t)p.n_pad * 4);
    p.state = take(c->max_rows);
    p.part = take((half ? whole / BF16_BLOCK * 2 : in_planes(c) ? whole / BF16_BLOCK : whole / F32_BLOCK * 2) * p.n_pad * sizeof(float2));
    p.value = take((size_t)p.n_pad * c->max_entries * 4);
    p.G = take((size_t)p.n_pad * p.g_ld * g_size);
    // bf16, rows of all splits (bf16_splits): blocks * splits <= 256 where there are fewer than 32 blocks, 8 splits up to 1024 blocks, one from there on
    const size_t sums = (size_t)p.splits * p.n_pad, most = std::max({(size_t)std::min(p.splits, 8) * std::min<size_t>(p.n_pad, 1024 / mb * BF16_BLOCK + BF16_BLOCK),
                                                                     (size_t)(256 / mb + 1) * BF16_BLOCK, (size_t)p.n_pad});
    p.acc = take((half ? std::min(sums, most) : sums) * p.d_pad * 4);
    if (half || in_planes(c)) {
        p.hp = take((size_t)p.n_pad * (half ? 1 : 3) * steps * 2);
        p.wp = take((size_t)p.packed * steps * 2);
        p.row = take((size_t)p.n_pad * sizeof(LossRow));
    }
    p.total = at;
    return p;
}

// Checks what every call has in common and fills in the arguments; TR_OK or an error, before anything is enqueued.
int arguments(const tr_loss_config *c, const tr_loss_rows *in, void *ws, size_t ws_bytes, bool teacher, bool gradient, LossArgs &a, Plan &p)
{
    if (!c || !in || !ws) return TR_ERR_INVALID_ARG;
    if (!config_ok(c)) return TR_ERR_SHAPE;
    p = plan_of(c);
    if (ws_bytes < p.total) return TR_ERR_CAPACITY;
    if (in->rows > c->max_rows) return TR_ERR_CAPACITY;
    if (in->rows < 0 || (reinterpret_cast<uintptr_t>(ws) & 255)) return TR_ERR_INVALID_ARG;
    if (!in->weight || (in->rows && (!in->hidden || !in->ids || (teacher && !in->teacher)))) return TR_ERR_INVALID_ARG;
    if (in->hidden_stride < c->dim || in->weight_stride < c->dim) return TR_ERR_INVALID_ARG;
    if (teacher && (in->entries < 1 || !(in->temperature > 0.f) || !std::isfinite(in->temperature))) return TR_ERR_INVALID_ARG;
    if (teacher && in->entries > c->max_entries) return TR_ERR_CAPACITY;
    const auto size = [](int dt) { return dt == TR_BF16 ? 2u : 4u; };
    if (reinterpret_cast<uintptr_t>(in->hidden) % size(c->hidden_dtype) || reinterpret_cast<uintptr_t>(in->weight) % size(c->weight_dtype)) return TR_ERR_INVALID_ARG;
    char *const b = (char *)ws;
    a = LossArgs{};
    a.hidden = in->hidden; a.weight = in->weight; a.hs = in->hidden_stride; a.ws = in->weight_stride;
    a.hdt = c->hidden_dtype == TR_BF16 ? DT_BF16 : DT_F32; a.wdt = c->weight_dtype == TR_BF16 ? DT_BF16 : DT_F32;
    a.rows = in->rows; a.dim = c->dim; a.vocab = c->vocab;
    a.entries = teacher ? in->entries : 1; a.ids = in->ids; a.teacher = teacher ? in->teacher : nullptr; a.temperature = teacher ? in->temperature : 1.f;
    a.head = (LossHead *)(b + p.head); a.idx = (int *)(b + p.idx); a.state = (unsigned char *)(b + p.state); a.part = (float2 *)(b + p.part);
    a.value = (float *)(b + p.value); a.G = b + p.G; a.acc = (float *)(b + p.acc);
    a.n_pad = a.part_ld = p.n_pad; a.d_pad = p.d_pad; a.piece = p.piece; a.g_ld = p.g_ld; a.splits = p.splits;
    a.direct = a.dim % 64 == 0 && a.ws % 8 == 0 && a.ws < (1 << 22) && (reinterpret_cast<uintptr_t>(a.weight) & 15) == 0;
    if (is_bf16(c) || in_planes(c)) {
        a.hp = b + p.hp; a.wp = b + p.wp; a.row = (LossRow *)(b + p.row);
        a.pairs = gradient && is_bf16(c);
        const int rows = gradient && a.rows <= PAIR_ROWS ? 2 * a.rows : a.rows;
        // Few rows in blocks of 256 entries x 64 or 128 rows, up to 256 rows (151936 x 896, 160 rows, blocks of 256 instead: gradients 316 us against 297; 300 rows 423 against 425).
        // Losses of small heads, where that leaves most compute units without a block, in small ones (100 rows x 30000 x 512: 21 -> 17 us; gradients would be 53 -> 59).
        const bool small = !gradient && c->vocab <= 128 * BF16_BLOCK;
        a.n_block = rows <= 64 || in_planes(c) ? 64 : rows <= 256 && !small ? 128 : 256;
        if (rows <= a.n_block && a.n_block < 256 && !in_planes(c)) a.part_ld = a.n_block;
        if (!a.direct) a.piece = std::min(p.piece, p.packed);
    }
    return TR_OK;
}

int enqueued() { return hipGetLastError() == hipSuccess ? TR_OK : TR_ERR_HIP; }

int forward(const tr_loss_config *c, void *ws, size_t ws_bytes, void *stream, const tr_loss_rows *in, float *loss, float *lse, bool teacher)
{
    LossArgs a;
    Plan p;
    if (const int e = arguments(c, in, ws, ws_bytes, teacher, false, a, p)) return e;
    if (a.rows && (!loss || !lse)) return TR_ERR_INVALID_ARG;
    if (!a.rows) return TR_OK;
    a.loss = loss; a.lse = lse;
    hipStream_t s = (hipStream_t)stream;
    launch_loss_rows(s, a);
    const bool bf16_products = a.hp != nullptr;
    if (bf16_products) {
        const int most = a.direct ? a.vocab : std::min(a.piece, a.vocab);
        const bool along = bf16_takes_entries(a, most);
        for (int v0 = 0, vn; v0 < a.vocab; v0 += vn) {
            vn = std::min(most, a.vocab - v0);
            if (!a.direct) launch_bf16_pack_head(s, a, v0, vn);
            launch_bf16_softmax(s, a, v0, vn, along && v0 == 0);
        }
        if (!along) launch_bf16_entries(s, a, !a.direct && a.piece >= a.vocab);
    } else {
        launch_f32_softmax(s, a);
    }
    launch_loss_finish(s, a, bf16_products ? bf16_softmax_parts(a) : f32_softmax_parts(a));
    return enqueued();
}

int backward(const tr_loss_config *c, void *ws, size_t ws_bytes, void *stream, const tr_loss_rows *in, const float *lse, const float *grad_loss, const tr_loss_grads *out, bool teacher)
{
    LossArgs a;
    Plan p;
    if (const int e = arguments(c, in, ws, ws_bytes, teacher, true, a, p)) return e;
    if (!out || (a.rows && (!lse || !grad_loss))) return TR_ERR_INVALID_ARG;
    if ((out->d_hidden && out->d_hidden_stride < c->dim) || (out->d_weight && out->d_weight_stride < c->dim)) return TR_ERR_INVALID_ARG;
    const auto size = [](int dt) { return dt == TR_BF16 ? 2u : 4u; };
    if (reinterpret_cast<uintptr_t>(out->d_hidden) % size(c->hidden_dtype) || reinterpret_cast<uintptr_t>(out->d_weight) % size(c->weight_dtype)) return TR_ERR_INVALID_ARG;
    if (!out->d_hidden && !out->d_weight) return TR_OK;
    a.lse = const_cast<float *>(lse); a.grad = grad_loss;
    a.d_hidden = out->d_hidden; a.dhs = out->d_hidden_stride; a.d_weight = out->d_weight; a.dws = out->d_weight_stride;
    hipStream_t s = (hipStream_t)stream;
    launch_loss_rows(s, a);
    // a teacher's entries are placed in G; cross entropy's one a row falls to whoever computes that place
    const bool half = is_bf16(c), bf16_products = a.hp != nullptr, one = a.piece >= a.vocab;
    const bool along = bf16_products && teacher && bf16_takes_entries(a, std::min(a.piece, a.vocab));
    const bool whole = bf16_products && a.rows && !a.direct && one;      // the head is packed once, whole
    if (whole) launch_bf16_pack_head(s, a, 0, a.vocab);
    if (a.rows && bf16_products && teacher && !along) launch_bf16_entries(s, a, whole);
    for (int v0 = 0; v0 < a.vocab; v0 += a.piece) {
        const int vn = std::min(a.piece, a.vocab - v0);
        if (a.rows) {
            if (bf16_products) {
                if (!a.direct && !whole) launch_bf16_pack_head(s, a, v0, vn);
                launch_bf16_probabilities(s, a, v0, vn, along && v0 == 0);
            } else launch_f32_probabilities(s, a, v0, vn);
            if (teacher && v0 == 0) launch_loss_values(s, a, one);
            if (teacher && !one) launch_loss_scatter(s, a, v0, vn);
            if (half && a.d_hidden) launch_bf16_hidden_grad(s, a, v0, vn, v0 == 0);
        }
        if (!half) launch_f32_gradients(s, a, v0, vn, v0 == 0);
        else if (a.d_weight) launch_bf16_weight_grad(s, a, v0, vn);
    }
    if (a.d_hidden) launch_loss_hidden_grad(s, a);
    return enqueued();
}

}  // namespace

extern "C" {

size_t tr_loss_workspace_bytes(const tr_loss_config *cfg) { return config_ok(cfg) ? plan_of(cfg).total : 0; }

int tr_cross_entropy(const tr_loss_config *cfg, void *workspace, size_t workspace_bytes, void *hip_stream, const tr_loss_rows *in, float *loss, float *lse)
{
    return forward(cfg, workspace, workspace_bytes, hip_stream, in, loss, lse, false);
}

int tr_cross_entropy_grad(const tr_loss_config *cfg, void *workspace, size_t workspace_bytes, void *hip_stream, const tr_loss_rows *in, const float *lse,
                          const float *grad_loss, const tr_loss_grads *out)
{
    return backward(cfg, workspace, workspace_bytes, hip_stream, in, lse, grad_loss, out, false);
}

int tr_distill(const tr_loss_config *cfg, void *workspace, size_t workspace_bytes, void *hip_stream, const tr_loss_rows *in, float *loss, float *lse)
{
    return forward(cfg, workspace, workspace_bytes, hip_stream, in, loss, lse, true);
}

int tr_distill_grad(const tr_loss_config *cfg, void *workspace, size_t workspace_bytes, void *hip_stream, const tr_loss_rows *in, const float *lse,
                    const float *grad_loss, const tr_loss_grads *out)
{
    return backward(cfg, workspace, workspace_bytes, hip_stream, in, lse, grad_loss, out, true);
}

}  // extern "C"
