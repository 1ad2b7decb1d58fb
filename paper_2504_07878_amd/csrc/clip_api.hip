// Host side of tr_grad_norm and tr_grad_clip: checks, before anything is enqueued, and lists of gradients for the kernels.
#include "../../include/tokroute.h"
#include "clip.h"

#include <algorithm>
#include <new>
#include <vector>

using namespace tr;

namespace {

struct Span { uintptr_t from, to; int of; bool written; };

size_t size_of(int dtype) { return dtype == TR_BF16 ? 2 : 4; }

// Whether memory that is written is also another gradient's, or lies across its own
bool overlap(int n, const void *const *in, void *const *out, const int64_t *counts, const int32_t *dtypes)
{
    std::vector<Span> spans;
    spans.reserve(2 * (size_t)n);
    for (int i = 0; i < n; ++i) {
        if (!counts[i]) continue;
        const size_t bytes = (size_t)counts[i] * size_of(dtypes[i]);
        const uintptr_t a = reinterpret_cast<uintptr_t>(in[i]), b = reinterpret_cast<uintptr_t>(out[i]);
        spans.push_back(Span{b, b + bytes, i, true});
        if (a != b) spans.push_back(Span{a, a + bytes, i, false});
    }
    std::sort(spans.begin(), spans.end(), [](const Span &x, const Span &y) { return x.from < y.from; });
    uintptr_t read_to = 0, written_to = 0;     // how far the spans before reach
    for (const Span &x : spans) {
        if (x.from < written_to || (x.written && x.from < read_to)) return true;
        (x.written ? written_to : read_to) = std::max(x.written ? written_to : read_to, x.to);
    }
    return false;
}

// f(list) for all gradients that have elements, from the last on where asked
template <class F> void lists(bool back, int n, const void *const *in, void *const *out, const int64_t *counts, const int32_t *dtypes, F f)
{
    ClipList l{};
    for (int k = 0; k < n; ++k) {
        const int i = back ? n - 1 - k : k;
        if (!counts[i]) continue;
        const uint64_t bytes = (uint64_t)counts[i] * size_of(dtypes[i]), tiles = (bytes + CLIP_TILE - 1) / CLIP_TILE;
        if (l.n == CLIP_LIST || l.tile[l.n] + tiles > 0x7fffffffu) {      // (one gradient alone has fewer)
            f(l);
            l.n = 0;
        }
        l.in[l.n] = in[i]; l.out[l.n] = out ? out[i] : nullptr; l.count[l.n] = counts[i]; l.half[l.n] = dtypes[i] == TR_BF16;
        l.tile[l.n + 1] = l.tile[l.n] + (uint32_t)tiles;
        ++l.n;
    }
    if (l.n) f(l);
}

int run(void *ws, size_t ws_bytes, void *stream, int n, const void *const *in, void *const *out, const int64_t *counts, const int32_t *dtypes, double max_norm, float *norm)
{
    if (!ws || !norm || n < 0 || (n && (!in || !counts || !dtypes))) return TR_ERR_INVALID_ARG;
    if (ws_bytes < CLIP_SUMS * sizeof(double)) return TR_ERR_CAPACITY;
    if ((reinterpret_cast<uintptr_t>(ws) & 255) || (reinterpret_cast<uintptr_t>(norm) & 3) || !(max_norm >= 0)) return TR_ERR_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        if (dtypes[i] != TR_F32 && dtypes[i] != TR_BF16) return TR_ERR_SHAPE;
        if (counts[i] < 0 || counts[i] > (int64_t)1 << 40) return TR_ERR_SHAPE;
        const size_t size = size_of(dtypes[i]);
        if (counts[i] && (!in[i] || reinterpret_cast<uintptr_t>(in[i]) % size || (out && (!out[i] || reinterpret_cast<uintptr_t>(out[i]) % size)))) return TR_ERR_INVALID_ARG;
    }
    if (out) {
        try {
            if (overlap(n, in, out, counts, dtypes)) return TR_ERR_INVALID_ARG;
        } catch (const std::bad_alloc &) {
            return TR_ERR_CAPACITY;
        }
    }
    hipStream_t s = (hipStream_t)stream;
    double *const sums = (double *)ws;
    int have = 0;                          // sums so far
    // tiles that are read again while the cache may still have them, the last ones, and those before them
    uint64_t kept = 0, past = 0;
    for (int i = 0; i < n; ++i) past += ((uint64_t)counts[i] * size_of(dtypes[i]) + CLIP_TILE - 1) / CLIP_TILE;
    if (out) kept = std::min<uint64_t>(past, CLIP_KEEP / CLIP_TILE);
    past -= kept;
    uint64_t left = past;
    lists(false, n, in, out, counts, dtypes, [&](ClipList &l) {
        l.past = (uint32_t)std::min<uint64_t>(left, l.tile[l.n]);
        left -= l.past;
        if (have + clip_groups(l) > CLIP_SUMS) {
            launch_clip_join(s, sums, have, sums, nullptr);
            have = 1;
        }
        launch_clip_squares(s, l, sums + have);
        have += clip_groups(l);
    });
    if (!out || !have) launch_clip_join(s, sums, have, nullptr, norm);
    else {
        // every workgroup of the scaling adds the sums up by itself, which saves a launch; many are added up once
        if (have > CLIP_GROUPS) {
            launch_clip_join(s, sums, have, sums, nullptr);
            have = 1;
        }
        lists(true, n, in, out, counts, dtypes, [&](ClipList &l) {
            l.past = (uint32_t)std::min<uint64_t>(kept, l.tile[l.n]);
            kept -= l.past;
            launch_clip_scale(s, l, sums, have, max_norm, norm);
            norm = nullptr;
        });
    }
    return hipGetLastError() == hipSuccess ? TR_OK : TR_ERR_HIP;
}

}  // namespace

extern "C" {

size_t tr_grad_workspace_bytes(void) { return CLIP_SUMS * sizeof(double); }

int tr_grad_norm(void *workspace, size_t workspace_bytes, void *hip_stream, int32_t n, const void *const *grads, const int64_t *counts, const int32_t *dtypes, float *norm)
{
    return run(workspace, workspace_bytes, hip_stream, n, grads, nullptr, counts, dtypes, 0.0, norm);
}

int tr_grad_clip(void *workspace, size_t workspace_bytes, void *hip_stream, int32_t n, const void *const *grads, void *const *out, const int64_t *counts, const int32_t *dtypes,
                 float max_norm, float *norm)
{
    if (n > 0 && !out) return TR_ERR_INVALID_ARG;
    return run(workspace, workspace_bytes, hip_stream, n, grads, out, counts, dtypes, (double)max_norm, norm);
}

}  // extern "C"
