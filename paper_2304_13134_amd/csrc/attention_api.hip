// C ABI of the layer's calls in which frames see each other (see include/last.h): argument validation, choice of the kernels,
// workspace planning and launches.  No allocation, no synchronisation.
#include "../../include/last.h"

#include <hip/hip_runtime.h>

#include "layer.hpp"
#include "layer_host.hpp"
#include "heads_kernels.hpp"
#include "attention_kernels.hpp"
#include "cached_kernels.hpp"
#include <algorithm>
#include <cmath>
#include <limits.h>

using namespace last;

namespace {

constexpr int kMostWidth = 128, kMostHeads = 1 << 16, kMostPage = 1 << 20;
constexpr int kMostFrames = 1 << 28;                  // of an item: sums of two of them and a position stay in 32 bits

last_status_t check_heads(const last_heads_t* h)
{
    if (!h) return LAST_ERR_NULL;
    if (h->heads < 1 || h->kv_heads < 1 || h->width < 1 || h->heads > kMostHeads) return LAST_ERR_SHAPE;
    if (h->heads % h->kv_heads != 0) return LAST_ERR_SHAPE;
    if (h->width % 8 != 0 || h->width > kMostWidth) return LAST_ERR_UNSUPPORTED;
    return LAST_OK;
}

// seen: of a call in which frames see each other, whose workgroups, at most one for each head of each frame, are numbered in 32 bits; an item's heads of
// frames in blocks of 32 are counted in 31
last_status_t check_items(const last_frames_t* f, const last_heads_t* h, bool seen, long long* rows)
{
    LAST_TRY(check_frames(f, rows));
    LAST_TRY(check_heads(h));
    if (f->T > kMostFrames || *rows * h->heads > (seen ? (1ll << 31) - 1 : 1ll << 36) || (long long)f->T * h->heads > 1ll << 30) return LAST_ERR_SHAPE;
    return LAST_OK;
}

last_status_t check_rotation(const last_rotation_t* r, int width)
{
    if (!r || r->columns == 0) return LAST_OK;
    if (r->columns < 0 || r->columns > width) return LAST_ERR_SHAPE;
    if (r->columns % 8 != 0) return LAST_ERR_UNSUPPORTED;
    return r->frequencies ? LAST_OK : LAST_ERR_NULL;
}

last_status_t check_band(const last_band_t* b)
{
    if (!b) return LAST_ERR_NULL;
    if (b->left < -1 || b->right < -1 || b->sinks < 0 || !(b->scale > 0.f) || !std::isfinite(b->scale)) return LAST_ERR_SHAPE;
    return b->sinks > kMostSinks ? LAST_ERR_UNSUPPORTED : LAST_OK;
}

last_status_t check_cache(const last_cache_t* c)
{
    if (!c || !c->k || !c->v || !c->table || !c->used) return LAST_ERR_NULL;
    if (c->pages < 1 || c->page < 1 || c->page > kMostPage || c->entries < 1) return LAST_ERR_SHAPE;
    if ((long long)c->page * c->entries > kMostUsed) return LAST_ERR_SHAPE;
    if ((uintptr_t)c->k % 16 != 0 || (uintptr_t)c->v % 16 != 0) return LAST_ERR_SHAPE;
    return LAST_OK;
}

Turn turn_of(const last_rotation_t* r)
{
    if (!r || r->columns == 0) return Turn{nullptr, nullptr, 0};
    return Turn{r->frequencies, r->first, r->columns};
}

Pages pages_of(const last_cache_t* c)
{
    return Pages{c->table, c->used, c->pages, c->page, c->entries, divisor_of((unsigned)c->page)};
}

// In frames that are there, no limit is one of T.
Band band_of(const last_band_t* b, int T)
{
    const auto within = [&](int n) { return n < 0 || n > T ? T : n; };
    return Band{within(b->left), within(b->right), b->sinks, b->scale};
}

HeadSide side_of(const last_matrix_t* x, const last_matrix_t* y, const float* gain, int heads)
{
    HeadSide s{};
    s.x = x->data;
    s.px = x->pitch;
    if (y) { s.y = y->data; s.py = y->pitch; }
    s.gain = gain;
    s.heads = heads;
    return s;
}

template <typename E, int LN>
void launch_heads(const HeadArgs& a, hipStream_t st)
{
    int groups = 0;
    for (const HeadSide& side : a.side) groups += (side.heads + kWave / LN - 1) / (kWave / LN);
    // A wavefront takes all heads of a frame, whose angles it forms once, but where that leaves compute units without work.
    const int split = (int)std::max(1ll, std::min<long long>(groups, 4096 / a.rows));
    const dim3 grid((unsigned)std::min<long long>(((long long)a.rows + 3) / 4, 2048), (unsigned)split);
    if (a.cache.table) hipLaunchKernelGGL((heads_kernel<E, LN, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((heads_kernel<E, LN, false>), grid, dim3(256), 0, st, a);
}

template <typename E>
void launch_heads(const HeadArgs& a, hipStream_t st)
{
    const int lanes = a.D / 8;
    if (lanes > 8) launch_heads<E, 16>(a, st);
    else if (lanes > 4) launch_heads<E, 8>(a, st);
    else if (lanes > 2) launch_heads<E, 4>(a, st);
    else if (lanes > 1) launch_heads<E, 2>(a, st);
    else launch_heads<E, 1>(a, st);
}

void launch_heads_of(int type, const HeadArgs& a, hipStream_t st)
{
    if (type == LAST_F32) launch_heads<float>(a, st);
    else if (type == LAST_BF16) launch_heads<bf16_t>(a, st);
    else launch_heads<f16_t>(a, st);
}

// Workgroups of the gradient: each leaves a row of partial sums of the gains' gradients.
int head_grad_groups(long long rows) { return (int)std::min<long long>((rows + 3) / 4, 1024); }

template <typename E>
void launch_heads_grad(const HeadGradArgs& a, hipStream_t st)
{
    const dim3 grid((unsigned)head_grad_groups(a.rows)), block(256);
    const int lanes = a.D / 8;
    if (lanes > 8) hipLaunchKernelGGL((heads_grad_kernel<E, 16>), grid, block, 0, st, a);
    else if (lanes > 4) hipLaunchKernelGGL((heads_grad_kernel<E, 8>), grid, block, 0, st, a);
    else if (lanes > 2) hipLaunchKernelGGL((heads_grad_kernel<E, 4>), grid, block, 0, st, a);
    else if (lanes > 1) hipLaunchKernelGGL((heads_grad_kernel<E, 2>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((heads_grad_kernel<E, 1>), grid, block, 0, st, a);
}

// `count` workgroups of 256 threads in launches of as many as one takes
template <typename Launch>
void in_launches(long long count, Launch launch)
{
    constexpr long long kMost = kMaxThreads / 256;
    for (long long i = 0; i < count; i += kMost) launch(i, dim3((unsigned)std::min(count - i, kMost)));
}

int padded(int width) { return width <= 32 ? 32 : width <= 64 ? 64 : 128; }

#define LAST_BY_WIDTH(D, call)                                      \
    do {                                                            \
        if (padded(D) == 32) { constexpr int DP = 32; call; }       \
        else if (padded(D) == 64) { constexpr int DP = 64; call; }  \
        else { constexpr int DP = 128; call; }                      \
    } while (0)

// Heads that share keys go to one XCD together where that gives each as many.
unsigned heads_together(const AttentionArgs& a) { return a.B * a.kv_heads % 8 == 0 ? (unsigned)(a.heads / a.kv_heads) : 1u; }

// Two wavefronts for 32 frames where there are no more than two workgroups of 128 a compute unit: 1 x 4096, 16 heads of 128 on one (512 workgroups)
// 133 -> 111 us, 1 x 2048, 8 of 64 36 -> 29; of 1024 workgroups 16 x 1000, 8 of 64 48 -> 53, 1 x 8192, 16 of 128 109 -> 130.
bool in_halves(const AttentionArgs& a) { return (long long)((a.T + kOwn - 1) / kOwn) * a.heads * a.B <= 512; }

template <typename E>
void launch_attention(AttentionArgs a, hipStream_t st)
{
    const bool halves = in_halves(a);
    const int frames = halves ? kOwn / 2 : kOwn;
    a.tiles = (unsigned)((a.T + frames - 1) / frames);
    a.together = heads_together(a);
    in_launches((long long)a.tiles * a.heads * a.B, [&](long long first, dim3 grid) {
        a.first = (unsigned)first;
        if (halves) LAST_BY_WIDTH(a.D, hipLaunchKernelGGL((attention_kernel<E, DP, true>), grid, dim3(256), 0, st, a));
        else LAST_BY_WIDTH(a.D, hipLaunchKernelGGL((attention_kernel<E, DP, false>), grid, dim3(256), 0, st, a));
    });
}

// Chunks of the frames that see first ones from beyond the window: of 256 frames where that makes no more than 64 a head.
int sink_chunks(const Band& band, int T)
{
    if (band.sinks == 0 || band.left + 1 >= T) return 0;
    return std::max(1, std::min(64, (T - band.left - 1 + 255) / 256));
}

struct GradPlan {
    int chunks, shares, parts;
    float *delta, *part, *sums, *kept;
};

long long key_groups(int B, int T, int kv_heads, int width)
{
    return (long long)B * kv_heads * ((T + kOwn - 1) / kOwn) * (padded(width) == 128 ? 2 : 1);
}

// Two wavefronts for 32 keys where there is no more than one workgroup of 128 a compute unit: 1 x 2048, 8 heads of 64 on one 71 -> 60 us, 1 x 700, 8 of
// 64 31 -> 27; of 512 workgroups 2 x 4096, 16 of 128 on four 571 -> 599.
bool keys_in_halves(long long groups) { return groups <= 256; }

// Heads that share keys go in parts where there are fewer than 1024 workgroups, two rounds of what fits: before halves 1 x 4096, 16 heads of 128 on one 411
// us (503 with 512 workgroups, 2522 in one part), 2 x 4096, 16 on four 567 (582 in one part).
int grad_parts(const last_frames_t* f, const last_heads_t* h)
{
    long long groups = key_groups(f->B, f->T, h->kv_heads, h->width);
    if (keys_in_halves(groups)) groups *= 2;
    return (int)std::max(1ll, std::min<long long>(h->heads / h->kv_heads, 1024 / std::max(1ll, groups)));
}

GradPlan plan_grad(Carver& cv, long long rows, const last_frames_t* f, const last_heads_t* h, const Band& band)
{
    GradPlan p{};
    p.chunks = sink_chunks(band, f->T);
    p.shares = h->heads / h->kv_heads * p.chunks * 2;
    p.delta = (float*)cv.take(sizeof(float) * (size_t)rows * h->heads);
    if (p.chunks) {
        const size_t row = sizeof(float) * 2 * kMostSinks * padded(h->width), units = (size_t)f->B * h->kv_heads;
        p.part = (float*)cv.take(row * units * p.shares);
        p.sums = (float*)cv.take(row * units);
    }
    p.parts = grad_parts(f, h);
    if (p.parts > 1) p.kept = (float*)cv.take(sizeof(float) * 2 * p.parts * (size_t)rows * h->kv_heads * padded(h->width));
    return p;
}

template <typename E>
void launch_attention_grad(AttentionArgs a, int chunks, hipStream_t st)
{
    const bool halves = in_halves(a);
    const int frames = halves ? kOwn / 2 : kOwn;
    a.tiles = (unsigned)((a.T + frames - 1) / frames);
    a.together = heads_together(a);
    in_launches((long long)a.tiles * a.heads * a.B, [&](long long first, dim3 grid) {
        a.first = (unsigned)first;
        if (halves) LAST_BY_WIDTH(a.D, hipLaunchKernelGGL((grad_query_kernel<E, DP, true>), grid, dim3(256), 0, st, a));
        else LAST_BY_WIDTH(a.D, hipLaunchKernelGGL((grad_query_kernel<E, DP, false>), grid, dim3(256), 0, st, a));
    });
    a.together = 1;
    if (chunks) {
        a.tiles = (unsigned)chunks;
        in_launches((long long)a.tiles * a.heads * a.B, [&](long long first, dim3 grid) {
            a.first = (unsigned)first;
            LAST_BY_WIDTH(a.D, hipLaunchKernelGGL((grad_first_kernel<E, DP>), grid, dim3(256), 0, st, a));
        });
        in_launches((long long)a.B * a.kv_heads * 2 * a.band.sinks, [&](long long first, dim3 grid) {
            hipLaunchKernelGGL(first_join_kernel, grid, dim3(128), 0, st, (const float*)a.part, a.sums, a.shares, padded(a.D), a.band.sinks, first);
        });
    }
    const bool keys_halved = keys_in_halves(key_groups(a.B, a.T, a.kv_heads, a.D));
    const int keys = keys_halved ? kOwn / 2 : kOwn;
    a.tiles = (unsigned)((a.T + keys - 1) / keys);
    a.half = a.tiles * (unsigned)(a.kv_heads * a.parts * a.B);
    in_launches((long long)a.half * (padded(a.D) == 128 ? 2 : 1), [&](long long first, dim3 grid) {
        a.first = (unsigned)first;
        if (keys_halved) LAST_BY_WIDTH(a.D, hipLaunchKernelGGL((grad_key_kernel<E, DP, DP == 128, true>), grid, dim3(256), 0, st, a));
        else LAST_BY_WIDTH(a.D, hipLaunchKernelGGL((grad_key_kernel<E, DP, DP == 128, false>), grid, dim3(256), 0, st, a));
    });
    if (a.parts > 1) {
        in_launches((2ll * a.B * a.T * a.kv_heads * (padded(a.D) / 4) + 255) / 256, [&](long long first, dim3 grid) {
            hipLaunchKernelGGL((grad_join_kernel<E>), grid, dim3(256), 0, st, a, padded(a.D), first);
        });
    }
}

// Blocks of 32 rows, and over how many workgroups a block's frames are split: so that there are some 1024, each with at least 256 frames of the window, or of
// what the table has room for where there is none (how many there are is known on the device alone; a split without frames ends at once).
struct CachedPlan {
    int row_blocks, splits;
    float *part, *part_ml;
};

CachedPlan plan_cached(Carver& cv, long long rows, const last_frames_t* f, const last_heads_t* h, const last_band_t* band, const last_cache_t* c)
{
    CachedPlan p;
    const long long block_rows = (long long)f->T * (h->heads / h->kv_heads);
    p.row_blocks = (int)((block_rows + 31) / 32);
    const long long groups = (long long)f->B * h->kv_heads * p.row_blocks;
    long long seen = (long long)c->page * c->entries;
    if (band->left >= 0) seen = std::min(seen, (long long)band->left + band->sinks + 33);
    p.splits = (int)std::max(1ll, std::min({1024ll / std::max(1ll, groups), seen / 256, (long long)kMostSplits}));
    p.part = p.part_ml = nullptr;
    if (p.splits > 1) {
        p.part = (float*)cv.take(sizeof(float) * (size_t)rows * h->heads * p.splits * h->width);
        p.part_ml = (float*)cv.take(sizeof(float) * (size_t)rows * h->heads * p.splits * 2);
    }
    return p;
}

template <typename E>
void launch_cached(CachedArgs a, hipStream_t st)
{
    in_launches((long long)a.splits * a.row_blocks * a.kv_heads * a.B, [&](long long first, dim3 grid) {
        a.first = (unsigned)first;
        LAST_BY_WIDTH(a.D, hipLaunchKernelGGL((cached_kernel<E, DP>), grid, dim3(256), 0, st, a));
    });
    if (a.splits == 1) return;
    in_launches((long long)a.B * a.T * a.heads, [&](long long first, dim3 grid) {
        hipLaunchKernelGGL((cached_join_kernel<E>), grid, dim3(256), 0, st, a, first);
    });
}

}  // namespace

extern "C" {

size_t last_attention_workspace_bytes(int32_t op, const last_frames_t* frames, const last_heads_t* heads, const last_band_t* band,
                                      const last_cache_t* cache)
{
    long long rows;
    if (check_items(frames, heads, op != LAST_OP_HEAD_NORM_GRAD, &rows) != LAST_OK) return 0;
    Carver cv(nullptr);
    if (op == LAST_OP_HEAD_NORM_GRAD) {
        cv.take(sizeof(float) * 2 * (size_t)head_grad_groups(rows) * heads->width);
    } else if (op == LAST_OP_ATTENTION_GRAD) {
        if (check_band(band) != LAST_OK) return 0;
        plan_grad(cv, rows, frames, heads, band_of(band, frames->T));
    } else if (op == LAST_OP_CACHED_ATTENTION) {
        if (check_band(band) != LAST_OK || check_cache(cache) != LAST_OK) return 0;
        plan_cached(cv, rows, frames, heads, band, cache);
    } else {
        return 0;
    }
    return std::max(kAlign, cv.used);
}

last_status_t last_head_norm(const last_frames_t* frames, const last_heads_t* heads, const last_matrix_t* q, const last_matrix_t* k,
                             const float* gain_q, const float* gain_k, float eps, const last_rotation_t* rotation,
                             const last_matrix_t* yq, const last_matrix_t* yk, void* hip_stream)
{
    long long rows;
    LAST_TRY(check_items(frames, heads, false, &rows));
    if ((!q && !k) || (q && !yq) || (k && !yk)) return LAST_ERR_NULL;
    if (!(eps >= 0.f)) return LAST_ERR_SHAPE;
    LAST_TRY(check_rotation(rotation, heads->width));
    const int type = q ? q->type : k->type;
    HeadArgs a{};
    if (q) {
        LAST_TRY(check_matrix(q, (long long)heads->heads * heads->width, plain(type)));
        LAST_TRY(check_matrix(yq, (long long)heads->heads * heads->width, yq->type == type));
        a.side[0] = side_of(q, yq, gain_q, heads->heads);
    }
    if (k) {
        LAST_TRY(check_matrix(k, (long long)heads->kv_heads * heads->width, plain(type) && k->type == type));
        LAST_TRY(check_matrix(yk, (long long)heads->kv_heads * heads->width, yk->type == type));
        a.side[1] = side_of(k, yk, gain_k, heads->kv_heads);
    }
    if (rows == 0) return LAST_OK;
    a.frames = frames_of(frames);
    a.rows = (int)rows;
    a.B = frames->B;
    a.D = heads->width;
    a.eps = eps;
    a.turn = turn_of(rotation);
    launch_heads_of(type, a, (hipStream_t)hip_stream);
    return hip_done();
}

last_status_t last_head_norm_grad(const last_frames_t* frames, const last_heads_t* heads, const last_matrix_t* dyq, const last_matrix_t* dyk,
                                  const last_matrix_t* q, const last_matrix_t* k, const float* gain_q, const float* gain_k, float eps,
                                  const last_rotation_t* rotation, const last_matrix_t* dq, const last_matrix_t* dk, float* dgain_q,
                                  float* dgain_k, void* ws, size_t ws_bytes, void* hip_stream)
{
    long long rows;
    LAST_TRY(check_items(frames, heads, false, &rows));
    if ((!dyq && !dyk) || (dyq && (!dq || !q)) || (dyk && (!dk || !k))) return LAST_ERR_NULL;
    if ((dgain_q && (!gain_q || !dyq)) || (dgain_k && (!gain_k || !dyk))) return LAST_ERR_NULL;
    if (!(eps >= 0.f)) return LAST_ERR_SHAPE;
    LAST_TRY(check_rotation(rotation, heads->width));
    const int type = dyq ? dyq->type : dyk->type;
    HeadGradArgs a{};
    const last_matrix_t *dys[2] = {dyq, dyk}, *xs[2] = {q, k}, *dxs[2] = {dq, dk};
    const float* gains[2] = {gain_q, gain_k};
    for (int i = 0; i < 2; ++i) {
        if (!dys[i]) continue;
        const int n = i == 0 ? heads->heads : heads->kv_heads;
        const long long columns = (long long)n * heads->width;
        LAST_TRY(check_matrix(dys[i], columns, plain(type) && dys[i]->type == type));
        LAST_TRY(check_matrix(xs[i], columns, xs[i]->type == type));
        LAST_TRY(check_matrix(dxs[i], columns, dxs[i]->type == type));
        a.side[i] = HeadGradSide{dys[i]->data, xs[i]->data, dys[i]->pitch, xs[i]->pitch, dxs[i]->pitch, dxs[i]->data, gains[i], n};
    }
    const bool gain = dgain_q || dgain_k;
    if (rows == 0 && !gain) return LAST_OK;
    if (gain) LAST_TRY(check_ws(ws, ws_bytes, last_attention_workspace_bytes(LAST_OP_HEAD_NORM_GRAD, frames, heads, nullptr, nullptr)));
    a.frames = frames_of(frames);
    a.rows = (int)rows;
    a.D = heads->width;
    a.eps = eps;
    a.turn = turn_of(rotation);
    a.part = gain ? (float*)ws : nullptr;
    hipStream_t st = (hipStream_t)hip_stream;
    if (rows > 0) {
        if (type == LAST_F32) launch_heads_grad<float>(a, st);
        else if (type == LAST_BF16) launch_heads_grad<bf16_t>(a, st);
        else launch_heads_grad<f16_t>(a, st);
    }
    if (gain)
        hipLaunchKernelGGL(heads_gain_kernel, dim3((unsigned)((2 * a.D + 15) / 16)), dim3(1024), 0, st, (const float*)a.part,
                           head_grad_groups(rows), a.D, dgain_q, dgain_k);
    return hip_done();
}

last_status_t last_attention(const last_frames_t* frames, const last_heads_t* heads, const last_band_t* band, const last_matrix_t* q,
                             const last_matrix_t* k, const last_matrix_t* v, const last_matrix_t* y, float* lse, void* hip_stream)
{
    long long rows;
    LAST_TRY(check_items(frames, heads, true, &rows));
    if (!q || !k || !v || !y) return LAST_ERR_NULL;
    LAST_TRY(check_band(band));
    const long long cq = (long long)heads->heads * heads->width, ck = (long long)heads->kv_heads * heads->width;
    LAST_TRY(check_matrix(q, cq, half_width(q->type)));
    LAST_TRY(check_matrix(k, ck, k->type == q->type));
    LAST_TRY(check_matrix(v, ck, v->type == q->type));
    LAST_TRY(check_matrix(y, cq, y->type == q->type));
    if (rows == 0) return LAST_OK;
    AttentionArgs a{};
    a.len = frames->lengths;
    a.T = frames->T;
    a.B = frames->B;
    a.heads = heads->heads;
    a.kv_heads = heads->kv_heads;
    a.D = heads->width;
    a.q = q->data;
    a.k = k->data;
    a.v = v->data;
    a.y = y->data;
    a.pq = q->pitch;
    a.pk = k->pitch;
    a.pv = v->pitch;
    a.py = y->pitch;
    a.lse = lse;
    a.band = band_of(band, frames->T);
    hipStream_t st = (hipStream_t)hip_stream;
    if (q->type == LAST_BF16) launch_attention<bf16_t>(a, st);
    else launch_attention<f16_t>(a, st);
    return hip_done();
}

last_status_t last_attention_grad(const last_frames_t* frames, const last_heads_t* heads, const last_band_t* band, const last_matrix_t* dy,
                                  const last_matrix_t* q, const last_matrix_t* k, const last_matrix_t* v, const last_matrix_t* y,
                                  const float* lse, const last_matrix_t* dq, const last_matrix_t* dk, const last_matrix_t* dv, void* ws,
                                  size_t ws_bytes, void* hip_stream)
{
    long long rows;
    LAST_TRY(check_items(frames, heads, true, &rows));
    if (!dy || !q || !k || !v || !y || !lse || !dq || !dk || !dv) return LAST_ERR_NULL;
    LAST_TRY(check_band(band));
    const long long cq = (long long)heads->heads * heads->width, ck = (long long)heads->kv_heads * heads->width;
    const int type = q->type;
    const last_matrix_t *wide[4] = {dy, q, y, dq}, *narrow[4] = {k, v, dk, dv};
    for (const last_matrix_t* m : wide) LAST_TRY(check_matrix(m, cq, half_width(type) && m->type == type));
    for (const last_matrix_t* m : narrow) LAST_TRY(check_matrix(m, ck, m->type == type));
    LAST_TRY(check_ws(ws, ws_bytes, last_attention_workspace_bytes(LAST_OP_ATTENTION_GRAD, frames, heads, band, nullptr)));
    if (rows == 0) return LAST_OK;
    AttentionArgs a{};
    a.len = frames->lengths;
    a.T = frames->T;
    a.B = frames->B;
    a.heads = heads->heads;
    a.kv_heads = heads->kv_heads;
    a.D = heads->width;
    a.q = q->data;
    a.k = k->data;
    a.v = v->data;
    a.dy = dy->data;
    a.y = y->data;
    a.dq = dq->data;
    a.dk = dk->data;
    a.dv = dv->data;
    a.pq = q->pitch;
    a.pk = k->pitch;
    a.pv = v->pitch;
    a.pdy = dy->pitch;
    a.py = y->pitch;
    a.pdq = dq->pitch;
    a.pdk = dk->pitch;
    a.pdv = dv->pitch;
    a.lse = (float*)lse;
    a.band = band_of(band, frames->T);
    Carver cv(ws, ws_bytes);
    const GradPlan plan = plan_grad(cv, rows, frames, heads, a.band);
    a.delta = plan.delta;
    a.part = plan.part;
    a.sums = plan.sums;
    a.shares = plan.shares;
    a.parts = plan.parts;
    a.kept = plan.kept;
    hipStream_t st = (hipStream_t)hip_stream;
    if (type == LAST_BF16) launch_attention_grad<bf16_t>(a, plan.chunks, st);
    else launch_attention_grad<f16_t>(a, plan.chunks, st);
    return hip_done();
}

last_status_t last_cache_append(const last_frames_t* frames, const last_heads_t* heads, const last_matrix_t* q, const last_matrix_t* k,
                                const last_matrix_t* v, const float* gain_q, const float* gain_k, float eps, const last_rotation_t* rotation,
                                const last_cache_t* cache, const last_matrix_t* yq, int32_t* item_status, void* hip_stream)
{
    long long rows;
    LAST_TRY(check_items(frames, heads, false, &rows));
    if (!k || !v || (q && !yq)) return LAST_ERR_NULL;
    if (!(eps >= 0.f)) return LAST_ERR_SHAPE;
    LAST_TRY(check_rotation(rotation, heads->width));
    LAST_TRY(check_cache(cache));
    const long long cq = (long long)heads->heads * heads->width, ck = (long long)heads->kv_heads * heads->width;
    const int type = cache->type;
    HeadArgs a{};
    LAST_TRY(check_matrix(k, ck, half_width(type) && k->type == type));
    LAST_TRY(check_matrix(v, ck, v->type == type));
    if (q) {
        LAST_TRY(check_matrix(q, cq, q->type == type));
        LAST_TRY(check_matrix(yq, cq, yq->type == type));
        a.side[0] = side_of(q, yq, gain_q, heads->heads);
    }
    a.side[1] = side_of(k, nullptr, gain_k, heads->kv_heads);
    a.side[1].pages = (char*)cache->k;
    a.side[2] = side_of(v, nullptr, nullptr, heads->kv_heads);
    a.side[2].pages = (char*)cache->v;
    a.frames = frames_of(frames);
    a.rows = (int)rows;
    a.B = frames->B;
    a.D = heads->width;
    a.eps = eps;
    a.turn = turn_of(rotation);
    a.turn.first = nullptr;
    a.cache = pages_of(cache);
    a.status = item_status;
    hipStream_t st = (hipStream_t)hip_stream;
    if (rows == 0 && !item_status) return LAST_OK;
    if (rows > 0) launch_heads_of(type, a, st);
    else hipLaunchKernelGGL(no_frames_kernel, dim3((unsigned)((frames->B + 255) / 256)), dim3(256), 0, st, item_status, frames->B);
    return hip_done();
}

last_status_t last_cached_attention(const last_frames_t* frames, const last_heads_t* heads, const last_band_t* band, const last_matrix_t* q,
                                    const last_cache_t* cache, const last_matrix_t* y, int32_t* item_status, void* ws, size_t ws_bytes,
                                    void* hip_stream)
{
    long long rows;
    LAST_TRY(check_items(frames, heads, true, &rows));
    if (!q || !y) return LAST_ERR_NULL;
    LAST_TRY(check_band(band));
    LAST_TRY(check_cache(cache));
    const long long cq = (long long)heads->heads * heads->width;
    const int type = cache->type;
    LAST_TRY(check_matrix(q, cq, half_width(type) && q->type == type));
    LAST_TRY(check_matrix(y, cq, y->type == type));
    LAST_TRY(check_ws(ws, ws_bytes, last_attention_workspace_bytes(LAST_OP_CACHED_ATTENTION, frames, heads, band, cache)));
    Carver cv(ws, ws_bytes);
    const CachedPlan plan = plan_cached(cv, rows, frames, heads, band, cache);
    CachedArgs a{};
    a.len = frames->lengths;
    a.T = frames->T;
    a.B = frames->B;
    a.heads = heads->heads;
    a.kv_heads = heads->kv_heads;
    a.D = heads->width;
    a.q = q->data;
    a.y = y->data;
    a.pq = q->pitch;
    a.py = y->pitch;
    a.k = (const char*)cache->k;
    a.v = (const char*)cache->v;
    a.cache = pages_of(cache);
    // (past the new frames nothing is there to see)
    a.band = Band{band->left < 0 ? INT_MAX : band->left, band_of(band, frames->T).right, band->sinks, band->scale};
    a.status = item_status;
    a.part = plan.part;
    a.part_ml = plan.part_ml;
    a.splits = plan.splits;
    a.row_blocks = plan.row_blocks;
    hipStream_t st = (hipStream_t)hip_stream;
    if (rows == 0 && !item_status) return LAST_OK;
    if (rows == 0) {
        hipLaunchKernelGGL(no_frames_kernel, dim3((unsigned)((frames->B + 255) / 256)), dim3(256), 0, st, item_status, frames->B);
    } else if (type == LAST_BF16) {
        launch_cached<bf16_t>(a, st);
    } else {
        launch_cached<f16_t>(a, st);
    }
    return hip_done();
}

}  // extern "C"
