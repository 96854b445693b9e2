// C ABI of the layer between an encoder's frames and the lattice (see include/last.h): argument validation, choice of the
// kernels, workspace planning and launches.  No allocation, no synchronisation.
#include "../../include/last.h"

#include <hip/hip_runtime.h>

#include "layer.hpp"
#include "norm_kernels.hpp"
#include "keep_kernels.hpp"
#include "product_kernels.hpp"
#include <algorithm>
#include <type_traits>

using namespace last;

namespace last {
void note_hip_error(hipError_t e);
int option(int o);
}

namespace {

constexpr long long kMaxRows = 1ll << 30;
constexpr long long kMaxColumns = 1ll << 20;
constexpr long long kMaxPitchBytes = 4ll << 20;      // 256 rows of a tile stay within 32-bit offsets
constexpr int kMaxNormColumns = 16384;
constexpr long long kFewRows = 32;
constexpr size_t kAlign = 256;
constexpr long long kMaxThreads = 1ll << 31;         // of a launch, which takes fewer than 2^32: what has more to do goes out in pieces

size_t align_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }

last_status_t hip_done()
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return LAST_OK;
    note_hip_error(e);
    return LAST_ERR_HIP;
}

bool plain(int t) { return t == LAST_F32 || t == LAST_BF16 || t == LAST_F16; }
bool half_width(int t) { return t == LAST_BF16 || t == LAST_F16; }
bool eight(int t) { return t == LAST_I8 || t == LAST_E4M3; }
int size_of(int t) { return t == LAST_F32 ? 4 : half_width(t) ? 2 : 1; }

last_status_t check_frames(const last_frames_t* f, long long* rows)
{
    if (!f) return LAST_ERR_NULL;
    if (f->B < 1 || f->T < 0 || (long long)f->B * f->T > kMaxRows) return LAST_ERR_SHAPE;
    *rows = (long long)f->B * f->T;
    return LAST_OK;
}

last_status_t check_matrix(const last_matrix_t* m, long long columns, bool types)
{
    if (!m || !m->data) return LAST_ERR_NULL;
    if (!types) return LAST_ERR_UNSUPPORTED;
    if (m->pitch < columns || m->pitch > kMaxPitchBytes / size_of(m->type)) return LAST_ERR_SHAPE;
    if ((uintptr_t)m->data % size_of(m->type) != 0) return LAST_ERR_SHAPE;
    if (eight(m->type)) {
        if (!m->scales) return LAST_ERR_NULL;
        if (m->scale_pitch < (columns + kBlock - 1) / kBlock || m->scale_pitch > kMaxPitchBytes) return LAST_ERR_SHAPE;
    }
    return LAST_OK;
}

#define LAST_TRY(call)                                  \
    do {                                                \
        const last_status_t rc_ = (call);               \
        if (rc_ != LAST_OK) return rc_;                 \
    } while (0)

Frames frames_of(const last_frames_t* f) { return Frames{f->lengths, f->T, divisor_of((unsigned)f->T)}; }

Eight eight_of(const last_matrix_t* m)
{
    Eight e{};
    if (!m) return e;
    e.q = (uint8_t*)m->data;
    e.scales = m->scales;
    e.pitch = m->pitch;
    e.scale_pitch = m->scale_pitch;
    e.e4m3 = m->type == LAST_E4M3;
    return e;
}

bool bad_activation(int act) { return act < LAST_ACT_NONE || act > LAST_ACT_TANH; }

// ---------------------------------------------------------------- norm

template <typename X, bool KEEP>
void launch_norm(NormArgs a, hipStream_t st)
{
    const int rows = a.rows, most = (int)(kMaxThreads / (a.H <= 2048 ? 64 : a.H <= 8192 ? 256 : 1024));
    for (int row0 = 0; row0 < rows; row0 = a.rows) {
        a.row0 = row0;
        a.rows = rows - row0 < most ? rows : row0 + most;
        const dim3 each(a.rows - row0), four((a.rows - row0 + 3) / 4);
        if (a.H <= 512) hipLaunchKernelGGL((norm_kernel<X, 1, 1, KEEP>), four, dim3(256), 0, st, a);
        else if (a.H <= 1024) hipLaunchKernelGGL((norm_kernel<X, 1, 2, KEEP>), four, dim3(256), 0, st, a);
        else if (a.H <= 2048) hipLaunchKernelGGL((norm_kernel<X, 1, 4, KEEP>), four, dim3(256), 0, st, a);
        else if (a.H <= 4096) hipLaunchKernelGGL((norm_kernel<X, 4, 2, KEEP>), each, dim3(256), 0, st, a);
        else if (a.H <= 8192) hipLaunchKernelGGL((norm_kernel<X, 4, 4, KEEP>), each, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((norm_kernel<X, 16, 2, KEEP>), each, dim3(1024), 0, st, a);
    }
}

template <typename X>
void launch_norm(const NormArgs& a, hipStream_t st)
{
    if (a.kept.q) launch_norm<X, true>(a, st);
    else launch_norm<X, false>(a, st);
}

// Workgroups of the gradient: as many as are resident, since each leaves a row of partial sums of dgain.
int norm_grad_groups(long long rows, int H)
{
    if (H <= 1024) return (int)std::min<long long>((rows + 3) / 4, 1024);
    return (int)std::min<long long>(rows, H <= 4096 ? 1024 : 512);
}

template <typename DY, typename S, bool DS>
void launch_norm_grad(const NormGradArgs& a, int groups, hipStream_t st)
{
    if (a.H <= 512) hipLaunchKernelGGL((norm_grad_kernel<DY, S, 1, 1, DS>), dim3(groups), dim3(256), 0, st, a);
    else if (a.H <= 1024) hipLaunchKernelGGL((norm_grad_kernel<DY, S, 1, 2, DS>), dim3(groups), dim3(256), 0, st, a);
    else if (a.H <= 2048) hipLaunchKernelGGL((norm_grad_kernel<DY, S, 4, 1, DS>), dim3(groups), dim3(256), 0, st, a);
    else if (a.H <= 4096) hipLaunchKernelGGL((norm_grad_kernel<DY, S, 4, 2, DS>), dim3(groups), dim3(256), 0, st, a);
    else if (a.H <= 8192) hipLaunchKernelGGL((norm_grad_kernel<DY, S, 16, 1, DS>), dim3(groups), dim3(1024), 0, st, a);
    else hipLaunchKernelGGL((norm_grad_kernel<DY, S, 16, 2, DS>), dim3(groups), dim3(1024), 0, st, a);
}

template <typename DY, typename S>
void launch_norm_grad(const NormGradArgs& a, int groups, hipStream_t st)
{
    if (a.ds) launch_norm_grad<DY, S, true>(a, groups, st);
    else launch_norm_grad<DY, S, false>(a, groups, st);
}

// dy and s of one plain type, dy in 32 bits beside s in 16, or s in 8 bits
bool norm_grad_types(int dy, int s)
{
    return plain(dy) && (dy == s || eight(s) || (dy == LAST_F32 && half_width(s)));
}

template <typename DY>
void launch_norm_grad_on(int s, const NormGradArgs& a, int groups, hipStream_t st)
{
    if (s == LAST_I8) return launch_norm_grad<DY, i8_t>(a, groups, st);
    if (s == LAST_E4M3) return launch_norm_grad<DY, e4m3_t>(a, groups, st);
    if (s == Elt<DY>::type) return launch_norm_grad<DY, DY>(a, groups, st);
    if constexpr (Elt<DY>::type == LAST_F32) {
        if (s == LAST_BF16) return launch_norm_grad<DY, bf16_t>(a, groups, st);
        launch_norm_grad<DY, f16_t>(a, groups, st);
    }
}

// ---------------------------------------------------------------- 8 bits

// rows of the element-wise calls in launches of at most 2^29 places
template <typename Launch>
last_status_t in_pieces(KeepArgs a, long long rows, Launch launch)
{
    a.groups = (a.H + kBlock - 1) / kBlock * 4;
    a.by_groups = divisor_of((unsigned)a.groups);
    const long long most = std::max(1ll, (1ll << 29) / a.groups);
    for (long long r = 0; r < rows; r += most) {
        a.row0 = (int)r;
        a.rows = (int)std::min(most, rows - r);
        launch(a, dim3((unsigned)(((long long)a.rows * a.groups + 256 * kKeepDeep - 1) / (256 * kKeepDeep))));
    }
    return hip_done();
}

KeepArgs kept_values_args(const last_frames_t* f, int H, const last_matrix_t* kept, int act, const last_matrix_t* y)
{
    KeepArgs a{};
    a.frames = frames_of(f);
    a.H = H;
    a.y = y->data;
    a.py = y->pitch;
    a.act = act;
    a.ytype = y->type;
    a.kept = eight_of(kept);
    return a;
}

// ---------------------------------------------------------------- products

struct ProductPlan {
    int variant;                     // 0: few rows, 1: tiles of 64, 2: of 128, 3: of 256; -1: more results than a launch takes
    int splits;
    long long share;                 // of the reduction, in bytes (kAlong) or rows
};

// Tiles and shares of a reduction of `steps` steps (128 bytes, or 64 rows).  Up to 32 rows of a forward product go to the
// kernel that reads w once and keeps nothing in LDS: 16, 32, 48, 64 rows of 2048 results over 512 terms in bfloat16 take it 4.5, 5.5, 7.1, 7.5 us,
// of 512 over 2048 6.4, 8.4, 10.9, 12.2, of 1024 over 4096 10.2, 13.8, 19.0, 21.1; tiles of 64 6.5, 10.8 and 11 to 12, whatever the rows (8-bit
// operands: 4.0 to 5.9, 6.0 to 11.1, 8.5 to 16.8; 5.7, 9.0, 9.3).  Beyond, the cheapest of what these would take, from measurements on
// MI355X: a workgroup with a compute unit to itself takes 1.2, 0.5 and 0.2 us a step with tiles of 256, 128 and 64 (the first 1.5 on a
// full chip), two that share one 0.95 and 0.4 us (tiles of 128 and 64), three 0.55 (of 64), and 9, 5 and 3.5 us beside its steps;
// operands that run across the reduction (none, one, both) take up to 1.8 times as long (transposing reads), less where others fill the
// time.  Tiles of 256 win from a full chip on (16384 x 1024 on 4096: 105 us, with tiles of 128 129), tiles of 64 up to about half a million
// results (512 x 1024 on 4096: 20 us, 37 and 80).  Shares are written and read in 32 bits at about 5 TB/s and cost a launch:
// 16384 x 1024 x 4096 rows of weight gradient in 4 shares 152 us, in one 350 us.  Measured with operands of 16 bits and without an activation;
// of 180 products of drawn sizes, 8-bit operands among them, the tiles it names were 1 % slower than the best of the three in
// the mean, 26 % at worst, and of 20 with activations, residuals and kept sums 1 %, 7 %.
ProductPlan plan_product(bool forward, int across, long long P, long long Q, long long steps, int largest = 3)
{
    ProductPlan best{0, 1, steps};
    const int asked = std::min(option(LAST_OPT_PRODUCT_TILES), largest);
    if (forward && P <= kFewRows && !asked) return best;
    best.variant = -1;
    static const double alone[4] = {0, 0.2, 0.5, 1.2}, two[4] = {0, 0.4, 0.95, 0}, many[4] = {0, 0.55, 0.95, 1.5}, beside[4] = {0, 3.5, 5, 9};
    static const double alone_by[3][3] = {{0, 1, 1}, {0, 1.4, 1.15}, {0, 1.8, 1.5}};
    static const double many_by[3][4] = {{0, 1, 1, 1}, {0, 1.05, 1.05, 1}, {0, 1.1, 1.1, 1.15}};
    double least = 1e30;
    for (int variant = 1; variant <= largest; ++variant) {
        const long long tile = 32 << variant;
        const long long tiles = ((P + tile - 1) / tile) * ((Q + tile - 1) / tile);
        if (asked && variant != asked) continue;
        if (tiles * (variant == 3 ? 512 : 256) > kMaxThreads) continue;
        for (int splits = 1; splits <= 64; splits *= 2) {
            const long long part = std::max(1ll, (steps + splits - 1) / splits);
            if (splits > 1 && (part < 4 || (steps + part - 1) / part != splits)) continue;
            const long long blocks = tiles * splits, at_once = variant == 1 ? 768 : variant == 2 ? 512 : 256;
            double step, rounds = std::max(1.0, (double)blocks / at_once);
            if (variant == 3) {
                step = (alone[3] + (many[3] - alone[3]) * std::min(1.0, blocks / 256.0)) * many_by[across][3];
                rounds = (double)((blocks + 255) / 256);
            } else if (blocks <= 256) {
                step = alone[variant] * alone_by[across][variant];
            } else {
                step = (blocks <= 512 ? two : many)[variant] * many_by[across][variant];
            }
            double us = rounds * (part * step + beside[variant]);
            if (splits > 1) us += 4 + (double)splits * P * Q * 8 / 5e6;
            if (us < least) {
                least = us;
                best = ProductPlan{variant, splits, part};
            }
        }
    }
    return best;
}

template <typename E, int LP, int LQ>
void launch_tiles(ProductArgs a, const ProductPlan& p, hipStream_t st)
{
    const int tile = 32 << p.variant;
    a.tiles_p = (a.P + tile - 1) / tile;
    a.tiles_q = (a.Q + tile - 1) / tile;
    const dim3 grid((unsigned)(a.tiles_p * a.tiles_q), (unsigned)p.splits);
    const ProductArgs j = a;
    if (p.splits > 1) {                              // the epilogue comes with the joining
        Epilogue none{};
        none.part = a.e.part;
        none.part_bias = a.e.part_bias;
        a.e = none;
    }
    constexpr bool kEight = Elt<E>::size == 1;
    if constexpr (!std::is_same_v<E, wide_t>) {      // (no registers for widened fragments of 128 x 64 results a wavefront)
        if (p.variant == 3) hipLaunchKernelGGL((product_kernel<E, LP, LQ, 256, 256, 2, 4, kEight ? 2 : 3, 2>), grid, dim3(512), 0, st, a);
    }
    if (p.variant == 2) hipLaunchKernelGGL((product_kernel<E, LP, LQ, 128, 128, 2, 2, kEight ? 2 : 3, 2>), grid, dim3(256), 0, st, a);
    if (p.variant == 1) hipLaunchKernelGGL((product_kernel<E, LP, LQ, 64, 64, 2, 2, 3, 3>), grid, dim3(256), 0, st, a);
    if (p.splits > 1) {
        const long long waves = (long long)((a.P + 15) / 16) * ((a.Q + 31) / 32);
        hipLaunchKernelGGL(product_join_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, j, p.splits);
    }
}

template <typename E>
void launch_few(const ProductArgs& a, hipStream_t st)
{
    // values in 8 bits need the 32 columns of a block in one wavefront
    const bool two = a.e.kept.q || a.e.out.q || a.Q > 16 * 1024;
    const dim3 grid((unsigned)(two ? (a.Q + 31) / 32 : (a.Q + 15) / 16)), block(kFewWaves * kWave);
    if (two) {
        if (a.P <= 16) hipLaunchKernelGGL((few_kernel<E, 1, 2>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((few_kernel<E, 2, 2>), grid, block, 0, st, a);
    } else {
        if (a.P <= 16) hipLaunchKernelGGL((few_kernel<E, 1, 1>), grid, block, 0, st, a);
        else hipLaunchKernelGGL((few_kernel<E, 2, 1>), grid, block, 0, st, a);
    }
}

// 16-byte pieces of rows of `columns` elements can be loaded as they stand
bool direct(const last_matrix_t* m, long long columns)
{
    const long long es = size_of(m->type);
    return (uintptr_t)m->data % 16 == 0 && m->pitch * es % 16 == 0 && columns * es % 16 == 0;
}

// a row's scales of 128 columns are 4 aligned bytes
bool direct_scales(const last_matrix_t* m, long long columns)
{
    return columns % 128 == 0 && (uintptr_t)m->scales % 4 == 0 && m->scale_pitch % 4 == 0;
}

long long packed_pitch(long long columns, int type) { return (columns * size_of(type) + 15) / 16 * 16; }
long long packed_scale_pitch(long long columns) { return ((columns + 127) / 128 * 4 + 15) / 16 * 16; }

// Where an operand is read from: as it stands, or laid out in the workspace.
struct Operand {
    const char* data;
    long long pitch;                 // bytes
    const uint8_t* scales;
    long long scale_pitch;
};

struct Carver {
    char* base;
    size_t have, used = 0;
    explicit Carver(void* p, size_t n = 0) : base((char*)p), have(n) {}
    // a plan that went by another setting of an option than the size that was checked (set in between, by another thread)
    bool over() const { return base && used > have; }
    char* take(size_t bytes)
    {
        char* p = base ? base + used : nullptr;
        used += align_up(bytes);
        return p;
    }
};

// What has to be laid out before a product, collected and launched at once.
struct Preparation {
    PrepareArgs a{};
    int n = 0;
    unsigned mask_groups = 0;
    void rows(const void* in, long long pitch, long long bytes, char* out, long long out_pitch, long long count)
    {
        if (count == 0) return;
        auto& r = a.rows[n++];
        r = PrepareArgs::Rows{(const uint8_t*)in, (uint8_t*)out, pitch, out_pitch, count, (int)bytes,
                              (unsigned)((count * (out_pitch / 16) + 255) / 256)};
        a.groups += r.groups;
    }
    void values(const KeepArgs& k, dim3 grid)
    {
        a.values = k;
        a.values_groups = grid.x;
    }
    void mask(const last_frames_t* f, long long count, unsigned long long* out)
    {
        a.frames = frames_of(f);
        a.frame_rows = (int)count;
        a.mask = out;
        mask_groups = (unsigned)((count + 255) / 256);
    }
    void launch(hipStream_t st)
    {
        const unsigned n = a.groups + a.values_groups + mask_groups, most = (unsigned)(kMaxThreads / 256);
        for (a.first = 0; a.first < n; a.first += most)
            hipLaunchKernelGGL(prepare_kernel, dim3(std::min(most, n - a.first)), dim3(256), 0, st, a);
    }
};

// With a workspace that only measures (cv.base null) nothing is prepared.
Operand lay_out(Carver& cv, Preparation& pre, const last_matrix_t* m, long long rows, long long columns)
{
    const long long es = size_of(m->type);
    Operand o{(const char*)m->data, m->pitch * es, m->scales, m->scale_pitch};
    if (!direct(m, columns)) {
        o.pitch = packed_pitch(columns, m->type);
        char* at = cv.take((size_t)(rows * o.pitch));
        if (at) pre.rows(m->data, m->pitch * es, columns * es, at, o.pitch, rows);
        o.data = at;
    }
    if (eight(m->type) && !direct_scales(m, columns)) {
        o.scale_pitch = packed_scale_pitch(columns);
        char* at = cv.take((size_t)(rows * o.scale_pitch));
        if (at) pre.rows(m->scales, m->scale_pitch, (columns + kBlock - 1) / kBlock, at, o.scale_pitch, rows);
        o.scales = (const uint8_t*)at;
    }
    return o;
}

void set_plan(Carver& cv, ProductArgs& a, const ProductPlan& p, long long unit, float* dbias)
{
    a.share = p.share * unit;
    a.e.part = p.splits > 1 ? (float*)cv.take(sizeof(float) * (size_t)p.splits * a.P * a.Q) : nullptr;
    a.e.part_bias = nullptr;
    if (dbias) a.e.part_bias = p.splits > 1 ? (float*)cv.take(sizeof(float) * (size_t)p.splits * a.P) : dbias;
    a.e.sum_bias = dbias;
}

void set_result(Epilogue& e, const last_matrix_t* y, const last_matrix_t* res)
{
    if (eight(y->type)) {
        e.out = eight_of(y);
        e.type = res ? res->type : LAST_F32;
    } else {
        e.y = y->data;
        e.py = y->pitch;
        e.type = y->type;
    }
    if (res) {
        e.res = res->data;
        e.pres = res->pitch;
    }
}

// The call's plan, the same for measuring the workspace and for the call itself.  wide: 8-bit operands' products are added in 32 bits.
last_status_t run_product(Carver& cv, const last_frames_t* f, long long rows, int N, int K, const last_matrix_t* x, const last_matrix_t* w, bool wide,
                          const float* bias, int act, const last_matrix_t* res, const last_matrix_t* y, const last_matrix_t* kept, hipStream_t st)
{
    ProductArgs a{};
    const long long bytes = packed_pitch(K, x->type);
    Preparation pre;
    const Operand p = lay_out(cv, pre, x, rows, K), q = lay_out(cv, pre, w, N, K);
    a.p = p.data;
    a.q = q.data;
    a.pp = p.pitch;
    a.pq = q.pitch;
    a.sp = p.scales;
    a.sq = q.scales;
    a.psp = p.scale_pitch;
    a.psq = q.scale_pitch;
    a.P = (int)rows;
    a.Q = N;
    a.K = bytes;
    a.frames = frames_of(f);
    const ProductPlan plan = plan_product(true, 0, rows, N, (bytes + kStep - 1) / kStep, wide ? 2 : 3);
    if (plan.variant < 0) return LAST_ERR_SHAPE;
    set_plan(cv, a, plan, kStep, nullptr);
    if (cv.over()) return LAST_ERR_WORKSPACE;
    if (!cv.base || rows == 0) return LAST_OK;
    pre.launch(st);
    a.e.bias = bias;
    a.e.act = act;
    set_result(a.e, y, res);
    a.e.kept = eight_of(kept);
    if (plan.variant == 0) {
        if (x->type == LAST_BF16) launch_few<bf16_t>(a, st);
        else if (x->type == LAST_F16) launch_few<f16_t>(a, st);
        else if (wide) launch_few<wide_t>(a, st);
        else launch_few<e4m3_t>(a, st);
    } else {
        if (x->type == LAST_BF16) launch_tiles<bf16_t, kAlong, kAlong>(a, plan, st);
        else if (x->type == LAST_F16) launch_tiles<f16_t, kAlong, kAlong>(a, plan, st);
        else if (wide) launch_tiles<wide_t, kAlong, kAlong>(a, plan, st);
        else launch_tiles<e4m3_t, kAlong, kAlong>(a, plan, st);
    }
    return hip_done();
}

last_status_t run_grad_input(Carver& cv, const last_frames_t* f, long long rows, int N, int K, const last_matrix_t* dy, const last_matrix_t* w,
                             const last_matrix_t* kept, int act, const last_matrix_t* dx, hipStream_t st)
{
    ProductArgs a{};
    const long long bytes = packed_pitch(N, dy->type);
    Preparation pre;
    const Operand p = lay_out(cv, pre, dy, rows, N), q = lay_out(cv, pre, w, N, K);
    a.p = p.data;
    a.q = q.data;
    a.pp = p.pitch;
    a.pq = q.pitch;
    a.P = (int)rows;
    a.Q = K;
    a.K = bytes;
    a.q_rows = N;
    a.frames = frames_of(f);
    const ProductPlan plan = plan_product(false, 1, rows, K, (bytes + kStep - 1) / kStep);
    if (plan.variant < 0) return LAST_ERR_SHAPE;
    set_plan(cv, a, plan, kStep, nullptr);
    if (cv.over()) return LAST_ERR_WORKSPACE;
    if (!cv.base || rows == 0) return LAST_OK;
    pre.launch(st);
    set_result(a.e, dx, nullptr);
    a.e.kept_act = act;
    if (act != LAST_ACT_NONE) a.e.kept = eight_of(kept);
    if (dy->type == LAST_BF16) launch_tiles<bf16_t, kAlong, kAcross>(a, plan, st);
    else launch_tiles<f16_t, kAlong, kAcross>(a, plan, st);
    return hip_done();
}

last_status_t run_grad_weight(Carver& cv, const last_frames_t* f, long long rows, int N, int K, const last_matrix_t* dy, const last_matrix_t* x,
                              int act, const last_matrix_t* dw, float* dbias, hipStream_t st)
{
    ProductArgs a{};
    Preparation pre;
    const Operand p = lay_out(cv, pre, dy, rows, N);
    Operand q;
    if (eight(x->type)) {
        // the activation formed again, once, instead of by every tile that reads it; rounded to dy's type, as the product that it was the
        // input of had it: what dw is the gradient of, whatever the type of dw
        last_matrix_t v{};
        v.type = dy->type;
        v.pitch = packed_pitch(K, dy->type) / 2;
        v.data = cv.take((size_t)(rows * v.pitch * 2));
        if (cv.base && rows > 0) {
            // in the launch that prepares, but for what is left of rows that are more than one takes
            KeepArgs all = kept_values_args(f, K, x, act, &v);
            LAST_TRY(in_pieces(all, rows, [&](const KeepArgs& k, dim3 grid) {
                if (k.row0 == 0) pre.values(k, grid);
                else hipLaunchKernelGGL(kept_values_kernel, grid, dim3(256), 0, st, k);
            }));
        }
        q = Operand{(const char*)v.data, v.pitch * 2, nullptr, 0};
    } else {
        q = lay_out(cv, pre, x, rows, K);
    }
    a.p = p.data;
    a.q = q.data;
    a.pp = p.pitch;
    a.pq = q.pitch;
    a.P = N;
    a.Q = K;
    a.K = rows;
    const ProductPlan plan = plan_product(false, 2, N, K, (rows + 63) / 64);
    if (plan.variant < 0) return LAST_ERR_SHAPE;
    set_plan(cv, a, plan, 64, dbias);
    unsigned long long* mask = f->lengths ? (unsigned long long*)cv.take((size_t)((rows + 63) / 64 * 8)) : nullptr;
    if (cv.over()) return LAST_ERR_WORKSPACE;
    if (!cv.base) return LAST_OK;
    if (mask) pre.mask(f, rows, mask);
    pre.launch(st);
    a.mask = mask;
    set_result(a.e, dw, nullptr);
    if (dy->type == LAST_BF16) launch_tiles<bf16_t, kAcross, kAcross>(a, plan, st);
    else launch_tiles<f16_t, kAcross, kAcross>(a, plan, st);
    return hip_done();
}

// (the last: so that tiles are counted in 32 bits)
bool bad_sizes(long long rows, int N, int K)
{
    return N < 1 || K < 1 || N > kMaxColumns || K > kMaxColumns || rows * std::max(N, K) > 1ll << 42;
}

// need 0: sizes that no plan takes (the rest is checked by then)
last_status_t check_ws(void* ws, size_t have, size_t need)
{
    if (need == 0) return LAST_ERR_SHAPE;
    if (!ws || ((uintptr_t)ws % kAlign) != 0 || have < need) return LAST_ERR_WORKSPACE;
    return LAST_OK;
}

size_t part_bytes(long long rows, int H) { return sizeof(float) * (size_t)norm_grad_groups(rows, H) * H; }

}  // namespace

extern "C" {

size_t last_layer_workspace_bytes(int32_t op, const last_frames_t* frames, int32_t N, int32_t K, const last_matrix_t* a, const last_matrix_t* b)
{
    long long rows;
    if (check_frames(frames, &rows) != LAST_OK || bad_sizes(rows, N, K)) return 0;
    if (op == LAST_OP_RESIDUAL_NORM_GRAD) return K > kMaxNormColumns ? 0 : align_up(std::max<size_t>(1, part_bytes(rows, K)));
    if (op != LAST_OP_PRODUCT && op != LAST_OP_PRODUCT_GRAD_INPUT && op != LAST_OP_PRODUCT_GRAD_WEIGHT) return 0;
    if (!a || !b) return 0;
    const bool weight = op == LAST_OP_PRODUCT_GRAD_WEIGHT;
    const bool types = op == LAST_OP_PRODUCT ? a->type == b->type && (half_width(a->type) || a->type == LAST_E4M3)
                                             : half_width(a->type) && (a->type == b->type || (weight && eight(b->type)));
    if (!types) return 0;
    if (a->pitch < (op == LAST_OP_PRODUCT ? K : N) || b->pitch < K) return 0;
    Carver cv(nullptr);
    last_status_t rc;
    if (op == LAST_OP_PRODUCT) {
        rc = run_product(cv, frames, rows, N, K, a, b, false, nullptr, 0, nullptr, nullptr, nullptr, nullptr);
        if (rc == LAST_OK && a->type == LAST_E4M3) {                  // (the type of the result is not known here)
            Carver wide(nullptr);
            rc = run_product(wide, frames, rows, N, K, a, b, true, nullptr, 0, nullptr, nullptr, nullptr, nullptr);
            cv.used = std::max(cv.used, wide.used);
        }
    }
    else if (weight) rc = run_grad_weight(cv, frames, rows, N, K, a, b, 0, nullptr, (float*)kAlign, nullptr);
    else rc = run_grad_input(cv, frames, rows, N, K, a, b, nullptr, 0, nullptr, nullptr);
    return rc == LAST_OK ? std::max(kAlign, cv.used) : 0;
}

last_status_t last_residual_norm(const last_frames_t* frames, int32_t H, const last_matrix_t* x, const last_matrix_t* residual,
                                 const float* gain, float eps, const last_matrix_t* s, const last_matrix_t* y,
                                 const last_matrix_t* kept, float* inv, void* hip_stream)
{
    long long rows;
    LAST_TRY(check_frames(frames, &rows));
    if (!gain || !x || (!s && !y && !kept && !inv)) return LAST_ERR_NULL;
    if (H < 1) return LAST_ERR_SHAPE;
    if (H > kMaxNormColumns) return LAST_ERR_UNSUPPORTED;
    if (!(eps >= 0.f)) return LAST_ERR_SHAPE;
    LAST_TRY(check_matrix(x, H, plain(x->type)));
    if (residual) LAST_TRY(check_matrix(residual, H, residual->type == x->type));
    if (s) LAST_TRY(check_matrix(s, H, s->type == x->type));
    if (y) LAST_TRY(check_matrix(y, H, plain(y->type)));
    if (kept) LAST_TRY(check_matrix(kept, H, eight(kept->type)));
    if (rows == 0) return LAST_OK;
    NormArgs a{};
    a.frames = frames_of(frames);
    a.rows = (int)rows;
    a.H = H;
    a.x = x->data;
    a.px = x->pitch;
    if (residual) { a.res = residual->data; a.pr = residual->pitch; }
    if (s) { a.s = s->data; a.ps = s->pitch; }
    if (y) { a.y = y->data; a.py = y->pitch; a.ytype = y->type; }
    a.kept = eight_of(kept);
    a.gain = gain;
    a.inv = inv;
    a.eps = eps;
    hipStream_t st = (hipStream_t)hip_stream;
    if (x->type == LAST_F32) launch_norm<float>(a, st);
    else if (x->type == LAST_BF16) launch_norm<bf16_t>(a, st);
    else launch_norm<f16_t>(a, st);
    return hip_done();
}

last_status_t last_residual_norm_grad(const last_frames_t* frames, int32_t H, const last_matrix_t* dy, const last_matrix_t* s,
                                      const float* gain, const float* inv, const last_matrix_t* ds, const last_matrix_t* dx,
                                      float* dgain, void* ws, size_t ws_bytes, void* hip_stream)
{
    long long rows;
    LAST_TRY(check_frames(frames, &rows));
    if (!gain || !inv || !dy || !s || !dx) return LAST_ERR_NULL;
    if (H < 1) return LAST_ERR_SHAPE;
    if (H > kMaxNormColumns) return LAST_ERR_UNSUPPORTED;
    LAST_TRY(check_matrix(dy, H, plain(dy->type)));
    LAST_TRY(check_matrix(s, H, norm_grad_types(dy->type, s->type)));
    LAST_TRY(check_matrix(dx, H, plain(dx->type)));
    if (ds) LAST_TRY(check_matrix(ds, H, ds->type == dx->type));
    if (dgain) LAST_TRY(check_ws(ws, ws_bytes, last_layer_workspace_bytes(LAST_OP_RESIDUAL_NORM_GRAD, frames, 1, H, nullptr, nullptr)));
    NormGradArgs a{};
    a.frames = frames_of(frames);
    a.rows = (int)rows;
    a.H = H;
    a.dy = dy->data;
    a.pdy = dy->pitch;
    a.s = s->data;
    a.ps = s->pitch;
    a.s_scales = s->scales;
    a.pss = s->scale_pitch;
    if (ds) { a.ds = ds->data; a.pds = ds->pitch; }
    a.dx = dx->data;
    a.pdx = dx->pitch;
    a.dxtype = dx->type;
    a.gain = gain;
    a.inv = inv;
    a.part = dgain ? (float*)ws : nullptr;
    hipStream_t st = (hipStream_t)hip_stream;
    const int groups = norm_grad_groups(rows, H);
    if (rows > 0) {
        if (dy->type == LAST_F32) launch_norm_grad_on<float>(s->type, a, groups, st);
        else if (dy->type == LAST_BF16) launch_norm_grad_on<bf16_t>(s->type, a, groups, st);
        else launch_norm_grad_on<f16_t>(s->type, a, groups, st);
    }
    if (dgain)
        hipLaunchKernelGGL(column_sum_kernel, dim3((unsigned)((H + 31) / 32)), dim3(1024), 0, st, (const float*)a.part, groups, H, dgain);
    return hip_done();
}

last_status_t last_product(const last_frames_t* frames, int32_t N, int32_t K, const last_matrix_t* x, const last_matrix_t* w,
                           const float* bias, last_activation_t act, const last_matrix_t* residual, const last_matrix_t* y,
                           const last_matrix_t* kept, void* ws, size_t ws_bytes, void* hip_stream)
{
    long long rows;
    LAST_TRY(check_frames(frames, &rows));
    if (!x || !w || !y) return LAST_ERR_NULL;
    if (bad_sizes(rows, N, K)) return LAST_ERR_SHAPE;
    if (bad_activation(act)) return LAST_ERR_UNSUPPORTED;
    LAST_TRY(check_matrix(x, K, half_width(x->type) || x->type == LAST_E4M3));
    LAST_TRY(check_matrix(w, K, w->type == x->type));
    LAST_TRY(check_matrix(y, N, plain(y->type) || eight(y->type)));
    if (residual) LAST_TRY(check_matrix(residual, N, plain(residual->type) && (eight(y->type) || residual->type == y->type)));
    if (kept) LAST_TRY(check_matrix(kept, N, eight(kept->type)));
    LAST_TRY(check_ws(ws, ws_bytes, last_layer_workspace_bytes(LAST_OP_PRODUCT, frames, N, K, x, w)));
    Carver cv(ws, ws_bytes);
    const bool wide = x->type == LAST_E4M3 && y->type == LAST_F32;
    return run_product(cv, frames, rows, N, K, x, w, wide, bias, act, residual, y, kept, (hipStream_t)hip_stream);
}

last_status_t last_product_grad_input(const last_frames_t* frames, int32_t N, int32_t K, const last_matrix_t* dy, const last_matrix_t* w,
                                      const last_matrix_t* kept, last_activation_t act, const last_matrix_t* dx, void* ws,
                                      size_t ws_bytes, void* hip_stream)
{
    long long rows;
    LAST_TRY(check_frames(frames, &rows));
    if (!dy || !w || !dx || (act != LAST_ACT_NONE && !kept)) return LAST_ERR_NULL;
    if (bad_sizes(rows, N, K)) return LAST_ERR_SHAPE;
    if (bad_activation(act)) return LAST_ERR_UNSUPPORTED;
    LAST_TRY(check_matrix(dy, N, half_width(dy->type)));
    LAST_TRY(check_matrix(w, K, w->type == dy->type));
    LAST_TRY(check_matrix(dx, K, plain(dx->type)));
    if (kept) LAST_TRY(check_matrix(kept, K, eight(kept->type)));
    LAST_TRY(check_ws(ws, ws_bytes, last_layer_workspace_bytes(LAST_OP_PRODUCT_GRAD_INPUT, frames, N, K, dy, w)));
    Carver cv(ws, ws_bytes);
    return run_grad_input(cv, frames, rows, N, K, dy, w, kept, act, dx, (hipStream_t)hip_stream);
}

last_status_t last_product_grad_weight(const last_frames_t* frames, int32_t N, int32_t K, const last_matrix_t* dy, const last_matrix_t* x,
                                       last_activation_t act, const last_matrix_t* dw, float* dbias, void* ws, size_t ws_bytes,
                                       void* hip_stream)
{
    long long rows;
    LAST_TRY(check_frames(frames, &rows));
    if (!dy || !x || !dw) return LAST_ERR_NULL;
    if (bad_sizes(rows, N, K)) return LAST_ERR_SHAPE;
    if (bad_activation(act)) return LAST_ERR_UNSUPPORTED;
    LAST_TRY(check_matrix(dy, N, half_width(dy->type)));
    LAST_TRY(check_matrix(x, K, eight(x->type) || (x->type == dy->type && act == LAST_ACT_NONE)));
    LAST_TRY(check_matrix(dw, K, plain(dw->type)));
    LAST_TRY(check_ws(ws, ws_bytes, last_layer_workspace_bytes(LAST_OP_PRODUCT_GRAD_WEIGHT, frames, N, K, dy, x)));
    Carver cv(ws, ws_bytes);
    return run_grad_weight(cv, frames, rows, N, K, dy, x, act, dw, dbias, (hipStream_t)hip_stream);
}

last_status_t last_keep(const last_frames_t* frames, int32_t H, const last_matrix_t* x, const last_matrix_t* kept, void* hip_stream)
{
    long long rows;
    LAST_TRY(check_frames(frames, &rows));
    if (!x || !kept) return LAST_ERR_NULL;
    if (H < 1 || H > kMaxColumns) return LAST_ERR_SHAPE;
    LAST_TRY(check_matrix(x, H, plain(x->type)));
    LAST_TRY(check_matrix(kept, H, eight(kept->type)));
    KeepArgs a{};
    a.frames = frames_of(frames);
    a.H = H;
    a.x = x->data;
    a.px = x->pitch;
    a.kept = eight_of(kept);
    hipStream_t st = (hipStream_t)hip_stream;
    const int type = x->type;
    return in_pieces(a, rows, [&](const KeepArgs& k, dim3 grid) {
        if (type == LAST_F32) hipLaunchKernelGGL(keep_kernel<float>, grid, dim3(256), 0, st, k);
        else if (type == LAST_BF16) hipLaunchKernelGGL(keep_kernel<bf16_t>, grid, dim3(256), 0, st, k);
        else hipLaunchKernelGGL(keep_kernel<f16_t>, grid, dim3(256), 0, st, k);
    });
}

last_status_t last_kept_values(const last_frames_t* frames, int32_t H, const last_matrix_t* kept, last_activation_t act,
                               const last_matrix_t* y, void* hip_stream)
{
    long long rows;
    LAST_TRY(check_frames(frames, &rows));
    if (!kept || !y) return LAST_ERR_NULL;
    if (H < 1 || H > kMaxColumns) return LAST_ERR_SHAPE;
    if (bad_activation(act)) return LAST_ERR_UNSUPPORTED;
    LAST_TRY(check_matrix(kept, H, eight(kept->type)));
    LAST_TRY(check_matrix(y, H, plain(y->type)));
    hipStream_t st = (hipStream_t)hip_stream;
    return in_pieces(kept_values_args(frames, H, kept, act, y), rows,
                     [&](const KeepArgs& k, dim3 grid) { hipLaunchKernelGGL(kept_values_kernel, grid, dim3(256), 0, st, k); });
}

last_status_t last_kept_grad(const last_frames_t* frames, int32_t H, const last_matrix_t* dy, const last_matrix_t* kept,
                             last_activation_t act, const last_matrix_t* dx, void* hip_stream)
{
    long long rows;
    LAST_TRY(check_frames(frames, &rows));
    if (!dy || !kept || !dx) return LAST_ERR_NULL;
    if (H < 1 || H > kMaxColumns) return LAST_ERR_SHAPE;
    if (bad_activation(act)) return LAST_ERR_UNSUPPORTED;
    LAST_TRY(check_matrix(dy, H, plain(dy->type)));
    LAST_TRY(check_matrix(kept, H, eight(kept->type)));
    LAST_TRY(check_matrix(dx, H, plain(dx->type)));
    KeepArgs a{};
    a.frames = frames_of(frames);
    a.H = H;
    a.x = dy->data;
    a.px = dy->pitch;
    a.y = dx->data;
    a.py = dx->pitch;
    a.act = act;
    a.ytype = dx->type;
    a.kept = eight_of(kept);
    hipStream_t st = (hipStream_t)hip_stream;
    const int type = dy->type;
    return in_pieces(a, rows, [&](const KeepArgs& k, dim3 grid) {
        if (type == LAST_F32) hipLaunchKernelGGL(kept_grad_kernel<float>, grid, dim3(256), 0, st, k);
        else if (type == LAST_BF16) hipLaunchKernelGGL(kept_grad_kernel<bf16_t>, grid, dim3(256), 0, st, k);
        else hipLaunchKernelGGL(kept_grad_kernel<f16_t>, grid, dim3(256), 0, st, k);
    });
}

}  // extern "C"
