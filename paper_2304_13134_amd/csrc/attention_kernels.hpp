// Attention of frames to a band of frames around them and to a few first ones, and its gradient.
//     s is seen by t  <=>  s < len,  s <= t + right,  s >= t - left or s < sinks
//     S = scale q k^T,  P = softmax over what is seen,  y = P v,  L = log sum exp S
//     delta = dy . y,  dS = P (dy v^T - delta),  dq = scale dS k,  dk = scale dS^T q,  dv = P^T dy
//
// Every kernel has frames of its own, 32 a wavefront, one a lane (both halves of a wavefront have the same), and goes over tiles of 64 of
// the other ones, which stand in LDS.  Products are of 32 x 32 results: the tile's frames are the rows, the wavefront's
// own the columns.  So a lane has 16 scores of its own frame: softmax sums stay in the lane, but for the other half's; a factor
// of a frame is a number of the lane's; and the scores, rounded to 16 bits, are as they stand the second operand of the product that
// sums over the tile's frames, whose first one is read from LDS by transposing reads (ds_read_b64_tr_b16) in the order in which the
// scores lie: rows 4 h .. 4 h + 3 and 8 + 4 h .. of 16, h being the half.
//
// Scores, P and sums are in 32 bits; P and dS are rounded to the operands' type for the matrix cores, which adds as much to the
// result as its own rounding does (half a step of each term).
#pragma once
#include "heads_kernels.hpp"
#include "layer.hpp"

namespace last {

typedef float f16x __attribute__((ext_vector_type(16)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 64;            // frames of a tile in LDS
constexpr int kOwn = 128;            // frames of a workgroup
constexpr float kLog2e = 1.4426950408889634f;

struct Band {
    int left, right, sinks;
    float scale;
};

struct AttentionArgs {
    const int* len;
    int T, B, heads, kv_heads, D;
    const void *q, *k, *v, *dy;
    void *y, *dq, *dk, *dv;
    long long pq, pk, pv, py, pdy, pdq, pdk, pdv;
    float *lse, *delta;              // [B * T][heads]
    float* part;                     // first frames' sums of dk and dv, see sinks_kernel
    int shares;
    Band band;
    unsigned first, tiles;           // of the launch; a workgroup's own frames are tile `id % tiles`
};

template <typename E> struct Mma;
template <> struct Mma<bf16_t> {
    static __device__ __forceinline__ f16x go(u4 a, u4 b, f16x c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned pair(float lo, float hi) { return bf16_pair(lo, hi); }
};
template <> struct Mma<f16_t> {
    static __device__ __forceinline__ f16x go(u4 a, u4 b, f16x c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ unsigned pair(float lo, float hi) { return f16_pair(lo, hi); }
};

__device__ __forceinline__ f16x zeros16()
{
    f16x v;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = 0.f;
    return v;
}

// A tile in LDS: rows of DP columns of 16 bits.
template <int DP> struct Rows {
    static constexpr int kPitch = DP * 2 + 16;
    static constexpr int kBytes = kTile * kPitch;
    static constexpr int kPieces = DP / 8;                   // of 16 bytes a row
    static constexpr int kEach = kTile * kPieces / 256;      // of a thread of 256
    static constexpr int kApart = 256 / kPieces;             // rows between a thread's pieces
};

// a thread's pieces of a tile, sent for ahead
template <int DP> struct Sent {
    u4 v[Rows<DP>::kEach];
};

// Rows s0 .. s0 + 63 of a head from `p` (its row 0); what `exists(row)` denies and columns beyond D are zeros.
template <int DP, typename Exists>
__device__ __forceinline__ void send(Sent<DP>& r, const char* p, long long pitch, int D, int s0, Exists exists)
{
    const int c = (int)threadIdx.x % Rows<DP>::kPieces * 8;
#pragma unroll
    for (int i = 0; i < Rows<DP>::kEach; ++i) {
        const int s = s0 + (int)threadIdx.x / Rows<DP>::kPieces + i * Rows<DP>::kApart;
        r.v[i] = u4{0u, 0u, 0u, 0u};
        if (c < D && exists(s)) r.v[i] = *(const u4_any*)(p + ((size_t)s * pitch + c) * 2);
    }
}

template <int DP>
__device__ __forceinline__ void lay(const Sent<DP>& r, char* lds)
{
    const int at = (int)threadIdx.x / Rows<DP>::kPieces * Rows<DP>::kPitch + (int)threadIdx.x % Rows<DP>::kPieces * 16;
#pragma unroll
    for (int i = 0; i < Rows<DP>::kEach; ++i) *(u4*)(lds + at + i * Rows<DP>::kApart * Rows<DP>::kPitch) = r.v[i];
}

// first operand, rows 32 block .. of the tile, columns 16 k ..
template <int DP>
__device__ __forceinline__ u4 along_rows(const char* lds, int block, int k)
{
    const int lane = (int)threadIdx.x % kWave;
    return *(const u4*)(lds + (lane & 31) * Rows<DP>::kPitch + (lane >> 5) * 16 + block * 32 * Rows<DP>::kPitch + k * 32);
}

// first operand, columns 32 block .. of the tile, rows 16 k .. in the order of the scores
template <int DP>
__device__ __forceinline__ u4 along_columns(const char* lds, int block, int k)
{
    typedef __attribute__((address_space(3))) s4* at;
    const int lane = (int)threadIdx.x % kWave;
    const char* p = lds + (4 * (lane >> 5) + (lane & 15) / 4) * Rows<DP>::kPitch + ((lane >> 4 & 1) * 16 + (lane & 3) * 4) * 2 +
                    16 * k * Rows<DP>::kPitch + block * 64;
    const u2 lo = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)p));
    const u2 hi = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(p + 8 * Rows<DP>::kPitch)));
    return u4{lo[0], lo[1], hi[0], hi[1]};
}

// 16 sums of a lane to two second operands
template <typename E>
__device__ __forceinline__ void to_operands(const f16x& p, u4* r)
{
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) r[i][k] = Mma<E>::pair(p[8 * i + 2 * k], p[8 * i + 2 * k + 1]);
}

// the frame of the tile's 32 that a lane's i-th result belongs to
__device__ __forceinline__ int result_row(int i) { return 8 * (i >> 2) + 4 * ((int)threadIdx.x % kWave >> 5) + (i & 3); }

// second operands of a wavefront's own 32 rows: a lane's own row `p` (null: zeros)
template <int DP>
__device__ __forceinline__ void own_rows(const char* p, int D, u4* r)
{
    const int h = (int)threadIdx.x % kWave >> 5;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        const int c = 16 * k + 8 * h;
        r[k] = u4{0u, 0u, 0u, 0u};
        if (p && c < D) r[k] = *(const u4_any*)(p + c * 2);
    }
}

// a lane's own row of results, columns 32 block + result_row(i); zeros of a frame that is not there
template <typename E, int DP>
__device__ __forceinline__ void put_rows(char* p, int D, const f16x* acc, float factor, bool there)
{
    const int h = (int)threadIdx.x % kWave >> 5;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = 32 * d + 8 * j + 4 * h;
            if (c >= D) continue;
            float v[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) v[k] = there ? acc[d][4 * j + k] * factor : 0.f;
            store4<E>(p, c, v);
        }
}

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32, kWave); }

// frames of an item: lengths as clamped
__device__ __forceinline__ int frames_of_item(const int* len, int T, int b) { return len ? clamped(len[b], T) : T; }

template <typename E> __device__ __forceinline__ float value_at(const char* p, int c)
{
    if constexpr (Elt<E>::type == LAST_BF16) return bf16_to_float(((const uint16_t*)p)[c]);
    else return (float)((const _Float16*)p)[c];
}

// One frame's attention without matrix cores, by a wavefront, the head's columns over its lanes.  The products of the kernels multiply what is not
// seen by zero, which is no number for an infinity or a NaN; rows that come out so are formed again here, over what they see alone.
// seen(s): whether s in [from, to) is; row(p, s): where its keys and values are.
template <typename E, typename Seen, typename KeyRow, typename ValueRow>
__device__ void plain_row(const char* q, int D, float c2, int from, int to, Seen seen, KeyRow key, ValueRow value, float* m, float* l, float* o)
{
    const int lane = (int)threadIdx.x % kWave;
    float x[2], top = LAST_NEG_INF, sum = 0.f;
    o[0] = o[1] = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = lane + 64 * i < D ? value_at<E>(q, lane + 64 * i) : 0.f;
    for (int s = from; s < to; ++s) {
        if (!seen(s)) continue;
        const char *k = key(s), *v = value(s);
        float dot = 0.f, w[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (lane + 64 * i < D) {
                dot += x[i] * (k ? value_at<E>(k, lane + 64 * i) : __uint_as_float(0x7fc00000u));
                w[i] = v ? value_at<E>(v, lane + 64 * i) : 0.f;
            }
        dot = wave_sum(dot);
        const float higher = fmaxf(top, dot), by = higher == LAST_NEG_INF ? 0.f : higher;
        const float old = __builtin_amdgcn_exp2f((top - by) * c2), p = __builtin_amdgcn_exp2f((dot - by) * c2);
        top = higher;
        sum = sum * old + p;
#pragma unroll
        for (int i = 0; i < 2; ++i) o[i] = o[i] * old + p * w[i];
    }
    *m = top;
    *l = sum;
}

// the running maximum and sum of a lane's frame, its results so far
template <int DP> struct Softmax {
    f16x acc[DP / 32];
    float m, l;                      // l of this half of the wavefront
    __device__ void init()
    {
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) acc[d] = zeros16();
        m = LAST_NEG_INF;
        l = 0.f;
    }
    // scores of N blocks of 32 frames, -inf where not seen, become probabilities relative to m
    template <int N>
    __device__ __forceinline__ void take(f16x* s, float c2)
    {
        float top = s[0][0];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
        top = fmaxf(top, other_half(top));
        // The maximum is only a reference: as long as no score passes it by a factor of 2^8 the sums keep it, which saves their scaling.
        if (__any((top - m) * c2 > 8.f || (m == LAST_NEG_INF && top > m))) {
            const float higher = fmaxf(m, top), old = m == LAST_NEG_INF ? 0.f : __builtin_amdgcn_exp2f((m - higher) * c2);
            m = higher;
            l *= old;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] *= old;
        }
        const float by = m == LAST_NEG_INF ? 0.f : m * c2;
        float sum = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][i], c2, -by));
                sum += s[n][i];
            }
        l += sum;
    }
    // whether a result is no number (or would be for another frame's sake)
    __device__ __forceinline__ bool not_finite() const
    {
        float t = l * 0.f;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) t += acc[d][i] * 0.f;
        t += other_half(t);
        return !(t == 0.f);
    }
};

// what a workgroup works on
struct Place {
    int tile, head, kv, item, len;
    size_t row0;                     // of the item
};

__device__ __forceinline__ Place place_of(const AttentionArgs& a, int heads)
{
    Place p;
    const unsigned id = a.first + blockIdx.x, hb = id / a.tiles;
    p.tile = (int)(id % a.tiles);
    p.head = (int)(hb % (unsigned)heads);
    p.item = (int)(hb / (unsigned)heads);
    p.kv = p.head / (heads / a.kv_heads);
    p.len = frames_of_item(a.len, a.T, p.item);
    p.row0 = (size_t)p.item * a.T;
    return p;
}

template <typename E, int DP>
__global__ __launch_bounds__(256) void attention_kernel(AttentionArgs a)
{
    __shared__ __attribute__((aligned(16))) char lds[2 * Rows<DP>::kBytes];
    char *const kt = lds, *const vt = lds + Rows<DP>::kBytes;
    const Place at = place_of(a, a.heads);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x % kWave;
    const int g0 = at.tile * kOwn, t0 = g0 + wave * 32, t = t0 + (lane & 31);
    const Band band = a.band;
    const float c2 = band.scale * kLog2e;
    const bool there = t < at.len;
    const char* const q = (const char*)a.q + (((at.row0 + t) * a.pq) + (size_t)at.head * a.D) * 2;
    const char* const k = (const char*)a.k + (at.row0 * a.pk + (size_t)at.kv * a.D) * 2;
    const char* const v = (const char*)a.v + (at.row0 * a.pv + (size_t)at.kv * a.D) * 2;
    u4 qf[DP / 16];
    own_rows<DP>(there ? q : nullptr, a.D, qf);
    // frames that the workgroup's see: first ones, and [lo, hi)
    const int lo = g0 - band.left > 0 ? g0 - band.left : 0;
    const int hi = g0 >= at.len ? 0 : g0 + kOwn + band.right < at.len ? g0 + kOwn + band.right : at.len;
    const int first_tiles = band.sinks > 0 && hi > 0 ? 1 : 0;
    const int first = lo / kTile > first_tiles ? lo / kTile : first_tiles, last = (hi + kTile - 1) / kTile;
    const int tiles = first_tiles + (last > first ? last - first : 0);
    const auto start = [&](int j) { return (j < first_tiles ? j : first + j - first_tiles) * kTile; };
    const auto exists = [&](int s) { return s < hi && (s >= lo || s < band.sinks); };
    const int seen_lo = t - band.left, seen_hi = there ? (t + band.right + 1 < at.len ? t + band.right + 1 : at.len) : 0;
    Softmax<DP> soft;
    soft.init();
    Sent<DP> ks, vs;
    if (tiles > 0) {
        send<DP>(ks, k, a.pk, a.D, start(0), exists);
        send<DP>(vs, v, a.pv, a.D, start(0), exists);
    }
    for (int j = 0; j < tiles; ++j) {
        const int s0 = start(j);
        __syncthreads();
        lay<DP>(ks, kt);
        lay<DP>(vs, vt);
        __syncthreads();
        if (j + 1 < tiles) {
            send<DP>(ks, k, a.pk, a.D, start(j + 1), exists);
            send<DP>(vs, v, a.pv, a.D, start(j + 1), exists);
        }
        if (s0 >= t0 + 32 + band.right || t0 >= at.len || (s0 + kTile <= t0 - band.left && s0 >= band.sinks)) continue;
        f16x s[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            s[n] = zeros16();
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) s[n] = Mma<E>::go(along_rows<DP>(kt, n, i), qf[i], s[n]);
        }
        if (!(s0 >= t0 + 31 - band.left && s0 + kTile - 1 <= t0 + band.right && s0 + kTile <= at.len && t0 + 32 <= at.len)) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int f = s0 + 32 * n + result_row(i);
                    s[n][i] = f < seen_hi && (f >= seen_lo || f < band.sinks) ? s[n][i] : LAST_NEG_INF;
                }
        }
        soft.template take<2>(s, c2);
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            u4 p[2];
            to_operands<E>(s[n], p);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) soft.acc[d] = Mma<E>::go(along_columns<DP>(vt, d, 2 * n + i), p[i], soft.acc[d]);
        }
    }
    const float l = soft.l + other_half(soft.l);
    const bool odd = there && soft.not_finite();
    if (t < a.T && !odd) {
        char* const y = (char*)a.y + (((at.row0 + t) * a.py) + (size_t)at.head * a.D) * 2;
        put_rows<E, DP>(y, a.D, soft.acc, 1.f / l, there);
        if (a.lse && lane < 32) a.lse[(at.row0 + t) * a.heads + at.head] = there ? (soft.m * c2 + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : 0.f;
    }
    for (unsigned long long rows = __ballot(odd) & 0xffffffffull; rows; rows &= rows - 1) {
        const int tr = t0 + __ffsll(rows) - 1;
        const int end = tr + band.right + 1 < at.len ? tr + band.right + 1 : at.len;
        const char* const qr = (const char*)a.q + (((at.row0 + tr) * a.pq) + (size_t)at.head * a.D) * 2;
        float m, sum, o[2];
        plain_row<E>(qr, a.D, c2, 0, end, [&](int s) { return s >= tr - band.left || s < band.sinks; },
                     [&](int s) { return k + (size_t)s * a.pk * 2; }, [&](int s) { return v + (size_t)s * a.pv * 2; }, &m, &sum, o);
        char* const y = (char*)a.y + (((at.row0 + tr) * a.py) + (size_t)at.head * a.D) * 2;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (lane + 64 * i < a.D) Elt<E>::put(y, lane + 64 * i, o[i] / sum);
        if (a.lse && lane == 0) a.lse[(at.row0 + tr) * a.heads + at.head] = (m * c2 + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
    }
}

// delta[t][head] = dy . y, 0 where there is no frame: eight columns a lane, LN lanes a head
template <typename E, int LN>
__global__ __launch_bounds__(256) void delta_kernel(AttentionArgs a, long long first)
{
    const int lane = (int)threadIdx.x % LN;
    const long long i = first + ((long long)blockIdx.x * 256 + threadIdx.x) / LN;
    if (i >= (long long)a.B * a.T * a.heads) return;
    const long long row = i / a.heads;
    const int head = (int)(i - row * a.heads), b = (int)(row / a.T), c = 8 * lane;
    float sum = 0.f;
    if ((int)(row - (long long)b * a.T) < frames_of_item(a.len, a.T, b) && c < a.D) {
        float x[8], z[8];
        load8<E>(a.dy, (size_t)row * a.pdy + (size_t)head * a.D + c, 8, x);
        load8<E>(a.y, (size_t)row * a.py + (size_t)head * a.D + c, 8, z);
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += x[k] * z[k];
    }
    sum = head_sum<LN>(sum);
    if (lane == 0) a.delta[i] = sum;
}

// The gradient of queries: a wavefront's own frames are queries, the tiles keys and values.
template <typename E, int DP>
__global__ __launch_bounds__(256) void grad_query_kernel(AttentionArgs a)
{
    __shared__ __attribute__((aligned(16))) char lds[2 * Rows<DP>::kBytes];
    char *const kt = lds, *const vt = lds + Rows<DP>::kBytes;
    const Place at = place_of(a, a.heads);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x % kWave;
    const int g0 = at.tile * kOwn, t0 = g0 + wave * 32, t = t0 + (lane & 31);
    const Band band = a.band;
    const float c2 = band.scale * kLog2e;
    const bool there = t < at.len;
    const size_t row = at.row0 + t;
    const char* const k = (const char*)a.k + (at.row0 * a.pk + (size_t)at.kv * a.D) * 2;
    const char* const v = (const char*)a.v + (at.row0 * a.pv + (size_t)at.kv * a.D) * 2;
    u4 qf[DP / 16], df[DP / 16];
    own_rows<DP>(there ? (const char*)a.q + (row * a.pq + (size_t)at.head * a.D) * 2 : nullptr, a.D, qf);
    own_rows<DP>(there ? (const char*)a.dy + (row * a.pdy + (size_t)at.head * a.D) * 2 : nullptr, a.D, df);
    const float l2 = there ? a.lse[row * a.heads + at.head] * kLog2e : 0.f, delta = there ? a.delta[row * a.heads + at.head] : 0.f;
    const int lo = g0 - band.left > 0 ? g0 - band.left : 0;
    const int hi = g0 >= at.len ? 0 : g0 + kOwn + band.right < at.len ? g0 + kOwn + band.right : at.len;
    const int first_tiles = band.sinks > 0 && hi > 0 ? 1 : 0;
    const int first = lo / kTile > first_tiles ? lo / kTile : first_tiles, last = (hi + kTile - 1) / kTile;
    const int tiles = first_tiles + (last > first ? last - first : 0);
    const auto start = [&](int j) { return (j < first_tiles ? j : first + j - first_tiles) * kTile; };
    const auto exists = [&](int s) { return s < hi && (s >= lo || s < band.sinks); };
    const int seen_lo = t - band.left, seen_hi = there ? (t + band.right + 1 < at.len ? t + band.right + 1 : at.len) : 0;
    f16x acc[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) acc[d] = zeros16();
    Sent<DP> ks, vs;
    if (tiles > 0) {
        send<DP>(ks, k, a.pk, a.D, start(0), exists);
        send<DP>(vs, v, a.pv, a.D, start(0), exists);
    }
    for (int j = 0; j < tiles; ++j) {
        const int s0 = start(j);
        __syncthreads();
        lay<DP>(ks, kt);
        lay<DP>(vs, vt);
        __syncthreads();
        if (j + 1 < tiles) {
            send<DP>(ks, k, a.pk, a.D, start(j + 1), exists);
            send<DP>(vs, v, a.pv, a.D, start(j + 1), exists);
        }
        if (s0 >= t0 + 32 + band.right || t0 >= at.len || (s0 + kTile <= t0 - band.left && s0 >= band.sinks)) continue;
        const bool all = s0 >= t0 + 31 - band.left && s0 + kTile - 1 <= t0 + band.right && s0 + kTile <= at.len && t0 + 32 <= at.len;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            f16x s = zeros16(), p = zeros16();
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                s = Mma<E>::go(along_rows<DP>(kt, n, i), qf[i], s);
                p = Mma<E>::go(along_rows<DP>(vt, n, i), df[i], p);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c2, -l2)) * (p[i] - delta);
                const int f = s0 + 32 * n + result_row(i);
                s[i] = all || (f < seen_hi && (f >= seen_lo || f < band.sinks)) ? e : 0.f;
            }
            u4 d[2];
            to_operands<E>(s, d);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int x = 0; x < DP / 32; ++x) acc[x] = Mma<E>::go(along_columns<DP>(kt, x, 2 * n + i), d[i], acc[x]);
        }
    }
    if (t < a.T) put_rows<E, DP>((char*)a.dq + (row * a.pdq + (size_t)at.head * a.D) * 2, a.D, acc, band.scale, there);
}

// The gradients of keys and values: a wavefront's own frames are keys, the tiles queries and their dy, of all heads that share
// the keys.  SINKS: the part that first frames s < sinks have in frames t > s + left, a share of these a workgroup; its sums go to
// `part`, [item][kv head][share][2][64][DP], and are added by the workgroup that has these frames for its own.
template <typename E, int DP, bool SINKS>
__global__ __launch_bounds__(256) void grad_key_kernel(AttentionArgs a)
{
    __shared__ __attribute__((aligned(16))) char lds[2 * Rows<DP>::kBytes];
    __shared__ float stats[2][kTile];
    char *const qt = lds, *const yt = lds + Rows<DP>::kBytes;
    const Place at = place_of(a, a.kv_heads);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x % kWave;
    const Band band = a.band;
    const int g0 = SINKS ? 0 : at.tile * kOwn, s0 = g0 + wave * 32, s = s0 + (lane & 31);
    const float c2 = band.scale * kLog2e;
    const bool there = s < at.len && (!SINKS || s < band.sinks);
    const size_t row = at.row0 + s;
    const int group = a.heads / a.kv_heads;
    u4 kf[DP / 16], vf[DP / 16];
    own_rows<DP>(there ? (const char*)a.k + (row * a.pk + (size_t)at.kv * a.D) * 2 : nullptr, a.D, kf);
    own_rows<DP>(there ? (const char*)a.v + (row * a.pv + (size_t)at.kv * a.D) * 2 : nullptr, a.D, vf);
    // frames that see the workgroup's
    int lo = g0 - band.right > 0 ? g0 - band.right : 0;
    int hi = g0 >= at.len ? 0 : (long long)g0 + kOwn + band.left < at.len ? g0 + kOwn + band.left : at.len;
    if (SINKS) {
        lo = band.left + 1 < at.len ? band.left + 1 : at.len;
        hi = at.len;
    }
    int first = lo / kTile, last = (hi + kTile - 1) / kTile;
    if (SINKS) {
        const int n = last > first ? last - first : 0;
        last = first + (int)((long long)n * (at.tile + 1) / a.shares);
        first = first + (int)((long long)n * at.tile / a.shares);
    }
    const int per = last > first ? last - first : 0, tiles = per * group;
    const auto exists = [&](int t) { return t >= lo && t < hi; };
    // t sees s: s - right <= t, t <= s + left (or, of first frames, beyond)
    const int seen_lo = SINKS ? s + band.left + 1 : s - band.right;
    const int seen_hi = !there ? 0 : SINKS ? at.len : (long long)s + band.left + 1 < at.len ? s + band.left + 1 : at.len;
    const bool idle = SINKS ? s0 >= band.sinks : s0 >= at.len;
    f16x dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) dk[d] = dv[d] = zeros16();
    Sent<DP> qs, ys;
    float stat = 0.f;
    const auto get = [&](int j) {
        const int head = at.kv * group + j / per, t0 = (first + j % per) * kTile;
        send<DP>(qs, (const char*)a.q + (at.row0 * a.pq + (size_t)head * a.D) * 2, a.pq, a.D, t0, exists);
        send<DP>(ys, (const char*)a.dy + (at.row0 * a.pdy + (size_t)head * a.D) * 2, a.pdy, a.D, t0, exists);
        const int t = t0 + (int)threadIdx.x % kTile;
        stat = 0.f;
        if (threadIdx.x < 2 * kTile && exists(t)) {
            const size_t i = (at.row0 + t) * a.heads + head;
            stat = threadIdx.x < kTile ? a.lse[i] * kLog2e : a.delta[i];
        }
    };
    if (tiles > 0) get(0);
    for (int j = 0; j < tiles; ++j) {
        const int t0 = (first + j % per) * kTile;
        __syncthreads();
        lay<DP>(qs, qt);
        lay<DP>(ys, yt);
        if (threadIdx.x < 2 * kTile) stats[threadIdx.x / kTile][threadIdx.x % kTile] = stat;
        __syncthreads();
        if (j + 1 < tiles) get(j + 1);
        if (idle || t0 + kTile <= s0 - band.right || (!SINKS && t0 > (long long)s0 + 31 + band.left)) continue;
        const bool all = !SINKS && t0 >= s0 + 31 - band.right && t0 + kTile - 1 <= (long long)s0 + band.left && t0 + kTile <= at.len && s0 + 32 <= at.len;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            f16x p = zeros16(), e = zeros16();
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                p = Mma<E>::go(along_rows<DP>(qt, n, i), kf[i], p);
                e = Mma<E>::go(along_rows<DP>(yt, n, i), vf[i], e);
            }
            const int h = lane >> 5;
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const f4 l2 = *(const f4*)&stats[0][32 * n + 2 * i + 4 * h], delta = *(const f4*)&stats[1][32 * n + 2 * i + 4 * h];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int f = t0 + 32 * n + result_row(i + x);
                    const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i + x], c2, -l2[x]));
                    const bool sees = all || (f >= seen_lo && f < seen_hi);
                    p[i + x] = sees ? w : 0.f;
                    e[i + x] = sees ? w * (e[i + x] - delta[x]) : 0.f;
                }
            }
            u4 pf[2], ef[2];
            to_operands<E>(p, pf);
            to_operands<E>(e, ef);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) {
                    dv[d] = Mma<E>::go(along_columns<DP>(yt, d, 2 * n + i), pf[i], dv[d]);
                    dk[d] = Mma<E>::go(along_columns<DP>(qt, d, 2 * n + i), ef[i], dk[d]);
                }
        }
    }
    const size_t all_parts = ((size_t)at.item * a.kv_heads + at.kv) * a.shares;
    if constexpr (SINKS) {
        if (s >= 64) return;
        float* const out = a.part + ((all_parts + at.tile) * 2 * 64 + s) * DP;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                *(f4*)(out + 32 * d + result_row(i)) = f4{dk[d][i], dk[d][i + 1], dk[d][i + 2], dk[d][i + 3]};
                *(f4*)(out + 64 * DP + 32 * d + result_row(i)) = f4{dv[d][i], dv[d][i + 1], dv[d][i + 2], dv[d][i + 3]};
            }
    } else {
        if (a.part && s < band.sinks && there) {
            for (int share = 0; share < a.shares; ++share) {
                const float* const in = a.part + ((all_parts + share) * 2 * 64 + s) * DP;
#pragma unroll
                for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const f4 x = *(const f4*)(in + 32 * d + result_row(i)), z = *(const f4*)(in + 64 * DP + 32 * d + result_row(i));
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            dk[d][i + c] += x[c];
                            dv[d][i + c] += z[c];
                        }
                    }
            }
        }
        if (s < a.T) {
            put_rows<E, DP>((char*)a.dk + (row * a.pdk + (size_t)at.kv * a.D) * 2, a.D, dk, band.scale, there);
            put_rows<E, DP>((char*)a.dv + (row * a.pdv + (size_t)at.kv * a.D) * 2, a.D, dv, 1.f, there);
        }
    }
}

}  // namespace last
