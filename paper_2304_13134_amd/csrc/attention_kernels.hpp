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
#include <type_traits>

namespace last {

typedef float f16x __attribute__((ext_vector_type(16)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));

constexpr int kTile = 64;            // frames of a tile in LDS
constexpr int kOwn = 128;            // frames of a workgroup
constexpr int kMostSinks = 64;       // first frames
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

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
    float *lse, *delta;              // [B * T][heads]; delta of frames that exist
    float *part, *sums;              // first frames' sums of dk and dv (grad_first_kernel, first_join_kernel), or null
    int shares;
    float* kept;                     // sums of dk and dv of parts of the heads that share them (grad_join_kernel)
    int parts;
    Band band;
    unsigned half;                   // workgroups of grad_key_kernel that form keys' gradients alone
    unsigned first, tiles, together; // of the launch: its first workgroup, tiles of a head, heads that go to one XCD together
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

// A value that a branch changes, in the registers where the other way has it: else the compiler lets the branch write others, and copies on the way
// that does not change it, which is the usual one.
template <typename V>
__device__ __forceinline__ void in_place(V& v) { asm volatile("" : "+v"(v)); }

// A tile in LDS: rows of DP columns of 16 bits.  16-byte piece c of row r stands at c ^ spread(r) of its row, so that the 256 bytes that
// the banks give at a time are different ones for a column of 16 rows (reads along rows) and for four pieces of 4 rows (transposing reads).
template <int DP> struct Rows {
    static constexpr int kPitch = DP * 2;
    static constexpr int kBytes = kTile * kPitch;
    static __device__ __forceinline__ int spread(int r)
    {
        return (r >> 2 & 3) | (DP == 128 ? (r & 3) << 2 : DP == 64 ? (r >> 1 & 1) << 2 : 0);
    }
};

// A tile's way from memory to LDS, by THREADS threads: sent for ahead to registers.
template <int DP, int THREADS> struct Tile {
    static constexpr int kPieces = DP / 8;                   // of 16 bytes a row
    static constexpr int kApart = THREADS / kPieces;         // rows between a thread's pieces
    static constexpr int kEach = kTile / kApart;
    static_assert(kTile % kApart == 0 && kApart % 16 == 0, "whole tiles, the same spread for a thread's pieces");
    u4 v[kEach];
    bool all;

    // Rows s0 .. s0 + 63 of a head from `p` (its row 0).  all_: all of them are there; else what `exists(row)` denies is asked for at row `other`
    // instead, which exists, and laid as zeros, as are columns beyond D.
    template <typename Exists>
    __device__ __forceinline__ void send(const char* p, long long pitch, int D, int s0, bool all_, int other, Exists exists)
    {
        all = all_ && D == DP;
        if (all_) {
            send_all(p, pitch, D, s0);
        } else {
            const int piece = (int)threadIdx.x % kPieces * 8, c = piece < D ? piece : 0, r = (int)threadIdx.x / kPieces;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int s = s0 + r + i * kApart;
                v[i] = *(const u4_any*)(p + ((size_t)(unsigned)(exists(s) ? s : other) * pitch + c) * 2);
            }
        }
    }
    __device__ __forceinline__ void send_all(const char* p, long long pitch, int D, int s0)
    {
        const int piece = (int)threadIdx.x % kPieces * 8, c = piece < D ? piece : 0, r = (int)threadIdx.x / kPieces;
        const char* const base = p + (size_t)(unsigned)s0 * pitch * 2;
        const unsigned off = (unsigned)(r * pitch + c) * 2u;                       // (64 pitches of at most 4 MiB)
#pragma unroll
        for (int i = 0; i < kEach; ++i) v[i] = *(const u4_any*)(base + (size_t)i * kApart * pitch * 2 + off);
    }

    template <typename Exists>
    __device__ __forceinline__ void lay(char* lds, int D, int s0, Exists exists)
    {
        const int r = (int)threadIdx.x / kPieces, c = (int)threadIdx.x % kPieces;
        if (!all) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const unsigned keep = ((c * 8 < D) & exists(s0 + r + i * kApart)) ? ~0u : 0u;
                v[i] &= u4{keep, keep, keep, keep};
                in_place(v[i]);
            }
        }
        lay(lds);
    }
    __device__ __forceinline__ void lay(char* lds) const
    {
        const int r = (int)threadIdx.x / kPieces, c = (int)threadIdx.x % kPieces;
        const int at = r * Rows<DP>::kPitch + (c ^ Rows<DP>::spread(r)) * 16;
#pragma unroll
        for (int i = 0; i < kEach; ++i) *(u4*)(lds + at + i * kApart * Rows<DP>::kPitch) = v[i];
    }
    // zeros in columns beyond D
    __device__ __forceinline__ void clear(int D)
    {
        const unsigned keep = (int)threadIdx.x % kPieces * 8 < D ? ~0u : 0u;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            v[i] &= u4{keep, keep, keep, keep};
            in_place(v[i]);
        }
    }
};

// First operands from a tile: where a lane reads.
template <int DP> struct Reads {
    int rows[DP / 16];               // along rows: of columns 16 k ..
    int columns[DP / 32][2];         // along columns 32 d ..: rows 4 h .. and 8 + 4 h ..
    __device__ __forceinline__ void init()
    {
        const int lane = (int)threadIdx.x % kWave, h = lane >> 5, r = lane & 31;
        const int c = 4 * h + (lane & 15) / 4, piece = 2 * (lane >> 4 & 1) + (lane & 3) / 2;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) rows[k] = r * Rows<DP>::kPitch + ((2 * k + h) ^ Rows<DP>::spread(r)) * 16;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                columns[d][i] = (c + 8 * i) * Rows<DP>::kPitch + ((4 * d + piece) ^ Rows<DP>::spread(c + 8 * i)) * 16 + (lane & 1) * 8;
    }
    // rows 32 block .. of the tile, columns 16 k ..
    __device__ __forceinline__ u4 along_rows(const char* lds, int block, int k) const
    {
        return *(const u4*)(lds + rows[k] + block * 32 * Rows<DP>::kPitch);
    }
    // columns 32 d .. of the tile, rows 16 k .. in the order of the scores
    __device__ __forceinline__ u4 along_columns(const char* lds, int d, int k) const
    {
        typedef __attribute__((address_space(3))) s4* at;
        const u2 lo = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(lds + columns[d][0] + 16 * k * Rows<DP>::kPitch)));
        const u2 hi = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(lds + columns[d][1] + 16 * k * Rows<DP>::kPitch)));
        return u4{lo[0], lo[1], hi[0], hi[1]};
    }
};

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

// Waits for what a loop reads of its own before the loop: where that is left to the first use in it, every turn waits there for all loads under way.
template <int N>
__device__ __forceinline__ void have(u4 (&r)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("" : "+v"(r[k]));
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

// maximum and sum over both halves
__device__ __forceinline__ float max_of_halves(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

__device__ __forceinline__ float sum_of_halves(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// frames of an item, which is the same one for all lanes: lengths as clamped
__device__ __forceinline__ int frames_of_item(const int* len, int T, int b) { return len ? clamped(same_for_all(len, b), T) : T; }

// where a frame's keys and values are; null: nowhere, which makes NaN of what sees it
struct KeyValue {
    const char *k, *v;
};

// lane j's pointer
__device__ __forceinline__ const char* of_lane(const char* p, int j)
{
    const uintptr_t at = (uintptr_t)p;
    const unsigned lo = (unsigned)__shfl((int)(unsigned)at, j, kWave), hi = (unsigned)__shfl((int)(unsigned)(at >> 32), j, kWave);
    return (const char*)((uintptr_t)lo | (uintptr_t)hi << 32);
}

// One frame's attention without matrix cores, by a wavefront, to frames [from0, to0) and then [from, to).  The products of the kernels multiply what is not
// seen by zero, which is no number for an infinite value or a NaN; rows that come out so, though their sums of probabilities are numbers, are formed again
// here, over what they see alone.  64 frames at a time: scores with a frame a lane, then eight columns of a frame a lane; o: columns 8 (lane % (DP / 8)) ...
// It ends should the sum be no number, which all results then are.  A bad value makes such rows of all that see it, 32 of them one after the other, and
// each waits for its loads, so that many are under way at once: 8192 frames, 8 heads of 64, an infinite value among all that a frame sees: 7.8 ms (46 with
// four frames' values under way), 0.13 without.
template <typename E, int DP, typename Where>
__device__ void plain_row(const char* q, int D, float c2, int from0, int to0, int from, int to, Where where, float* m, float* l, float* o)
{
    constexpr int kPieces = DP / 8, kAtOnce = kWave / kPieces, kAhead = kPieces < 8 ? kPieces : 8;
    const int lane = (int)threadIdx.x % kWave;
    const int piece = lane % kPieces, row = lane / kPieces, column = piece * 8 < D ? piece * 8 : 0;
    float top = LAST_NEG_INF, sum = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = 0.f;
    for (int part = 0; part < 2 && sum == sum; ++part) {
        const int end = part ? to : to0;
        for (int s0 = part ? from : from0; s0 < end; s0 += kWave) {
            const int n = end - s0 < kWave ? end - s0 : kWave;
            const KeyValue at = where(s0 + (lane < n ? lane : n - 1));
            float dot = 0.f;
            if (at.k) {
#pragma unroll kAhead
                for (int j = 0; j < kPieces; ++j) {
                    const int c = j * 8 < D ? j * 8 : 0;
                    float x[8], y[8];
                    unpack<E>(Raw<E>{*(const u4_any*)(q + c * 2)}, x);
                    unpack<E>(Raw<E>{*(const u4_any*)(at.k + c * 2)}, y);
                    float t = dot;
#pragma unroll
                    for (int k = 0; k < 8; ++k) t = __builtin_fmaf(x[k], y[k], t);
                    dot = j * 8 < D ? t : dot;
                }
            }
            dot = lane >= n ? LAST_NEG_INF : at.k ? dot : __uint_as_float(0x7fc00000u);
            const float higher = fmaxf(top, wave_max(dot)), by = higher == LAST_NEG_INF ? 0.f : higher;
            const float old = __builtin_amdgcn_exp2f((top - by) * c2), p = __builtin_amdgcn_exp2f((dot - by) * c2);
            top = higher;
            sum = sum * old + wave_sum(p);
            if (__any(!(sum == sum))) break;
            u4 w[kPieces];
#pragma unroll
            for (int i = 0; i < kPieces; ++i) w[i] = *(const u4_any*)(of_lane(at.v, row + i * kAtOnce) + column * 2);
#pragma unroll
            for (int k = 0; k < 8; ++k) o[k] *= old;
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int r = row + i * kAtOnce;
                const unsigned keep = r < n ? ~0u : 0u;
                const float pr = __shfl(p, r, kWave);
                float v[8];
                unpack<E>(Raw<E>{w[i] & u4{keep, keep, keep, keep}}, v);
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = __builtin_fmaf(pr, v[k], o[k]);
            }
        }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
#pragma unroll
        for (int x = kPieces; x < kWave; x <<= 1) o[k] += __shfl_xor(o[k], x, kWave);
    *m = top;
    *l = sum;
}

// What a lane's frame sees: [lo, hi) and first frames.  Frames are told apart by one unsigned comparison; first ones only in tiles that have any.
struct Sight {
    int lo, hi, sinks;
    // scores of 32 frames from s0 on; what is not seen becomes `other`
    template <bool FIRSTS = true>
    __device__ __forceinline__ void apply(f16x& s, int s0, float other) const
    {
        const unsigned span = hi > lo ? (unsigned)(hi - lo) : 0u;
        const int from = s0 + result_row(0) - lo;
        if (FIRSTS && s0 < sinks) {
            const int end = hi < sinks ? hi : sinks;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int c = 8 * (i >> 2) + (i & 3);
                s[i] = (unsigned)(from + c) < span || c < end - (s0 + result_row(0)) ? s[i] : other;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = (unsigned)(from + 8 * (i >> 2) + (i & 3)) < span ? s[i] : other;
        }
    }
};

// frame t of an item of len frames, in a band
__device__ __forceinline__ Sight sight_of(int t, int len, const Band& band)
{
    Sight s;
    s.lo = t - band.left;
    s.hi = t >= len ? 0 : t + band.right + 1 < len ? t + band.right + 1 : len;
    s.sinks = band.sinks;
    return s;
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
    // raises m to the maximum of scores of N blocks of 32 frames, -inf where not seen, if they pass it
    template <int N>
    __device__ __forceinline__ void raise(const f16x* s, float c2)
    {
        float top = s[0][0];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
        top = max_of_halves(top);
        // The maximum is only a reference: as long as no score passes it by a factor of 2^8 the sums keep it, which saves their scaling.
        if (__any(((top - m) * c2 > 8.f) | ((m == LAST_NEG_INF) & (top > m)))) {
            const float higher = fmaxf(m, top), old = m == LAST_NEG_INF ? 0.f : __builtin_amdgcn_exp2f((m - higher) * c2);
            m = higher;
            l *= old;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) {
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] *= old;
                in_place(acc[d]);
            }
        }
    }
    // the scores become probabilities relative to m
    template <int N>
    __device__ __forceinline__ void take(f16x* s, float c2)
    {
        raise<N>(s, c2);
        l += powers<N>(s, c2, m == LAST_NEG_INF ? 0.f : m * c2);
    }
    // scores become probabilities relative to an exponent; their sum
    template <int N>
    __device__ __forceinline__ float powers(f16x* s, float c2, float by) const
    {
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][i], c2, -by));
                sum[i % 4] += s[n][i];
            }
        return (sum[0] + sum[1]) + (sum[2] + sum[3]);
    }
    // whether a result is no number (or would be for another frame's sake)
    __device__ __forceinline__ bool not_finite() const
    {
        float t = 0.f;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) t += acc[d][i] * 0.f;
        t = sum_of_halves(t);
        return !(t == 0.f);
    }
};

// what a workgroup works on
struct Place {
    int tile, head, kv, item, len;
    size_t row0;                     // of the item
};

// Workgroups i, i + 8, ... run on one XCD: those of a head do, eight heads (or heads that share keys) at a time, so that its keys and values are
// in one L2; what is left of fewer than eight goes over all.  Those that have most to do where there is no window come first: the last queries, the first keys.
__device__ __forceinline__ Place place_of(const AttentionArgs& a, unsigned id, int heads, bool keys = false)
{
    Place p;
    const unsigned units = (unsigned)(a.B * heads) / a.together, per = a.tiles * a.together;
    unsigned unit, rest;
    if (id < units / 8 * 8 * per) {
        unit = id / (8 * per) * 8 + id % 8;
        rest = id % (8 * per) / 8;
    } else {
        unit = id / per;
        rest = id % per;
    }
    const unsigned hb = unit * a.together + rest / a.tiles;
    p.tile = (int)(keys ? rest % a.tiles : a.tiles - 1 - rest % a.tiles);
    p.head = (int)(hb % (unsigned)heads);
    p.item = (int)(hb / (unsigned)heads);
    p.kv = p.head / (heads / a.kv_heads);
    p.len = frames_of_item(a.len, a.T, p.item);
    p.row0 = (size_t)p.item * a.T;
    return p;
}

// The order of a workgroup's tiles: first those of which some of its frames see not all, in order, then in a loop of its own, which looks at no limits, the
// others, tiles low .. low + full - 1.  (Limits looked at for each tile: a third of the vector instructions of a tile that needs none, since
// the compiler forms masks before it branches, and copies what they may change.)
struct Order {
    int firsts, first, low, full, some;          // firsts: 1 if tile 0 is there for first frames, before those from `first` on
    // own frames [g0, end) see, or are seen by, frames from - t .. to + t, of which [lo, hi) are there for any of them
    __device__ __forceinline__ Order(int g0, int end, long long from, long long to, int lo, int hi, int len, int firsts_)
    {
        firsts = hi > 0 ? firsts_ : 0;
        first = lo / kTile > firsts ? lo / kTile : firsts;
        const int last = (hi + kTile - 1) / kTile, tiles = firsts + (last > first ? last - first : 0);
        const long long all_from = end - 1 - from, all_to = g0 + to + 1;
        low = all_from > 0 ? (int)((all_from + kTile - 1) / kTile) : 0;
        low = low > first ? low : first;
        const int high = (int)(all_to < len ? all_to : len) / kTile;
        full = last > first && high > low ? high - low : 0;
        some = tiles - full;
    }
    __device__ __forceinline__ int tiles() const { return some + full; }
    // where tile i of the order begins
    __device__ __forceinline__ int start(int i) const
    {
        if (i < firsts) return i * kTile;
        const int n = i - firsts + first;
        return (i >= some ? low + i - some : n < low ? n : n + full) * kTile;
    }
};

// HALVES: a workgroup has 64 frames instead of 128, and two wavefronts for each 32 of them, one for either half of each tile, whose sums are joined at the end:
// twice as many workgroups of half the length.
// A tile of 64 columns is 16 products of 32 clocks for a SIMD, and 133 vector instructions beside them, 32 of them exponentials of 8 clocks.  Of 128
// columns: 900 TF (8 x 2048 frames, 16 heads, all seen; the matrix cores are busy 42% of the time, at 1.8 GHz); of 64: 660 TF (64 x 1024, 8 heads; 38%).
// At 128 columns neither the vector units (0.08 instructions a clock) nor LDS (31 %) is what that waits for, but the order of a wavefront's work: products, exponentials
// and products of a tile one after the other, nothing of the next one meanwhile.
// Measured and left: 64 frames a wavefront, half the LDS reads but one wavefront a SIMD (8192 frames, 16 heads of 128: 182 us, so 110); a
// block of 32 of the tile at a time (16 x 1000, 8 heads of 64: 59 us, so 53).
template <typename E, int DP, bool HALVES>
__global__ __launch_bounds__(256, DP == 128 ? 2 : 3) void attention_kernel(AttentionArgs a)
{
    constexpr int kGroup = HALVES ? 64 : 128, kBlocks = HALVES ? 1 : 2;
    __shared__ __attribute__((aligned(16))) char lds[2][2 * Rows<DP>::kBytes];
    __shared__ float stats[HALVES ? 2 : 1][2][32];
    const Place at = place_of(a, a.first + blockIdx.x, a.heads);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x % kWave;
    const int half = HALVES ? wave / 2 : 0;
    const int g0 = at.tile * kGroup, t0 = g0 + (HALVES ? wave % 2 : wave) * 32, t = t0 + (lane & 31);
    const Band band = a.band;
    const float c2 = band.scale * kLog2e;
    const bool there = t < at.len;
    const size_t row = at.row0 + t;
    const char* const q = (const char*)a.q + (at.row0 * a.pq + (size_t)at.head * a.D) * 2;
    const char* const k = (const char*)a.k + (at.row0 * a.pk + (size_t)at.kv * a.D) * 2;
    const char* const v = (const char*)a.v + (at.row0 * a.pv + (size_t)at.kv * a.D) * 2;
    u4 qf[DP / 16];
    own_rows<DP>(there ? q + (size_t)t * a.pq * 2 : nullptr, a.D, qf);
    // frames that the workgroup's see: first ones, and [lo, hi)
    const int lo = g0 - band.left > 0 ? g0 - band.left : 0;
    const int hi = g0 >= at.len ? 0 : g0 + kGroup + band.right < at.len ? g0 + kGroup + band.right : at.len;
    const Order order(g0, g0 + kGroup < at.len ? g0 + kGroup : at.len, band.left, band.right, lo, hi, at.len, band.sinks > 0);
    const int some = order.some, tiles = order.tiles();
    const auto exists = [&](int s) { return (s < hi) & ((s >= lo) | (s < band.sinks)); };
    const Sight sight = sight_of(t, at.len, band);
    Softmax<DP> soft;
    soft.init();
    Tile<DP, 256> ks, vs;
    Reads<DP> reads;
    reads.init();
    const auto get = [&](int s0) {
        const bool all = s0 >= lo && s0 + kTile <= hi;
        ks.send(k, a.pk, a.D, s0, all, hi - 1, exists);
        vs.send(v, a.pv, a.D, s0, all, hi - 1, exists);
    };
    if (tiles > 0) get(order.start(0));
    have(qf);
    // N blocks of 32 of a tile's frames, from block `n0` on
    const auto scores = [&](const char* kt, int n0, auto N, f16x* s) {
#pragma unroll
        for (int n = 0; n < N; ++n) s[n] = zeros16();
#pragma unroll
        for (int i = 0; i < DP / 16; ++i)
#pragma unroll
            for (int n = 0; n < N; ++n) s[n] = Mma<E>::go(reads.along_rows(kt, n0 + n, i), qf[i], s[n]);
    };
    const auto multiply = [&](const char* vt, int n0, auto N, f16x* s) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            u4 p[2];
            to_operands<E>(s[n], p);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) soft.acc[d] = Mma<E>::go(reads.along_columns(vt, d, 2 * (n0 + n) + i), p[i], soft.acc[d]);
        }
    };
    typedef std::integral_constant<int, 1> One;
    typedef std::integral_constant<int, kBlocks> All;
    for (int j = 0; j < some; ++j) {
        const int s0 = order.start(j);
        char *const kt = lds[j & 1], *const vt = kt + Rows<DP>::kBytes;
        ks.lay(kt, a.D, s0, exists);
        vs.lay(vt, a.D, s0, exists);
        __syncthreads();                             // (the other buffer is written again after the next one)
        if (j + 1 < tiles) get(order.start(j + 1));
        if (t0 >= at.len) continue;
        // blocks of which anything is seen
        const auto unseen = [&](int n) { return s0 + 32 * n >= t0 + 32 + band.right || (s0 + 32 * n + 32 <= t0 - band.left && s0 + 32 * n >= band.sinks); };
        int n = HALVES ? half : 0, end = HALVES ? half + 1 : 2;
        if (unseen(n)) ++n;
        if (n < end && unseen(end - 1)) --end;
#pragma unroll 1
        for (; n < end; ++n) {
            f16x s;
            scores(kt, n, One{}, &s);
            sight.apply(s, s0 + 32 * n, LAST_NEG_INF);
            soft.template take<1>(&s, c2);
            multiply(vt, n, One{}, &s);
        }
    }
    // Relative to the reference there is, without a look at the maximum.  Where that gives a sum that is none (no reference yet: the exponent is
    // -inf) or beyond 2^15, which a type of 16 bits holds, the loop is left to raise the reference, and entered again with the same tile.
    const bool whole = a.D == DP;
    float by = soft.m * c2;
    bool raised = false;
    for (int j = some; j < tiles;) {
        char *kt = lds[j & 1], *vt = kt + Rows<DP>::kBytes;
        f16x s[kBlocks];
        for (; j < tiles; ++j) {
            kt = lds[j & 1];
            vt = kt + Rows<DP>::kBytes;
            if (!raised) {
                if (!whole) {
                    ks.clear(a.D);
                    vs.clear(a.D);
                }
                ks.lay(kt);
                vs.lay(vt);
                __syncthreads();
                if (j + 1 < tiles) {
                    const int s0 = (order.low + j + 1 - some) * kTile;
                    ks.send_all(k, a.pk, a.D, s0);
                    vs.send_all(v, a.pv, a.D, s0);
                }
            }
            scores(kt, half, All{}, s);
            const float sum = soft.template powers<kBlocks>(s, c2, by);
            if (!raised && __any(!(sum <= 0x1p15f))) break;
            raised = false;
            by = soft.m * c2;                        // (again -inf where all scores were)
            soft.l += sum;
            multiply(vt, half, All{}, s);
        }
        if (j >= tiles) break;
        scores(kt, half, All{}, s);
        soft.template raise<kBlocks>(s, c2);
        by = soft.m == LAST_NEG_INF ? 0.f : soft.m * c2;
        raised = true;
    }
    float l = sum_of_halves(soft.l);
    if constexpr (HALVES) {
        // the second half's sums, relative to the larger maximum
        float* const sums = (float*)lds[0] + wave % 2 * (DP / 32 * 16 * kWave);
        __syncthreads();
        if (half == 1) {
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[(d * 16 + i) * kWave + lane] = soft.acc[d][i];
            if (lane < 32) {
                stats[wave % 2][0][lane] = soft.m;
                stats[wave % 2][1][lane] = l;
            }
        }
        __syncthreads();
        if (half == 1) return;
        const float m1 = stats[wave % 2][0][lane & 31], l1 = stats[wave % 2][1][lane & 31];
        const float m = fmaxf(soft.m, m1), by = m == LAST_NEG_INF ? 0.f : m;
        const float f0 = __builtin_amdgcn_exp2f((soft.m - by) * c2), f1 = __builtin_amdgcn_exp2f((m1 - by) * c2);
        soft.m = m;
        l = l * f0 + l1 * f1;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) soft.acc[d][i] = soft.acc[d][i] * f0 + sums[(d * 16 + i) * kWave + lane] * f1;
    }
    // (a sum has no part of what is not seen: one that is no number makes a row that is none, as it stands)
    const bool odd = there && l == l && soft.not_finite();
    if (t < a.T && !odd) {
        put_rows<E, DP>((char*)a.y + (row * a.py + (size_t)at.head * a.D) * 2, a.D, soft.acc, 1.f / l, there);
        if (a.lse && lane < 32) a.lse[row * a.heads + at.head] = there ? (soft.m * c2 + __builtin_amdgcn_logf(l)) * kLn2 : 0.f;
    }
    for (unsigned long long rows = __ballot(odd) & 0xffffffffull; rows; rows &= rows - 1) {
        const int tr = t0 + __ffsll(rows) - 1;
        const int end = tr + band.right + 1 < at.len ? tr + band.right + 1 : at.len;
        float m, sum, o[8];
        const int firsts = band.sinks < end ? band.sinks : end, from = tr - band.left > firsts ? tr - band.left : firsts;
        plain_row<E, DP>(q + (size_t)tr * a.pq * 2, a.D, c2, 0, firsts, from, end, [&](int s) { return KeyValue{k + (size_t)s * a.pk * 2, v + (size_t)s * a.pv * 2}; },
                     &m, &sum, o);
        char* const y = (char*)a.y + (((at.row0 + tr) * a.py) + (size_t)at.head * a.D) * 2;
        if (lane < DP / 8 && lane * 8 < a.D) {
#pragma unroll
            for (int c = 0; c < 8; ++c) Elt<E>::put(y, lane * 8 + c, o[c] / sum);
        }
        if (a.lse && lane == 0) a.lse[(at.row0 + tr) * a.heads + at.head] = (m * c2 + __builtin_amdgcn_logf(sum)) * kLn2;
    }
}

// a lane's own row's scalar product of two rows of 16 bits that both halves have alternate pieces of
template <typename E, int N>
__device__ __forceinline__ float row_product(const u4 (&x)[N], const u4 (&y)[N])
{
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float a[8], b[8];
        unpack<E>(Raw<E>{x[k]}, a);
        unpack<E>(Raw<E>{y[k]}, b);
#pragma unroll
        for (int c = 0; c < 8; ++c) sum = __builtin_fmaf(a[c], b[c], sum);
    }
    return sum_of_halves(sum);
}

// The gradient of queries: a wavefront's own frames are queries, the tiles keys and values.  It comes first, and leaves delta for the others (a kernel of its
// own for delta: 7 us of 81 at 16 x 1024 frames, 8 heads of 64 in a band).  Three products a tile; 225 to 242 us at 2 x 4096, 16 heads of 128 that see 2047
// back (660 TF), bound by waits for LDS: with 253 registers in use nothing is read more than a product ahead (43 complete waits among 48 products).  In float16
// 128 columns spill 196 registers: the whole gradient 677 us where it is 560 in bfloat16.
template <typename E, int DP, bool HALVES>
__global__ __launch_bounds__(256, 2) void grad_query_kernel(AttentionArgs a)
{
    constexpr int kGroup = HALVES ? 64 : kOwn;
    __shared__ __attribute__((aligned(16))) char lds[2][2 * Rows<DP>::kBytes];
    const Place at = place_of(a, a.first + blockIdx.x, a.heads);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x % kWave;
    const int half = HALVES ? wave / 2 : 0;
    const int g0 = at.tile * kGroup, t0 = g0 + (HALVES ? wave % 2 : wave) * 32, t = t0 + (lane & 31);
    const Band band = a.band;
    const float c2 = band.scale * kLog2e;
    const bool there = t < at.len;
    const size_t row = at.row0 + t;
    const char* const k = (const char*)a.k + (at.row0 * a.pk + (size_t)at.kv * a.D) * 2;
    const char* const v = (const char*)a.v + (at.row0 * a.pv + (size_t)at.kv * a.D) * 2;
    u4 qf[DP / 16], df[DP / 16];
    own_rows<DP>(there ? (const char*)a.q + (row * a.pq + (size_t)at.head * a.D) * 2 : nullptr, a.D, qf);
    own_rows<DP>(there ? (const char*)a.dy + (row * a.pdy + (size_t)at.head * a.D) * 2 : nullptr, a.D, df);
    float l2 = there ? a.lse[row * a.heads + at.head] * kLog2e : 0.f, delta;
    {
        u4 yf[DP / 16];
        own_rows<DP>(there ? (const char*)a.y + (row * a.py + (size_t)at.head * a.D) * 2 : nullptr, a.D, yf);
        delta = row_product<E>(df, yf);
        if (there && lane < 32 && half == 0) a.delta[row * a.heads + at.head] = delta;
    }
    const int lo = g0 - band.left > 0 ? g0 - band.left : 0;
    const int hi = g0 >= at.len ? 0 : g0 + kGroup + band.right < at.len ? g0 + kGroup + band.right : at.len;
    const Order order(g0, g0 + kGroup < at.len ? g0 + kGroup : at.len, band.left, band.right, lo, hi, at.len, band.sinks > 0);
    const int some = order.some, tiles = order.tiles();
    const auto exists = [&](int s) { return (s < hi) & ((s >= lo) | (s < band.sinks)); };
    const Sight sight = sight_of(t, at.len, band);
    f16x acc[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) acc[d] = zeros16();
    Tile<DP, 256> ks, vs;
    Reads<DP> reads;
    reads.init();
    const auto get = [&](int s0) {
        const bool all = s0 >= lo && s0 + kTile <= hi;
        ks.send(k, a.pk, a.D, s0, all, hi - 1, exists);
        vs.send(v, a.pv, a.D, s0, all, hi - 1, exists);
    };
    if (tiles > 0) get(order.start(0));
    have(qf);
    have(df);
    asm volatile("" : "+v"(l2), "+v"(delta));
    const auto turn = [&](const char* kt, const char* vt, auto limits, bool all, int s0, int from, int to) {
        constexpr int kAtOnce = limits || HALVES ? 1 : 2;
#pragma unroll kAtOnce
        for (int n = from; n < to; ++n) {
            f16x s = zeros16(), p = zeros16();
#pragma unroll
            for (int i = 0; i < DP / 16; ++i) {
                s = Mma<E>::go(reads.along_rows(kt, n, i), qf[i], s);
                p = Mma<E>::go(reads.along_rows(vt, n, i), df[i], p);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c2, -l2)) * (p[i] - delta);
            }
            if constexpr (limits) {
                in_place(s);
                if (!all) {
                    sight.apply(s, s0 + 32 * n, 0.f);
                    in_place(s);
                }
            }
            u4 d[2];
            to_operands<E>(s, d);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int x = 0; x < DP / 32; ++x) acc[x] = Mma<E>::go(reads.along_columns(kt, x, 2 * n + i), d[i], acc[x]);
        }
    };
    for (int j = 0; j < some; ++j) {
        const int s0 = order.start(j);
        char *const kt = lds[j & 1], *const vt = kt + Rows<DP>::kBytes;
        ks.lay(kt, a.D, s0, exists);
        vs.lay(vt, a.D, s0, exists);
        __syncthreads();
        if (j + 1 < tiles) get(order.start(j + 1));
        if (s0 >= t0 + 32 + band.right || t0 >= at.len || (s0 + kTile <= t0 - band.left && s0 >= band.sinks)) continue;
        const bool all = s0 >= t0 + 31 - band.left && s0 + kTile - 1 <= t0 + band.right && s0 + kTile <= at.len;
        int from = s0 + 32 <= t0 - band.left && s0 >= band.sinks ? 1 : 0, to = s0 + 32 >= t0 + 32 + band.right ? 1 : 2;
        if (HALVES) {
            from = from > half ? from : half;
            to = to < half + 1 ? to : half + 1;
        }
        turn(kt, vt, std::true_type{}, all, s0, from, to);
    }
    for (int j = some; j < tiles; ++j) {
        char *const kt = lds[j & 1], *const vt = kt + Rows<DP>::kBytes;
        if (a.D != DP) {
            ks.clear(a.D);
            vs.clear(a.D);
        }
        ks.lay(kt);
        vs.lay(vt);
        __syncthreads();
        if (j + 1 < tiles) {
            const int s0 = (order.low + j + 1 - some) * kTile;
            ks.send_all(k, a.pk, a.D, s0);
            vs.send_all(v, a.pv, a.D, s0);
        }
        turn(kt, vt, std::false_type{}, true, 0, half, HALVES ? half + 1 : 2);
    }
    if constexpr (HALVES) {
        float* const sums = (float*)lds[0] + wave % 2 * (DP / 32 * 16 * kWave);
        __syncthreads();
        if (half == 1) {
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[(d * 16 + i) * kWave + lane] = acc[d][i];
        }
        __syncthreads();
        if (half == 1) return;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[d][i] += sums[(d * 16 + i) * kWave + lane];
    }
    if (t < a.T) put_rows<E, DP>((char*)a.dq + (row * a.pdq + (size_t)at.head * a.D) * 2, a.D, acc, band.scale, there);
}

// What a tile of 64 queries and their dy adds to the gradients of a wavefront's 32 keys (DK) and values (DV); of blocks from .. to - 1 of its 32 queries.
// LIMITS: not all of them may see the wavefront's.
template <typename E, int DP, bool DK, bool DV, bool LIMITS>
__device__ __forceinline__ void key_tile(const char* qt, const char* yt, const float* st, const Reads<DP>& reads, const u4 (&kf)[DP / 16],
                                         const u4 (&vf)[DP / 16], float c2, const Sight& sight, int t0, int from, int to, f16x* dk, f16x* dv)
{
    const int h = (int)threadIdx.x % kWave >> 5;
    // (both gradients' sums and operands leave no registers for two blocks at a time)
#pragma unroll 1
    for (int n = from; n < to; ++n) {
        f16x p = zeros16(), e = zeros16();
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            p = Mma<E>::go(reads.along_rows(qt, n, i), kf[i], p);
            if constexpr (DK) e = Mma<E>::go(reads.along_rows(yt, n, i), vf[i], e);
        }
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const f4 l2 = *(const f4*)&st[32 * n + 2 * i + 4 * h];
            f4 delta{};
            if constexpr (DK) delta = *(const f4*)&st[kTile + 32 * n + 2 * i + 4 * h];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                p[i + x] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[i + x], c2, -l2[x]));
                if constexpr (DK) e[i + x] = p[i + x] * (e[i + x] - delta[x]);
            }
        }
        if constexpr (LIMITS) {
            if constexpr (DV) sight.apply<false>(p, t0 + 32 * n, 0.f);
            if constexpr (DK) sight.apply<false>(e, t0 + 32 * n, 0.f);
        }
        u4 f[2];
        if constexpr (DV) {
            to_operands<E>(p, f);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) dv[d] = Mma<E>::go(reads.along_columns(yt, d, 2 * n + i), f[i], dv[d]);
        }
        if constexpr (DK) {
            to_operands<E>(e, f);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) dk[d] = Mma<E>::go(reads.along_columns(qt, d, 2 * n + i), f[i], dk[d]);
        }
    }
}

// The gradients of keys (DK) and values (DV): a wavefront's own frames are keys, the tiles queries and their dy, of the heads that share the keys, or
// of a part of them, whose sums grad_join_kernel adds (1 x 4096, 16 heads of 128 on one: the whole gradient 2522 us undivided, 434 in 16 parts).  No
// atomics: every sum has one order.
template <typename E, int DP, bool DK, bool DV, bool HALVES>
__device__ __forceinline__ void grad_key(const AttentionArgs& a, const Place& at, char (*lds)[2 * Rows<DP>::kBytes], float (*stats)[2][kTile])
{
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x % kWave;
    const Band band = a.band;
    constexpr int kGroup = HALVES ? 64 : kOwn;
    const int half = HALVES ? wave / 2 : 0;
    const int g0 = at.tile * kGroup, s0 = g0 + (HALVES ? wave % 2 : wave) * 32, s = s0 + (lane & 31);
    const float c2 = band.scale * kLog2e;
    const bool there = s < at.len;
    const size_t row = at.row0 + s;
    const int group = a.heads / a.kv_heads, part = at.head % a.parts;
    const int from = at.kv * group + group * part / a.parts, to = at.kv * group + group * (part + 1) / a.parts;
    u4 kf[DP / 16], vf[DP / 16];
    own_rows<DP>(there ? (const char*)a.k + (row * a.pk + (size_t)at.kv * a.D) * 2 : nullptr, a.D, kf);
    if constexpr (DK) own_rows<DP>(there ? (const char*)a.v + (row * a.pv + (size_t)at.kv * a.D) * 2 : nullptr, a.D, vf);
    // frames that see the workgroup's
    const int lo = g0 - band.right > 0 ? g0 - band.right : 0;
    const int hi = g0 >= at.len ? 0 : (long long)g0 + kGroup + band.left < at.len ? g0 + kGroup + band.left : at.len;
    const Order order(g0, g0 + kGroup < at.len ? g0 + kGroup : at.len, band.right, band.left, lo, hi, at.len, 0);
    const int some = order.some;
    const auto exists = [&](int t) { return (t >= lo) & (t < hi); };
    // t sees s: s - right <= t <= s + left
    const Sight sight{s - band.right, !there ? 0 : (long long)s + band.left + 1 < at.len ? s + band.left + 1 : at.len, 0};
    f16x dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) dk[d] = dv[d] = zeros16();
    Tile<DP, 256> qs, ys;
    Reads<DP> reads;
    reads.init();
    float stat = 0.f;
    const auto get_stat = [&](int head, int t) {
        const size_t i = (at.row0 + t) * a.heads + head;
        stat = *(threadIdx.x < kTile ? a.lse + i : a.delta + i);
    };
    const auto lay_stat = [&](float* st) {
        if (threadIdx.x < 2 * kTile) st[threadIdx.x] = threadIdx.x < kTile ? stat * kLog2e : stat;
    };
    const auto get = [&](int head, int t0) {
        const bool all = t0 >= lo && t0 + kTile <= hi;
        qs.send((const char*)a.q + (at.row0 * a.pq + (size_t)head * a.D) * 2, a.pq, a.D, t0, all, hi - 1, exists);
        ys.send((const char*)a.dy + (at.row0 * a.pdy + (size_t)head * a.D) * 2, a.pdy, a.D, t0, all, hi - 1, exists);
        const int t = t0 + (int)threadIdx.x % kTile;
        stat = 0.f;
        if (threadIdx.x < 2 * kTile && exists(t)) get_stat(head, t);
    };
    // (of all heads first the tiles of which not all is seen, then the others)
    const int turns = some * (to - from), all_turns = order.full * (to - from);
    if (turns + all_turns > 0) get(from, order.start(0));
    have(kf);
    if constexpr (DK) have(vf);
    int head = from, i = 0;
    for (int j = 0; j < turns; ++j) {
        const int t0 = order.start(i);
        char *const qt = lds[j & 1], *const yt = qt + Rows<DP>::kBytes;
        float* const st = stats[j & 1][0];
        qs.lay(qt, a.D, t0, exists);
        ys.lay(yt, a.D, t0, exists);
        lay_stat(st);
        __syncthreads();
        if (++i == some) {
            i = 0;
            ++head;
        }
        const bool more = j + 1 < turns;
        if (more || all_turns > 0) get(more ? head : from, more ? order.start(i) : order.low * kTile);
        if (s0 >= at.len || t0 + kTile <= s0 - band.right || t0 > (long long)s0 + 31 + band.left) continue;
        int from_block = t0 + 32 <= s0 - band.right ? 1 : 0, to_block = t0 + 32 > (long long)s0 + 31 + band.left ? 1 : 2;
        if (HALVES) {
            from_block = from_block > half ? from_block : half;
            to_block = to_block < half + 1 ? to_block : half + 1;
        }
        key_tile<E, DP, DK, DV, true>(qt, yt, st, reads, kf, vf, c2, sight, t0, from_block, to_block, dk, dv);
    }
    head = from;
    i = 0;
    for (int j = turns; j < turns + all_turns; ++j) {
        char *const qt = lds[j & 1], *const yt = qt + Rows<DP>::kBytes;
        float* const st = stats[j & 1][0];
        if (a.D != DP) {
            qs.clear(a.D);
            ys.clear(a.D);
        }
        qs.lay(qt);
        ys.lay(yt);
        lay_stat(st);
        __syncthreads();
        if (++i == order.full) {
            i = 0;
            ++head;
        }
        if (j + 1 < turns + all_turns) {
            const int t0 = (order.low + i) * kTile;
            qs.send_all((const char*)a.q + (at.row0 * a.pq + (size_t)head * a.D) * 2, a.pq, a.D, t0);
            ys.send_all((const char*)a.dy + (at.row0 * a.pdy + (size_t)head * a.D) * 2, a.pdy, a.D, t0);
            if (threadIdx.x < 2 * kTile) get_stat(head, t0 + (int)threadIdx.x % kTile);
        }
        key_tile<E, DP, DK, DV, false>(qt, yt, st, reads, kf, vf, c2, sight, 0, half, HALVES ? half + 1 : 2, dk, dv);
    }
    if constexpr (HALVES) {
        const auto join = [&](float* all, f16x* sums) {
            float* const other = all + wave % 2 * (DP / 32 * 16 * kWave);
            if (half == 1) {
#pragma unroll
                for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) other[(d * 16 + i) * kWave + lane] = sums[d][i];
            }
            __syncthreads();
            if (half == 1) return;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[d][i] += other[(d * 16 + i) * kWave + lane];
        };
        __syncthreads();
        if constexpr (DK) join((float*)lds[0], dk);
        if constexpr (DV) join((float*)lds[1], dv);
        if (half == 1) return;
    }
    if (s >= a.T) return;
    if (a.parts > 1) {
        if (!there) return;
        const size_t at_k = (((size_t)part * a.B * a.T + row) * a.kv_heads + at.kv) * DP, to_v = (size_t)a.parts * a.B * a.T * a.kv_heads * DP;
        const auto keep = [&](float* out, const f16x* sums) {
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4) *(f4*)(out + 32 * d + result_row(i)) = f4{sums[d][i], sums[d][i + 1], sums[d][i + 2], sums[d][i + 3]};
        };
        if constexpr (DK) keep(a.kept + at_k, dk);
        if constexpr (DV) keep(a.kept + to_v + at_k, dv);
        return;
    }
    // what frames beyond the window add to first ones
    const auto add_first = [&](f16x* sums, int which) {
        if (!a.part || !(there && s < band.sinks)) return;
        const float* const in = a.sums + ((((size_t)at.item * a.kv_heads + at.kv) * 2 + which) * kMostSinks + s) * DP;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const f4 x = *(const f4*)(in + 32 * d + result_row(i));
#pragma unroll
                for (int c = 0; c < 4; ++c) sums[d][i + c] += x[c];
            }
    };
    if constexpr (DK) {
        add_first(dk, 0);
        put_rows<E, DP>((char*)a.dk + (row * a.pdk + (size_t)at.kv * a.D) * 2, a.D, dk, band.scale, there);
    }
    if constexpr (DV) {
        add_first(dv, 1);
        put_rows<E, DP>((char*)a.dv + (row * a.pdv + (size_t)at.kv * a.D) * 2, a.D, dv, 1.f, there);
    }
}

// HALVES: as in attention_kernel.  APART: workgroups of a second half form the values' gradients, those of the first the keys', since both sums and operands of 128 columns do not leave
// registers for two wavefronts on a SIMD; the scores are formed twice, which is a product of five (8 x 2048 frames, 16 heads: the whole gradient
// 1503 us with both in one, 1185 apart).  368 to 389 us at 2 x 4096, 16 heads that see 2047 back: 660 TF with the scores counted twice; bound by waits for LDS
// (25 among 24 products).  HALVES and APART spill 14 registers (15 in float16).
template <typename E, int DP, bool APART, bool HALVES>
__global__ __launch_bounds__(256, 2) void grad_key_kernel(AttentionArgs a)
{
    __shared__ __attribute__((aligned(16))) char lds[2][2 * Rows<DP>::kBytes];
    __shared__ float stats[2][2][kTile];
    const unsigned id = a.first + blockIdx.x;
    if constexpr (APART) {
        if (id >= a.half) grad_key<E, DP, false, true, HALVES>(a, place_of(a, id - a.half, a.kv_heads * a.parts, true), lds, stats);
        else grad_key<E, DP, true, false, HALVES>(a, place_of(a, id, a.kv_heads * a.parts, true), lds, stats);
    } else {
        grad_key<E, DP, true, true, HALVES>(a, place_of(a, id, a.kv_heads * a.parts, true), lds, stats);
    }
}

// The part that first frames s < sinks have in frames t > s + left: a workgroup takes a chunk of these of one head, a wavefront 32 first frames and half
// of each tile (in grad_key_kernel's workgroup of the first frames, which then goes over all of the item, 146 us at 2 x 4096; here 24, and 5 for the
// join).  Sums go to `part`, [item][kv head][share][2][64][DP], a share for each head of the group, chunk and half.
template <typename E, int DP>
__global__ __launch_bounds__(256, DP == 128 ? 1 : 2) void grad_first_kernel(AttentionArgs a)
{
    __shared__ __attribute__((aligned(16))) char lds[2][2 * Rows<DP>::kBytes];
    __shared__ float stats[2][2][kTile];
    const Place at = place_of(a, a.first + blockIdx.x, a.heads);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x % kWave;
    const Band band = a.band;
    const int s0 = wave % 2 * 32, s = s0 + (lane & 31), half = wave / 2, group = a.heads / a.kv_heads;
    const float c2 = band.scale * kLog2e;
    const bool there = s < at.len && s < band.sinks;
    const size_t row = at.row0 + s;
    u4 kf[DP / 16], vf[DP / 16];
    own_rows<DP>(there ? (const char*)a.k + (row * a.pk + (size_t)at.kv * a.D) * 2 : nullptr, a.D, kf);
    own_rows<DP>(there ? (const char*)a.v + (row * a.pv + (size_t)at.kv * a.D) * 2 : nullptr, a.D, vf);
    const int lo = band.left + 1 < at.len ? band.left + 1 : at.len, hi = at.len;
    const int all_first = lo / kTile, n = lo < hi ? (hi + kTile - 1) / kTile - all_first : 0;
    const int first = all_first + (int)((long long)n * at.tile / (int)a.tiles), last = all_first + (int)((long long)n * (at.tile + 1) / (int)a.tiles);
    const auto exists = [&](int t) { return (t >= lo) & (t < hi); };
    const Sight sight{s + band.left + 1, there ? at.len : 0, 0};
    f16x dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) dk[d] = dv[d] = zeros16();
    Tile<DP, 256> qs, ys;
    Reads<DP> reads;
    reads.init();
    float stat = 0.f;
    const auto get = [&](int t0) {
        const bool all = t0 >= lo && t0 + kTile <= hi;
        qs.send((const char*)a.q + (at.row0 * a.pq + (size_t)at.head * a.D) * 2, a.pq, a.D, t0, all, hi - 1, exists);
        ys.send((const char*)a.dy + (at.row0 * a.pdy + (size_t)at.head * a.D) * 2, a.pdy, a.D, t0, all, hi - 1, exists);
        const int t = t0 + (int)threadIdx.x % kTile;
        stat = 0.f;
        if (threadIdx.x < 2 * kTile && exists(t)) {
            const size_t i = (at.row0 + t) * a.heads + at.head;
            stat = *(threadIdx.x < kTile ? a.lse + i : a.delta + i);
        }
    };
    if (first < last) get(first * kTile);
    have(kf);
    have(vf);
    for (int j = first; j < last; ++j) {
        const int t0 = j * kTile;
        char *const qt = lds[j & 1], *const yt = qt + Rows<DP>::kBytes;
        float* const st = stats[j & 1][0];
        qs.lay(qt, a.D, t0, exists);
        ys.lay(yt, a.D, t0, exists);
        if (threadIdx.x < 2 * kTile) st[threadIdx.x] = threadIdx.x < kTile ? stat * kLog2e : stat;
        __syncthreads();
        if (j + 1 < last) get(t0 + kTile);
        if (s0 >= band.sinks) continue;
        key_tile<E, DP, true, true, true>(qt, yt, st, reads, kf, vf, c2, sight, t0, half, half + 1, dk, dv);
    }
    if (s >= band.sinks) return;
    const int share = ((at.head % group) * (int)a.tiles + at.tile) * 2 + half;
    float* const out = a.part + ((((size_t)at.item * a.kv_heads + at.kv) * a.shares + share) * 2 * kMostSinks + s) * DP;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            *(f4*)(out + 32 * d + result_row(i)) = f4{dk[d][i], dk[d][i + 1], dk[d][i + 2], dk[d][i + 3]};
            *(f4*)(out + kMostSinks * DP + 32 * d + result_row(i)) = f4{dv[d][i], dv[d][i + 1], dv[d][i + 2], dv[d][i + 3]};
        }
}

// Gradients of keys and values from the parts' sums [2][part][row][kv head][DP], in order: four columns a thread.  Bound by reading them: 15 us for two
// parts of 8192 x 4 heads of 128 (75 MB).
template <typename E>
__global__ __launch_bounds__(256) void grad_join_kernel(AttentionArgs a, int DP, long long first)
{
    const int fours = DP / 4;
    const long long i = (first + blockIdx.x) * 256 + threadIdx.x, units = (long long)a.B * a.T * a.kv_heads;
    const long long u = i / fours;
    const int c = (int)(i - u * fours) * 4;
    if (u >= 2 * units || c >= a.D) return;
    const int which = u >= units ? 1 : 0;
    const long long unit = u - which * units, row = unit / a.kv_heads;
    const int kv = (int)(unit - row * a.kv_heads), b = (int)(row / a.T), s = (int)(row - (long long)b * a.T);
    f4 v{};
    if (s < (a.len ? clamped(a.len[b], a.T) : a.T)) {
        for (int part = 0; part < a.parts; ++part) v += *(const f4*)(a.kept + (((size_t)which * a.parts + part) * units + unit) * DP + c);
        if (a.part && s < a.band.sinks) v += *(const f4*)(a.sums + ((((size_t)b * a.kv_heads + kv) * 2 + which) * kMostSinks + s) * DP + c);
        if (which == 0) v *= a.band.scale;
    }
    const float x[4] = {v[0], v[1], v[2], v[3]};
    store4<E>(which ? a.dv : a.dk, (size_t)row * (which ? a.pdv : a.pdk) + (size_t)kv * a.D + c, x);
}

// sums [item][kv head][2][64][DP] of the shares, in order; a workgroup a row
__global__ __launch_bounds__(128) void first_join_kernel(const float* part, float* sums, int shares, int DP, int sinks, long long first)
{
    const long long i = first + blockIdx.x, unit = i / (2 * sinks);
    const int r = (int)(i - unit * 2 * sinks), which = r / sinks, s = r - which * sinks, c = (int)threadIdx.x;
    if (c >= DP) return;
    const float* in = part + ((size_t)unit * shares * 2 * kMostSinks + (size_t)which * kMostSinks + s) * DP + c;
    float t = 0.f;
#pragma unroll 8
    for (int k = 0; k < shares; ++k) t += in[(size_t)k * 2 * kMostSinks * DP];
    sums[(((size_t)unit * 2 + which) * kMostSinks + s) * DP + c] = t;
}

}  // namespace last
