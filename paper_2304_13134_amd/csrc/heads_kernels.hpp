// Norms of the heads' queries and keys with the rotation by their frame's position, and their gradient; the same with its
// results laid into the pages of a cache.
//     inv = 1 / sqrt(mean_c x^2 + eps),  n = x inv gain  (n = x where there is no gain)
//     y_i = n_i cos(p w_i) - n_(i+R/2) sin(p w_i),  y_(i+R/2) = n_(i+R/2) cos(p w_i) + n_i sin(p w_i)  for i < R/2,  y_c = n_c beyond
//     dn = dy rotated back,  u = gain dn,  dx = inv (u - x inv^2 mean_c(u x)),  dgain[c] = sum over frames and heads of dn x inv
// A head's row stands in LN neighbouring lanes, eight columns a lane: four of the first half of the rotated columns with the four
// that they are rotated with, or eight of the rest, so that no column changes lanes.  A wavefront takes 64 / LN heads of a frame at
// a time and keeps the frame's angles, which are the same for all heads.
#pragma once
#include "layer.hpp"

namespace last {

// one of queries, keys and values
struct HeadSide {
    const void* x;
    long long px;
    void* y;                         // null: to the pages
    long long py;
    const float* gain;               // null: not normed
    int heads;
    int turned;                      // whether it is rotated
    char* pages;
};

struct Turn {
    const float* frequencies;        // radians a frame, R / 2 of them
    const int* first;                // position of an item's first frame, or null for 0
    int R;
};

// pages of a cache: [page][kv head][frame of the page][column]
struct Pages {
    const int* table;                // [B][entries]: the page of an item's frames j page ..
    const int* used;                 // [B] frames before this call's
    int pages, page, entries;
    Divisor by_page;
};

struct HeadArgs {
    Frames frames;
    int rows, B;
    int D;
    float eps;
    Turn turn;
    HeadSide side[3];
    int sides, split;                // wavefronts a frame
    Pages cache;
    int* status;                     // [B] or null
};

constexpr int kMostUsed = 1 << 30;   // positions stay in 32 bits

__device__ __forceinline__ int used_frames(const int* used, int b)
{
    const int n = used[b];
    return n < 0 ? 0 : n > kMostUsed ? kMostUsed : n;
}

__device__ __forceinline__ int clamped(int n, int most) { return n < 0 ? 0 : n > most ? most : n; }

// The page that frame s of item b is on, -1 if the table names none that exists.
__device__ __forceinline__ int page_of(const Pages& c, int b, int s, int* row)
{
    const int j = (int)quotient((unsigned)s, c.by_page);
    *row = s - j * c.page;
    if (j >= c.entries) return -1;
    const int p = c.table[(size_t)b * c.entries + j];
    return (unsigned)p < (unsigned)c.pages ? p : -1;
}

// sine and cosine of t turns.  The angle's part beyond whole quarter turns is formed in 64 bits (a position times a frequency has
// more digits than 32 bits hold), at most an eighth of a turn, on which the Taylor series to x^9 and x^8 are good to 3e-8.
__device__ __forceinline__ void sine_cosine(double t, float* sine, float* cosine)
{
    const double f = t - floor(t), k = rint(f * 4.0);
    const int quarter = (int)k;
    const float x = (float)((f - k * 0.25) * 6.283185307179586), s = x * x;
    const float sn = x * (1.f + s * (-1.6666667e-1f + s * (8.3333333e-3f + s * (-1.9841270e-4f + s * 2.7557319e-6f))));
    const float cs = 1.f + s * (-0.5f + s * (4.1666667e-2f + s * (-1.3888889e-3f + s * 2.4801587e-5f)));
    const float a = quarter & 1 ? cs : sn, b = quarter & 1 ? sn : cs;
    *sine = quarter & 2 ? -a : a;
    *cosine = (quarter + 1) & 2 ? -b : b;
}

// which columns a lane of a head holds: c0 .. c0 + 3 and c1 .. c1 + 3
struct HeadLane {
    int c0, c1;
    bool here, turned;
    __device__ HeadLane(int lane, int D, int R)
    {
        here = lane * 8 < D;
        turned = lane * 8 < R;
        c0 = turned ? 4 * lane : 8 * lane;
        c1 = turned ? R / 2 + 4 * lane : 8 * lane + 4;
    }
};

template <typename E> struct Four {
    u2 a;
};
template <> struct Four<float> {
    u4 a;
};
typedef u2 u2_two __attribute__((aligned(2)));
typedef u4 u4_four __attribute__((aligned(4)));

template <typename E>
__device__ __forceinline__ Four<E> raw4(const void* p, size_t i)
{
    Four<E> r;
    if constexpr (Elt<E>::size == 4) r.a = *(const u4_four*)((const float*)p + i);
    else r.a = *(const u2_two*)((const uint16_t*)p + i);
    return r;
}

template <typename E>
__device__ __forceinline__ void unpack4(const Four<E>& r, float* v)
{
    if constexpr (Elt<E>::type == LAST_F32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = __uint_as_float(r.a[k]);
    } else if constexpr (Elt<E>::type == LAST_BF16) {
#pragma unroll
        for (int k = 0; k < 2; ++k) { v[2 * k] = bf16_to_float(r.a[k] & 0xffffu); v[2 * k + 1] = __uint_as_float(r.a[k] & 0xffff0000u); }
    } else {
        typedef _Float16 h4 __attribute__((ext_vector_type(4)));
        const h4 h = __builtin_bit_cast(h4, r.a);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = (float)h[k];
    }
}

template <typename E>
__device__ __forceinline__ void store4(void* p, size_t i, const float* v)
{
    if constexpr (Elt<E>::type == LAST_F32) *(u4_four*)((float*)p + i) = __builtin_bit_cast(u4, f4{v[0], v[1], v[2], v[3]});
    else if constexpr (Elt<E>::type == LAST_BF16) *(u2_two*)((uint16_t*)p + i) = u2{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
    else *(u2_two*)((uint16_t*)p + i) = u2{f16_pair(v[0], v[1]), f16_pair(v[2], v[3])};
}

template <int LN>
__device__ __forceinline__ float head_sum(float v)
{
#pragma unroll
    for (int o = LN / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

// the angles of a frame: of the lane's four pairs
__device__ __forceinline__ void angles(const double* turns, double position, bool turned, float* sn, float* cs)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        sn[k] = 0.f;
        cs[k] = 1.f;
        if (turned) sine_cosine(position * turns[k], &sn[k], &cs[k]);
    }
}

__device__ __forceinline__ void own_turns(const Turn& t, const HeadLane& at, double* turns)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) turns[k] = at.turned ? (double)t.frequencies[at.c0 + k] * 0.15915494309189535 : 0.0;
}

__device__ __forceinline__ void load_gain(const float* gain, const HeadLane& at, float* g)
{
#pragma unroll
    for (int k = 0; k < 8; ++k) g[k] = gain && at.here ? gain[(k < 4 ? at.c0 : at.c1 - 4) + k] : 1.f;
}

__device__ __forceinline__ void rotate8(const float* sn, const float* cs, float sign, float* v)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float a = v[k], b = v[4 + k], s = sign * sn[k];
        v[k] = a * cs[k] - b * s;
        v[4 + k] = b * cs[k] + a * s;
    }
}

// status of the items of a call without frames
__global__ void no_frames_kernel(int* status, int B)
{
    const int b = (int)(blockIdx.x * 256 + threadIdx.x);
    if (b < B) status[b] = kItemOk;
}

// LN: lanes of a head.  A unit of work is every split-th group of 64 / LN heads of a frame.
template <typename E, int LN>
__global__ __launch_bounds__(256) void heads_kernel(HeadArgs a)
{
    constexpr int kAtOnce = kWave / LN;
    const int lane = (int)threadIdx.x % LN, group = (int)threadIdx.x % kWave / LN;
    const int wave = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), waves = (int)gridDim.x * 4;
    const HeadLane at(lane, a.D, a.turn.R);
    double turns[4];
    own_turns(a.turn, at, turns);
    float gq[8], gk[8];
    load_gain(a.side[0].gain, at, gq);
    load_gain(a.side[1].gain, at, gk);
    const int n0 = a.side[0].heads, n1 = n0 + a.side[1].heads, n2 = n1 + a.side[2].heads;
    for (long long unit = wave; unit < (long long)a.rows * a.split; unit += waves) {
        const int row = a.split == 1 ? (int)unit : (int)(unit / a.split), part = (int)(unit - (long long)row * a.split);
        const int b = (int)quotient((unsigned)row, a.frames.by), t = row - b * a.frames.T;
        const int exist = a.frames.len ? a.frames.len[b] : a.frames.T;
        const bool there = t < exist;
        const int first = a.turn.first ? a.turn.first[b] : 0;
        int page = 0, in_page = 0;
        if (a.cache.table) {
            const int used = used_frames(a.cache.used, b);
            page = page_of(a.cache, b, used + t, &in_page);
            if (a.status && t == 0 && part == 0) {
                // every page that the item's new frames go to
                int bad = 0, n = clamped(exist, a.frames.T), r;
                for (int i = (int)threadIdx.x % kWave; i < n; i += kWave) bad |= page_of(a.cache, b, used + i, &r) < 0;
                const bool any = __any(bad);
                if (threadIdx.x % kWave == 0) a.status[b] = any ? kItemBadPage : kItemOk;
            }
        }
        float sn[4], cs[4];
        angles(turns, (double)(a.cache.table ? used_frames(a.cache.used, b) : first) + t, at.turned, sn, cs);
        for (int h0 = part * kAtOnce; h0 < n2; h0 += a.split * kAtOnce) {
            const int head = h0 + group;
            const int which = head < n0 ? 0 : head < n1 ? 1 : 2;
            const HeadSide& s = a.side[which];
            const int h = head - (which == 0 ? 0 : which == 1 ? n0 : n1);
            const bool on = head < n2 && at.here;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0.f;
            if (on && there) {
                const size_t x = (size_t)row * s.px + (size_t)h * a.D;
                unpack4<E>(raw4<E>(s.x, x + at.c0), v);
                unpack4<E>(raw4<E>(s.x, x + at.c1), v + 4);
            }
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += v[k] * v[k];
            sum = head_sum<LN>(sum);
            if (!on) continue;
            if (there && s.gain) {
                const float inv = 1.f / sqrtf(sum / (float)a.D + a.eps);
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] *= inv * (which == 0 ? gq[k] : gk[k]);
            }
            if (there && s.turned) rotate8(sn, cs, 1.f, v);
            if (s.y) {
                const size_t y = (size_t)row * s.py + (size_t)h * a.D;
                store4<E>(s.y, y + at.c0, v);
                store4<E>(s.y, y + at.c1, v + 4);
            } else if (there && page >= 0) {
                const size_t y = (((size_t)page * s.heads + h) * a.cache.page + in_page) * a.D;
                store4<E>(s.pages, y + at.c0, v);
                store4<E>(s.pages, y + at.c1, v + 4);
            }
        }
    }
}

struct HeadGradSide {
    const void *dy, *x;
    long long pdy, px, pdx;
    void* dx;
    const float* gain;
    int heads;
};

struct HeadGradArgs {
    Frames frames;
    int rows, D;
    float eps;
    Turn turn;
    HeadGradSide side[2];
    float* part;                     // [workgroups][2][D] partial sums of the gains' gradients, or null
};

template <typename E, int LN>
__global__ __launch_bounds__(256) void heads_grad_kernel(HeadGradArgs a)
{
    constexpr int kAtOnce = kWave / LN;
    const int lane = (int)threadIdx.x % LN, group = (int)threadIdx.x % kWave / LN;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const HeadLane at(lane, a.D, a.turn.R);
    double turns[4];
    own_turns(a.turn, at, turns);
    float g[2][8], dg[2][8];
    load_gain(a.side[0].gain, at, g[0]);
    load_gain(a.side[1].gain, at, g[1]);
#pragma unroll
    for (int k = 0; k < 8; ++k) dg[0][k] = dg[1][k] = 0.f;
    const int n0 = a.side[0].heads, n1 = n0 + a.side[1].heads;
    for (long long r = (long long)blockIdx.x * 4 + wave; r < a.rows; r += (long long)gridDim.x * 4) {
        const int row = (int)r, b = (int)quotient((unsigned)row, a.frames.by), t = row - b * a.frames.T;
        const bool there = frame_exists(a.frames, row);
        float sn[4], cs[4];
        angles(turns, (double)(a.turn.first ? a.turn.first[b] : 0) + t, at.turned, sn, cs);
        for (int h0 = 0; h0 < n1; h0 += kAtOnce) {
            const int head = h0 + group, which = head < n0 ? 0 : 1;
            const HeadGradSide& s = a.side[which];
            const int h = head - (which ? n0 : 0);
            const bool on = head < n1 && at.here;
            float u[8], x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) u[k] = x[k] = 0.f;
            if (on && there) {
                const size_t i = (size_t)row * s.pdy + (size_t)h * a.D, j = (size_t)row * s.px + (size_t)h * a.D;
                unpack4<E>(raw4<E>(s.dy, i + at.c0), u);
                unpack4<E>(raw4<E>(s.dy, i + at.c1), u + 4);
                if (s.gain) {
                    unpack4<E>(raw4<E>(s.x, j + at.c0), x);
                    unpack4<E>(raw4<E>(s.x, j + at.c1), x + 4);
                }
                rotate8(sn, cs, -1.f, u);
            }
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) sum += x[k] * x[k];
            const float inv = 1.f / sqrtf(head_sum<LN>(sum) / (float)a.D + a.eps);
            float dot = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float d = on && there && s.gain ? u[k] * x[k] * inv : 0.f;
                dg[0][k] += which == 0 ? d : 0.f;
                dg[1][k] += which == 1 ? d : 0.f;
                u[k] *= which == 0 ? g[0][k] : g[1][k];
                dot += u[k] * x[k];
            }
            const float m = inv * inv * (head_sum<LN>(dot) / (float)a.D);
            if (!on) continue;
            if (s.gain) {
#pragma unroll
                for (int k = 0; k < 8; ++k) u[k] = there ? inv * (u[k] - x[k] * m) : 0.f;
            }
            const size_t i = (size_t)row * s.pdx + (size_t)h * a.D;
            store4<E>(s.dx, i + at.c0, u);
            store4<E>(s.dx, i + at.c1, u + 4);
        }
    }
    if (!a.part) return;
    // over the heads of the wavefront, then over the wavefronts
    __shared__ float red[4][2][LN * 8];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float v = dg[i][k];
#pragma unroll
            for (int o = LN; o < kWave; o <<= 1) v += __shfl_xor(v, o, kWave);
            if (group == 0) red[wave][i][lane * 8 + k] = v;
        }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < 2 * LN * 8; i += 256) {
        const int side = i / (LN * 8), slot = i % (LN * 8);
        const HeadLane of(slot / 8, a.D, a.turn.R);
        if (!of.here) continue;
        const int c = slot % 8 < 4 ? of.c0 + slot % 8 : of.c1 + slot % 8 - 4;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) v += red[w][side][slot];
        a.part[((size_t)blockIdx.x * 2 + side) * a.D + c] = v;
    }
}

// dgain of both from n workgroups' partial sums, in a fixed order: 16 columns a workgroup, 64 groups of rows
__global__ __launch_bounds__(1024) void heads_gain_kernel(const float* part, int n, int D, float* dq, float* dk)
{
    __shared__ float red[64][17];
    const int c = threadIdx.x & 15, g = threadIdx.x >> 4, i = (int)blockIdx.x * 16 + c;
    float t = 0.f;
    if (i < 2 * D) {
#pragma unroll 4
        for (int k = g; k < n; k += 64) t += part[(size_t)k * 2 * D + i];
    }
    red[g][c] = t;
    __syncthreads();
    if (g == 0 && i < 2 * D) {
        t = 0.f;
#pragma unroll
        for (int k = 0; k < 64; ++k) t += red[k][c];
        float* out = i < D ? dq : dk;
        if (out) out[i < D ? i : i - D] = t;
    }
}

}  // namespace last
