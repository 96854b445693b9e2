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
    Pages cache;
    int* status;                     // [B] or null
};

constexpr int kMostUsed = 1 << 30;   // positions stay in 32 bits

// p[i] where both are the same for all lanes: by the scalar unit, whose loads wait for no others
__device__ __forceinline__ int same_for_all(const int* p, int i)
{
    typedef const __attribute__((address_space(4))) int* at;
    return *((at)(uintptr_t)p + i);
}

__device__ __forceinline__ int used_frames(const int* used, int b)
{
    const int n = same_for_all(used, b);
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
    float sn = __builtin_fmaf(s, 2.7557319e-6f, -1.9841270e-4f), cs = __builtin_fmaf(s, 2.4801587e-5f, -1.3888889e-3f);
    sn = x * __builtin_fmaf(s, __builtin_fmaf(s, __builtin_fmaf(s, sn, 8.3333333e-3f), -1.6666667e-1f), 1.f);
    cs = __builtin_fmaf(s, __builtin_fmaf(s, __builtin_fmaf(s, cs, 4.1666667e-2f), -0.5f), 1.f);
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

// 1 / sqrt(v), to an ulp (the instruction knows no subnormal numbers)
__device__ __forceinline__ float inverse_root(float v)
{
    const bool small = v < 0x1p-64f;
    const float r = __builtin_amdgcn_rsqf(small ? v * 0x1p64f : v);
    return small ? r * 0x1p32f : r;
}

// in one instruction each: `p` is the same for all lanes
template <typename E>
__device__ __forceinline__ void get8(const char* p, unsigned o0, unsigned o1, Four<E>* r)
{
    r[0] = raw4<E>(p + o0, 0);
    r[1] = raw4<E>(p + o1, 0);
}

template <int LN>
__device__ __forceinline__ float head_sum(float v)
{
#pragma unroll
    for (int o = LN / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}

// The angles of a frame: a lane forms one pair's, and has its own four from LDS (`turned`: 2 x 64 floats of the wavefront's).
struct Angles {
    float frequency;                 // of the pair that the lane forms
    float* at;
    __device__ __forceinline__ void init(const Turn& t, float* lds)
    {
        const int lane = (int)threadIdx.x % kWave;
        at = lds + (int)threadIdx.x / kWave * 2 * kWave;
        frequency = lane < t.R / 2 ? t.frequencies[lane] : 0.f;
    }
    __device__ __forceinline__ void get(double position, const HeadLane& of, float* sn, float* cs) const
    {
        const int lane = (int)threadIdx.x % kWave;
        float s, c;
        sine_cosine(position * ((double)frequency * 0.15915494309189535), &s, &c);
        asm volatile("" ::: "memory");
        at[lane] = s;
        at[kWave + lane] = c;
        asm volatile("" ::: "memory");                       // (one wavefront's accesses to LDS stay in order)
        const f4 x = *(const f4*)(at + (of.turned ? of.c0 : 0)), y = *(const f4*)(at + kWave + (of.turned ? of.c0 : 0));
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            sn[k] = of.turned ? x[k] : 0.f;
            cs[k] = of.turned ? y[k] : 1.f;
        }
    }
};

// (two instructions: a compute unit takes about 33 clocks for one that addresses memory by lane, whatever its width, and sixteen of a value each
// were most of a wavefront's)
__device__ __forceinline__ void load_gain(const float* gain, const HeadLane& at, float* g)
{
    f4 a{1.f, 1.f, 1.f, 1.f}, b = a;
    if (gain && at.here) {
        a = *(const f4_any*)(gain + at.c0);
        b = *(const f4_any*)(gain + at.c1);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        g[k] = a[k];
        g[4 + k] = b[k];
    }
}

// (which products are fused is written out, here and in the sums, so that a row has the same bits from every kernel)
__device__ __forceinline__ void rotate8(const float* sn, const float* cs, float sign, float* v)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float a = v[k], b = v[4 + k], s = sign * sn[k];
        v[k] = __builtin_fmaf(a, cs[k], -(b * s));
        v[4 + k] = __builtin_fmaf(b, cs[k], a * s);
        asm("" : "+v"(v[k]), "+v"(v[4 + k]));                // (else they may be rounded to 16 bits in the same instruction, or not)
    }
}

// status of the items of a call without frames
__global__ void no_frames_kernel(int* status, int B)
{
    const int b = (int)(blockIdx.x * 256 + threadIdx.x);
    if (b < B) status[b] = kItemOk;
}

// LN: lanes of a head.  A group is 64 / LN heads of a frame, of queries, keys or values alone, so that pointers are the same for all lanes; a wavefront
// takes every split-th group of a frame.  PAGES: keys and values go to the pages of a cache.  The code is kept short: with four groups unrolled, and
// loads sent for ahead, its 17 KB took longer to arrive than a frame does.
// 16384 x 16 heads of 64 in bfloat16, three quarters of the frames existing (59 MB): 13 us, of which the memory takes 9
template <typename E, int LN, bool PAGES>
__global__ __launch_bounds__(256) void heads_kernel(HeadArgs a)
{
    constexpr int kAtOnce = kWave / LN;
    constexpr unsigned kSize = Elt<E>::size;
    __shared__ __attribute__((aligned(16))) float lds[4 * 2 * kWave];
    const int lane = (int)threadIdx.x % LN, group = (int)threadIdx.x % kWave / LN;
    const int wave = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + (int)threadIdx.x / kWave), waves = (int)gridDim.x * 4;
    const HeadLane at(lane, a.D, a.turn.R);
    const unsigned o0 = (unsigned)(group * a.D + at.c0) * kSize, o1 = (unsigned)(group * a.D + at.c1) * kSize;
    const HeadSide s0 = a.side[0], s1 = a.side[1], s2 = a.side[2];
    const int g0 = (s0.heads + kAtOnce - 1) / kAtOnce, g1 = g0 + (s1.heads + kAtOnce - 1) / kAtOnce;
    const int groups = g1 + (PAGES ? (s2.heads + kAtOnce - 1) / kAtOnce : 0), part = (int)blockIdx.y, split = (int)gridDim.y;
    Angles angles;
    angles.init(a.turn, lds);
    float gq[8], gk[8];
    load_gain(s0.gain, at, gq);
    load_gain(s1.gain, at, gk);
    const float by_width = 1.f / (float)a.D;
    for (int row = wave; row < a.rows; row += waves) {
        const int b = (int)quotient((unsigned)row, a.frames.by), t = row - b * a.frames.T;
        const int exist = a.frames.len ? same_for_all(a.frames.len, b) : a.frames.T;
        const bool there = t < exist;
        double position = t;
        int page = 0, in_page = 0;
        if constexpr (PAGES) {
            const int used = used_frames(a.cache.used, b);
            page = page_of(a.cache, b, used + t, &in_page);
            position += used;
            if (a.status && t == 0 && part == 0) {
                // every page that the item's new frames go to
                int bad = 0, n = clamped(exist, a.frames.T), r;
                for (int i = (int)threadIdx.x % kWave; i < n; i += kWave) bad |= page_of(a.cache, b, used + i, &r) < 0;
                const bool any = __any(bad);
                if (threadIdx.x % kWave == 0) a.status[b] = any ? kItemBadPage : kItemOk;
            }
        } else if (a.turn.first) {
            position += same_for_all(a.turn.first, b);
        }
        // (a frame that is not there has zeros, whatever the gains and frequencies are)
        if (!there) {
            const float zeros[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int i = part; i < (PAGES ? g0 : g1); i += split) {
                const bool of_q = i < g0;
                const int h = (of_q ? i : i - g0) * kAtOnce;
                if (!at.here || group >= (of_q ? s0.heads : s1.heads) - h) continue;
                char* const y = (char*)(of_q ? s0.y : s1.y) + ((size_t)row * (of_q ? s0.py : s1.py) + (size_t)h * a.D) * kSize;
                store4<E>(y + o0, 0, zeros);
                store4<E>(y + o1, 0, zeros);
            }
            continue;
        }
        float sn[4], cs[4];
#pragma unroll 1
        for (int i = part; i < groups; i += split) {
            const bool of_q = i < g0, of_k = !of_q && i < g1;
            const int h = (of_q ? i : of_k ? i - g0 : i - g1) * kAtOnce, heads = of_q ? s0.heads : of_k ? s1.heads : s2.heads;
            const bool on = at.here && group < heads - h;
            const size_t column = (size_t)h * a.D;
            Four<E> x[2]{};
            if (on)
                get8<E>((const char*)(of_q ? s0.x : of_k ? s1.x : s2.x) + ((size_t)row * (of_q ? s0.px : of_k ? s1.px : s2.px) + column) * kSize, o0, o1, x);
            if (i == part) angles.get(position, at, sn, cs);
            float v[8];
            unpack4<E>(x[0], v);
            unpack4<E>(x[1], v + 4);
            if (of_q || of_k) {
                if (of_q ? s0.gain : s1.gain) {
                    float sum = 0.f;
#pragma unroll
                    for (int c = 0; c < 8; ++c) sum = __builtin_fmaf(v[c], v[c], sum);
                    const float inv = inverse_root(__builtin_fmaf(head_sum<LN>(sum), by_width, a.eps));
#pragma unroll
                    for (int c = 0; c < 8; ++c) v[c] *= inv * (of_q ? gq[c] : gk[c]);
                }
                rotate8(sn, cs, 1.f, v);
            }
            if (!on) continue;
            if (!PAGES || of_q) {
                char* const y = (char*)(of_q ? s0.y : s1.y) + ((size_t)row * (of_q ? s0.py : s1.py) + column) * kSize;
                store4<E>(y + o0, 0, v);
                store4<E>(y + o1, 0, v + 4);
            } else if (page >= 0) {
                char* const y = (of_k ? s1.pages : s2.pages) + (((size_t)page * heads + h + group) * a.cache.page + in_page) * a.D * kSize;
                store4<E>(y, at.c0, v);
                store4<E>(y, at.c1, v + 4);
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

// 16384 x 20 heads of 128 in bfloat16, three quarters of the frames existing (210 MB): 43 us (4.9 TB/s)
template <typename E, int LN>
__global__ __launch_bounds__(256) void heads_grad_kernel(HeadGradArgs a)
{
    constexpr int kAtOnce = kWave / LN;
    constexpr unsigned kSize = Elt<E>::size;
    __shared__ __attribute__((aligned(16))) float lds[4 * 2 * kWave];
    const int lane = (int)threadIdx.x % LN, group = (int)threadIdx.x % kWave / LN;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const HeadLane at(lane, a.D, a.turn.R);
    const unsigned o0 = (unsigned)(group * a.D + at.c0) * kSize, o1 = (unsigned)(group * a.D + at.c1) * kSize;
    const HeadGradSide s0 = a.side[0], s1 = a.side[1];
    Angles angles;
    angles.init(a.turn, lds);
    float gq[8], gk[8], dgq[8], dgk[8];
    load_gain(s0.gain, at, gq);
    load_gain(s1.gain, at, gk);
#pragma unroll
    for (int k = 0; k < 8; ++k) dgq[k] = dgk[k] = 0.f;
    const float by_width = 1.f / (float)a.D;
    const int g0 = (s0.heads + kAtOnce - 1) / kAtOnce, groups = g0 + (s1.heads + kAtOnce - 1) / kAtOnce;
    // u = dy rotated back to dx, d[k] += what the gain's gradient gets
    // (lanes without a head have zeros, and no factor: it would be infinite without an eps)
    const auto norm_grad = [&](float* u, const float* x, const float* gain, float* d, bool on) {
        float sum = 0.f, dot = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) sum += x[k] * x[k];
        float inv = inverse_root(head_sum<LN>(sum) * by_width + a.eps);
        inv = on ? inv : 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            d[k] += u[k] * (x[k] * inv);
            u[k] *= gain[k];
            dot += u[k] * x[k];
        }
        const float m = inv * inv * (head_sum<LN>(dot) * by_width);
#pragma unroll
        for (int k = 0; k < 8; ++k) u[k] = inv * (u[k] - x[k] * m);
    };
    for (long long r = (long long)blockIdx.x * 4 + wave; r < a.rows; r += (long long)gridDim.x * 4) {
        const int row = __builtin_amdgcn_readfirstlane((int)r), b = (int)quotient((unsigned)row, a.frames.by), t = row - b * a.frames.T;
        const bool there = t < (a.frames.len ? same_for_all(a.frames.len, b) : a.frames.T);
        const double position = (double)(a.turn.first ? same_for_all(a.turn.first, b) : 0) + t;
        float sn[4], cs[4];
#pragma unroll 1
        for (int i = 0; i < groups; ++i) {
            const bool of_q = i < g0;
            const int h = (of_q ? i : i - g0) * kAtOnce;
            const bool on = at.here && group < (of_q ? s0.heads : s1.heads) - h;
            const size_t column = (size_t)h * a.D;
            Four<E> raw[4]{};
            if (there && on) {
                get8<E>((const char*)(of_q ? s0.dy : s1.dy) + ((size_t)row * (of_q ? s0.pdy : s1.pdy) + column) * kSize, o0, o1, raw);
                if (of_q ? s0.gain : s1.gain)
                    get8<E>((const char*)(of_q ? s0.x : s1.x) + ((size_t)row * (of_q ? s0.px : s1.px) + column) * kSize, o0, o1, raw + 2);
            }
            if (i == 0) angles.get(position, at, sn, cs);
            float u[8], x[8];
            unpack4<E>(raw[0], u);
            unpack4<E>(raw[1], u + 4);
            unpack4<E>(raw[2], x);
            unpack4<E>(raw[3], x + 4);
            if (there) {
                rotate8(sn, cs, -1.f, u);
                if (of_q) {
                    if (s0.gain) norm_grad(u, x, gq, dgq, on);
                } else {
                    if (s1.gain) norm_grad(u, x, gk, dgk, on);
                }
            }
            if (!on) continue;
            char* const dx = (char*)(of_q ? s0.dx : s1.dx) + ((size_t)row * (of_q ? s0.pdx : s1.pdx) + column) * kSize;
            store4<E>(dx + o0, 0, u);
            store4<E>(dx + o1, 0, u + 4);
        }
    }
    if (!a.part) return;
    // over the heads of the wavefront, then over the wavefronts
    __shared__ float red[4][2][LN * 8];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float v = i == 0 ? dgq[k] : dgk[k];
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
