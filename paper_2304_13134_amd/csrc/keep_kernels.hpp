// Activations kept in 8 bits: a row in blocks of 32 columns, each with a power of two 2^e, the smallest at which no value
// passes the largest code, and codes v 2^-e to nearest even.  A power of two makes both products exact: the one rounding
// is the code's, and what a code stands for has at most 7 bits, so bfloat16 results hold it without another (float16 ones at
// scales from 2^-24 for int8, 2^-15 for e4m3, up to what passes 65504).  (A scale of top / 127 would use up to a bit more of the codes'
// range, 0.5 % instead of 0.8 % of the rms for normal values, and round three times.)  All are bound by memory: 8 columns a thread, four neighbouring threads hold a block.  16384 x 2048
// from bfloat16 to int8 17.7 us (84 MB, three quarters of the frames existing), the activation formed again 17.6 us (93 MB); 32768 x
// 4096 formed again 61 us (406 MB: 6.6 TB/s), the gradient of silu alone 27.8 us (16384 x 2048, all frames, 169 MB).  Instructions are a third of the time, so places are found without a division.
#pragma once
#include "layer.hpp"

namespace last {

struct KeepArgs {
    Frames frames;
    int row0, rows, H;               // rows row0 .. row0 + rows of the matrices
    int groups;                      // threads of a row: 4 for each block
    Divisor by_groups;
    const void* x;                   // keep: values; grad: dy
    void* y;                         // values, grad: results
    long long px, py;
    int act, ytype;
    Eight kept;
};

// Eight columns in each of kKeepDeep places, the loads of all under way before the first is worked on.
constexpr int kKeepDeep = 4;

struct KeepPlace {
    int row, h;
    bool in;                         // of the matrix's rows
    int n;                           // columns to read: 0 past the end, or where no frame is
};

__device__ __forceinline__ KeepPlace keep_place(const KeepArgs& a, unsigned group, int d)
{
    const unsigned i = (group * kKeepDeep + d) * 256u + threadIdx.x;
    const unsigned r = quotient(i, a.by_groups);
    KeepPlace p;
    p.row = a.row0 + (int)r;
    p.h = (int)(i - r * a.groups) * 8;
    p.in = r < (unsigned)a.rows;
    p.n = p.in && frame_exists(a.frames, p.row) ? a.H - p.h : 0;
    return p;
}

template <typename X>
__global__ __launch_bounds__(256) void keep_kernel(KeepArgs a)
{
    KeepPlace p[kKeepDeep];
    Raw<X> x[kKeepDeep];
#pragma unroll
    for (int d = 0; d < kKeepDeep; ++d) p[d] = keep_place(a, blockIdx.x, d);
#pragma unroll
    for (int d = 0; d < kKeepDeep; ++d) x[d] = raw8<X>(a.x, (size_t)p[d].row * a.px + p[d].h, p[d].n);
#pragma unroll
    for (int d = 0; d < kKeepDeep; ++d) {
        float v[8] = {};
        unsigned top = 0;
        if (__any(p[d].n > 0)) {                             // (some frame of the wavefront exists)
            unpack<X>(x[d], v);
            top = quad_max(top8(v));
        }
        if (p[d].in) store_eight(a.kept, p[d].row, p[d].h, a.H - p[d].h, (p[d].h & (kBlock - 1)) == 0, top, v);
    }
}

struct RawEight {
    Raw<i8_t> q;
    unsigned scale;
};

__device__ __forceinline__ RawEight raw_eight(const Eight& k, const KeepPlace& p)
{
    RawEight r{};
    r.q = raw8<i8_t>(k.q, (size_t)p.row * k.pitch + p.h, p.n);
    if (p.n > 0) r.scale = k.scales[(size_t)p.row * k.scale_pitch + p.h / kBlock];
    return r;
}

__device__ __forceinline__ void unpack_eight(bool e4m3, const RawEight& r, float* v)
{
    const float sc = scale_value(r.scale);
    if (e4m3) {
        decode4<true>(r.q.a[0], sc, v);
        decode4<true>(r.q.a[1], sc, v + 4);
    } else {
        decode4<false>(r.q.a[0], sc, v);
        decode4<false>(r.q.a[1], sc, v + 4);
    }
}

// y = act(kept)
__device__ __forceinline__ void kept_values(const KeepArgs& a, unsigned group)
{
    KeepPlace p[kKeepDeep];
    RawEight x[kKeepDeep];
#pragma unroll
    for (int d = 0; d < kKeepDeep; ++d) p[d] = keep_place(a, group, d);
#pragma unroll
    for (int d = 0; d < kKeepDeep; ++d) x[d] = raw_eight(a.kept, p[d]);
#pragma unroll
    for (int d = 0; d < kKeepDeep; ++d) {
        float v[8] = {};
        if (__any(p[d].n > 0)) {
            unpack_eight(a.kept.e4m3, x[d], v);              // (act(0) = 0 for each)
            activate8(a.act, v);
        }
        store8_as(a.ytype, a.y, (size_t)p[d].row * a.py + p[d].h, p[d].in ? a.H - p[d].h : 0, v);
    }
}

__global__ __launch_bounds__(256) void kept_values_kernel(KeepArgs a) { kept_values(a, blockIdx.x); }

// y = dy act'(kept)
template <typename X>
__global__ __launch_bounds__(256) void kept_grad_kernel(KeepArgs a)
{
    KeepPlace p[kKeepDeep];
    RawEight x[kKeepDeep];
    Raw<X> dy[kKeepDeep];
#pragma unroll
    for (int d = 0; d < kKeepDeep; ++d) p[d] = keep_place(a, blockIdx.x, d);
#pragma unroll
    for (int d = 0; d < kKeepDeep; ++d) {
        x[d] = raw_eight(a.kept, p[d]);
        dy[d] = raw8<X>(a.x, (size_t)p[d].row * a.px + p[d].h, p[d].n);
    }
#pragma unroll
    for (int d = 0; d < kKeepDeep; ++d) {
        float h[8], v[8] = {};
        if (__any(p[d].n > 0)) {
            unpack_eight(a.kept.e4m3, x[d], h);
            unpack<X>(dy[d], v);
            times_slope(a.act, h, v);
        }
        store8_as(a.ytype, a.y, (size_t)p[d].row * a.py + p[d].h, p[d].in ? a.H - p[d].h : 0, v);
    }
}

}  // namespace last
