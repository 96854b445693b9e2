// Activations kept in 8 bits: a row in blocks of 32 columns, each with a power of two 2^e, the smallest at which no value
// passes the largest code, and codes v 2^-e to nearest even.  A power of two makes both products exact: the one rounding
// is the code's, and what a code stands for has at most 7 bits, so 16-bit results hold it without another.  (A scale of
// top / 127 would use up to a bit more of the codes' range, 0.5 % instead of 0.8 % of the rms for normal values, and
// round three times.)  All are bound by memory: 8 columns a thread, four neighbouring threads hold a block.
#pragma once
#include "layer.hpp"

namespace last {

struct KeepArgs {
    Frames frames;
    int row0, rows, H;               // rows row0 .. row0 + rows of the matrices
    int groups;                      // threads of a row: 4 for each block
    const void* x;                   // keep: values; grad: dy
    void* y;                         // values, grad: results
    long long px, py;
    int act, ytype;
    Eight kept;
};

__device__ __forceinline__ bool keep_place(const KeepArgs& a, int* row, int* h)
{
    const unsigned i = blockIdx.x * 256u + threadIdx.x;
    const unsigned r = i / (unsigned)a.groups;
    *row = a.row0 + (int)r;
    *h = (int)(i - r * a.groups) * 8;
    return r < (unsigned)a.rows;
}

template <typename X>
__global__ __launch_bounds__(256) void keep_kernel(KeepArgs a)
{
    int row, h;
    const bool in = keep_place(a, &row, &h);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (in && h < a.H && frame_exists(a.frames, row)) load8<X>(a.x, (size_t)row * a.px + h, a.H - h, v);
    const unsigned top = quad_max(top8(v));
    if (in) store_eight(a.kept, row, h, a.H - h, (h & (kBlock - 1)) == 0, top, v);
}

__device__ __forceinline__ void load_eight(const Eight& k, size_t row, int h, int n, float* v)
{
    unsigned lo, hi;
    load_codes(k.q + row * k.pitch, h, n, &lo, &hi);
    const float sc = scale_value(k.scales[row * k.scale_pitch + h / kBlock]);
    if (k.e4m3) {
        decode4<true>(lo, sc, v);
        decode4<true>(hi, sc, v + 4);
    } else {
        decode4<false>(lo, sc, v);
        decode4<false>(hi, sc, v + 4);
    }
}

// y = act(kept)
__global__ __launch_bounds__(256) void kept_values_kernel(KeepArgs a)
{
    int row, h;
    if (!keep_place(a, &row, &h) || h >= a.H) return;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (frame_exists(a.frames, row)) {
        load_eight(a.kept, row, h, a.H - h, v);
        activate8(a.act, v);
    }
    store8_as(a.ytype, a.y, (size_t)row * a.py + h, a.H - h, v);
}

// y = dy act'(kept)
template <typename X>
__global__ __launch_bounds__(256) void kept_grad_kernel(KeepArgs a)
{
    int row, h;
    if (!keep_place(a, &row, &h) || h >= a.H) return;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, d[8];
    if (frame_exists(a.frames, row)) {
        load8<X>(a.x, (size_t)row * a.px + h, a.H - h, d);
        load_eight(a.kept, row, h, a.H - h, v);
        times_slope(a.act, v, d);
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) d[k] = 0.f;
    }
    store8_as(a.ytype, a.y, (size_t)row * a.py + h, a.H - h, d);
}

}  // namespace last
