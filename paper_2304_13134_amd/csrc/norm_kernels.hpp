// Root-mean-square norm of the sum of a row and a residual, and its gradient.
//     s = x + residual,  inv = 1 / sqrt(mean_h s^2 + eps),  y = s inv gain
//     u = gain dy,  dx = inv (u - s inv^2 mean_h(u s)) + ds,  dgain[h] = sum over rows of dy s inv
// Both read and write every value once and are bound by memory: a row stays in registers between the sum and its use
// (8 columns a lane in each of CH places), in one wavefront up to 2048 columns, so that no barrier separates them, and in
// 4 or 16 wavefronts beyond.  16384 x 512 in bfloat16 with a residual, three quarters of the frames existing: 10.9 us (59 MB), one row
// 2.1 us; with all frames in float32 23.9 us (134 MB: 5.6 TB/s), 2048 x 16384 in bfloat16 46 us (268 MB: 5.8 TB/s).  To 8 bits: 16384 x 512
// from bfloat16 22 us (59 MB: 2.7 TB/s, bound by the instructions in 64 bits), 2331 x 257 from float32 7.2 us (a chain of latencies: the
// row, its sum, a root and a division in 64 bits, the gain).
#pragma once
#include "layer.hpp"

#include <type_traits>

namespace last {

struct NormArgs {
    Frames frames;
    int row0, rows, H;               // rows row0 .. rows of the matrices
    const void *x, *res;             // res: null, or of the type of x
    const float* gain;
    void *s, *y;                     // each may be null; s of the type of x
    float* inv;
    long long px, pr, ps, py;
    int ytype;
    float eps;
    Eight kept;
};

// sum over the WPR wavefronts of a row; `red`: 2 x WPR places of LDS, `turn` alternates between their halves so that one
// barrier a sum is enough
template <int WPR, typename F>
__device__ __forceinline__ F row_sum(F v, F* red, int turn)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
    if constexpr (WPR > 1) {
        red += (turn & 1) * WPR;
        if ((threadIdx.x & (kWave - 1)) == 0) red[threadIdx.x / kWave] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int i = 0; i < WPR; ++i) v += red[i];
    }
    return v;
}

// to 32 bits, inexact values to the neighbour whose last bit is 1: rounding that again, to fewer bits, is rounding once.
// near: v to nearest, which is infinite where v passes what 32 bits hold
__device__ __forceinline__ float to_odd(double v, float near)
{
    const float f = __double2float_rz(v);
    return (double)f == v || !(fabsf(near) < __builtin_huge_valf()) ? near : __uint_as_float(__float_as_uint(f) | 1u);
}

// KEEP: with the result in 8 bits.  Its codes are those of the exact row: where 32 bits are enough for a result that is
// rounded by 2^-8 of itself, a code moves by 2^-4 where a sum in another order falls on the other side of a half, so these rows
// are formed in 64 bits (the sum of x and residual as its rounded value and the rest), a few operations a value beside its bytes.
template <typename X, int WPR, int CH, bool KEEP>
__global__ __launch_bounds__(WPR == 1 ? 256 : WPR * kWave) void norm_kernel(NormArgs a)
{
    constexpr int kRows = WPR == 1 ? 4 : 1;                  // rows of a workgroup
    using F = std::conditional_t<KEEP, double, float>;
    __shared__ F red[2 * WPR];
    const int row = a.row0 + (int)blockIdx.x * kRows + (WPR == 1 ? (int)threadIdx.x / kWave : 0);
    const int lane = WPR == 1 ? (int)threadIdx.x % kWave : (int)threadIdx.x;
    if (WPR == 1 && row >= a.rows) return;
    const bool there = frame_exists(a.frames, row);
    float v[CH][8], rest[KEEP ? CH : 1][8];
    F sum = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            v[c][k] = 0.f;
            if constexpr (KEEP) rest[c][k] = 0.f;
        }
    if (there) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int h = (c * WPR * kWave + lane) * 8;
            load8<X>(a.x, (size_t)row * a.px + h, a.H - h, v[c]);
        }
        if (a.res) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int h = (c * WPR * kWave + lane) * 8;
                float r[8];
                load8<X>(a.res, (size_t)row * a.pr + h, a.H - h, r);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const float x = v[c][k], s = x + r[k];
                    if constexpr (KEEP) {
                        const float t = s - x;
                        rest[c][k] = fabsf(s) < __builtin_huge_valf() ? (x - (s - t)) + (r[k] - t) : 0.f;   // (of an infinity: NaN)
                    }
                    v[c][k] = s;
                }
            }
        }
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                F s = v[c][k];
                if constexpr (KEEP) s += (double)rest[c][k];
                sum += s * s;
            }
    }
    sum = row_sum<WPR>(sum, red, 0);
    F inv = 0;
    if (there) {
        if constexpr (KEEP) inv = 1.0 / sqrt(sum / a.H + (double)a.eps);
        else inv = 1.f / sqrtf(sum / (float)a.H + a.eps);
    }
    if (lane == 0 && a.inv) a.inv[row] = (float)inv;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int h = (c * WPR * kWave + lane) * 8;
        if (a.s) store8<X>(a.s, (size_t)row * a.ps + h, a.H - h, v[c]);
        float g[8];
        load8<float>(a.gain, h, a.H - h, g);
        if constexpr (KEEP) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const double d = there ? ((double)v[c][k] + (double)rest[c][k]) * inv * (double)g[k] : 0.0;
                g[k] = (float)d;                             // a result in 32 bits is rounded to nearest, the codes and 16 bits once more
                v[c][k] = to_odd(d, g[k]);
            }
            store_eight(a.kept, row, h, a.H - h, (lane & 3) == 0, quad_max(top8(v[c])), v[c]);
            if (a.y && a.ytype == LAST_F32) {
                store8<float>(a.y, (size_t)row * a.py + h, a.H - h, g);
                continue;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[c][k] = there ? v[c][k] * inv * g[k] : 0.f;
        }
        if (a.y) store8_as(a.ytype, a.y, (size_t)row * a.py + h, a.H - h, v[c]);
    }
}

struct NormGradArgs {
    Frames frames;
    int rows, H;
    const void *dy, *s, *ds;         // ds: null, or of the type of dx
    const uint8_t* s_scales;         // s in 8 bits only
    const float *gain, *inv;
    void* dx;
    float* part;                     // [workgroups][H] partial sums of dgain, or null
    long long pdy, ps, pds, pdx, pss;
    int dxtype;
};

// Every wavefront (WPR = 1) or workgroup goes over its rows and keeps the sums of its columns of dgain in registers;
// they meet in LDS and go out as one row of partial sums a workgroup, added in order by column_sum_kernel.  The next row
// is sent for before this one is worked on, always, so that the wait for this one is not one for it too: in the place of a
// row that does not exist this one is read again, from cache.  From turn to turn a workgroup moves on by 0.618 of their number,
// so that one that meets the end of an item does not meet those of all, T being a multiple of that number or close to it.
// 16384 x 2048 in bfloat16 with ds, three quarters of the frames existing (218 MB): 42 us, and 4.7 us for the sums over the
// workgroups; in the same place every turn 45 us; a row a wavefront, nothing sent for ahead, 70 us.  With all frames: in float32 105 us
// (537 MB: 5.1 TB/s), s in 8 bits 46 us (236 MB); 16384 x 512 15.5 us (67 MB), 4096 x 8192 60 us (268 MB: 4.5 TB/s).  Beyond 8192 columns the two
// rows in registers spill (up to 86 of them): 2048 x 16384 117 us (268 MB: 2.3 TB/s).
template <typename DY, typename S, int WPR, int CH, bool DS>
__global__ __launch_bounds__(WPR == 1 ? 256 : WPR * kWave) void norm_grad_kernel(NormGradArgs a)
{
    constexpr int kRows = WPR == 1 ? 4 : 1;
    constexpr bool kEight = Elt<S>::size == 1;
    __shared__ float red[2 * WPR];
    __shared__ float cols[WPR == 1 ? 4 * kWave * 8 : 1];
    const int lane = WPR == 1 ? (int)threadIdx.x % kWave : (int)threadIdx.x;
    const int wave = WPR == 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave) : 0;
    struct Row {
        Raw<DY> dy[CH];
        Raw<S> s[CH];
        Raw<float> ds[DS ? CH : 1];
        unsigned scale[kEight ? CH : 1];
        float inv;
    };
    const auto get = [&](int row) {
        Row r;
        r.inv = a.inv[row];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int h = (c * WPR * kWave + lane) * 8;
            r.dy[c] = raw8<DY>(a.dy, (size_t)row * a.pdy + h, a.H - h);
            r.s[c] = raw8<S>(a.s, (size_t)row * a.ps + h, a.H - h);
            if constexpr (kEight) r.scale[c] = h < a.H ? a.s_scales[(size_t)row * a.pss + h / kBlock] : 0u;
            if constexpr (DS) {
                if (a.dxtype == LAST_F32) r.ds[c] = raw8<float>(a.ds, (size_t)row * a.pds + h, a.H - h);
                else r.ds[c].a = raw8<bf16_t>(a.ds, (size_t)row * a.pds + h, a.H - h).a;
            }
        }
        return r;
    };
    float dg[CH][8];
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int k = 0; k < 8; ++k) dg[c][k] = 0.f;
    const auto exists = [&](long long row) { return row < a.rows && frame_exists(a.frames, (int)row); };
    const int groups = (int)gridDim.x, shift = (int)(0.618f * (float)groups);
    int place = (int)blockIdx.x;
    long long first = 0;                                     // of the turn that is looked at
    const auto later = [&]() {
        first += groups;
        place += shift;
        place -= place >= groups ? groups : 0;
        return (first + place) * kRows + wave;
    };
    long long row = (long long)place * kRows + wave, row_next = later();
    bool there = exists(row), there_next = exists(row_next);
    Row next{};
    if (row < a.rows) next = get((int)row);
    for (int turn = 0; row < a.rows; ++turn) {
        const Row now = next;
        next = get((int)(there_next ? row_next : row));
        const long long row_later = later();
        const bool there_later = exists(row_later);
        float u[CH][8], s[CH][8];
        float dot = 0.f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int h = (c * WPR * kWave + lane) * 8;
            unpack<DY>(now.dy[c], u[c]);
            unpack<S>(now.s[c], s[c]);
            if constexpr (kEight) {
                const float sc = scale_value(now.scale[c]);
#pragma unroll
                for (int k = 0; k < 8; ++k) s[c][k] *= sc;
            }
            float g[8];
            load8<float>(a.gain, h, a.H - h, g);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                dg[c][k] += there ? u[c][k] * s[c][k] * now.inv : 0.f;
                u[c][k] *= g[k];
                dot += u[c][k] * s[c][k];
            }
        }
        dot = row_sum<WPR>(dot, red, turn);
        const float m = now.inv * now.inv * (dot / (float)a.H);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int h = (c * WPR * kWave + lane) * 8;
#pragma unroll
            for (int k = 0; k < 8; ++k) u[c][k] = now.inv * (u[c][k] - s[c][k] * m);
            if constexpr (DS) {
                float d[8];
                if (a.dxtype == LAST_F32) unpack<float>(now.ds[c], d);
                else if (a.dxtype == LAST_BF16) unpack<bf16_t>(Raw<bf16_t>{now.ds[c].a}, d);
                else unpack<f16_t>(Raw<f16_t>{now.ds[c].a}, d);
#pragma unroll
                for (int k = 0; k < 8; ++k) u[c][k] += d[k];
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) u[c][k] = there ? u[c][k] : 0.f;
            store8_as(a.dxtype, a.dx, (size_t)row * a.pdx + h, a.H - h, u[c]);
        }
        row = row_next;
        row_next = row_later;
        there = there_next;
        there_next = there_later;
    }
    if (!a.part) return;
    float* out = a.part + (size_t)blockIdx.x * a.H;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int h = (c * WPR * kWave + lane) * 8;
        if constexpr (WPR == 1) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < 8; ++k) cols[(wave * 8 + k) * kWave + lane] = dg[c][k];
            __syncthreads();
            // wavefront w sums columns 2w, 2w + 1 of every lane's eight
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int k = 2 * wave + j;
                float t = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) t += cols[(w * 8 + k) * kWave + lane];
                if (h + k < a.H) out[h + k] = t;
            }
        } else {
            store8<float>(out, h, a.H - h, dg[c]);
        }
    }
}

// out[h] = sum over n rows of part[n][H], in a fixed order: 32 columns a workgroup, 32 groups of rows
__global__ __launch_bounds__(1024) void column_sum_kernel(const float* part, int n, int H, float* out)
{
    __shared__ float red[32][33];
    const int c = threadIdx.x & 31, g = threadIdx.x >> 5, h = (int)blockIdx.x * 32 + c;
    float t = 0.f;
    if (h < H) {
#pragma unroll 4
        for (int i = g; i < n; i += 32) t += part[(size_t)i * H + h];
    }
    red[g][c] = t;
    __syncthreads();
    if (g == 0 && h < H) {
        t = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += red[i][c];
        out[h] = t;
    }
}

}  // namespace last
