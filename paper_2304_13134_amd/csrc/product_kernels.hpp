// Products of the layer between an encoder's frames and the lattice, on the matrix cores, with their epilogues.
//
//     forward       y[m][n]  = act(sum_k x[m][k] w[n][k] + bias[n]) + residual[m][n]       both operands along k
//     of the input  dx[m][k] = (sum_n dy[m][n] w[n][k]) act'(kept[m][k])                   w across n
//     of weights    dw[n][k] = sum_m dy[m][n] x[m][k],  dbias[n] = sum_m dy[m][n]          both across m
//
// One kernel does all: an output of P rows and Q columns, operands P and Q whose reduction index runs along their rows in
// memory (kAlong) or across them (kAcross).  A workgroup computes a tile of BP x BQ, a wavefront a part of it in
// accumulators of 16 x 16; 128 bytes of the reduction index (64 values of 16 bits, 128 of 8) of both operands at a time go
// from memory to LDS without passing registers, the next ones while these are multiplied.  The Q operand is given to the
// matrix instruction as its first, so that a lane's four results are neighbours in a row of the output.
//
// LDS.  A load writes 64 lanes' 16 bytes in a row, so the swizzle that spreads rows over the banks is one of the addresses
// that are read: along, 16-byte piece c of row r stands at c ^ along_swizzle(r) of its 128 bytes, which gives the 16 rows
// of an operand 16 different places; across, 32-byte granules of row r stand at g ^ across_swizzle(r), and the transposing read
// (ds_read_b64_tr_b16: 16 lanes read four rows of 16 values and get four values of a column each) brings the reduction
// index into a lane.  Out-of-range pieces have an offset that the buffer's bounds check turns into zeros, in memory order
// that is: rows past the end, frames that do not exist, the rest of the reduction.
//
// Tiles of 256 x 256 on eight wavefronts of 128 x 64: 128 sums a lane leave registers for one set of fragments and a bit.
// Measured (16384 x 1024 results, bfloat16): over 1024, 4096, 8192 terms 37, 107, 205 us = 930, 1285, 1340 TFLOP/s; a large library
// product of these sizes 31, 90, 176 us.  8-bit operands: 28.6, 66, 118 us = 1200, 2080, 2330; with results in float32, on tiles of
// 128 x 128 of widened codes, 8000 x 4096 over 4096 280 us = 960 (145 us = 1850 with results in bfloat16).  Input gradients as forward; weight
// gradients 4096 x 4096 over 16384 rows 428 us = 1285 TFLOP/s.  The matrix cores are busy 65 % of the cycles at 2.0 GHz (the
// library's: 80 % at 1.87, the clock follows the power); LDS 25 %, without bank conflicts.  A step of 128 bytes takes 1.53 us on the
// whole chip, 1.45 without the reads of LDS, 1.08 without the loads to it, and 1.10 on a chip with 16 such workgroups: what is
// left is bound by the feed from L2 and memory, 16.8 MB a step.  Tried and slower or the same: four wavefronts of 128 x 128,
// tiles of 128 x 256, starting each XCD at another place of the reduction, two buffers for P, whole 512-byte rows of results in a
// wavefront.  Tiles of 64 have three buffers, so that three workgroups share a compute unit: 8000 x 257 on 512 in float16 10.1 us,
// with four buffers and two 13.6, with two buffers the same, but 31 instead of 20 us for 512 x 1024 on 4096.  The epilogue's activations are bound by instructions: a slope of silu takes 9 a value, two of them at a quarter of
// the rate, 8 us a tile of 256 x 256; rows that do not exist skip them.
#pragma once
#include "keep_kernels.hpp"
#include "layer.hpp"

#include <type_traits>

namespace last {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef int i8x __attribute__((ext_vector_type(8)));
typedef int i4x __attribute__((ext_vector_type(4)));

typedef __attribute__((address_space(3))) void* lds_t;

// e4m3 codes that are multiplied as bfloat16
struct wide_t { uint8_t bits; };
template <> struct Elt<wide_t> : EltCodes<true> {};

enum { kAlong = 0, kAcross = 1 };
constexpr unsigned kNowhere = 0x80000000u;       // beyond every buffer
constexpr int kStep = 128;                       // bytes of the reduction index at a time (kAlong), 64 rows (kAcross)

// what becomes of the sums of a tile
struct Epilogue {
    const float* bias;                           // [Q] or null
    int act;
    const void* res;                             // residual of type `type`, or null
    long long pres;
    void* y;                                     // null: 8-bit values `out` instead
    long long py;
    int type;
    Eight out;                                   // result in 8 bits
    Eight kept;                                  // forward: written with the sums + bias; of the input: read
    int kept_act;                                // of the input: times act' of what is kept (LAST_ACT_NONE: nothing is)
    float* part;                                 // [splits][P][Q] sums of a share of the reduction, or null
    float* part_bias;                            // [splits][P] row sums of the P operand, or null
    float* sum_bias;                             // [P] their sum (product_join_kernel)
};

struct ProductArgs {
    const char *p, *q;
    long long pp, pq;                            // bytes from a row to the next
    const uint8_t *sp, *sq;                      // scales of 8-bit operands, four blocks to 4 aligned bytes
    long long psp, psq;
    int P, Q;
    long long K;                                 // of the reduction: bytes of a row (kAlong) or rows (kAcross)
    long long q_rows;                            // kAlong with kAcross: rows of Q (P's rows may be padded beyond)
    long long share;                             // of the reduction that a split takes, a multiple of kStep or 64
    int tiles_p, tiles_q;
    Frames frames;                               // rows of P exist or not (kAlong)
    const unsigned long long* mask;              // kAcross on both: bits of the rows that exist, or null for all
    Epilogue e;
};

__device__ __forceinline__ int along_swizzle(int r) { return (r >> 1) & 7; }
template <int ROWS>
__device__ __forceinline__ int across_swizzle(int r)         // (rows of 64 columns have four granules only)
{
    return ((r & 3) | ((r >> 3) & 1) << 2) & (ROWS / 16 - 1);
}


__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* base)
{
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0x7fffffff, 0x00020000);
}

// a buffer's descriptor for the assembly below; base + offsets stay below 2^31, kNowhere is out of range whatever is added
__device__ __forceinline__ u4 descriptor(const void* base)
{
    const uint64_t p = (uint64_t)base;
    return u4{(unsigned)p, (unsigned)(p >> 32) & 0xffffu, 0x7fffffffu, 0x00020000u};
}

__device__ __forceinline__ unsigned lds_byte(const void* p) { return (unsigned)(uintptr_t)(lds_t)p; }

// 64 lanes' 16 (4) bytes at offset o + more of the buffer to LDS from byte `to` on.  In assembly, since the compiler makes every
// later read of LDS wait for its own form of this; whoever reads waits with arrived().  (m0 is a register that the compiler
// keeps nothing in: it sets it right before an instruction that reads it.)
template <int BYTES>
__device__ __forceinline__ void to_lds(u4 b, unsigned o, unsigned more, unsigned to)
{
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(to), "v"(o), "s"(b), "s"(more) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(to), "v"(o), "s"(b), "s"(more) : "memory");
}

// what this wavefront asked from LDS has come, and what it sent there but for the last LATER loads; then the same of the whole
// workgroup
template <int LATER>
__device__ __forceinline__ void arrived()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LATER) : "memory");
}

// ---- one operand's tile: ROWS rows or columns of the output
template <int L, int ROWS, int THREADS>
struct Tile {
    static constexpr int kBytes = ROWS * kStep;
    static constexpr int kLoads = kBytes / 16 / THREADS;                 // of a thread, kApart rows from each other
    static constexpr int kPieces = L == kAlong ? 8 : ROWS / 8;           // 16-byte pieces of a row in LDS
    static constexpr int kApart = THREADS / kPieces;
    static_assert(kBytes % (16 * THREADS) == 0, "whole loads");
    static_assert(L == kAlong || ROWS >= 64, "granules to swizzle");
    static_assert(kApart % 16 == 0, "the same swizzle for all loads of a thread");
    unsigned off;                                                        // of the first load, from the tile's first byte
    unsigned valid;                                                      // kAlong: bits of the loads whose row exists
    unsigned apart;                                                      // bytes from a load to the next
    unsigned wave_at;                                                    // of the wavefront's part of a load in LDS
    int row, piece;                                                      // of the first load

    // first: first row or column of the tile; count: how many the matrix has
    __device__ void init(int first, int count, long long pitch, const Frames* frames)
    {
        row = (int)threadIdx.x / kPieces;
        const int c = (int)threadIdx.x % kPieces;
        valid = 0;
        apart = (unsigned)(kApart * pitch);
        wave_at = (unsigned)__builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave) * kWave * 16;
        if constexpr (L == kAlong) {
            piece = c ^ along_swizzle(row);
            off = (unsigned)(row * pitch) + 16u * (unsigned)piece;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int r = first + row + j * kApart;
                if (r < count && (!frames || frame_exists(*frames, r))) valid |= 1u << j;
            }
        } else {
            const int col = ((c >> 1) ^ across_swizzle<ROWS>(row)) * 16 + (c & 1) * 8;
            off = first + col < count ? (unsigned)(row * pitch) + 2u * (unsigned)col : kNowhere;
        }
    }

    // bits of a step's loads that read what exists.  left: how many bytes the reduction still has (kAlong), mask: which rows
    // exist (kAcross)
    __device__ __forceinline__ unsigned bits(long long left, unsigned long long mask) const
    {
        if constexpr (L == kAlong) {
            return left >= kStep || 16 * piece < left ? valid : 0u;
        } else {
            if (mask == ~0ull) return (1u << kLoads) - 1;
            unsigned b = 0;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) b |= (unsigned)(mask >> (row + j * kApart) & 1) << j;
            return b;
        }
    }

    // load j of the tile's 128 bytes or 64 rows from the buffer's base on, to LDS byte `to`
    __device__ __forceinline__ void load(int j, u4 buffer, unsigned bits, unsigned to) const
    {
        to_lds<16>(buffer, bits >> j & 1 ? off : kNowhere, j * apart, to + wave_at + j * THREADS * 16);
    }
};

template <typename E> struct Mfma;
template <> struct Mfma<bf16_t> {
    static __device__ __forceinline__ f4 go(u4 a, u4 b, f4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
    }
};
template <> struct Mfma<f16_t> {
    static __device__ __forceinline__ f4 go(u4 a, u4 b, f4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
    }
};

__device__ __forceinline__ i8x join8(u4 a, u4 b)
{
    return i8x{(int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)b[0], (int)b[1], (int)b[2], (int)b[3]};
}

// lane: values 16 g .. and 64 + 16 g .. of 128 of its row or column, and the scale of values 32 g ..  The instruction adds the 32
// products of a block with 13 bits below the largest (1 + 2^-13 is exact, 1 + 2^-14 is 1) and blocks in 32 bits: at most 32
// 2^-13 of a block's largest product, typically 2^-16 of the sum's terms, where each code is already 2^-5 off.  A choice for results
// of 16 bits and fewer, whose last bit is 2^-8 or 2^-11; those of 32 bits are of codes turned into bfloat16 (widen).
__device__ __forceinline__ f4 mfma_scaled(i8x a, i8x b, f4 c, int sa, int sb)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
}

// 16 codes and their scale to bfloat16, which holds them (values under 2^-126 as far as its subnormal numbers do): products of
// these are added in 32 bits throughout, at half the rate of the codes' own and with the conversions on top
__device__ __forceinline__ void widen(u4 q, unsigned byte, u4* w)
{
    const float scale = scale_value(byte);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i >> 1][(i & 1) * 2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[i], scale, false));
        w[i >> 1][(i & 1) * 2 + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(q[i], scale, true));
    }
}

// a lane's 32 codes of 128; scales: of values 32 (g / 2) .. in the first byte, of 64 + 32 (g / 2) .. in the second
__device__ __forceinline__ void widen(i8x q, int scales, u4* w)
{
    widen(u4{(unsigned)q[0], (unsigned)q[1], (unsigned)q[2], (unsigned)q[3]}, scales & 255, w);
    widen(u4{(unsigned)q[4], (unsigned)q[5], (unsigned)q[6], (unsigned)q[7]}, scales >> 8, w + 2);
}

__device__ __forceinline__ u4 across_read(const char* lds, int a0, int a1)
{
    typedef __attribute__((address_space(3))) s4* at;
    const u2 lo = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(lds + a0)));
    const u2 hi = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((at)(lds + a1)));
    return u4{lo[0], lo[1], hi[0], hi[1]};
}

// ---- epilogue of eight neighbouring columns n.. of row m; four neighbouring lanes hold a block of 32 columns between them.
// All lanes call; columns past Q and rows past P, or that do not exist, are not written or are zeros.

// what it reads, sent for ahead of its use: the residual, or the codes and the scale of what was kept
struct Fetched {
    u4 a, b;
    unsigned scale;
};

__device__ __forceinline__ Fetched fetch(const Epilogue& e, int m, int n, int P, int Q, bool there)
{
    Fetched f{};
    const int left = m < P && there ? Q - n : 0;
    if (left > 0) {
        if (e.kept_act != LAST_ACT_NONE) {
            unsigned lo, hi;
            load_codes(e.kept.q + (size_t)m * e.kept.pitch, n, left, &lo, &hi);
            f.a[0] = lo;
            f.a[1] = hi;
            f.scale = e.kept.scales[(size_t)m * e.kept.scale_pitch + n / kBlock];
        } else if (e.res) {
            const size_t at = (size_t)m * e.pres + n;
            if (e.type == LAST_F32) {
                const Raw<float> r = raw8<float>(e.res, at, left);
                f.a = r.a;
                f.b = r.b;
            } else {
                f.a = raw8<bf16_t>(e.res, at, left).a;
            }
        }
    }
    return f;
}

__device__ __forceinline__ void finish(const Epilogue& e, int m, int n, int P, int Q, bool there, const float* bias, const Fetched& f, float* v)
{
    const int left = m < P ? Q - n : 0;
    if (e.kept_act != LAST_ACT_NONE) {
        const float sc = scale_value(f.scale);
        float h[8];
        if (e.kept.e4m3) {
            decode4<true>(f.a[0], sc, h);
            decode4<true>(f.a[1], sc, h + 4);
        } else {
            decode4<false>(f.a[0], sc, h);
            decode4<false>(f.a[1], sc, h + 4);
        }
        times_slope(e.kept_act, h, v);
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = there && u < left ? v[u] + bias[u] : 0.f;
    if (e.kept_act == LAST_ACT_NONE && e.kept.q)
        store_eight(e.kept, m, n, left, (n & (kBlock - 1)) == 0, quad_max(top8(v)), v);
    activate8(e.act, v);
    if (e.res) {
        float r[8];
        if (e.type == LAST_F32) unpack<float>(Raw<float>{f.a, f.b}, r);
        else if (e.type == LAST_BF16) unpack<bf16_t>(Raw<bf16_t>{f.a}, r);
        else unpack<f16_t>(Raw<f16_t>{f.a}, r);
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] += r[u];
    }
    if (e.out.q) store_eight(e.out, m, n, left, (n & (kBlock - 1)) == 0, quad_max(top8(v)), v);
    if (e.y && left > 0) store8_as(e.type, e.y, (size_t)m * e.py + n, left, v);
}

__device__ __forceinline__ void load_bias(const Epilogue& e, int n, int Q, float* b)
{
    load8<float>(e.bias, n, e.bias ? Q - n : 0, b);
}

// Eight columns that are all inside of rows that all are, the common case, without a branch around a load or a store, so that no
// store is waited for (they count with the loads, in order).  What is read beside the sums is sent for four rows at a time, a
// batch ahead, and also where no frame is, whose results are zeros.
enum { kRowsPlain = 0, kRowsResidual = 1, kRowsSlope = 2, kRowsKeep = 3, kRowsWide = 4, kRowsEight = 5, kRowsNone = 6, kRowsAny = 7 };

__device__ __forceinline__ int rows_kind(const Epilogue& e)
{
    if (e.out.q) return !e.res && !e.kept.q ? kRowsEight : kRowsAny;
    if (e.type == LAST_F32) return !e.res && !e.kept.q ? kRowsWide : kRowsAny;
    if (e.kept_act != LAST_ACT_NONE) return kRowsSlope;
    if (e.res) return !e.kept.q ? kRowsResidual : kRowsAny;
    return e.kept.q ? kRowsKeep : kRowsPlain;
}

__device__ __forceinline__ u4 pack8(int type, const float* v)
{
    if (type == LAST_BF16) return u4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
    return u4{f16_pair(v[0], v[1]), f16_pair(v[2], v[3]), f16_pair(v[4], v[5]), f16_pair(v[6], v[7])};
}

__device__ __forceinline__ unsigned encode_block(bool e4m3, const float* v, unsigned* lo, unsigned* hi)
{
    const unsigned top = quad_max(top8(v));
    const unsigned byte = e4m3 ? scale_byte<true>(top) : scale_byte<false>(top);
    *lo = e4m3 ? encode4<true>(v, byte) : encode4<false>(v, byte);
    *hi = e4m3 ? encode4<true>(v + 4, byte) : encode4<false>(v + 4, byte);
    return byte;
}

// m: this lane's first row, every `step`-th of which it has, COUNT in all, and bit step * i of `exist` tells whether the i-th
// exists; n: its columns.  get(i, v): the sums of its i-th row.
template <int KIND, int COUNT, typename Get>
__device__ __forceinline__ void fast_rows(const Epilogue& e, size_t m, int n, int step, unsigned long long exist, const float* bias, Get get)
{
    constexpr bool kExtra = KIND == kRowsResidual || KIND == kRowsSlope;
    constexpr int kBatch = !kExtra ? 1 : COUNT < 4 ? COUNT : 4;
    static_assert(COUNT % kBatch == 0, "whole batches");
    struct Extra {
        u4 w;
        unsigned scale;
    };
    const auto extra = [&](int i) {
        const size_t row = m + (size_t)(i < COUNT ? i : COUNT - 1) * step;
        Extra x{};
        if constexpr (KIND == kRowsResidual) x.w = *(const u4_any*)((const uint16_t*)e.res + row * e.pres + n);
        if constexpr (KIND == kRowsSlope) {
            const u2 q = *(const u2_any*)(e.kept.q + row * e.kept.pitch + n);
            x.w[0] = q[0];
            x.w[1] = q[1];
            x.scale = e.kept.scales[row * e.kept.scale_pitch + n / kBlock];
        }
        return x;
    };
    const auto finish_row = [&](int i, const Extra& x) {
        const size_t row = m + (size_t)i * step;
        if constexpr (KIND == kRowsNone) {                   // no frame: nothing to read or to compute
            *(u4_any*)((uint16_t*)e.y + row * e.py + n) = u4{0, 0, 0, 0};
            return;
        }
        const bool there = exist >> (i * step) & 1;
        float v[8];
        get(i, v);
        if constexpr (KIND == kRowsSlope) {
            float h[8];
            const float sc = scale_value(x.scale);
            if (e.kept.e4m3) {
                decode4<true>(x.w[0], sc, h);
                decode4<true>(x.w[1], sc, h + 4);
            } else {
                decode4<false>(x.w[0], sc, h);
                decode4<false>(x.w[1], sc, h + 4);
            }
            times_slope(e.kept_act, h, v);
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] += bias[u];
        }
        if constexpr (KIND == kRowsKeep) {
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = there ? v[u] : 0.f;
            unsigned lo, hi;
            const unsigned byte = encode_block(e.kept.e4m3, v, &lo, &hi);
            *(u2_any*)(e.kept.q + row * e.kept.pitch + n) = u2{lo, hi};
            e.kept.scales[row * e.kept.scale_pitch + n / kBlock] = (uint8_t)byte;    // (all four lanes of the block, the same)
        }
        activate8(e.act, v);
        if constexpr (KIND == kRowsResidual) {
            float r[8];
            if (e.type == LAST_BF16) unpack<bf16_t>(Raw<bf16_t>{x.w}, r);
            else unpack<f16_t>(Raw<f16_t>{x.w}, r);
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] += r[u];
        }
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = there ? v[u] : 0.f;
        if constexpr (KIND == kRowsEight) {
            unsigned lo, hi;
            const unsigned byte = encode_block(e.out.e4m3, v, &lo, &hi);
            *(u2_any*)(e.out.q + row * e.out.pitch + n) = u2{lo, hi};
            e.out.scales[row * e.out.scale_pitch + n / kBlock] = (uint8_t)byte;
        } else if constexpr (KIND == kRowsWide) {
            Elt<float>::put8(e.y, row * e.py + n, v);
        } else {
            *(u4_any*)((uint16_t*)e.y + row * e.py + n) = pack8(e.type, v);
        }
    };
    Extra now[kBatch], next[kBatch];
#pragma unroll
    for (int j = 0; j < kBatch; ++j) next[j] = extra(j);
#pragma unroll 1
    for (int i = 0; i < COUNT; i += kBatch) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) now[j] = next[j];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) next[j] = extra(i + kBatch + j);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) finish_row(i + j, now[j]);
    }
}

// tiles in the order of the workgroups: workgroups i = j (mod 8) share an XCD and its L2, so each XCD gets a stretch of
// the tiles; within it, columns of eight tiles
__device__ __forceinline__ void tile_of(int id, int n, int tiles_p, int tiles_q, int* tp, int* tq)
{
    const int full = n / 8 * 8;
    if (id < full) id = (id & 7) * (n / 8) + (id >> 3);
    const int per = 8 * tiles_q, g = id / per, first = g * 8;
    const int h = tiles_p - first < 8 ? tiles_p - first : 8, in = id - g * per;
    *tp = first + in % h;
    *tq = in / h;
}

// The loop.  A step's 128 bytes are multiplied in two phases: the halves of its reduction, or, with 8-bit operands, whose
// instruction takes 128 values at once, the halves of the rows of P.  A fragment of the next phase is read from LDS into the
// registers of one that was just used, so that the matrix cores wait for LDS as little as there are few registers for copies.
// One barrier a step, between the phases: all fragments of the step have then been read, its buffers are free, and the loads
// that fill them are sent one by one between the matrix instructions of the second phase, SP steps of P and SQ of Q ahead of
// their use.
template <typename E, int LP, int LQ, int BP, int BQ, int WP, int WQ, int SP, int SQ>
__global__ __launch_bounds__(WP * WQ * kWave, 2) void product_kernel(ProductArgs a)
{
    constexpr int kThreads = WP * WQ * kWave;
    constexpr bool kEight = Elt<E>::size == 1, kWide = std::is_same_v<E, wide_t>;
    constexpr int NP = BP / WP / 16, NQ = BQ / WQ / 16;                   // accumulators of a wavefront
    using TP = Tile<LP, BP, kThreads>;
    using TQ = Tile<LQ, BQ, kThreads>;
    constexpr unsigned kAtQ = SP * TP::kBytes, kLds = kAtQ + SQ * TQ::kBytes;
    constexpr int kScaleRows = (BP + BQ + kThreads - 1) / kThreads * kThreads, kScaleLoads = kEight ? kScaleRows / kThreads : 0;
    static_assert(SQ >= 2 && (SP == SQ || (SP == SQ + 1 && !kEight)), "the order of the loads");
    __shared__ __align__(1024) char lds[kLds];
    __shared__ __align__(4) uint8_t scales[kEight ? SQ : 1][kEight ? kScaleRows * 4 : 1];

    const int lane = (int)threadIdx.x % kWave, g = lane >> 4, i16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), wp = wave / WQ, wq = wave % WQ;
    int tp, tq;
    tile_of((int)blockIdx.x, a.tiles_p * a.tiles_q, a.tiles_p, a.tiles_q, &tp, &tq);
    const int p0 = tp * BP, q0 = tq * BQ;
    const long long k0 = (long long)blockIdx.y * a.share, k1 = k0 + a.share < a.K ? k0 + a.share : a.K;

    TP P;
    TQ Q;
    P.init(p0, a.P, a.pp, LP == kAlong ? &a.frames : nullptr);
    Q.init(q0, a.Q, a.pq, nullptr);
    bool work = true;                                                     // a row of the tile exists
    if (LP == kAlong && a.frames.len) {
        unsigned* some = (unsigned*)lds;
        const unsigned long long b = __ballot(P.valid != 0);
        if (lane == 0) some[wave] = b != 0;
        __syncthreads();
        work = false;
        for (int w = 0; w < WP * WQ; ++w) work |= __builtin_amdgcn_readfirstlane((int)some[w]) != 0;
        __syncthreads();
    }
    const int steps = work ? (int)((k1 - k0 + (LP == kAlong ? kStep : 64) - 1) / (LP == kAlong ? kStep : 64)) : 0;

    f4 acc[NP][NQ];
    constexpr int NB = NP / WQ;                                           // row sums of P: the WQ wavefronts of the same rows share them
    f4 accb[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) accb[j] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < NP; ++x) {
#pragma unroll
        for (int y = 0; y < NQ; ++y) acc[x][y] = f4{0.f, 0.f, 0.f, 0.f};
    }
    const bool bias_too = LP == kAcross && a.e.part_bias && tq == 0;

    const char* bp = a.p + (LP == kAlong ? (long long)p0 * a.pp + k0 : (long long)p0 * 2 + k0 * a.pp);
    const char* bq = a.q + (LQ == kAlong ? (long long)q0 * a.pq + k0 : (long long)q0 * 2 + (LP == kAlong ? k0 / 2 : k0) * a.pq);

    // Loads of step s of P and s of Q; beyond the last step they are sent all the same, from nowhere, so that their number
    // always tells which have come.
    const auto left_of = [&](int s) { return s < steps ? k1 - k0 - (long long)s * (LP == kAlong ? kStep : 64) : 0ll; };
    const auto mask_of = [&](int s) {
        if constexpr (LP == kAcross) {
            const long long left = left_of(s);
            unsigned long long m = left >= 64 ? ~0ull : (1ull << left) - 1;
            // (constant memory to the compiler: a scalar load, which is not counted with those that are waited for)
            typedef const __attribute__((address_space(4))) unsigned long long* constant_t;
            if (a.mask && s < steps) m &= ((constant_t)(uintptr_t)a.mask)[(k0 >> 6) + s];
            return m;
        } else if constexpr (LQ == kAcross) {
            const long long rows = s < steps ? a.q_rows - k0 / 2 - 64ll * s : 0;
            return rows < 64 ? (1ull << rows) - 1 : ~0ull;
        } else {
            return ~0ull;
        }
    };
    struct Sent {                                                         // a step's loads of an operand
        u4 buffer;
        unsigned bits, to;
    };
    const unsigned lds_at = lds_byte(lds);
    const auto sent_p = [&](int s, int buf, unsigned long long mask) {
        return Sent{descriptor(bp + (long long)s * (LP == kAlong ? kStep : 64 * a.pp)), P.bits(left_of(s), mask), lds_at + buf * TP::kBytes};
    };
    const auto sent_q = [&](int s, int buf, unsigned long long mask) {
        return Sent{descriptor(bq + (long long)s * (LQ == kAlong ? kStep : 64 * a.pq)), Q.bits(left_of(s), mask), lds_at + kAtQ + buf * TQ::kBytes};
    };
    const auto send_scales = [&](int j, int s, int buf) {                 // a row's four scales of the step
        const int r = j * kThreads + (int)threadIdx.x, first = j * kThreads + wave * kWave;
        const bool isp = first < BP;
        const int row = isp ? r : r - BP;
        const bool ok = s < steps && (isp ? p0 + row < a.P : row < BQ && q0 + row < a.Q);
        const unsigned o = ok ? (unsigned)(row * (isp ? a.psp : a.psq)) + (unsigned)(k0 / kBlock) + 4u * (unsigned)s : kNowhere;
        to_lds<4>(descriptor(isp ? a.sp + (long long)p0 * a.psp : a.sq + (long long)q0 * a.psq), o, 0, lds_byte(&scales[buf][first * 4]));
    };

    // LDS byte of a wavefront's first fragment of a step's first half.  Along: fragment x is 16 rows on, half h at piece ^ 4 h.
    // Across: half h is 32 rows on, the second four rows of a lane four on, and fragment x at granule ^ x (a wavefront's first
    // column is a multiple of its 16 NP, NQ, powers of two, so the sum is an exclusive or).
    const int kr = 8 * g + (i16 >> 2), swizzled = (g ^ along_swizzle(i16)) << 4;
    const unsigned at_p = LP == kAlong ? (wp * (BP / WP) + i16) * kStep + swizzled
                                       : kr * (BP * 2) + ((wp * NP ^ across_swizzle<BP>(kr)) << 5) + (i16 & 3) * 8;
    const unsigned at_q = kAtQ + (LQ == kAlong ? (wq * (BQ / WQ) + i16) * kStep + swizzled
                                               : kr * (BQ * 2) + ((wq * NQ ^ across_swizzle<BQ>(kr)) << 5) + (i16 & 3) * 8);
    const auto read_p = [&](unsigned at, int half, int x) {
        if constexpr (LP == kAlong) return *(const u4*)(lds + (at ^ half * 64) + x * 16 * kStep);
        else return across_read(lds + (at ^ x * 32) + half * 32 * BP * 2, 0, 4 * BP * 2);
    };
    const auto read_q = [&](unsigned at, int half, int y) {
        if constexpr (LQ == kAlong) return *(const u4*)(lds + (at ^ half * 64) + y * 16 * kStep);
        else return across_read(lds + (at ^ y * 32) + half * 32 * BQ * 2, 0, 4 * BQ * 2);
    };
    // an address that the compiler computes here and does not keep for all fragments from step to step
    const auto here = [&](unsigned at) {
        asm volatile("" : "+v"(at));
        return at;
    };

    if (steps > 0) {
        unsigned long long mask = ~0ull, mask_last = ~0ull;
#pragma unroll
        for (int s = 0; s < SP; ++s) {
            mask_last = mask;
            mask = mask_of(s);
            const Sent p = sent_p(s, s, mask);
#pragma unroll
            for (int j = 0; j < TP::kLoads; ++j) P.load(j, p.buffer, p.bits, p.to);
            if (s < SQ) {
                const Sent q = sent_q(s, s, mask);
#pragma unroll
                for (int j = 0; j < TQ::kLoads; ++j) Q.load(j, q.buffer, q.bits, q.to);
#pragma unroll
                for (int j = 0; j < kScaleLoads; ++j) send_scales(j, s, s);
            }
        }
        arrived<TP::kLoads * (SP - 1) + (TQ::kLoads + kScaleLoads) * (SQ - 1)>();

        // of those sent, a step's Q before its P, what may still be on its way when the next step's fragments are read
        constexpr int kLater = (SQ - 2) * (TP::kLoads + TQ::kLoads + kScaleLoads) + (SP > SQ ? TP::kLoads : 0);
        int buf_p = 0, buf_q = 0;                                         // of step s
        const auto after = [&](int b, int n) { return b + 1 == n ? 0 : b + 1; };
        if constexpr (kEight) {
            constexpr int H = NP / 2, kSends = (TP::kLoads + TQ::kLoads + kScaleLoads + H - 1) / H;
            i8x fp[NP], fq[NQ];
            int cp[NP], cq[NQ];
            u4 vp[kWide ? 4 : 1], vq[kWide ? NQ : 1][kWide ? 4 : 1];      // widened: a row of P, all columns of Q
            const auto scale_of = [&](int buf, int r) {
                if constexpr (kWide) return scales[buf][r * 4 + (g >> 1)] | scales[buf][r * 4 + 2 + (g >> 1)] << 8;
                else return (int)scales[buf][r * 4 + g];
            };
            const auto take_p = [&](int buf, int x) {
                const unsigned at = here(at_p + buf * TP::kBytes);
                fp[x] = join8(read_p(at, 0, x), read_p(at, 1, x));
                cp[x] = scale_of(buf, wp * (BP / WP) + x * 16 + i16);
            };
            const auto take_q = [&](int buf, int y) {
                const unsigned at = here(at_q + buf * TQ::kBytes);
                fq[y] = join8(read_q(at, 0, y), read_q(at, 1, y));
                cq[y] = scale_of(buf, BP + wq * (BQ / WQ) + y * 16 + i16);
            };
            const auto multiply = [&](int x, int y) {
                if constexpr (kWide) {
                    if (y == 0) widen(fp[x], cp[x], vp);
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[x][y] = Mfma<bf16_t>::go(vq[y][k], vp[k], acc[x][y]);
                } else {
                    acc[x][y] = mfma_scaled(fq[y], fp[x], acc[x][y], cq[y], cp[x]);
                }
            };
#pragma unroll
            for (int y = 0; y < NQ; ++y) take_q(0, y);
#pragma unroll
            for (int x = 0; x < H; ++x) take_p(0, x);
            for (int s = 0; s < steps; ++s) {
                if constexpr (kWide) {
#pragma unroll
                    for (int y = 0; y < NQ; ++y) widen(fq[y], cq[y], vq[y]);
                }
#pragma unroll
                for (int x = 0; x < H; ++x) {
                    take_p(buf_q, H + x);
#pragma unroll
                    for (int y = 0; y < NQ; ++y) multiply(x, y);
                    __builtin_amdgcn_sched_barrier(0);
                }
                arrived<kLater>();
                const int next = after(buf_q, SQ);
                const Sent p = sent_p(s + SP, buf_q, ~0ull), q = sent_q(s + SQ, buf_q, ~0ull);
#pragma unroll
                for (int x = 0; x < H; ++x) {
#pragma unroll
                    for (int j = kSends * x; j < kSends * x + kSends; ++j) {
                        if (j < TP::kLoads) P.load(j, p.buffer, p.bits, p.to);
                        else if (j < TP::kLoads + TQ::kLoads) Q.load(j - TP::kLoads, q.buffer, q.bits, q.to);
                        else if (j < TP::kLoads + TQ::kLoads + kScaleLoads) send_scales(j - TP::kLoads - TQ::kLoads, s + SQ, buf_q);
                    }
                    take_p(next, x);
                    if (x + 1 < H) {
#pragma unroll
                        for (int y = 0; y < NQ; ++y) multiply(H + x, y);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
#pragma unroll
                for (int y = 0; y < NQ; ++y) {
                    multiply(NP - 1, y);
                    take_q(next, y);
                    __builtin_amdgcn_sched_barrier(0);
                }
                buf_q = next;
            }
        } else {
            // Of P's fragments the last kTwice have two places, so that the next phase's can be read while they are used, and the last
            // read of a phase has the products of as many rows to come.
            constexpr int kTwice = NP >= 8 ? 2 : 1, kOwn = NP - kTwice;
            u4 fp[kOwn], fe[2][kTwice], fq[2][NQ];
            const unsigned one = Elt<E>::type == LAST_BF16 ? 0x3f803f80u : 0x3c003c00u;
            const auto multiply = [&](int half, int x) {
                const u4 f = x < kOwn ? fp[x < kOwn ? x : 0] : fe[half][x < kOwn ? 0 : x - kOwn];
#pragma unroll
                for (int y = 0; y < NQ; ++y) acc[x][y] = Mfma<E>::go(fq[half][y], f, acc[x][y]);
                if constexpr (LP == kAcross) {
                    if (bias_too && x / NB == wq) accb[x % NB] = Mfma<E>::go(u4{one, one, one, one}, f, accb[x % NB]);
                }
            };
            // what is read for the phase of `half` beside the products of row x of the phase before
            const auto read = [&](unsigned ap, unsigned aq, int half, int x) {
#pragma unroll
                for (int y = 2 * x; y < 2 * x + 2; ++y)
                    if (y < NQ) fq[half][y] = read_q(aq, half, y);
                if (x < kTwice) fe[half][x] = read_p(ap, half, kOwn + x);
                if (x < kOwn) fp[x] = read_p(ap, half, x);
            };
            static_assert(2 * NP >= NQ && kOwn >= kTwice, "all fragments are read");
            {
                const unsigned ap = here(at_p), aq = here(at_q);
#pragma unroll
                for (int x = 0; x < NP; ++x) read(ap, aq, 0, x);
            }
            for (int s = 0; s < steps; ++s) {
                const int next_p = after(buf_p, SP), next_q = after(buf_q, SQ);
                mask_last = mask;
                mask = mask_of(s + SP);
                const Sent q = sent_q(s + SQ, buf_q, SP > SQ ? mask_last : mask), p = sent_p(s + SP, buf_p, mask);
                {
                    const unsigned ap = here(at_p + buf_p * TP::kBytes), aq = here(at_q + buf_q * TQ::kBytes);
#pragma unroll
                    for (int x = 0; x < NP; ++x) {
                        multiply(0, x);
                        read(ap, aq, 1, x);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                arrived<kLater>();
                {
                    const unsigned ap = here(at_p + next_p * TP::kBytes), aq = here(at_q + next_q * TQ::kBytes);
                    constexpr int kSends = (TP::kLoads + TQ::kLoads + NP - 1) / NP;
#pragma unroll
                    for (int x = 0; x < NP; ++x) {
                        multiply(1, x);
#pragma unroll
                        for (int j = kSends * x; j < kSends * x + kSends; ++j) {
                            if (j < TQ::kLoads) Q.load(j, q.buffer, q.bits, q.to);
                            else if (j < TQ::kLoads + TP::kLoads) P.load(j - TQ::kLoads, p.buffer, p.bits, p.to);
                        }
                        read(ap, aq, 0, x);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                buf_p = next_p;
                buf_q = next_q;
            }
        }
        arrived<0>();                                                     // the loads from nowhere, before LDS is used again
    }

    // A lane has row 16 x + i16 of P and columns 16 y + 4 g .. of Q.  The epilogue wants eight columns of a row in a lane and
    // whole lines of rows in a wavefront: 64 rows at a time change places in the wavefront's own part of LDS, whose 16-byte
    // pieces of a row are swizzled by the row.
    constexpr int kCols = BQ / WQ, kPieces = kCols / 4, kLanes = kCols / 8, kRows = kWave / kLanes, XS = NP < 4 ? NP : 4;
    static_assert((size_t)XS * 16 * kCols * 4 * WP * WQ <= sizeof(lds), "room for the epilogue");
    char* mine = lds + wave * (XS * 16 * kCols * 4);
    const int c = (lane % kLanes) * 8, n = q0 + wq * kCols + c;
    Epilogue e = a.e;
    if (e.part) {                                                         // sums of a share go out as they are
        e.y = e.part + (size_t)blockIdx.y * a.P * a.Q;
        e.py = a.Q;
        e.type = LAST_F32;
    }
    const int kind = rows_kind(e);
    float bias[8];
    load_bias(e, n, a.Q, bias);
#pragma unroll 1
    for (int part = 0; part < NP / XS; ++part) {
#pragma unroll
        for (int p = 0; p < NP / XS; ++p)
            if (p == part) {
#pragma unroll
                for (int x = 0; x < XS; ++x)
#pragma unroll
                    for (int y = 0; y < NQ; ++y)
                        *(f4*)(mine + (x * 16 + i16) * (kCols * 4) + (((4 * y + g) ^ (i16 & (kPieces - 1))) << 4)) = acc[p * XS + x][y];
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();                     // (the reads follow the writes in the wavefront's order)
        const int first = p0 + wp * (BP / WP) + part * XS * 16;
        const auto get = [&](int r, float* v) {
            const f4 lo = *(const f4*)(mine + r * (kCols * 4) + (((c / 4) ^ (r & (kPieces - 1))) << 4));
            const f4 hi = *(const f4*)(mine + r * (kCols * 4) + (((c / 4 + 1) ^ (r & (kPieces - 1))) << 4));
#pragma unroll
            for (int u = 0; u < 4; ++u) { v[u] = lo[u]; v[4 + u] = hi[u]; }
        };
        const auto get_mine = [&](int i, float* v) { get(lane / kLanes + i * kRows, v); };
        // bits of the rows that exist
        const int mine_row = first + lane % (XS * 16);
        const unsigned long long rows = __ballot(mine_row < a.P && (LP == kAcross || frame_exists(a.frames, mine_row)));
        const size_t m0 = (size_t)first + lane / kLanes;
        constexpr int kCount = XS * 16 / kRows;
        // blocks in 8 bits need all their lanes, else a lane goes by its own columns
        const int last = kind == kRowsKeep || kind == kRowsEight ? q0 + (wq + 1) * kCols : n + 8;
        const unsigned long long exist = rows >> (lane / kLanes);
        if (first + XS * 16 <= a.P && last <= a.Q && kind != kRowsAny) {
            if (rows == 0 && kind <= kRowsSlope) fast_rows<kRowsNone, kCount>(e, m0, n, kRows, exist, bias, get_mine);
            else if (kind == kRowsPlain) fast_rows<kRowsPlain, kCount>(e, m0, n, kRows, exist, bias, get_mine);
            else if (kind == kRowsResidual) fast_rows<kRowsResidual, kCount>(e, m0, n, kRows, exist, bias, get_mine);
            else if (kind == kRowsSlope) fast_rows<kRowsSlope, kCount>(e, m0, n, kRows, exist, bias, get_mine);
            else if (kind == kRowsKeep) fast_rows<kRowsKeep, kCount>(e, m0, n, kRows, exist, bias, get_mine);
            else if (kind == kRowsEight) fast_rows<kRowsEight, kCount>(e, m0, n, kRows, exist, bias, get_mine);
            else fast_rows<kRowsWide, kCount>(e, m0, n, kRows, exist, bias, get_mine);
        } else if (n - c < a.Q) {                            // (some column of the wavefront)
            bool there = rows >> (lane / kLanes) & 1;
            Fetched f = fetch(e, (int)m0, n, a.P, a.Q, there);
#pragma unroll 1
            for (int r = lane / kLanes; r < XS * 16; r += kRows) {
                const int m = first + r;
                const bool there_next = r + kRows < XS * 16 && (rows >> (r + kRows) & 1) != 0;
                const Fetched f_next = fetch(e, m + kRows, n, a.P, a.Q, there_next);
                float v[8];
                get(r, v);
                finish(e, m, n, a.P, a.Q, there, bias, f, v);
                f = f_next;
                there = there_next;
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    if (bias_too && g == 0) {
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int m = p0 + wp * (BP / WP) + (wq * NB + j) * 16 + i16;
            if (m < a.P) a.e.part_bias[(size_t)blockIdx.y * a.P + m] = accb[j][0];
        }
    }
}

// ---- few rows: y = act(x w^T + bias) + residual for at most 16 MT rows, bound by the bytes of w, which go from memory to
// registers once.  One row of 512 x 2048 in bfloat16 4.4 us, four of 4096 x 4096 in 8 bits 7.0 us (2.5 TB/s: a launch, a load, a
// sum through LDS and a store, one after the other), 10.7 us with results in float32.  A workgroup takes 16 QF columns, its wavefronts every kFewWaves-th 128 bytes of the rows, four (two) such
// steps' loads under way at a time; their sums meet in LDS.
constexpr int kFewWaves = 8;

template <typename E, int MT, int QF>
__global__ __launch_bounds__(kFewWaves * kWave) void few_kernel(ProductArgs a)
{
    constexpr bool kEight = Elt<E>::size == 1, kWide = std::is_same_v<E, wide_t>;
    constexpr int kDeep = kWide && MT * QF >= 4 ? 2 : 4;                 // (steps under way: as many as there are registers for)
    __shared__ f4 red[kFewWaves][MT][QF][kWave];
    const int lane = (int)threadIdx.x % kWave, g = lane >> 4, i16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
    const int q0 = (int)blockIdx.x * 16 * QF;
    const __amdgpu_buffer_rsrc_t bq = buffer_of(a.q + (long long)q0 * a.pq), bp = buffer_of(a.p);
    unsigned oq[QF], op[MT];
    int rq[QF];
#pragma unroll
    for (int f = 0; f < QF; ++f) {
        rq[f] = 16 * f + i16;
        oq[f] = q0 + rq[f] < a.Q ? (unsigned)(rq[f] * a.pq) + 16u * g : kNowhere;
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = t * 16 + i16;
        op[t] = m < a.P && frame_exists(a.frames, m) ? (unsigned)(m * a.pp) + 16u * g : kNowhere;
    }
    f4 acc[MT][QF];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int f = 0; f < QF; ++f) acc[t][f] = f4{0.f, 0.f, 0.f, 0.f};
    const int bytes = (int)a.K, steps = (bytes + kStep - 1) / kStep;
    for (int s0 = wave; s0 < steps; s0 += kFewWaves * kDeep) {
        u4 fq[kDeep][QF][2], fp[kDeep][MT][2];
        int cq[kDeep][QF], cp[kDeep][MT];
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
            const int k = (s0 + d * kFewWaves) * kStep;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int kh = k + 64 * h;
                const bool in = kh + 16 * g < bytes;
#pragma unroll
                for (int f = 0; f < QF; ++f)
                    fq[d][f][h] = __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(bq, in ? (int)(oq[f] + kh) : (int)kNowhere, 0, 0));
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    fp[d][t][h] = __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(bp, in ? (int)(op[t] + kh) : (int)kNowhere, 0, 0));
            }
            if constexpr (kEight) {
                const auto scale_of = [&](bool there, const uint8_t* row, int block) { return there && block * kBlock < bytes ? (int)row[block] : 0; };
                const auto scales_of = [&](bool there, const uint8_t* row) {
                    if constexpr (kWide) return scale_of(there, row, k / kBlock + (g >> 1)) | scale_of(there, row, k / kBlock + 2 + (g >> 1)) << 8;
                    else return scale_of(there, row, k / kBlock + g);
                };
#pragma unroll
                for (int f = 0; f < QF; ++f) cq[d][f] = scales_of(oq[f] < kNowhere, a.sq + (q0 + rq[f]) * a.psq);
#pragma unroll
                for (int t = 0; t < MT; ++t) cp[d][t] = scales_of(op[t] < kNowhere, a.sp + (t * 16 + i16) * a.psp);
            }
        }
#pragma unroll
        for (int d = 0; d < kDeep; ++d) {
            u4 vq[kWide ? QF : 1][kWide ? 4 : 1];
            if constexpr (kWide) {
#pragma unroll
                for (int f = 0; f < QF; ++f) widen(join8(fq[d][f][0], fq[d][f][1]), cq[d][f], vq[f]);
            }
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                u4 vp[kWide ? 4 : 1];
                if constexpr (kWide) widen(join8(fp[d][t][0], fp[d][t][1]), cp[d][t], vp);
#pragma unroll
                for (int f = 0; f < QF; ++f) {
                    if constexpr (kWide) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) acc[t][f] = Mfma<bf16_t>::go(vq[f][j], vp[j], acc[t][f]);
                    } else if constexpr (kEight) {
                        acc[t][f] = mfma_scaled(join8(fq[d][f][0], fq[d][f][1]), join8(fp[d][t][0], fp[d][t][1]), acc[t][f], cq[d][f], cp[d][t]);
                    } else {
                        acc[t][f] = Mfma<E>::go(fq[d][f][0], fp[d][t][0], acc[t][f]);
                        acc[t][f] = Mfma<E>::go(fq[d][f][1], fp[d][t][1], acc[t][f]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int f = 0; f < QF; ++f) red[wave][t][f][lane] = acc[t][f];
    __syncthreads();
    if (wave >= MT) return;
    // lane: row lane / 4 of the wavefront's 16, columns 8 (lane & 3) .. of the workgroup's 16 QF
    const int r = lane >> 2, c = lane & 3, m = wave * 16 + r;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (c < 2 * QF) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            f4 t = red[0][wave][c >> 1][(2 * (c & 1) + h) * 16 + r];
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w) t += red[w][wave][c >> 1][(2 * (c & 1) + h) * 16 + r];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * h + i] = t[i];
        }
    }
    const int P = c < 2 * QF ? a.P : 0, n = q0 + 8 * c;
    const bool there = m < P && frame_exists(a.frames, m);
    float bias[8];
    load_bias(a.e, n, a.Q, bias);
    finish(a.e, m, n, P, a.Q, there, bias, fetch(a.e, m, n, P, a.Q, there), v);
}

// ---- shares of a reduction joined, in order, with the epilogue; a wavefront has 16 rows of 32 columns
__global__ __launch_bounds__(256) void product_join_kernel(ProductArgs a, int splits)
{
    const int lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave;
    const int across = (a.Q + 31) / 32;
    const unsigned id = blockIdx.x * 4u + wave;
    const int m = (int)(id / (unsigned)across) * 16 + (lane >> 2), n = (int)(id % (unsigned)across) * 32 + 8 * (lane & 3);
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (m < a.P) {
        for (int s = 0; s < splits; ++s) {
            float t[8];
            load8<float>(a.e.part + ((size_t)s * a.P + m) * a.Q, n, a.Q - n, t);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += t[k];
        }
        if (a.e.part_bias && n == 0) {
            float b = 0.f;
            for (int s = 0; s < splits; ++s) b += a.e.part_bias[(size_t)s * a.P + m];
            a.e.sum_bias[m] = b;
        }
    }
    const bool there = m < a.P && frame_exists(a.frames, m);
    float bias[8];
    load_bias(a.e, n, a.Q, bias);
    finish(a.e, m, n, a.P, a.Q, there, bias, fetch(a.e, m, n, a.P, a.Q, there), v);
}

// ---- before a product, in one launch: rows of operands laid out at multiples of 16 bytes with zeros behind them, 16 bytes a
// thread; an activation formed again from what was kept; which rows exist, a bit each
struct PrepareArgs {
    struct Rows {
        const uint8_t* in;
        uint8_t* out;
        long long pitch, out_pitch, count;       // bytes from a row to the next, rows
        int bytes;                               // of a row
        unsigned groups;                         // workgroups that do it
    } rows[4];
    unsigned groups;                             // of all four
    unsigned first;                              // of this launch's workgroups
    KeepArgs values;
    unsigned values_groups;
    Frames frames;
    int frame_rows;
    unsigned long long* mask;
};

__global__ __launch_bounds__(256) void prepare_kernel(PrepareArgs a)
{
    unsigned group = a.first + blockIdx.x;
    if (group >= a.groups && group - a.groups < a.values_groups) {
        kept_values(a.values, group - a.groups);
        return;
    }
    if (group >= a.groups) {
        const int row = (int)((group - a.groups - a.values_groups) * 256 + threadIdx.x);
        const unsigned long long m = __ballot(row < a.frame_rows && frame_exists(a.frames, row));
        if ((threadIdx.x & (kWave - 1)) == 0 && row < a.frame_rows) a.mask[row >> 6] = m;
        return;
    }
    int k = 0;
    while (group >= a.rows[k].groups) group -= a.rows[k++].groups;
    const auto& r = a.rows[k];
    const unsigned per = (unsigned)(r.out_pitch / 16);
    const unsigned long long i = (unsigned long long)group * 256 + threadIdx.x;
    const unsigned long long row = i >> 32 ? i / per : (unsigned)i / per;
    const int at = (int)(i - row * per) * 16;
    if (row >= (unsigned long long)r.count) return;
    const uint8_t* p = r.in + row * r.pitch + at;
    u4 w = {0u, 0u, 0u, 0u};
    if (at + 16 <= r.bytes) {
        w = *(const u4_byte*)p;
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (at + j < r.bytes) w[j >> 2] |= (unsigned)p[j] << (8 * (j & 3));
    }
    *(u4*)(r.out + row * r.out_pitch + at) = w;
}

}  // namespace last
