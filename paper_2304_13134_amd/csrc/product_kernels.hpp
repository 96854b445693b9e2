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
#pragma once
#include "layer.hpp"

namespace last {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef int i8x __attribute__((ext_vector_type(8)));
typedef int i4x __attribute__((ext_vector_type(4)));

typedef __attribute__((address_space(3))) void* lds_t;

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
    bool wide, wide_res, wide_bias;              // eight elements at a time are aligned
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
__device__ __forceinline__ int across_swizzle(int r) { return (r & 3) | ((r >> 3) & 1) << 2; }


__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* base)
{
    return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 0x7fffffff, 0x00020000);
}

// 64 lanes' 16 (4) bytes at offset `o` of the buffer at `base` to LDS from `to` on.  In assembly, since the compiler makes every
// later read of LDS wait for its own form of this; whoever reads waits with arrived().
template <int BYTES>
__device__ __forceinline__ void to_lds(const void* base, unsigned o, const void* to)
{
    const uint64_t p = (uint64_t)base;
    const u4 b = {(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)p), (unsigned)__builtin_amdgcn_readfirstlane((int)(p >> 32)) & 0xffffu,
                  0x7fffffffu, 0x00020000u};
    const unsigned m = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)(uintptr_t)(lds_t)to);
    if constexpr (BYTES == 16)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(m), "v"(o), "s"(b) : "memory");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(m), "v"(o), "s"(b) : "memory");
}

// what this wavefront sent to LDS and asked from it has come, then the same of the whole workgroup
__device__ __forceinline__ void arrived()
{
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// ---- one operand's tile: ROWS rows or columns of the output
template <int L, int ROWS, int THREADS>
struct Tile {
    static constexpr int kBytes = ROWS * kStep;
    static constexpr int kLoads = kBytes / 16 / THREADS;
    static constexpr int kPieces = L == kAlong ? 8 : ROWS / 8;           // 16-byte pieces of a row in LDS
    static_assert(kBytes % (16 * THREADS) == 0, "whole loads");
    static_assert(L == kAlong || ROWS >= 128, "eight granules to swizzle");
    unsigned off[kLoads];

    // first: first row or column of the tile; count: how many the matrix has
    __device__ void init(int first, int count, long long pitch, const Frames* frames, int* any)
    {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int i = j * THREADS + (int)threadIdx.x, r = i / kPieces, c = i % kPieces;
            if constexpr (L == kAlong) {
                bool ok = first + r < count;
                if (ok && frames) ok = frame_exists(*frames, first + r);
                if (any) *any |= ok;
                off[j] = ok ? (unsigned)(r * pitch) + 16u * (unsigned)(c ^ along_swizzle(r)) : kNowhere;
            } else {
                const int g = (c >> 1) ^ across_swizzle(r), col = g * 16 + (c & 1) * 8;
                off[j] = first + col < count ? (unsigned)(r * pitch) + 2u * (unsigned)col : kNowhere;
            }
        }
    }

    // the tile's 128 bytes or 64 rows from `base` on; left: how many of them the reduction still has
    __device__ __forceinline__ void load(const char* base, long long left, unsigned long long mask, char* lds)
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            unsigned o = off[j];
            if constexpr (L == kAlong) {
                if (left < kStep) {
                    const int i = j * THREADS + (int)threadIdx.x, r = i / kPieces, c = i % kPieces;
                    if (16 * (c ^ along_swizzle(r)) >= left) o = kNowhere;
                }
            } else {
                const int r = (j * THREADS + (int)threadIdx.x) / kPieces;
                if (!(mask >> r & 1)) o = kNowhere;
            }
            to_lds<16>(base, o, lds + (j * THREADS + wave * kWave) * 16);
        }
    }
};

// LDS byte of a piece of a row (kAlong)
__device__ __forceinline__ int along_at(int r, int piece) { return r * kStep + ((piece ^ along_swizzle(r)) << 4); }

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

__device__ __forceinline__ f4 mfma_scaled(const u4* a, const u4* b, f4 c, int sa, int sb)
{
    i8x x, y;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        x[k] = (int)a[0][k];
        x[4 + k] = (int)a[1][k];
        y[k] = (int)b[0][k];
        y[4 + k] = (int)b[1][k];
    }
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 0, 0, 0, sa, 0, sb);
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
__device__ __forceinline__ void finish(const Epilogue& e, int m, int n, int P, int Q, bool there, float* v)
{
    const int left = m < P ? Q - n : 0;
    if (e.kept_act != LAST_ACT_NONE) {
        if (there && left > 0) {
            unsigned lo, hi;
            load_codes(e.kept.q + (size_t)m * e.kept.pitch, n, left, e.kept.aligned, &lo, &hi);
            const float sc = scale_value(e.kept.scales[(size_t)m * e.kept.scale_pitch + n / kBlock]);
            float h[8];
            if (e.kept.e4m3) {
                decode4<true>(lo, sc, h);
                decode4<true>(hi, sc, h + 4);
            } else {
                decode4<false>(lo, sc, h);
                decode4<false>(hi, sc, h + 4);
            }
            times_slope(e.kept_act, h, v);
        }
    } else if (e.bias) {
        float b[8];
        load8<float>(e.bias, n, left, e.wide_bias, b);
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] += b[u];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u)
        if (!there || u >= left) v[u] = 0.f;
    if (e.kept_act == LAST_ACT_NONE && e.kept.q)
        store_eight(e.kept, m, n, left, (n & (kBlock - 1)) == 0, quad_max(top8(v)), v);
    activate8(e.act, v);
    if (e.res && there && left > 0) {
        const size_t at = (size_t)m * e.pres + n;
        float r[8];
        if (e.type == LAST_BF16) load8<bf16_t>(e.res, at, left, e.wide_res, r);
        else if (e.type == LAST_F16) load8<f16_t>(e.res, at, left, e.wide_res, r);
        else load8<float>(e.res, at, left, e.wide_res, r);
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] += r[u];
    }
    if (e.out.q) store_eight(e.out, m, n, left, (n & (kBlock - 1)) == 0, quad_max(top8(v)), v);
    if (e.y && left > 0) store8_as(e.type, e.y, (size_t)m * e.py + n, left, e.wide, v);
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

// The loop.  While a wavefront multiplies the first half of a step (32 of its 64 rows of the reduction) it reads the second
// half's operands from LDS, and while it multiplies the second half it reads those of the next step, so that the matrix cores
// do not wait for LDS; one barrier a step, in the middle, after which the step's own buffer is free and the step after the
// next is sent for.  The next step has then had a whole step's time to come.  With 8-bit operands one instruction takes
// 128 values of the reduction, and the halves are those of the rows of P.
template <typename E, int LP, int LQ, int BP, int BQ, int WP, int WQ>
__global__ __launch_bounds__(WP * WQ * kWave) void product_kernel(ProductArgs a)
{
    constexpr int kThreads = WP * WQ * kWave;
    constexpr bool kEight = Elt<E>::size == 1;
    constexpr int NP = BP / WP / 16, NQ = BQ / WQ / 16;                   // accumulators of a wavefront
    using TP = Tile<LP, BP, kThreads>;
    using TQ = Tile<LQ, BQ, kThreads>;
    __shared__ __align__(1024) char lds[2][TP::kBytes + TQ::kBytes];
    __shared__ unsigned scales[kEight ? 2 : 1][kEight ? BP + BQ : 1];

    const int lane = (int)threadIdx.x % kWave, g = lane >> 4, i16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), wp = wave / WQ, wq = wave % WQ;
    int tp, tq;
    tile_of((int)blockIdx.x, a.tiles_p * a.tiles_q, a.tiles_p, a.tiles_q, &tp, &tq);
    const int p0 = tp * BP, q0 = tq * BQ;
    const long long k0 = (long long)blockIdx.y * a.share, k1 = k0 + a.share < a.K ? k0 + a.share : a.K;

    TP P;
    TQ Q;
    int any = 0;
    P.init(p0, a.P, a.pp, LP == kAlong ? &a.frames : nullptr, LP == kAlong ? &any : nullptr);
    Q.init(q0, a.Q, a.pq, nullptr, nullptr);
    const bool work = LP == kAcross || __syncthreads_or(any);
    const int steps = work ? (int)((k1 - k0 + (LP == kAlong ? kStep : 64) - 1) / (LP == kAlong ? kStep : 64)) : 0;

    f4 acc[NP][NQ];
    f4 accb[(NP + WQ - 1) / WQ];                                          // row sums of P, shared by the wavefronts that read it
#pragma unroll
    for (int x = 0; x < NP; ++x) {
        accb[x / WQ] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int y = 0; y < NQ; ++y) acc[x][y] = f4{0.f, 0.f, 0.f, 0.f};
    }
    const bool bias_too = LP == kAcross && a.e.part_bias && tq == 0;

    const char* bp = a.p + (LP == kAlong ? (long long)p0 * a.pp + k0 : (long long)p0 * 2 + k0 * a.pp);
    const char* bq = a.q + (LQ == kAlong ? (long long)q0 * a.pq + k0 : (long long)q0 * 2 + (LP == kAlong ? k0 / 2 : k0) * a.pq);

    const auto send = [&](int s) {
        const int buf = s & 1;
        const long long left = k1 - k0 - (long long)s * (LP == kAlong ? kStep : 64);
        unsigned long long mask = ~0ull;
        if constexpr (LP == kAcross) {
            mask = left < 64 ? (1ull << left) - 1 : ~0ull;
            if (a.mask) mask &= a.mask[(k0 >> 6) + s];
        } else if constexpr (LQ == kAcross) {
            const long long rows = a.q_rows - k0 / 2 - 64ll * s;
            mask = rows < 64 ? (1ull << rows) - 1 : ~0ull;
        }
        P.load(bp + (long long)s * (LP == kAlong ? kStep : 64 * a.pp), left, mask, lds[buf]);
        Q.load(bq + (long long)s * (LQ == kAlong ? kStep : 64 * a.pq), left, mask, lds[buf] + TP::kBytes);
        if constexpr (kEight) {
            // a row's four scales of the step
            const int first = wave * kWave;
#pragma unroll
            for (int j = 0; j < (BP + BQ + kThreads - 1) / kThreads; ++j) {
                const int r = j * kThreads + (int)threadIdx.x;
                if (j * kThreads + first < BP + BQ) {
                    const bool isp = j * kThreads + first < BP;
                    const int row = isp ? r : r - BP;
                    const bool ok = isp ? p0 + row < a.P : q0 + row < a.Q;
                    const unsigned o = ok ? (unsigned)(row * (isp ? a.psp : a.psq)) + (unsigned)(k0 / kBlock) + 4u * (unsigned)s : kNowhere;
                    to_lds<4>(isp ? a.sp + (long long)p0 * a.psp : a.sq + (long long)q0 * a.psq, o, &scales[buf][j * kThreads + first]);
                }
            }
        }
    };
    const auto read_p = [&](int s, int half, int x) {
        const char* l = lds[s & 1];
        const int at = wp * (BP / WP) + x * 16, kr = half * 32 + 8 * g + (i16 >> 2);
        if constexpr (LP == kAlong) return *(const u4*)(l + along_at(at + i16, half * 4 + g));
        else
            return across_read(l, kr * (BP * 2) + ((at / 16 ^ across_swizzle(kr)) << 5) + (i16 & 3) * 8,
                               (kr + 4) * (BP * 2) + ((at / 16 ^ across_swizzle(kr + 4)) << 5) + (i16 & 3) * 8);
    };
    const auto read_q = [&](int s, int half, int y) {
        const char* l = lds[s & 1] + TP::kBytes;
        const int at = wq * (BQ / WQ) + y * 16, kr = half * 32 + 8 * g + (i16 >> 2);
        if constexpr (LQ == kAlong) return *(const u4*)(l + along_at(at + i16, half * 4 + g));
        else
            return across_read(l, kr * (BQ * 2) + ((at / 16 ^ across_swizzle(kr)) << 5) + (i16 & 3) * 8,
                               (kr + 4) * (BQ * 2) + ((at / 16 ^ across_swizzle(kr + 4)) << 5) + (i16 & 3) * 8);
    };

    if (steps > 0) {
        send(0);
        arrived();
        if (steps > 1) send(1);
        if constexpr (kEight) {
            u4 fp[NP][2], fq[NQ][2];
            int cp[NP], cq[NQ];
            for (int s = 0; s < steps; ++s) {
#pragma unroll
                for (int y = 0; y < NQ; ++y) {
                    fq[y][0] = read_q(s, 0, y);
                    fq[y][1] = read_q(s, 1, y);
                    cq[y] = (int)(scales[s & 1][BP + wq * (BQ / WQ) + y * 16 + i16] >> (8 * g));
                }
#pragma unroll
                for (int x = 0; x < NP; ++x) {
                    fp[x][0] = read_p(s, 0, x);
                    fp[x][1] = read_p(s, 1, x);
                    cp[x] = (int)(scales[s & 1][wp * (BP / WP) + x * 16 + i16] >> (8 * g));
                }
#pragma unroll
                for (int x = 0; x < NP; ++x)
#pragma unroll
                    for (int y = 0; y < NQ; ++y) acc[x][y] = mfma_scaled(fq[y], fp[x], acc[x][y], cq[y], cp[x]);
                arrived();
                if (s + 2 < steps) send(s + 2);
            }
        } else {
            u4 fp[2][NP], fq[2][NQ];
            const auto read = [&](int s, int half) {
#pragma unroll
                for (int y = 0; y < NQ; ++y) fq[half][y] = read_q(s, half, y);
#pragma unroll
                for (int x = 0; x < NP; ++x) fp[half][x] = read_p(s, half, x);
            };
            const auto multiply = [&](int half) {
#pragma unroll
                for (int x = 0; x < NP; ++x)
#pragma unroll
                    for (int y = 0; y < NQ; ++y) acc[x][y] = Mfma<E>::go(fq[half][y], fp[half][x], acc[x][y]);
                if constexpr (LP == kAcross) {
                    if (bias_too) {
                        const unsigned one = Elt<E>::type == LAST_BF16 ? 0x3f803f80u : 0x3c003c00u;
#pragma unroll
                        for (int x = 0; x < NP; ++x)
                            if (x % WQ == wq) accb[x / WQ] = Mfma<E>::go(u4{one, one, one, one}, fp[half][x], accb[x / WQ]);
                    }
                }
            };
            read(0, 0);
            for (int s = 0; s < steps; ++s) {
                read(s, 1);
                __builtin_amdgcn_sched_barrier(0);
                multiply(0);
                __builtin_amdgcn_sched_barrier(0);
                arrived();
                if (s + 2 < steps) send(s + 2);
                if (s + 1 < steps) read(s + 1, 0);
                __builtin_amdgcn_sched_barrier(0);
                multiply(1);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }

    // A lane has row 16 x + i16 of P and columns 16 y + 4 g .. of Q.  The epilogue wants eight columns of a row in a lane and
    // whole lines of rows in a wavefront: 64 rows at a time change places in the wavefront's own part of LDS, whose 16-byte
    // pieces of a row are swizzled by the row.
    constexpr int kCols = BQ / WQ, kPieces = kCols / 4, kLanes = kCols / 8, kRows = kWave / kLanes, XS = NP < 4 ? NP : 4;
    static_assert((size_t)XS * 16 * kCols * 4 * WP * WQ <= sizeof(lds), "room for the epilogue");
    __syncthreads();
    char* mine = &lds[0][0] + wave * (XS * 16 * kCols * 4);
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
        const int c = (lane % kLanes) * 8, n = q0 + wq * kCols + c;
#pragma unroll 1
        for (int r = lane / kLanes; r < XS * 16; r += kRows) {
            const int m = p0 + wp * (BP / WP) + part * XS * 16 + r;
            const f4 lo = *(const f4*)(mine + r * (kCols * 4) + (((c / 4) ^ (r & (kPieces - 1))) << 4));
            const f4 hi = *(const f4*)(mine + r * (kCols * 4) + (((c / 4 + 1) ^ (r & (kPieces - 1))) << 4));
            float v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            if (a.e.part) {
                if (m < a.P) store8<float>(a.e.part, ((size_t)blockIdx.y * a.P + m) * a.Q + n, a.Q - n, (a.Q & 3) == 0, v);
            } else {
                finish(a.e, m, n, a.P, a.Q, m < a.P && (LP == kAcross || frame_exists(a.frames, m)), v);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    if (bias_too) {
#pragma unroll
        for (int x = 0; x < NP; ++x) {
            const int m = p0 + wp * (BP / WP) + x * 16 + i16;
            if (x % WQ == wq && g == 0 && m < a.P) a.e.part_bias[(size_t)blockIdx.y * a.P + m] = accb[x / WQ][0];
        }
    }
}

// ---- few rows: y = act(x w^T + bias) + residual for at most 16 MT rows, bound by the bytes of w, which go from memory to
// registers once.  A workgroup takes 16 QF columns, its wavefronts every kFewWaves-th 128 bytes of the rows, four such
// steps' loads under way at a time; their sums meet in LDS.
constexpr int kFewWaves = 8;
constexpr int kFewDeep = 4;

template <typename E, int MT, int QF>
__global__ __launch_bounds__(kFewWaves * kWave) void few_kernel(ProductArgs a)
{
    constexpr bool kEight = Elt<E>::size == 1;
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
    for (int s0 = wave; s0 < steps; s0 += kFewWaves * kFewDeep) {
        u4 fq[kFewDeep][QF][2], fp[kFewDeep][MT][2];
        int cq[kFewDeep][QF], cp[kFewDeep][MT];
#pragma unroll
        for (int d = 0; d < kFewDeep; ++d) {
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
                const int block = k / kBlock + g;
                const bool in = block * kBlock < bytes;
#pragma unroll
                for (int f = 0; f < QF; ++f) cq[d][f] = in && oq[f] < kNowhere ? a.sq[(q0 + rq[f]) * a.psq + block] : 0;
#pragma unroll
                for (int t = 0; t < MT; ++t) cp[d][t] = in && op[t] < kNowhere ? a.sp[(t * 16 + i16) * a.psp + block] : 0;
            }
        }
#pragma unroll
        for (int d = 0; d < kFewDeep; ++d)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int f = 0; f < QF; ++f) {
                    if constexpr (kEight) {
                        acc[t][f] = mfma_scaled(fq[d][f], fp[d][t], acc[t][f], cq[d][f], cp[d][t]);
                    } else {
                        acc[t][f] = Mfma<E>::go(fq[d][f][0], fp[d][t][0], acc[t][f]);
                        acc[t][f] = Mfma<E>::go(fq[d][f][1], fp[d][t][1], acc[t][f]);
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
    const int P = c < 2 * QF ? a.P : 0;
    finish(a.e, m, q0 + 8 * c, P, a.Q, m < P && frame_exists(a.frames, m), v);
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
            load8<float>(a.e.part + ((size_t)s * a.P + m) * a.Q, n, a.Q - n, (a.Q & 3) == 0, t);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += t[k];
        }
        if (a.e.part_bias && n == 0) {
            float b = 0.f;
            for (int s = 0; s < splits; ++s) b += a.e.part_bias[(size_t)s * a.P + m];
            a.e.sum_bias[m] = b;
        }
    }
    finish(a.e, m, n, a.P, a.Q, m < a.P && frame_exists(a.frames, m), v);
}

// ---- rows of `bytes` bytes laid out at multiples of 16 with zeros behind them, 16 bytes a thread
__global__ __launch_bounds__(256) void repack_kernel(const uint8_t* in, long long pitch, int bytes, uint8_t* out, int out_pitch, long long pieces)
{
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= pieces) return;
    const int per = out_pitch / 16;
    const long long row = i / per;
    const int at = (int)(i - row * per) * 16;
    const uint8_t* p = in + row * pitch + at;
    unsigned w[4] = {0u, 0u, 0u, 0u};
    if (((uintptr_t)in & 1) == 0 && (pitch & 1) == 0 && (bytes & 1) == 0) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (at + 2 * k < bytes) w[k >> 1] |= (unsigned)*(const uint16_t*)(p + 2 * k) << (16 * (k & 1));
    } else {
#pragma unroll
        for (int k = 0; k < 16; ++k)
            if (at + k < bytes) w[k >> 2] |= (unsigned)p[k] << (8 * (k & 3));
    }
    *(u4*)(out + row * out_pitch + at) = u4{w[0], w[1], w[2], w[3]};
}

// ---- which rows exist, a bit each
__global__ __launch_bounds__(256) void frame_mask_kernel(Frames f, int rows, unsigned long long* mask)
{
    const int row = (int)(blockIdx.x * 256 + threadIdx.x);
    const unsigned long long m = __ballot(row < rows && frame_exists(f, row));
    if ((threadIdx.x & (kWave - 1)) == 0 && row < rows) mask[row >> 6] = m;
}

}  // namespace last
