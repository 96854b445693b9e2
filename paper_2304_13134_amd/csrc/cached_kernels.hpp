// Attention of new frames to the frames in a paged cache, the form of attention_kernels.hpp for streams.
//
// A wavefront's 32 rows are the new frames of a kv head, each with all heads that share it, so that a cache is read once for them.
// Bound by the bytes of keys and values: each wavefront goes over blocks of 32 frames of its own, whole rows from memory to registers, a block ahead,
// and on to LDS for the matrix cores' operands, with no barrier; the four of a workgroup, which take the blocks in turn, are joined at the end.  Few rows
// on a long cache are split over workgroups and joined by cached_join_kernel (one stream of 32768 frames, 16 heads of 128 on four: 117 us undivided, 37).
// 16 such streams: 149 us and 7 for the join, 5.7 TB/s of keys and values, where a copy's reads reach 6.7; 64 streams of 16384 frames, 8 heads of 64: 6.0.
// A lane's own rows straight from memory, with no LDS: 268 us, whole rows 239; queries in registers, which then do not hold the block ahead: 236.
#pragma once
#include "attention_kernels.hpp"

namespace last {

constexpr int kMostSplits = 128;

struct CachedArgs {
    const int* len;
    int T, B, heads, kv_heads, D;
    const void* q;
    void* y;
    long long pq, py;
    const char *k, *v;
    Pages cache;
    Band band;
    int* status;                     // [B] or null
    float *part, *part_ml;           // [item][kv head][row][split][D], [..][2]: sums, and their maximum and count; of more than one split
    int splits, row_blocks;
    unsigned first;
};

template <int DP> struct CachedRows {
    static constexpr int kBytes = 32 * Rows<DP>::kPitch;     // keys or values of a block
    static constexpr int kPieces = DP / 8;                   // lanes of a row when it is loaded
    static constexpr int kAtOnce = kWave / kPieces;          // rows a load
    static constexpr int kEach = 32 / kAtOnce;
};

// The rows of a block of 32 frames: in pages one after the other, or row by row where a page ends in it.
struct Block {
    size_t at;                       // elements: of the lane's own row (both halves the same), or of the block's first
    bool together;                   // the same for all lanes
    unsigned bad, there;             // bits of rows
};

template <typename E, int DP>
__global__ __launch_bounds__(256, 2) void cached_kernel(CachedArgs a)
{
    using C = CachedRows<DP>;
    __shared__ __attribute__((aligned(16))) char lds[9 * C::kBytes];          // the queries, then keys and values of each wavefront
    __shared__ float all_m[4][32], all_l[4][32];
    const unsigned id = a.first + blockIdx.x;
    const int split = (int)(id % (unsigned)a.splits), rb = (int)(id / (unsigned)a.splits % (unsigned)a.row_blocks);
    const unsigned ik = id / (unsigned)a.splits / (unsigned)a.row_blocks;
    const int kv = (int)(ik % (unsigned)a.kv_heads), b = (int)(ik / (unsigned)a.kv_heads);
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), lane = (int)threadIdx.x % kWave, h = lane >> 5;
    const int group = a.heads / a.kv_heads, rows = a.T * group, r = rb * 32 + (lane & 31);
    const int made = frames_of_item(a.len, a.T, b), used = used_frames(a.cache.used, b), total = used + made;
    const int t = r / group, head = kv * group + r % group;
    const bool there = t < made;
    const Band band = a.band;
    const float c2 = band.scale * kLog2e;
    const size_t row0 = (size_t)b * a.T;
    if (a.status && split == 0 && rb == 0 && kv == 0 && wave == 0) {
        // every page that the item's new frames look at
        int bad = 0, x;
        const int from = used - band.left > 0 ? used - band.left : 0;
        if (made > 0) {
            for (int s = from + lane * a.cache.page; s < total; s += kWave * a.cache.page) bad |= page_of(a.cache, b, s, &x) < 0;
            if (lane == 0) bad |= page_of(a.cache, b, total - 1, &x) < 0;
            if (lane < band.sinks && lane < total) bad |= page_of(a.cache, b, lane, &x) < 0;
        }
        const bool any = __any(bad);
        if (lane == 0) a.status[b] = any ? kItemBadPage : kItemOk;
    }
    // frames that the rows see: first ones, and [lo, hi), in blocks of 32
    const int t_lo = rb * 32 / group, t_hi = (rb * 32 + 31) / group < made - 1 ? (rb * 32 + 31) / group : made - 1;
    const int lo = used + t_lo - band.left > 0 ? used + t_lo - band.left : 0;
    const int hi = t_lo >= made ? 0 : used + t_hi + 1 + band.right < total ? used + t_hi + 1 + band.right : total;
    const int sinks = band.sinks < hi ? band.sinks : hi, sink_blocks = (sinks + 31) / 32;
    const int first = lo / 32 > sink_blocks ? lo / 32 : sink_blocks, last = (hi + 31) / 32;
    const int blocks = sink_blocks + (last > first ? last - first : 0);
    const int begin = (int)((long long)blocks * split / a.splits), end = (int)((long long)blocks * (split + 1) / a.splits);
    const auto start = [&](int j) { return (j < sink_blocks ? j : first + j - sink_blocks) * 32; };
    // element of frame s's row; -1: there is no such page
    const auto row_of = [&](int s) -> long long {
        int x;
        const int page = page_of(a.cache, b, s, &x);
        return page < 0 ? -1 : (long long)((((size_t)page * a.kv_heads + kv) * a.cache.page + x) * a.D);
    };
    const Sight sight{used + t - band.left > 0 ? used + t - band.left : 0, !there ? 0 : used + t + band.right + 1 < total ? used + t + band.right + 1 : total, sinks};
    Softmax<DP> soft;
    soft.init();
    char *const qt = lds, *const kt = lds + (1 + wave * 2) * C::kBytes, *const vt = kt + C::kBytes;
    Reads<DP> reads;
    reads.init();
    // a quarter of the queries' columns; they are read again for each block, to leave registers for what is under way
#pragma unroll
    for (int i = 0; i < DP / 16; i += 4) {
        const int k = i + wave, c = 16 * k + 8 * h;
        u4 x{0u, 0u, 0u, 0u};
        if (k < DP / 16 && there && c < a.D) x = *(const u4_any*)((const char*)a.q + ((row0 + t) * a.pq + (size_t)head * a.D + c) * 2);
        if (k < DP / 16) *(u4*)(qt + (lane & 31) * Rows<DP>::kPitch + ((2 * k + h) ^ Rows<DP>::spread(lane & 31)) * 16) = x;
    }
    const auto seen = [&](int s) { return (s < hi) & ((s >= lo) | (s < sinks)); };
    // What the table says about the lane's row of block j: sent for a turn before it is looked at, since a wavefront's loads return in order and the
    // next block's keys and values are under way behind it.
    const auto ask = [&](int j) {
        const int s = start(j) + (lane & 31), e = (int)quotient((unsigned)s, a.cache.by_page);
        return seen(s) && e < a.cache.entries ? a.cache.table[(size_t)b * a.cache.entries + e] : -1;
    };
    // where the rows of block j are
    const auto find = [&](int j, int page) {
        const int s0 = start(j), s = s0 + (lane & 31), size = a.cache.page, x = s - (int)quotient((unsigned)s, a.cache.by_page) * size;
        const bool known = (unsigned)page < (unsigned)a.cache.pages;
        Block k;
        k.at = known ? (((size_t)page * a.kv_heads + kv) * size + x) * a.D : 0;
        k.there = (unsigned)__ballot(seen(s) && known);
        k.bad = (unsigned)__ballot(seen(s) && !known);
        k.together = k.there == ~0u && __builtin_amdgcn_readfirstlane(x) + 32 <= size;
        return k;
    };
    const int piece = lane % C::kPieces, r0 = lane / C::kPieces;
    u4 ks[C::kEach], vs[C::kEach];
    unsigned there_now = 0, bad_now = 0;
    const auto get = [&](const Block& k) {
        const int c = piece * 8 < a.D ? piece * 8 : 0;
        there_now = k.there;
        bad_now = k.bad;
        if (k.together) {
            const size_t base = (size_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)k.at) |
                                (size_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(k.at >> 32)) << 32;
            const unsigned off = (unsigned)(r0 * a.D + c) * 2u, step = (unsigned)(C::kAtOnce * a.D) * 2u;
            const char *const k0 = a.k + base * 2, *const v0 = a.v + base * 2;
#pragma unroll
            for (int i = 0; i < C::kEach; ++i) {
                ks[i] = *(const u4*)(k0 + i * step + off);
                vs[i] = *(const u4*)(v0 + i * step + off);
            }
        } else if (k.there != 0) {
            // (rows that are not there: another one's, which is)
            const int other = __ffs((int)k.there) - 1;
#pragma unroll
            for (int i = 0; i < C::kEach; ++i) {
                const int r = r0 + i * C::kAtOnce, from = k.there >> r & 1 ? r : other;
                const size_t at = ((size_t)(unsigned)__shfl((int)(unsigned)k.at, from, kWave) | (size_t)(unsigned)__shfl((int)(k.at >> 32), from, kWave) << 32) + c;
                ks[i] = *(const u4*)(a.k + at * 2);
                vs[i] = *(const u4*)(a.v + at * 2);
            }
        }
    };
    int page = -1;
    if (begin + wave < end) {
        const int now = ask(begin + wave);
        if (begin + wave + 4 < end) page = ask(begin + wave + 4);
        get(find(begin + wave, now));
    }
    __syncthreads();
    for (int j = begin + wave; j < end; j += 4) {
        const int s0 = start(j);
        const bool all = there_now == ~0u && a.D == DP;
#pragma unroll
        for (int i = 0; i < C::kEach; ++i) {
            const int r = r0 + i * C::kAtOnce, at = r * Rows<DP>::kPitch + (piece ^ Rows<DP>::spread(r)) * 16;
            u4 k = ks[i], v = vs[i];
            if (!all) {
                // a frame whose page there is none of makes the rows that see it NaN
                const unsigned keep = ((there_now >> r & 1) & (piece * 8 < a.D)) ? ~0u : 0u, fill = bad_now >> r & 1 ? 0x7fff7fffu : 0u;
                k = (k & u4{keep, keep, keep, keep}) | u4{fill, fill, fill, fill};
                v = v & u4{keep, keep, keep, keep};
            }
            *(u4*)(kt + at) = k;
            *(u4*)(vt + at) = v;
        }
        if (j + 4 < end) {
            const Block next = find(j + 4, page);
            if (j + 8 < end) page = ask(j + 8);
            get(next);
        }
        asm volatile("" ::: "memory");
        f16x s = zeros16();
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) s = Mma<E>::go(reads.along_rows(kt, 0, i), reads.along_rows(qt, 0, i), s);
        sight.apply(s, s0, LAST_NEG_INF);
        soft.template take<1>(&s, c2);
        u4 p[2];
        to_operands<E>(s, p);
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) soft.acc[d] = Mma<E>::go(reads.along_columns(vt, d, i), p[i], soft.acc[d]);
        asm volatile("" ::: "memory");
    }
    // the four wavefronts' sums, relative to the largest maximum, in a fixed order
    float l = sum_of_halves(soft.l);
    if (lane < 32) {
        all_m[wave][lane] = soft.m;
        all_l[wave][lane] = l;
    }
    __syncthreads();
    float m = LAST_NEG_INF;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, all_m[w][lane & 31]);
    const float by = m == LAST_NEG_INF ? 0.f : m;
    l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) l += all_l[w][lane & 31] * __builtin_amdgcn_exp2f((all_m[w][lane & 31] - by) * c2);
    const float own = __builtin_amdgcn_exp2f((soft.m - by) * c2);
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) soft.acc[d][i] *= own;
    float* const sums = (float*)lds;
#pragma unroll
    for (int half = 2; half > 0; half >>= 1) {
        __syncthreads();
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) sums[(((wave - half) * (DP / 32) + d) * 16 + i) * kWave + lane] = soft.acc[d][i];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) soft.acc[d][i] += sums[((wave * (DP / 32) + d) * 16 + i) * kWave + lane];
        }
    }
    if (wave > 0) return;
    const bool odd = there && l == l && soft.not_finite();   // (as in attention_kernel)
    const size_t part_row = ((size_t)b * a.kv_heads + kv) * rows;
    if (r < rows && !odd) {
        if (a.splits == 1) {
            put_rows<E, DP>((char*)a.y + ((row0 + t) * a.py + (size_t)head * a.D) * 2, a.D, soft.acc, 1.f / l, there);
        } else {
            float* const out = a.part + ((part_row + r) * a.splits + split) * a.D;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    if (32 * d + result_row(i) < a.D)
                        *(f4*)(out + 32 * d + result_row(i)) = f4{soft.acc[d][i], soft.acc[d][i + 1], soft.acc[d][i + 2], soft.acc[d][i + 3]};
            if (lane < 32) {
                float* const ml = a.part_ml + ((part_row + r) * a.splits + split) * 2;
                ml[0] = m;
                ml[1] = l;
            }
        }
    }
    unsigned long long bits = __ballot(odd) & 0xffffffffull;
    if (__builtin_expect(bits == 0, 1)) return;              // (the usual end before that code, not behind it: 8 x 16 new frames 14.5 -> 14.2 us)
    for (; bits; bits &= bits - 1) {
        const int rr = rb * 32 + __ffsll(bits) - 1, tr = rr / group, hr = kv * group + rr % group, at = used + tr;
        // of what the row sees, the split's blocks: first frames and the others
        const int start0 = start(begin), stop = start(end - 1) + 32, last_seen = at + band.right + 1 < total ? at + band.right + 1 : total;
        const int to = last_seen < stop ? last_seen : stop, firsts = sinks < to ? sinks : to;
        const int low = at - band.left > firsts ? at - band.left : firsts;
        float pm, pl, o[8];
        plain_row<E, DP>((const char*)a.q + ((row0 + tr) * a.pq + (size_t)hr * a.D) * 2, a.D, c2, start0, firsts, low > start0 ? low : start0, to,
                     [&](int s) {
                         const long long p = row_of(s);
                         return p >= 0 ? KeyValue{a.k + p * 2, a.v + p * 2} : KeyValue{nullptr, nullptr};
                     },
                     &pm, &pl, o);
        if (lane < DP / 8 && lane * 8 < a.D) {
            char* const y = (char*)a.y + ((row0 + tr) * a.py + (size_t)hr * a.D) * 2;
            float* const out = a.part + ((part_row + rr) * a.splits + split) * a.D;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                if (a.splits == 1) Elt<E>::put(y, lane * 8 + c, o[c] / pl);
                else out[lane * 8 + c] = o[c];
            }
        }
        if (a.splits > 1 && lane == 0) {
            float* const ml = a.part_ml + ((part_row + rr) * a.splits + split) * 2;
            ml[0] = pm;
            ml[1] = pl;
        }
    }
}

// y of a row of a head from its splits: a workgroup a row, of which each wavefront adds every fourth split, two columns a lane, and the four are added in order
template <typename E>
__global__ __launch_bounds__(256) void cached_join_kernel(CachedArgs a, long long first_row)
{
    __shared__ float factors[kMostSplits], sums[4][128];
    const int lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave, group = a.heads / a.kv_heads, rows = a.T * group;
    const long long i = first_row + blockIdx.x;
    const int ik = (int)(i / rows), r = (int)(i - (long long)ik * rows), b = ik / a.kv_heads, kv = ik - b * a.kv_heads;
    const int t = r / group, head = kv * group + r % group;
    const bool there = t < frames_of_item(a.len, a.T, b);
    const float c2 = a.band.scale * kLog2e;
    const float* const ml = a.part_ml + (size_t)i * a.splits * 2;
    float m = LAST_NEG_INF, l = 0.f;
    if (there) {
        for (int s = lane; s < a.splits; s += kWave) m = fmaxf(m, ml[2 * s]);
        m = wave_max(m);
        for (int s = lane; s < a.splits; s += kWave) {
            const float f = __builtin_amdgcn_exp2f((ml[2 * s] - m) * c2);
            l += ml[2 * s + 1] * f;
            if (wave == 0) factors[s] = f;
        }
        l = wave_sum(l);
    }
    __syncthreads();
    float o[2] = {0.f, 0.f};
    if (there) {
        const float* const in = a.part + (size_t)i * a.splits * a.D + lane;
#pragma unroll 4
        for (int s = wave; s < a.splits; s += 4) {
            const float f = factors[s];
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (lane + 64 * c < a.D) o[c] += in[(size_t)s * a.D + 64 * c] * f;
        }
    }
    sums[wave][lane] = o[0];
    sums[wave][lane + 64] = o[1];
    __syncthreads();
    if ((int)threadIdx.x < a.D) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) v += sums[w][threadIdx.x];
        Elt<E>::put((char*)a.y + (((size_t)b * a.T + t) * a.py + (size_t)head * a.D) * 2, threadIdx.x, there ? v / l : 0.f);
    }
}

}  // namespace last
