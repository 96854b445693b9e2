// Attention of new frames to the frames in a paged cache, the form of attention_kernels.hpp for streams.
//
// A wavefront's 32 rows are the new frames of a kv head, each with all heads that share it, so that a cache is read once for them.
// Bound by the bytes of keys and values: each wavefront goes over blocks of 32 frames of its own, keys from memory to the matrix cores'
// first operand as they stand, values through LDS for the transposing reads, with no barrier; the four of a workgroup, which take the
// blocks in turn, are joined at the end.  Few rows on a long cache are split over workgroups and joined by cached_join_kernel.
#pragma once
#include "attention_kernels.hpp"

namespace last {

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

// Where the rows of a block stand, of which a lane has one (and both halves the same).
struct PageRow {
    size_t at;                       // elements
    bool exists, bad;
};

template <int DP> struct CachedRows {
    static constexpr int kBytes = 32 * Rows<DP>::kPitch;     // values of a block
    static constexpr int kSums = DP / 32 * 16 * kWave * 4;   // sums of a wavefront
    static constexpr int kAll = 4 * kBytes > 2 * kSums ? 4 * kBytes : 2 * kSums;
};

template <typename E, int DP>
__global__ __launch_bounds__(256) void cached_kernel(CachedArgs a)
{
    __shared__ __attribute__((aligned(16))) char lds[CachedRows<DP>::kAll];
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
    const auto find = [&](int s) {
        PageRow p{};
        if (s < hi && (s >= lo || s < sinks)) {
            int x;
            const int page = page_of(a.cache, b, s, &x);
            p.exists = page >= 0;
            p.bad = page < 0;
            p.at = (((size_t)(page < 0 ? 0 : page) * a.kv_heads + kv) * a.cache.page + x) * a.D;
        }
        return p;
    };
    const Sight sight{used + t - band.left, !there ? 0 : used + t + band.right + 1 < total ? used + t + band.right + 1 : total, sinks};
    u4 qf[DP / 16];
    own_rows<DP>(there ? (const char*)a.q + ((row0 + t) * a.pq + (size_t)head * a.D) * 2 : nullptr, a.D, qf);
    Softmax<DP> soft;
    soft.init();
    char* const vt = lds + wave * CachedRows<DP>::kBytes;
    Reads<DP> reads;
    reads.init();
    u4 kf[DP / 16], vf[DP / 16];
    const auto get = [&](int j) {
        const PageRow p = find(start(j) + (lane & 31));
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) {
            const int c = 16 * i + 8 * h;
            // a frame whose page there is none of makes the rows that see it NaN
            const unsigned fill = p.bad ? 0x7fff7fffu : 0u;
            kf[i] = u4{fill, fill, fill, fill};
            vf[i] = u4{0u, 0u, 0u, 0u};
            if (p.exists && c < a.D) {
                kf[i] = *(const u4_any*)(a.k + (p.at + c) * 2);
                vf[i] = *(const u4_any*)(a.v + (p.at + c) * 2);
            }
        }
    };
    if (begin + wave < end) get(begin + wave);
    for (int j = begin + wave; j < end; j += 4) {
        const int s0 = start(j);
        f16x s = zeros16();
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) s = Mma<E>::go(kf[i], qf[i], s);
#pragma unroll
        for (int i = 0; i < DP / 16; ++i) *(u4*)(vt + reads.rows[i]) = vf[i];
        if (j + 4 < end) get(j + 4);
        sight.apply(s, s0, LAST_NEG_INF);
        soft.template take<1>(&s, c2);
        u4 p[2];
        to_operands<E>(s, p);
        asm volatile("" ::: "memory");
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
    soft.m = m;
    soft.l = h ? 0.f : l;
    const bool odd = there && soft.not_finite();
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
    for (unsigned long long bits = __ballot(odd) & 0xffffffffull; bits; bits &= bits - 1) {
        const int rr = rb * 32 + __ffsll(bits) - 1, tr = rr / group, hr = kv * group + rr % group, at = used + tr;
        const int to = at + band.right + 1 < total ? at + band.right + 1 : total, stop = start(end - 1) + 32;
        const auto where = [&](const char* base, int s) -> const char* {
            const PageRow p = find(s);
            return p.exists ? base + p.at * 2 : nullptr;
        };
        float pm, pl, o[2];
        plain_row<E>((const char*)a.q + ((row0 + tr) * a.pq + (size_t)hr * a.D) * 2, a.D, c2, start(begin), to < stop ? to : stop,
                     [&](int s) { return s >= at - band.left || s < sinks; }, [&](int s) { return where(a.k, s); },
                     [&](int s) { return where(a.v, s); }, &pm, &pl, o);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int c = lane + 64 * i;
            if (c >= a.D) continue;
            if (a.splits == 1) Elt<E>::put((char*)a.y + ((row0 + tr) * a.py + (size_t)hr * a.D) * 2, c, o[i] / pl);
            else a.part[((part_row + rr) * a.splits + split) * a.D + c] = o[i];
        }
        if (a.splits > 1 && lane == 0) {
            float* const ml = a.part_ml + ((part_row + rr) * a.splits + split) * 2;
            ml[0] = pm;
            ml[1] = pl;
        }
    }
}

// y of a row from its splits: a wavefront a row, two columns a lane
template <typename E>
__global__ __launch_bounds__(256) void cached_join_kernel(CachedArgs a, long long first_row)
{
    const int lane = (int)threadIdx.x % kWave, group = a.heads / a.kv_heads, rows = a.T * group;
    const long long i = first_row + (long long)blockIdx.x * 4 + (int)threadIdx.x / kWave;
    if (i >= (long long)a.B * a.kv_heads * rows) return;
    const int ik = (int)(i / rows), r = (int)(i - (long long)ik * rows), b = ik / a.kv_heads, kv = ik - b * a.kv_heads;
    const int t = r / group, head = kv * group + r % group;
    const bool there = t < frames_of_item(a.len, a.T, b);
    const float c2 = a.band.scale * kLog2e;
    float m = LAST_NEG_INF, l = 0.f, o[2] = {0.f, 0.f};
    if (there) {
        const float* const ml = a.part_ml + (size_t)i * a.splits * 2;
        for (int s = 0; s < a.splits; ++s) m = fmaxf(m, ml[2 * s]);
        for (int s = 0; s < a.splits; ++s) {
            const float f = __builtin_amdgcn_exp2f((ml[2 * s] - m) * c2);
            l += ml[2 * s + 1] * f;
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if (lane + 64 * c < a.D) o[c] += a.part[((size_t)i * a.splits + s) * a.D + lane + 64 * c] * f;
        }
    }
    char* const y = (char*)a.y + (((size_t)b * a.T + t) * a.py + (size_t)head * a.D) * 2;
#pragma unroll
    for (int c = 0; c < 2; ++c)
        if (lane + 64 * c < a.D) Elt<E>::put(y, lane + 64 * c, there ? o[c] / l : 0.f);
}

}  // namespace last
