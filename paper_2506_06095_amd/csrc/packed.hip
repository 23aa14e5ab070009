// A cache held in 4 bits: keys and values packed as they are written, read back, and attended to.
//
// A packed row stands for the d columns of one key or value, 32 at a time (the last group may be shorter).  Each group has a step s and a base m, both binary16, and
// a code c of 0 .. 15 for every column, which stands for v = RN16(c s + m), the binary16 nearest to it: one rounding, that of a fused multiply and add
// in binary16, so that whoever unpacks a row, and however, has the same bits.
//   row: (s, m) of every group, 4 bytes each, then the codes; 8 columns are a word of 32 bits, columns 2i from bit 4i on, columns 2i + 1 from bit
//   16 + 4i, so that a mask of 0x000F000F leaves a pair of neighbours in the halves of a word.
// 5 bits a column where groups are whole: 80 bytes for 128 columns, where 16 bits take 256.
//
// Packing, per group: x limited to +-65280; m = the largest binary16 <= min x; s = the smallest binary16 with 15 s + m >= max x; c = the number of k in
// 0 .. 14 with x >= m + (k + 1/2) s (0 where s = 0).  No value is further from x than s / 2 and half its own last place; 15 s + m
// exceeds max x by less than 15 of s's last places, 120 at most, so that every code stands for something finite.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "device_common.hpp"
#include "smha.h"

namespace smha {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr float kPackedMost = 65280.f;

static int packed_groups(int d) { return (d + 31) / 32; }
static int packed_row_bytes(int d) { return 4 * packed_groups(d) + d / 2; }

// What eight codes stand for, as pairs of neighbours; `head`: s in the lower half, m in the upper.  0x6400 + c are the bits of 1024 + c and 0x5400 + 16 c those
// of 64 + c, so that a pair is three instructions and a shared shift: and-or, the bias off (exact), fused multiply and add.  (The first is written out: the
// compiler makes two of it, each with a constant in its encoding.)
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t bits) {
    uint32_t y;
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(y) : "v"(x), "s"(mask), "v"(bits));
    return y;
}
__device__ __forceinline__ u32x4 unpack8(uint32_t word, uint32_t head) {
    const f16x2 h = __builtin_bit_cast(f16x2, head), s = {h[0], h[0]}, m = {h[1], h[1]};
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? word : word >> 8;
        const f16x2 biased = __builtin_bit_cast(f16x2, i & 1 ? and_or(w, 0x00F000F0u, 0x54005400u) : and_or(w, 0x000F000Fu, 0x64006400u));
        const _Float16 bias = i & 1 ? (_Float16)64.f : (_Float16)1024.f;
        v[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(biased - f16x2{bias, bias}, s, m));
    }
    return v;
}

// n / d for 0 <= n <= 2^30, 0 < d < 2^30: in 32-bit floats, again for what that leaves, and by one for what that does.  (Rows and segments are found by chains of
// divisions; the compiler's take twice as many instructions.)
__device__ __forceinline__ int quotient(int n, int d) {
    const float inv = __builtin_amdgcn_rcpf((float)d);
    int q = (int)((float)n * inv);
    q += (int)((float)(n - q * d) * inv);
    const int rest = n - q * d;
    return q + (rest >= d ? 1 : 0) - (rest < 0 ? 1 : 0);
}

// Two binary16 values as a pair of bfloat16.
__device__ __forceinline__ uint32_t as_bf16(uint32_t pair) {
    const f16x2 h = __builtin_bit_cast(f16x2, pair);
    return pack2<true>((float)h[0], (float)h[1]);
}

// ---------------------------------------------------------------------------------------
// Writing and reading
// ---------------------------------------------------------------------------------------
struct PackParams {
    const uint16_t *x[2];  // keys and values of new tokens
    uint8_t *cache[2];
    uint16_t *values[2];   // what they stand for then, packed as tensors are, or null
    Strides xs[2], cs[2];
    const int32_t *lengths, *offsets;  // offsets: null for lengths - T
    int B, Hkv, T, Sk, d;
};

template <int CTRL> __device__ __forceinline__ float quad_moved(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float quad_min(float v) {
    v = fminf(v, quad_moved<0xB1>(v));  // lanes 1 0 3 2
    return fminf(v, quad_moved<0x4E>(v));  // lanes 2 3 0 1
}
__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, quad_moved<0xB1>(v));
    return fmaxf(v, quad_moved<0x4E>(v));
}

// The neighbour of a finite binary16 towards -inf, and that of one that is not negative towards +inf.
__device__ __forceinline__ uint32_t below16(uint32_t h) { return h == 0 ? 0x8001u : h & 0x8000u ? h + 1 : h - 1; }

// A lane takes 8 columns, four lanes a group: they share the group's least and largest value.
template <bool BF16>
__device__ __forceinline__ uint32_t pack8(u32x4 x, bool there, uint32_t &head) {
    float f[8], lo = __builtin_inff(), hi = -__builtin_inff(), bad = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float y = widen16<BF16>(e & 1 ? x[e / 2] >> 16 : x[e / 2] & 0xFFFFu);
        if (y != y) bad = 1.f;
        f[e] = fminf(fmaxf(y, -kPackedMost), kPackedMost);
        lo = fminf(lo, f[e]);
        hi = fmaxf(hi, f[e]);
    }
    if (!there) {
        lo = __builtin_inff();
        hi = -__builtin_inff();
        bad = 0.f;
    }
    lo = quad_min(lo) + 0.f;  // (no -0)
    hi = quad_max(hi);
    bad = quad_max(bad);
    uint32_t mb = __builtin_bit_cast(uint16_t, (_Float16)lo);
    if (BF16 && widen16<false>(mb) > lo) mb = below16(mb);
    const float m = widen16<false>(mb);
    // the quotient in 32 bits is no more than a step below the one that is wanted; compared in 64, where 15 s + m is exact
    uint32_t sb = __builtin_bit_cast(uint16_t, (_Float16)((hi - m) * (1.f / 15.f)));
    if (fma(15.0, (double)widen16<false>(sb), (double)m) < (double)hi) ++sb;
    const float s = widen16<false>(sb), inv = sb ? __builtin_amdgcn_rcpf(s) : 0.f;
    // The place among the borders: q is off by 15 (2^-24 + 2^-23) + 2^-21 = 3.2e-6 at most (the difference's rounding, the reciprocal's last place, the sum's rounding).  Where a
    // lane of the wave has a value that is closer to a border than 2^-16, borders are compared in 64 bits, where they are exact, so that equal inputs and ties give the same
    // code everywhere.  (Always so: 62 us for the call below.)
    uint32_t word = 0;
    float least = 1.f, most = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float q = fmaf(f[e] - m, inv, 0.5f), past = __builtin_amdgcn_fractf(q);
        word |= (uint32_t)(int)q << (4 * (e / 2) + 16 * (e & 1));
        least = fminf(least, past);
        most = fmaxf(most, past);
    }
    if (__builtin_amdgcn_ballot_w64(there && (least < 0x1p-16f || most > 1.f - 0x1p-16f)) != 0) {
        const double s64 = s, m64 = sb ? (double)m : (double)__builtin_inff();
        word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float k = truncf(fmaf(f[e] - m, inv, 0.5f - 0x1p-10f));  // the right code, or the one below it
            word |= ((uint32_t)(int)k + (fma((double)(k + 0.5f), s64, m64) <= (double)f[e] ? 1 : 0)) << (4 * (e / 2) + 16 * (e & 1));
        }
    }
    if (bad != 0.f) {
        sb = 0;
        mb = 0x7E00u;
        word = 0;
    }
    head = sb | mb << 16;
    return word;
}

// Where a row of a call is: token t of key head hk of sequence b, and its slot.
struct PackedRow {
    int b, hk, t;
    int64_t slot;
    bool kept;
    __device__ __forceinline__ PackedRow(int row, int T, int Hkv, int Sk, const int32_t *lengths, const int32_t *offsets, bool at_end) {
        const int bh = quotient(row, T);
        b = quotient(bh, Hkv);
        t = row - bh * T;
        hk = bh - b * Hkv;
        const int len = min(max(lengths[b], 0), Sk);
        slot = (offsets ? (int64_t)offsets[b] : at_end ? (int64_t)len - T : 0) + t;
        kept = slot >= 0 && slot < len;
    }
};

// A quad of lanes takes a group of a new token's key and of its value: 2 d bytes in and R out for each, 2 d more with `values`.  Issue of vector instructions (94 % of the
// cycles) and memory bound it, one as nearly as the other: 4 x 8 x 8192 x 128 with values, of 70 to 100 % of that length: 280 MB, 58.4 us, 4.8 TB/s, which is a copy's rate
// (6 us more with stores of values that stay in the caches, 4 and 6 more where a thread takes two and four tokens).
template <int G, bool BF16>
__global__ void __launch_bounds__(256) smha_packed_put(const PackParams p) {
    constexpr int ROWS = 64 / G;  // of a workgroup (of three groups one quad has nothing to do)
    const int quad = threadIdx.x >> 2, at = threadIdx.x & 3, first = quad / G, g = quad - first * G, col = 32 * g + 8 * at, row = (int)blockIdx.x * ROWS + first;
    if (first >= ROWS || row >= p.B * p.Hkv * p.T) return;
    const PackedRow to_row(row, p.T, p.Hkv, p.Sk, p.lengths, p.offsets, true);
    const bool there = col < p.d;
    u32x4 x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[i] = u32x4{0, 0, 0, 0};
        if (to_row.kept && there) x[i] = *reinterpret_cast<const u32x4 *>(p.x[i] + to_row.b * p.xs[i].b + to_row.hk * p.xs[i].h + to_row.t * p.xs[i].s + col);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t head;
        const uint32_t word = pack8<BF16>(x[i], there, head);
        if (to_row.kept) {
            uint8_t *const to = p.cache[i] + to_row.b * p.cs[i].b + to_row.hk * p.cs[i].h + to_row.slot * p.cs[i].s;
            if (at == 0) *reinterpret_cast<uint32_t *>(to + 4 * g) = head;
            if (there) *reinterpret_cast<uint32_t *>(to + 4 * G + 16 * g + 4 * at) = word;
        }
        if (p.values[i] && there) {
            u32x4 v = unpack8(word, head);
            if (BF16)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = as_bf16(v[e]);
            if (!to_row.kept) v = u32x4{0, 0, 0, 0};
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>(p.values[i] + (int64_t)row * p.d + col));
        }
    }
}

struct UnpackParams {
    const uint8_t *cache[2];
    void *out[2];
    Strides cs[2], os[2];
    const int32_t *lengths, *offsets;  // offsets: null for 0
    int B, Hkv, T, Sk, d;
};

// A lane takes 8 columns of a slot's key and of its value: R bytes in and d values out for each.  Issue of vector instructions (82 % of the cycles) and memory bound it: 4 x 8 x
// 16384 x 128 of 70 to 100 % of that length to bfloat16: 352 MB, 51 us a pass (of which the cache's 84 MB stay in the last level from call to call; 20 more with stores that
// do, 1 or 2 where a thread takes two and four slots).  To float32 608 MB, 218 us: its two stores of a lane lie 32 bytes apart between lanes, each half of what it touches.
template <int OUT>
__global__ void __launch_bounds__(256) smha_packed_get(const UnpackParams p) {
    const int chunks = p.d >> 3, G = (p.d + 31) >> 5, at_once = quotient(256, chunks), first = quotient(threadIdx.x, chunks), chunk = (int)threadIdx.x - first * chunks;
    const int row = (int)blockIdx.x * at_once + first;
    if (first >= at_once || row >= p.B * p.Hkv * p.T) return;
    const PackedRow of(row, p.T, p.Hkv, p.Sk, p.lengths, p.offsets, false);
    uint32_t head[2] = {0, 0}, word[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (of.kept) {
            const uint8_t *const from = p.cache[i] + of.b * p.cs[i].b + of.hk * p.cs[i].h + of.slot * p.cs[i].s;
            head[i] = *reinterpret_cast<const uint32_t *>(from + 4 * (chunk >> 2));
            word[i] = *reinterpret_cast<const uint32_t *>(from + 4 * G + 4 * chunk);
        }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        u32x4 v = unpack8(word[i], head[i]);
        const int64_t at = of.b * p.os[i].b + of.hk * p.os[i].h + of.t * p.os[i].s + 8 * chunk;
        if constexpr (OUT == SMHA_F32) {
            float *const to = (float *)p.out[i] + at;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                __builtin_nontemporal_store(f32x4{widen16<false>(v[2 * h] & 0xFFFFu), widen16<false>(v[2 * h] >> 16), widen16<false>(v[2 * h + 1] & 0xFFFFu), widen16<false>(v[2 * h + 1] >> 16)},
                                            reinterpret_cast<f32x4 *>(to + 4 * h));
        } else {
            if (OUT == SMHA_BF16)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = as_bf16(v[e]);
            __builtin_nontemporal_store(v, reinterpret_cast<u32x4 *>((uint16_t *)p.out[i] + at));
        }
    }
}

// ---------------------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------------------
// The rows that read the same keys, T tokens times G = H / Hkv heads, token by token, are taken 16, 32, 64 or 128 at a time; such a tile of rows and
// the tiles of keys that it sees are a group.  Memory bounds calls of few rows: a key's 10 d / 8 bytes meet 4 d G T operations.  There
// every compute unit has to read, whatever the lengths are, so the key tiles of all groups are counted on the device and cut into segments of about the same length, as many as
// workgroups fit the chip (twice as many where few rows read much, half where groups fill the chip by themselves); segments of one group are joined by a second kernel, in a fixed order.
struct PackedParams {
    const uint16_t *Q;
    const uint8_t *K, *V;
    uint16_t *O;
    Strides qs, ks, vs, os;
    const int32_t *lengths;
    int B, H, Hkv, G, T, Sk, d;
    int window, n_sink;
    int row_tiles;  // of a key head's G T rows
    float c;        // scale * log2(e)
    int slots;      // segments wanted; 0: a group is a segment
    int most_slots; // of calls that have much to do
    int2 *info;     // [groups]: first place, segments.  A place is what a segment of a cut group leaves:
    float *stats;   // [place][2][rows]: reference (log2 units), sum
    float *parts;   // [place][rows][D]
};

// The keys that rows of tokens t0 .. t1 of a sequence see: the tiles of the sinks, then those of the window.
template <int KT> struct PackedKeys {
    int len, end, head, first, n, gap0, gap1;
    __device__ __forceinline__ PackedKeys(int length, int T, int Sk, int window, int n_sink, int t0, int t1) {
        len = min(max(length, 0), Sk);
        end = max(0, len - T + t1 + 1);  // past the last token's
        const int from = max(0, max(len - T + t0, 0) - window + 1);  // the first key in the first token's window
        head = (min(n_sink, from) + KT - 1) / KT;
        first = max(from / KT, head);
        n = end > 0 ? max(head + (end - 1) / KT + 1 - first, 0) : 0;
        gap0 = n_sink < from ? n_sink : 0;
        gap1 = n_sink < from ? from : 0;
    }
    // of the rows rows0 .. rows0 + ROWS - 1
    static __device__ __forceinline__ PackedKeys of(const PackedParams &p, int length, int rows0, int rows_of_tile) {
        int t0 = 0, t1 = p.T - 1;
        if (p.row_tiles > 1) {
            t0 = quotient(rows0, p.G);
            t1 = quotient(min(rows0 + rows_of_tile, p.G * p.T) - 1, p.G);
        }
        return PackedKeys(length, p.T, p.Sk, p.window, p.n_sink, t0, t1);
    }
    __device__ __forceinline__ int key(int tile) const { return KT * (tile < head ? tile : first + tile - head); }
};

struct PackedSegment {
    int b, hk, rows0, length;  // b < 0: no segment
    int part, parts;
    int place, group;          // of its results
    __device__ __forceinline__ bool whole() const { return parts == 1; }
    // its share of n tiles
    __device__ __forceinline__ void share(int n, int &begin, int &end) const {
        const int each = parts > 1 ? quotient(n, parts) : n, rest = n - each * parts;
        begin = each * part + min(rest, part);
        end = begin + each + (part < rest ? 1 : 0);
    }
};

// Running sums over a wave's lanes without LDS, and the last of them.
template <int CTRL, int ROWS> __device__ __forceinline__ int plus_moved(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false); }
__device__ __forceinline__ int lanes_scan(int v) {
    v = plus_moved<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8: in rows of 16
    v = plus_moved<0x112, 0xF>(v);
    v = plus_moved<0x114, 0xF>(v);
    v = plus_moved<0x118, 0xF>(v);
    v = plus_moved<0x142, 0xA>(v);     // the first and third row's sums to the second and fourth
    return plus_moved<0x143, 0xC>(v);  // the first half's to the second
}
__device__ __forceinline__ int lanes_sum(int v) { return __builtin_amdgcn_readlane(lanes_scan(v), 63); }

// The segment of a workgroup.  Every workgroup of the launch computes the same cut: `most` tiles a segment at most, so many that all tiles make `wanted` segments.  A
// group's last segment is shorter, so that there are more of them then; where that is most of what is over, `most` is raised by it.  (Where groups fill the
// chip by themselves only those are cut that are longer than twice what a slot has to do.)  Where none are cut, row tiles that read the same keys are a multiple of Hkv
// segments apart, and so, with eight key heads or a multiple, on the same XCD.  Up to 64 entries (row tiles of all sequences) are a lane each, and every wave counts by itself; more are
// counted by the workgroup, in LDS, where its tiles come later.
constexpr int kPackedEntries = 4096;
template <int KT, int ROWS, int TURN> struct PackedCut {
    const PackedParams &p;
    const int E, lane;
    struct Entry {
        int b, rows0, length, n;
    };
    __device__ __forceinline__ Entry entry(int i) const {
        Entry e{0, 0, 0, 0};
        if (i < E) {
            e.b = p.row_tiles > 1 ? quotient(i, p.row_tiles) : i;
            e.rows0 = ROWS * (p.row_tiles - 1 - (i - e.b * p.row_tiles));  // a sequence's last rows, which see the most keys, come first
            e.length = p.lengths[e.b];
            e.n = PackedKeys<KT>::of(p, e.length, e.rows0, ROWS).n;
        }
        return e;
    }
    static __device__ __forceinline__ int parts_of(int n, int most) { return max(1, quotient(n + most - 1, most)); }
    static __device__ __forceinline__ int at_most(int total, int segments) { return max(4, (quotient(total + segments - 1, segments) + TURN - 1) / TURN * TURN); }
    // `count(most)`: segments then.  Where few rows read much (64 tiles a segment then), twice as many: workgroups start while others read (64 x 32 on 8 x 16384 x 128, of 10 to 100 %:
    // 162 us in segments of 188 tiles, 146 of 94; 256 groups of 10 to 100 % of 256 tiles 46.6 of 51, 48.1 of 26; a little more than there are slots is worst, 103 us for 84).
    template <typename Count> __device__ __forceinline__ void choose(int total, int &most, int &n, Count count) const {
        const int target = total >= 64 * p.most_slots ? p.most_slots : p.slots;
        int wanted = target;
        for (;;) {
            most = at_most(total, wanted);
            n = count(most);
            if (wanted < target || n <= target) break;
            wanted -= n - quotient(total, most);  // what is over
            if (2 * wanted <= target) break;
        }
    }
    __device__ __forceinline__ void set(PackedSegment &s, const Entry &e, int parts, int rest, int place) const {
        s.b = e.b;
        s.rows0 = e.rows0;
        s.length = e.length;
        s.parts = parts;
        s.hk = quotient(rest, parts);
        s.part = rest - s.hk * parts;
        s.place = place + rest;
        s.group = (s.b * p.Hkv + s.hk) * p.row_tiles + s.rows0 / ROWS;
    }
    __device__ __forceinline__ void few(PackedSegment &s, int at) const {
        const Entry e = entry(lane);
        auto parts = [&](int most) __attribute__((always_inline)) { return lane < E ? parts_of(e.n, most) : 0; };
        int most, n;
        choose(p.Hkv * lanes_sum(e.n), most, n, [&](int most) __attribute__((always_inline)) { return p.Hkv * lanes_sum(parts(most)); });
        if (at >= n) return;
        const int mine = parts(most), segs = p.Hkv * mine, upto = lanes_scan(segs), cut = mine > 1 ? segs : 0, cut_upto = lanes_scan(cut);
        const int who = __builtin_ctzll(__builtin_amdgcn_ballot_w64(upto > at));
        auto his = [&](int v) __attribute__((always_inline)) { return __builtin_amdgcn_readlane(v, who); };
        set(s, Entry{his(e.b), his(e.rows0), his(e.length), 0}, his(mine), at - his(upto - segs), his(cut_upto - cut));
    }
    __device__ __forceinline__ void many(PackedSegment &s, int at, int *tiles) const {
        __shared__ int sums[2][4];
        __shared__ int found[4];
        const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), per = (E + 255) / 256, first = (int)threadIdx.x * per, last = min(first + per, E);
        for (int i = threadIdx.x; i < E; i += 256) tiles[i] = entry(i).n;
        __syncthreads();
        // a value of every thread: the sum of those before it, and of all
        auto sum_of = [&](int v, int turn, int &before) __attribute__((always_inline)) {
            const int upto = lanes_scan(v);
            __syncthreads();  // (the sums of before are read)
            if (lane == 63) sums[turn][w] = upto;
            __syncthreads();
            int all = 0;
            before = upto - v;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int y = sums[turn][x];
                before += x < w ? y : 0;
                all += y;
            }
            return __builtin_amdgcn_readfirstlane(all);
        };
        int sum = 0, before, most, n;
        for (int i = first; i < last; ++i) sum += tiles[i];
        const int total = p.Hkv * sum_of(sum, 0, before);
        choose(total, most, n, [&](int most) __attribute__((always_inline)) {
            int sum = 0;
            for (int i = first; i < last; ++i) sum += parts_of(tiles[i], most);
            return p.Hkv * sum_of(sum, 0, before);
        });
        if (at >= n) return;  // (the whole workgroup)
        const int start = p.Hkv * before;  // of this thread's entries' segments (the last count was with this `most`)
        int cuts = 0, cuts_before;
        for (int i = first; i < last; ++i) {
            const int parts = parts_of(tiles[i], most);
            cuts += parts > 1 ? parts : 0;
        }
        sum_of(cuts, 1, cuts_before);
        int from = start, place = p.Hkv * cuts_before;
        for (int i = first; i < last && from <= at; ++i) {
            const int parts = parts_of(tiles[i], most);
            if (at < from + p.Hkv * parts) {
                found[0] = i;
                found[1] = parts;
                found[2] = at - from;
                found[3] = place;
            }
            from += p.Hkv * parts;
            place += parts > 1 ? p.Hkv * parts : 0;
        }
        __syncthreads();
        const int i = __builtin_amdgcn_readfirstlane(found[0]), parts = __builtin_amdgcn_readfirstlane(found[1]), rest = __builtin_amdgcn_readfirstlane(found[2]);
        const int b = __builtin_amdgcn_readfirstlane(quotient(i, p.row_tiles));
        set(s, Entry{b, ROWS * (p.row_tiles - 1 - (i - b * p.row_tiles)), uniform_load(p.lengths + b), 0}, parts, rest, __builtin_amdgcn_readfirstlane(found[3]));
    }
};
template <int KT, int ROWS, int TURN> __device__ __forceinline__ PackedSegment packed_segment(const PackedParams &p, int lane, char *lds) {
    PackedSegment s{-1, 0, 0, 0, 0, 1, 0, 0};
    if (p.slots) {
        const PackedCut<KT, ROWS, TURN> cut{p, p.B * p.row_tiles, lane};
        if (__builtin_expect(cut.E <= 64, 1)) cut.few(s, blockIdx.x);
        else cut.many(s, blockIdx.x, reinterpret_cast<int *>(lds));
        return s;
    }
    // groups as they are, an XCD a run of them, with sequences of all lengths
    const int n = p.B * p.Hkv * p.row_tiles, run = (n + 7) / 8, slot = (int)blockIdx.x >> 3, at = ((int)blockIdx.x & 7) * run + slot;
    if (slot >= run || at >= n) return s;
    const int hb = quotient(at, p.row_tiles);
    s.hk = quotient(hb, p.B);
    s.b = hb - s.hk * p.B;
    s.rows0 = ROWS * (p.row_tiles - 1 - (at - hb * p.row_tiles));
    s.length = uniform_load(p.lengths + s.b);
    return s;
}

// Probabilities are rounded to binary16 for the second product, whatever the inputs' type, relative to a reference that is about the row's largest score so far.  They are
// taken 2^7 times as large, as are their sums, so that the joins and the last division know nothing of it: below 2^-14 binary16 has fewer digits and
// below 2^-25 none, and where one key has nearly all of the weight (the first of a text often has) the others share what is down there.  Only what is
// below 2^-32 of the largest is lost so.  The reference is raised by a score 2^4 over it, not 2^8 as in the 16-bit operators: 2^11 times 2^4.99 is binary16's end, as far from
// the largest as there, where scores are so large that 32 bits leave their exponents whole numbers.
constexpr float kPackedShift = 7.f;
__device__ __forceinline__ float packed_raised_over(float c) { return fminf(4.0f / c, 3e38f); }
// The exponent's constant for a running reference (not yet multiplied by c): fmaf(score, c, this).
__device__ __forceinline__ float packed_from(float reference, float c) { return fmaf(reference == -__builtin_inff() ? 0.f : -reference, c, kPackedShift); }
// The reference in powers of two, as that constant has it after its rounding.
__device__ __forceinline__ float packed_reference(float reference, float c) { return reference == -__builtin_inff() ? reference : kPackedShift - packed_from(reference, c); }

// The reference that a row's segment leaves: -inf says that it has no keys.  (A row of NaN has no largest score either, and must not be passed over.)
__device__ __forceinline__ float reference_left(float m, float l) { return l == l ? m : 0.f; }

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// A row of queries as the B operand of the scores' product, in binary16: a lane holds N chunks of 8 columns, chunk i from column `col(i)` on, and the row's other
// columns are in lanes 16 (STEPS16: and 32) apart.  A row that does not exist and columns that the head does not have are zeros (something that exists is
// read in their place: loads without branches travel together).  bfloat16 rows are brought to 2^14 .. 2^15 by a power of two, by which they fit binary16
// without loss (but for columns below 2^-31 of the largest, which lose digits); returns what the scores have to be multiplied by.
template <int N, bool BF16, bool STEPS16, typename Col>
__device__ __forceinline__ float load_query(u32x4 (&qf)[N], const uint16_t *row, bool exists, const uint16_t *other, int d, Col col) {
    if (!exists) row = other;
#pragma unroll
    for (int i = 0; i < N; ++i) qf[i] = *reinterpret_cast<const u32x4 *>(row + (col(i) < d ? col(i) : 0));
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (!exists || col(i) >= d) qf[i] = u32x4{0, 0, 0, 0};
    if constexpr (!BF16) {
        return 1.f;
    } else {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(fabsf(widen16<true>(qf[i][e] & 0xFFFFu)), fabsf(widen16<true>(qf[i][e] >> 16))));
        if (STEPS16) top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const int e2 = min(15 - __builtin_amdgcn_frexp_expf(top), 100);
        const float power = __builtin_amdgcn_ldexpf(1.f, e2);
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) qf[i][e] = pack2<false>(widen16<true>(qf[i][e] & 0xFFFFu) * power, __builtin_bit_cast(float, qf[i][e] & 0xFFFF0000u) * power);
        return __builtin_amdgcn_ldexpf(1.f, -e2);
    }
}

// Packed rows as a lane reads them: D / 4 columns of a key, those from (D / 4) u on.  Keys past the buffer read as zeros, and so do those between the sinks
// and the window (which no row of the tile sees; a step and a base of 0 are enough) and the columns that the head does not have.
template <int D> struct PackedLoad {
    static constexpr int NW = D / 32;  // words of codes
    struct Raw {
        uint32_t head, code[NW];
    };
    __amdgpu_buffer_rsrc_t r;
    int pitch, head_at, codes_at, gap0, gap1;
    template <int KT> __device__ __forceinline__ PackedLoad(const uint8_t *rows, int64_t pitch_, const PackedKeys<KT> &keys, int d, int u) {
        const int groups = (d + 31) >> 5, mine = D == 128 ? u : u >> 1;
        r = make_rsrc(rows, keys.end > 0 ? (int64_t)(keys.end - 1) * pitch_ + 4 * groups + (d >> 1) : 0);
        pitch = (int)pitch_;
        head_at = mine < groups ? 4 * mine : (int)kPast;
        codes_at = 4 * groups + D / 8 * u;
        gap0 = keys.gap0;
        gap1 = keys.gap1;
    }
    __device__ __forceinline__ Raw operator()(int key) const {
        Raw x;
        const int at = key * pitch;
        x.head = __builtin_amdgcn_raw_buffer_load_b32(r, (key >= gap0 && key < gap1) || head_at == (int)kPast ? (int)kPast : at + head_at, 0, 0);
        if constexpr (NW == 4) {
            const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, at + codes_at, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) x.code[i] = v[i];
        } else {
            const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, at + codes_at, 0, 0));
            x.code[0] = v[0];
            x.code[1] = v[1];
        }
        return x;
    }
};

// Swizzle of a 32-row tile of values: writes of 16 rows at one chunk of 16 bytes, and transposing reads of 8 rows x 2 chunks (half a wave), all over the banks.
template <int D> __device__ __forceinline__ int swz_values(int row) {
    if constexpr (D == 128) return ((row & 7) << 1) | ((row >> 3) & 1);
    else return (((row >> 1) & 3) << 1) | ((row >> 3) & 1);
}

// Which of 16 rows lane j unpacks into LDS: a write of 8 lanes' 16 bytes goes without conflicts where these chunks are apart, modulo 8, of rows swizzled as above (D: as by
// swz_values; WIDE: as by swz_both).
template <int D, bool WIDE = false> __device__ __forceinline__ int mixed(int j) {
    if constexpr (D == 64) return ((j & 7) << 1) | (j >> 3);
    else if constexpr (WIDE) return (j & 1) | ((j & 6) << 1) | ((j & 8) >> 2);
    else return (j & 3) | ((j & 4) << 1) | ((j & 8) >> 1);
}

// Four waves take a segment's tiles of 32 keys in turn and join in LDS, as they read alone: what bounds it is memory (1024 x 32 on 8 x 2048 x 128: 2.7 GB in 513 us, 5.2 TB/s; 2 x 32 on
// 8 x 65536: 168 MB in 32 us), with vector instructions on more than half of the cycles.  A lane unpacks D / 4 columns of two keys: keys are an operand as they come out; values go
// through LDS once, for the transposing reads that make them the other product's.  NR tiles of 16 rows share what is unpacked.
constexpr int packed_workgroups(int D, int NR) { return D == 64 ? (NR == 1 ? 4 : 3) : NR == 1 ? 3 : 2; }  // of a compute unit
template <int D, int NR, bool BF16>
__global__ void __launch_bounds__(256, packed_workgroups(D, NR)) smha_packed_part(const PackedParams p) {
    constexpr int NS = D / 32, NC = D / 16, TB = 32 * D * 2, ROWS = 16 * NR;  // steps of the first product, tiles of columns, bytes of a tile
    __shared__ __attribute__((aligned(1024))) char all_tiles[4 * TB];
    __shared__ float team[4][2][ROWS];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 15, u = lane >> 4;
    char *const smem = all_tiles + w * TB;
    const float NEG_INF = -__builtin_inff();

    const PackedSegment s = packed_segment<32, ROWS, 4>(p, lane, all_tiles);
    if (s.b < 0) return;
    const int rows = p.G * p.T;
    const auto keys = PackedKeys<32>::of(p, s.length, s.rows0, ROWS);
    const PackedLoad<D> loadK(p.K + s.b * p.ks.b + s.hk * p.ks.h, p.ks.s, keys, p.d, u), loadV(p.V + s.b * p.vs.b + s.hk * p.vs.h, p.vs.s, keys, p.d, u);
    int begin, end;
    s.share(keys.n, begin, end);
    begin += w;
    const int vj = mixed<D>(j);  // the key of a value that this lane unpacks
    typename PackedLoad<D>::Raw k_raw[2], v_raw[2];  // refilled as soon as they are unpacked
    auto request_k = [&](int tile) __attribute__((always_inline)) {
        const int key = keys.key(tile) + j;
#pragma unroll
        for (int a = 0; a < 2; ++a) k_raw[a] = loadK(key + 16 * a);
    };
    auto request_v = [&](int tile) __attribute__((always_inline)) {
        const int key = keys.key(tile) + vj;
#pragma unroll
        for (int a = 0; a < 2; ++a) v_raw[a] = loadV(key + 16 * a);
    };
    if (begin < end) {
        request_k(begin);
        request_v(begin);
    }

    u32x4 qf[NR][NS];
    int pos[NR];  // below 0: no such query
    uint16_t *to[NR];
    float c[NR], thr[NR];
#pragma unroll
    for (int x = 0; x < NR; ++x) {
        const int row = s.rows0 + 16 * x + j, t = quotient(row, p.G), g = row - t * p.G, h = s.hk * p.G + g;
        pos[x] = row < rows ? keys.len - p.T + t : -1;
        to[x] = row < rows ? p.O + s.b * p.os.b + h * p.os.h + t * p.os.s : nullptr;
        // (never 0: -inf times it)
        const uint16_t *const q0 = p.Q + s.b * p.qs.b + s.hk * p.G * p.qs.h;
        c[x] = fmaxf(p.c * load_query<NS, BF16, true>(qf[x], q0 + g * p.qs.h + t * p.qs.s, pos[x] >= 0, q0, p.d, [&](int i) { return D / 4 * u + 8 * i; }), 0x1p-126f);
        thr[x] = packed_raised_over(c[x]);
    }
    float m_run[NR], l_run[NR];
    f32x4 o[NR][NC];
#pragma unroll
    for (int x = 0; x < NR; ++x) {
        m_run[x] = NEG_INF;
        l_run[x] = 0.f;
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) o[x][ct] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int tr_row = 4 * u + (j >> 2);
    for (int tile = begin; tile < end; tile += 4) {
        const int key = keys.key(tile);
        // acc[x][a][r]: the score of query j and key 16 a + 4 u + r
        f32x4 acc[NR][2];
#pragma unroll
        for (int x = 0; x < NR; ++x) acc[x][0] = acc[x][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const u32x4 kf = unpack8(k_raw[a].code[i], k_raw[a].head);
#pragma unroll
                for (int x = 0; x < NR; ++x) acc[x][a] = mfma16(kf, qf[x][i], acc[x][a]);
            }
        if (tile + 4 < end) request_k(tile + 4);
        // values go to LDS under that product
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int i = 0; i < NS; ++i)
                *reinterpret_cast<u32x4 *>(smem + (16 * a + vj) * D * 2 + (((D / 32 * u + i) ^ swz_values<D>(vj)) * 16)) = unpack8(v_raw[a].code[i], v_raw[a].head);
        if (tile + 4 < end) request_v(tile + 4);
        __builtin_amdgcn_s_setprio(1);  // (as in smha_packed_wide; 64 x 32 on 8 x 4096 x 128, 5 tokens: 82 us without, 81; of 10 to 100 % of that length 72, 70.5)
        u32x4 pf[NR];
#pragma unroll
        for (int x = 0; x < NR; ++x) {
            const uint32_t word = pos[x] >= 0 ? low_bits32(pos[x] - key + 1) & (~low_bits32(pos[x] - p.window + 1 - key) | low_bits32(p.n_sink - key)) : 0;
            if (__builtin_amdgcn_ballot_w64(word != ~0u) != 0) {
#pragma unroll
                for (int a = 0; a < 2; ++a)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[x][a][r] = (word >> (16 * a + 4 * u + r)) & 1 ? acc[x][a][r] : NEG_INF;
            }
            float mt = NEG_INF;
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int r = 0; r < 4; ++r) mt = fmaxf(mt, acc[x][a][r]);
            if (__builtin_amdgcn_ballot_w64(mt > m_run[x] + thr[x]) != 0) {
                mt = fmaxf(mt, __shfl_xor(mt, 16));
                mt = fmaxf(mt, __shfl_xor(mt, 32));
                const float m_new = fmaxf(m_run[x], mt), alpha = fast_exp2((m_run[x] - (m_new == NEG_INF ? 0.f : m_new)) * c[x]);
                m_run[x] = m_new;
                l_run[x] *= alpha;
#pragma unroll
                for (int ct = 0; ct < NC; ++ct) o[x][ct] *= alpha;
            }
            const float from = packed_from(m_run[x], c[x]);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float e0 = fast_exp2(fmaf(acc[x][q >> 1][2 * (q & 1)], c[x], from)), e1 = fast_exp2(fmaf(acc[x][q >> 1][2 * (q & 1) + 1], c[x], from));
                pf[x][q] = pack2<false>(e0, e1);
                l_run[x] += e0 + e1;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) {
            const int chunk = 2 * ct + ((j & 3) >> 1), at = tr_row * D * 2 + ((chunk ^ swz_values<D>(tr_row)) * 16) + (j & 1) * 8;
            const u32x2 lo = lds_read_tr(reinterpret_cast<const uint16_t *>(smem + at)), hi = lds_read_tr(reinterpret_cast<const uint16_t *>(smem + at + 16 * D * 2));
#pragma unroll
            for (int x = 0; x < NR; ++x) o[x][ct] = mfma16(u32x4{lo[0], lo[1], hi[0], hi[1]}, pf[x], o[x][ct]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tile is read
        __builtin_amdgcn_s_setprio(0);
    }

    // The team joins: every wave leaves its accumulators in its own tile's place and takes a quarter of the columns of all four.
    constexpr int NQ = NC / 4;
    if (p.slots && s.part == 0 && threadIdx.x == 0) p.info[s.group] = int2{s.place, s.parts};
#pragma unroll
    for (int x = 0; x < NR; ++x) {
        float l = l_run[x] + __shfl_xor(l_run[x], 16);
        l += __shfl_xor(l, 32);
        if (u == 0) {
            team[w][0][16 * x + j] = packed_reference(m_run[x], c[x]);
            team[w][1][16 * x + j] = l;
        }
    }
#pragma unroll
    for (int x = 0; x < NR; ++x) {
        if (x) __syncthreads();
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) *reinterpret_cast<f32x4 *>(smem + (ct * 64 + lane) * 16) = o[x][ct];
        __syncthreads();
        float m_all = NEG_INF, l_all = 0.f;
        f32x4 out[NQ];
#pragma unroll
        for (int v = 0; v < 4; ++v) m_all = fmaxf(m_all, team[v][0][16 * x + j]);
#pragma unroll
        for (int i = 0; i < NQ; ++i) out[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const float mu = team[v][0][16 * x + j], share = mu != NEG_INF ? fast_exp2(mu - m_all) : 0.f;
            l_all = fmaf(share, team[v][1][16 * x + j], l_all);
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                const f32x4 y = *reinterpret_cast<const f32x4 *>(all_tiles + v * TB + ((w * NQ + i) * 64 + lane) * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) out[i][e] = fmaf(share, y[e], out[i][e]);
            }
        }
        if (to[x]) {
            const float inv = l_all != 0.f ? 1.0f / l_all : 0.f;
            if (!s.whole() && w == 0 && u == 0) {
                p.stats[(int64_t)s.place * 2 * ROWS + 16 * x + j] = reference_left(m_all, l_all);
                p.stats[(int64_t)s.place * 2 * ROWS + ROWS + 16 * x + j] = l_all;
            }
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                const int col = 16 * (w * NQ + i) + 4 * u;
                if (s.whole()) {
                    if (col < p.d) store4<BF16 ? SMHA_BF16 : SMHA_F16>(to[x], col, out[i][0] * inv, out[i][1] * inv, out[i][2] * inv, out[i][3] * inv);
                } else {
                    *reinterpret_cast<f32x4 *>(p.parts + ((int64_t)s.place * ROWS + 16 * x + j) * D + col) = out[i];
                }
            }
        }
    }
}

// Many rows on the same keys: four waves share tiles of 64 keys, which all of them unpack into LDS, the next one before they use this one, from words that were
// requested two tiles before (one before: 538 us for the 522 of the call below on one card).  KH = 1: a wave takes 32 of 128 rows; KH = 2: a wave takes 32 of 64 rows and one half of the keys, and the halves are joined at the end.  From
// LDS on it is as in smha_sink_fwd, in binary16 throughout.  Waves with vector work go first, those in the mixed phase (masks, exponentials, second product) before those that
// unpack, so that the two of a SIMD are in different phases (2 x 1024 tokens x 32 on 8 x 16384 x 128: 579 us without, 537, of 70 to 100 % of that length 541, 507; 4 x 512 x 32 on 8 x 8192 x 64: 234, 205).
// Bound by issue (81 % of the cycles) and by power (1.95 GHz): the second of these calls 505 to 520 us, by the card, 0.9 PFLOP/s.
template <int D, int KH, bool BF16>
__global__ void __launch_bounds__(256, D == 64 ? 3 : 2) smha_packed_wide(const PackedParams p) {
    constexpr int NS = D / 16, NDT = D / 32, NL = D / 32, TB = 64 * D * 2, ROWS = 128 / KH, KTS = 2 / KH;  // KTS: halves of a tile that a wave takes
    constexpr int PF = KH == 1 && D == 128 ? 8 : 4;  // operands requested ahead
    __shared__ __attribute__((aligned(1024))) char smem[4 * TB];  // K[0], K[1], V[0], V[1]
    __shared__ float team[2][2][32];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 31, hh = lane >> 5;
    const int wr = KH == 1 ? w : w & 1, wk = KH == 1 ? 0 : w >> 1;  // the wave's rows, and its half of the keys
    const float NEG_INF = -__builtin_inff();

    const PackedSegment s = packed_segment<64, ROWS, 1>(p, lane, smem);
    if (s.b < 0) return;
    const int rows = p.G * p.T;
    const auto keys = PackedKeys<64>::of(p, s.length, s.rows0, ROWS);
    const PackedLoad<D> loadK(p.K + s.b * p.ks.b + s.hk * p.ks.h, p.ks.s, keys, p.d, lane >> 4), loadV(p.V + s.b * p.vs.b + s.hk * p.vs.h, p.vs.s, keys, p.d, lane >> 4);
    int begin, end;
    s.share(keys.n, begin, end);
    // this lane's part of a tile: D / 4 columns of one of the wave's 16 keys
    const int kj = 16 * w + mixed<D, true>(lane & 15);
    struct Raw {
        typename PackedLoad<D>::Raw k, v;
    } raw[2];  // of the next two tiles
    auto request = [&](Raw &x, int tile) __attribute__((always_inline)) {
        const int key = keys.key(tile) + kj;
        x.k = loadK(key);
        x.v = loadV(key);
    };
    if (begin < end) request(raw[0], begin);
    if (begin + 1 < end) request(raw[1], begin + 1);

    const int row0 = s.rows0 + 32 * wr, row = row0 + j, t = quotient(row, p.G), g = row - t * p.G, h = s.hk * p.G + g;
    const int pos = row < rows ? keys.len - p.T + t : -1;  // below 0: no such query
    const int wp0 = keys.len - p.T + quotient(row0, p.G), wp1 = row0 < rows ? keys.len - p.T + quotient(min(row0 + 32, rows) - 1, p.G) : -1;  // the wave's positions
    const bool every = wp0 >= 0 && row0 + 32 <= rows;
    u32x4 qf[NS];
    const uint16_t *const q0 = p.Q + s.b * p.qs.b + s.hk * p.G * p.qs.h;
    const float c = fmaxf(p.c * load_query<NS, BF16, false>(qf, q0 + g * p.qs.h + t * p.qs.s, pos >= 0, q0, p.d, [&](int i) { return 16 * i + 8 * hh; }), 0x1p-126f);
    const float thr = packed_raised_over(c);

    // the i-th of 2 NL chunks of a tile, keys' first
    const int lv = kj * D * 2 + ((NL * (lane >> 4) ^ (swz_both<D>(kj) & ~(NL - 1))) * 16), lx = swz_both<D>(kj) & (NL - 1);
    auto leave = [&](int at, int par, const Raw &x, int i) __attribute__((always_inline)) {
        char *const tile = smem + (i < NL ? par : 2 + par) * TB;
        const typename PackedLoad<D>::Raw &y = i < NL ? x.k : x.v;
        *reinterpret_cast<u32x4 *>(tile + at + (((i % NL) ^ lx) * 16)) = unpack8(y.code[i % NL], y.head);
    };
    if (begin < end) {
#pragma unroll
        for (int i = 0; i < 2 * NL; ++i) leave(lv, 0, raw[0], i);
    }
    if (begin + 2 < end) request(raw[0], begin + 2);

    const int rd = j * D * 2 + ((hh ^ swz_both<D>(j)) * 16);
    const int tr_row = 4 * hh + ((lane & 15) >> 2);
    const int tr = tr_row * D * 2 + ((swz_both<D>(tr_row) ^ (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1))) * 16) + (lane & 1) * 8;
    float m_run = NEG_INF, l_run = 0.f;
    f32x16 o[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) o[dt] = zeros16();
    __syncthreads();
    auto step = [&](int tile, Raw &next) __attribute__((always_inline)) {
        const int par = (tile - begin) & 1;
        const int key = keys.key(tile), key_w = key + 32 * wk;
        constexpr int KW = 32 * KTS;
        __builtin_amdgcn_s_setprio(1);
        if (tile + 1 < end) {
#pragma unroll
            for (int i = 0; i < 2 * NL; ++i) leave(lv, par ^ 1, next, i);
            if (tile + 3 < end) request(next, tile + 3);
        }
        if (wp1 >= 0 && key_w <= wp1 && (wp0 - key_w - (KW - 1) < p.window || key_w < p.n_sink)) {  // some row of the wave sees some key
            const char *const Kt = smem + par * TB + 32 * wk * D * 2, *const Vt = smem + (2 + par) * TB + 32 * wk * D * 2;
            __builtin_amdgcn_s_setprio(0);
            f32x16 acc[KTS];
#pragma unroll
            for (int kt = 0; kt < KTS; ++kt) acc[kt] = zeros16();
            auto k_frag = [&](int i) __attribute__((always_inline)) { return *reinterpret_cast<const u32x4 *>(Kt + ((rd ^ (32 * (i / KTS))) + 64 * (i % KTS) * D)); };
            u32x4 kf[PF];
#pragma unroll
            for (int i = 0; i < PF; ++i) kf[i] = k_frag(i);
#pragma unroll
            for (int i = 0; i < KTS * NS; ++i) {
                acc[i % KTS] = mfma32<false>(kf[i % PF], qf[i / KTS], acc[i % KTS]);
                if (i + PF < KTS * NS) kf[i % PF] = k_frag(i + PF);
            }
            __builtin_amdgcn_s_setprio(2);
            if (!(every && key_w + KW - 1 <= wp0 && (wp1 - key_w < p.window || key_w + KW - 1 < p.n_sink))) {  // not every row sees every key
                const uint64_t word = pos >= 0 ? low_bits(pos - key_w + 1) & (~low_bits(pos - p.window + 1 - key_w) | low_bits(p.n_sink - key_w)) : 0;
#pragma unroll
                for (int kt = 0; kt < KTS; ++kt) {
                    const u32x16 keep = keep_of((uint32_t)(word >> (32 * kt)) >> (4 * hh)), sc = __builtin_bit_cast(u32x16, acc[kt]);
                    acc[kt] = __builtin_bit_cast(f32x16, (sc & keep) | (~keep & 0xFF800000u));
                }
            }
            float mt = NEG_INF;
#pragma unroll
            for (int kt = 0; kt < KTS; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) mt = fmaxf(mt, acc[kt][r]);
            if (__builtin_amdgcn_ballot_w64(mt > m_run + thr) != 0) {
                mt = fmaxf(mt, __shfl_xor(mt, 32));
                const float m_new = fmaxf(m_run, mt), alpha = fast_exp2((m_run - (m_new == NEG_INF ? 0.f : m_new)) * c);
                m_run = m_new;
                l_run *= alpha;
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) o[dt] *= alpha;
            }
            const float from = packed_from(m_run, c);
            u32x4 pf[2 * KTS];
            auto p_pair = [&](int cu, int q) __attribute__((always_inline)) {
                const float e0 = fast_exp2(fmaf(acc[cu >> 1][8 * (cu & 1) + 2 * q], c, from)), e1 = fast_exp2(fmaf(acc[cu >> 1][8 * (cu & 1) + 2 * q + 1], c, from));
                pf[cu][q] = pack2<false>(e0, e1);
                l_run += e0 + e1;
            };
            auto v_frag = [&](int i) __attribute__((always_inline)) {
                const char *const at = Vt + ((tr ^ (64 * (i % NDT))) + 32 * (i / NDT) * D), *const at8 = Vt + ((tr ^ (64 * (i % NDT)) ^ 32) + 32 * (i / NDT) * D + 16 * D);
                const u32x2 lo = lds_read_tr(reinterpret_cast<const uint16_t *>(at)), hi = lds_read_tr(reinterpret_cast<const uint16_t *>(at8));
                return u32x4{lo[0], lo[1], hi[0], hi[1]};
            };
            u32x4 vf[PF];
#pragma unroll
            for (int i = 0; i < PF; ++i) vf[i] = v_frag(i);
#pragma unroll
            for (int q = 0; q < 4; ++q) p_pair(0, q);
#pragma unroll
            for (int i = 0; i < 2 * KTS * NDT; ++i) {
                const int cu = i / NDT, dt = i % NDT;
                o[dt] = mfma32<false>(vf[i % PF], pf[cu], o[dt]);
                if (i + PF < 2 * KTS * NDT) vf[i % PF] = v_frag(i + PF);
                if (cu < 2 * KTS - 1) {
#pragma unroll
                    for (int q = (4 * dt + NDT - 1) / NDT; q < (4 * dt + NDT + 3) / NDT; ++q) p_pair(cu + 1, q);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        // (not __syncthreads: that would wait for the words on their way)
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    for (int tile = begin; tile < end; tile += 2) {
        step(tile, raw[1]);
        if (tile + 1 < end) step(tile + 1, raw[0]);
    }
    float l = l_run + __shfl_xor(l_run, 32), m = packed_reference(m_run, c);
    if constexpr (KH == 2) {  // the keys' halves join: the second leaves its accumulators where the tiles were
        f32x4 *const left = reinterpret_cast<f32x4 *>(smem + wr * (32 * D * 4));
        if (wk == 1) {
#pragma unroll
            for (int i = 0; i < D / 8; ++i) left[i * 64 + lane] = f32x4{o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]};
            if (hh == 0) {
                team[wr][0][j] = m;
                team[wr][1][j] = l;
            }
        }
        __syncthreads();
        if (wk == 1) return;
        const float mu = team[wr][0][j], top = fmaxf(m, mu), mine = m != NEG_INF ? fast_exp2(m - top) : 0.f, his = mu != NEG_INF ? fast_exp2(mu - top) : 0.f;
        l = fmaf(his, team[wr][1][j], mine * l);
        m = top;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            const f32x4 y = left[i * 64 + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i / 4][4 * (i % 4) + e] = fmaf(his, y[e], mine * o[i / 4][4 * (i % 4) + e]);
        }
    }
    if (p.slots && s.part == 0 && threadIdx.x == 0) p.info[s.group] = int2{s.place, s.parts};
    if (row >= rows) return;
    if (s.whole()) {
        const float inv = l != 0.f ? 1.0f / l : 0.f;
        uint16_t *const to = p.O + s.b * p.os.b + h * p.os.h + t * p.os.s;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
            const int col = 8 * i + 4 * hh;
            if (col < p.d)
                store4<BF16 ? SMHA_BF16 : SMHA_F16>(to, col, o[i / 4][4 * (i % 4)] * inv, o[i / 4][4 * (i % 4) + 1] * inv, o[i / 4][4 * (i % 4) + 2] * inv, o[i / 4][4 * (i % 4) + 3] * inv);
        }
    } else {
        if (hh == 0) {
            p.stats[(int64_t)s.place * 2 * ROWS + 32 * wr + j] = reference_left(m, l);
            p.stats[(int64_t)s.place * 2 * ROWS + ROWS + 32 * wr + j] = l;
        }
        float *const part = p.parts + ((int64_t)s.place * ROWS + 32 * wr + j) * D + 4 * hh;
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
            *reinterpret_cast<f32x4 *>(part + 8 * i) = f32x4{o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]};
    }
}

// Joins the segments of a row, W waves a row: D / 4 lanes read a segment's result, four columns each, and as many segments are read at once as there are
// such lanes, four times over.  (What a row lasts is its chain of trips to memory.)
template <int D, int ROWS, int W, bool BF16>
__global__ void __launch_bounds__(256) smha_packed_join(const PackedParams p) {
    constexpr int CL = D / 4, SUB = 64 / CL, RPW = 4 / W;
    __shared__ float lds_ml[2][4];
    __shared__ __attribute__((aligned(16))) float lds_o[4][D];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rows = p.G * p.T, cl = lane % CL;
    // (a wave that has a row for itself takes several where there are many)
    for (int id = (int)blockIdx.x * RPW + w / W; id < p.B * p.Hkv * rows; id += (int)gridDim.x * RPW) {
        const int bh = quotient(id, rows), row = id - bh * rows, b = quotient(bh, p.Hkv), hk = bh - b * p.Hkv, t = quotient(row, p.G), g = row - t * p.G;
        const int2 info = uniform_load(p.info + (int64_t)bh * p.row_tiles + row / ROWS);
        if (info.y <= 1) continue;  // written whole
        const float *const stats = p.stats + (int64_t)info.x * 2 * ROWS + row % ROWS, *const parts = p.parts + ((int64_t)info.x * ROWS + row % ROWS) * D + 4 * cl;
        const float NEG_INF = -__builtin_inff();
        float m = NEG_INF, sum = 0.f;
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
        for (int i0 = (w % W) * SUB + lane / CL; i0 < info.y; i0 += 4 * W * SUB) {
            float ref[4], part[4], top = m;
            f32x4 x[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int i = i0 + W * SUB * q < info.y ? i0 + W * SUB * q : i0;
                ref[q] = stats[(int64_t)i * 2 * ROWS];
                part[q] = stats[(int64_t)i * 2 * ROWS + ROWS];
                x[q] = *reinterpret_cast<const f32x4 *>(parts + (int64_t)i * ROWS * D);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if (i0 + W * SUB * q >= info.y) ref[q] = NEG_INF;
                top = fmaxf(top, ref[q]);
            }
            const float old = m != NEG_INF ? fast_exp2(m - top) : 0.f;
            sum *= old;
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] *= old;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (ref[q] != NEG_INF) {
                    const float share = fast_exp2(ref[q] - top);
                    sum = fmaf(share, part[q], sum);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[e] = fmaf(share, x[q][e], acc[e]);
                }
            m = top;
        }
        // lanes with the same columns, in the order of a tree
#pragma unroll
        for (int far = CL; far < 64; far *= 2) {
            const float mu = __shfl_xor(m, far), top = fmaxf(m, mu), mine = m != NEG_INF ? fast_exp2(m - top) : 0.f, his = mu != NEG_INF ? fast_exp2(mu - top) : 0.f;
            sum = mine * sum + his * __shfl_xor(sum, far);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = mine * acc[e] + his * __shfl_xor(acc[e], far);
            m = top;
        }
        uint16_t *const to = p.O + b * p.os.b + (hk * p.G + g) * p.os.h + t * p.os.s;
        if constexpr (W == 4) {
            if (lane == 0) {
                lds_ml[0][w] = m;
                lds_ml[1][w] = sum;
            }
            if (lane < CL) *reinterpret_cast<f32x4 *>(&lds_o[w][4 * cl]) = acc;
            __syncthreads();
            if (w) return;  // (a workgroup has one row)
            const float top = fmaxf(fmaxf(lds_ml[0][0], lds_ml[0][1]), fmaxf(lds_ml[0][2], lds_ml[0][3]));
            sum = 0.f;
            acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float share = lds_ml[0][q] != NEG_INF ? fast_exp2(lds_ml[0][q] - top) : 0.f;
                const f32x4 y = *reinterpret_cast<const f32x4 *>(&lds_o[q][4 * cl]);
                sum = fmaf(share, lds_ml[1][q], sum);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(share, y[e], acc[e]);
            }
        }
        const float inv = sum != 0.f ? 1.0f / sum : 0.f;
        if (lane < CL && 4 * cl < p.d) store4<BF16 ? SMHA_BF16 : SMHA_F16>(to, 4 * cl, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
    }
}

// ---------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------
// Rows of packed bytes: whole words, none over another, a head within 2 GiB.
static bool packed_strides_fit(const int64_t *s, int64_t rows, int d) {
    const int row = packed_row_bytes(d);
    if (!s) return (rows + 64) * row < ((int64_t)1 << 31);
    return s[0] % 4 == 0 && s[1] % 4 == 0 && s[2] % 4 == 0 && s[0] >= 0 && s[1] >= 0 && s[2] >= row && s[2] < ((int64_t)1 << 31) && (rows + 64) * s[2] + row < ((int64_t)1 << 31);
}
static Strides packed_strides(const int64_t *s, int64_t heads, int64_t rows, int d) {
    const int64_t row = packed_row_bytes(d);
    return s ? Strides{s[0], s[1], s[2]} : Strides{heads * rows * row, rows * row, row};
}
// Rows of 16-bit values (of `size` bytes each, where they are written), aligned to 16 bytes.
static bool value_strides_fit(const int64_t *s, int64_t rows, int d, int size = 2) {
    if (!s) return (rows + 64) * d * size < ((int64_t)1 << 31);
    const int whole = 16 / size;
    return s[0] % whole == 0 && s[1] % whole == 0 && s[2] % whole == 0 && s[0] >= 0 && s[1] >= 0 && s[2] >= d && s[2] < ((int64_t)1 << 30) &&
           ((rows + 64) * s[2] + d) * size < ((int64_t)1 << 31);
}
static Strides value_strides(const int64_t *s, int64_t heads, int64_t rows, int d) {
    return s ? Strides{s[0], s[1], s[2]} : Strides{heads * rows * d, rows * d, d};
}

// Whether two tensors of B x H x n rows of `row` bytes have bytes in common; each one's rows are `apart`, strides are in bytes.  Exact where they are laid out alike (keys and
// values side by side, heads of one tensor); where they are not, those that reach into one another are taken to have.
struct Laid {
    uintptr_t at;
    int64_t n[3], step[3], row;  // (no step where there is one)
    Laid(const void *p, const int64_t *s, int64_t B, int64_t H, int64_t rows, int64_t row_, int64_t size) : at((uintptr_t)p), n{B, H, rows}, row(row_) {
        const int64_t packed[3] = {H * rows * row, rows * row, row};
        for (int i = 0; i < 3; ++i) step[i] = n[i] > 1 ? (s ? s[i] * size : packed[i]) : 0;
    }
    __int128 end() const {
        __int128 e = (__int128)at + row;
        for (int i = 0; i < 3; ++i) e += (__int128)step[i] * (n[i] - 1);
        return e;
    }
    bool alike(const Laid &o) const { return step[0] == o.step[0] && step[1] == o.step[1] && step[2] == o.step[2]; }
    bool reaches(const Laid &o) const { return (__int128)at < o.end() && (__int128)o.at < end(); }
    bool meets(const Laid &o) const {
        if (!reaches(o) || !alike(o)) return reaches(o);
        int order[3] = {0, 1, 2};
        std::sort(order, order + 3, [&](int x, int y) { return step[x] > step[y]; });
        return meets((__int128)at - (__int128)o.at, order, 0);
    }

  private:
    // Whether a whole number of every step brings two rows that are `far` apart over one another.  What the closer dimensions span is less than a step, which leaves two numbers.
    bool meets(__int128 far, const int *order, int i) const {
        if (i == 3) return far < row && -far < row;
        const __int128 s = step[order[i]], most = n[order[i]] - 1;
        if (s == 0) return meets(far, order, i + 1);
        const __int128 down = far / s - (far % s < 0 ? 1 : 0);
        for (__int128 times = down; times <= down + 1; ++times)
            if (times <= most && -times <= most && meets(far - times * s, order, i + 1)) return true;
        return false;
    }
};

// What all entry points refuse.
static smha_status_t packed_sizes(int B, int Hkv, int T, int Sk, int d) {
    if (B < 1 || Hkv < 1 || T < 1 || Sk < 1) return SMHA_ERR_INVALID_ARG;
    if (d < 8 || d > 128 || d % 8 || T >= kRowsEnd || Sk >= kRowsEnd) return SMHA_ERR_UNSUPPORTED;
    // (rows are counted in 32 bits, and a launch has less than 2^32 threads)
    if ((int64_t)B * Hkv > (1 << 24) || (int64_t)B * Hkv * T > SMHA_PACKED_MOST_ROWS) return SMHA_ERR_UNSUPPORTED;
    return SMHA_OK;
}

}  // namespace smha

using namespace smha;

extern "C" smha_status_t smha_packed_row(int d, int *bytes) {
    if (!bytes) return SMHA_ERR_INVALID_ARG;
    if (d < 8 || d > 128 || d % 8) return SMHA_ERR_UNSUPPORTED;
    *bytes = packed_row_bytes(d);
    return SMHA_OK;
}

extern "C" smha_status_t smha_packed_write(const void *K_new, const void *V_new, void *K, void *V, void *K_values, void *V_values, const int32_t *lengths,
                                           const int32_t *offsets, int B, int Hkv, int T, int Sk, int d, smha_dtype_t dtype, const int64_t kn_strides[3],
                                           const int64_t vn_strides[3], const int64_t k_strides[3], const int64_t v_strides[3], void *hip_stream) {
    if (!K_new || !V_new || !K || !V || !lengths || K == V || !K_values != !V_values) return SMHA_ERR_INVALID_ARG;
    const smha_status_t st = packed_sizes(B, Hkv, T, Sk, d);
    if (st != SMHA_OK) return st;
    if (dtype != SMHA_F16 && dtype != SMHA_BF16) return SMHA_ERR_UNSUPPORTED;
    if (((uintptr_t)K_new | (uintptr_t)V_new | (uintptr_t)K_values | (uintptr_t)V_values) & 15 || ((uintptr_t)K | (uintptr_t)V) & 3) return SMHA_ERR_UNSUPPORTED;
    if (!value_strides_fit(kn_strides, T, d) || !value_strides_fit(vn_strides, T, d) || !packed_strides_fit(k_strides, Sk, d) || !packed_strides_fit(v_strides, Sk, d))
        return SMHA_ERR_UNSUPPORTED;
    if (!apart(k_strides, B, Hkv, Sk, packed_row_bytes(d)) || !apart(v_strides, B, Hkv, Sk, packed_row_bytes(d))) return SMHA_ERR_UNSUPPORTED;
    // What is written twice, or read by one lane and written by another, would be as the order of workgroups has it.
    const Laid caches[2] = {{K, k_strides, B, Hkv, Sk, packed_row_bytes(d), 1}, {V, v_strides, B, Hkv, Sk, packed_row_bytes(d), 1}};
    if (caches[0].meets(caches[1])) return SMHA_ERR_INVALID_ARG;
    if (K_values) {
        const Laid values[2] = {{K_values, nullptr, B, Hkv, T, 2 * d, 2}, {V_values, nullptr, B, Hkv, T, 2 * d, 2}};
        const Laid tokens[2] = {{K_new, kn_strides, B, Hkv, T, 2 * d, 2}, {V_new, vn_strides, B, Hkv, T, 2 * d, 2}};
        if (values[0].reaches(values[1])) return SMHA_ERR_INVALID_ARG;
        for (const Laid &to : values) {
            for (const Laid &cache : caches)
                if (to.reaches(cache)) return SMHA_ERR_INVALID_ARG;
            for (const Laid &from : tokens)  // (a lane has read both of its tokens' columns when it writes theirs)
                if (to.reaches(from) && !(to.at == from.at && to.alike(from))) return SMHA_ERR_INVALID_ARG;
        }
    }
    PackParams pp{};
    pp.x[0] = (const uint16_t *)K_new; pp.x[1] = (const uint16_t *)V_new;
    pp.cache[0] = (uint8_t *)K; pp.cache[1] = (uint8_t *)V;
    pp.values[0] = (uint16_t *)K_values; pp.values[1] = (uint16_t *)V_values;
    pp.xs[0] = value_strides(kn_strides, Hkv, T, d); pp.xs[1] = value_strides(vn_strides, Hkv, T, d);
    pp.cs[0] = packed_strides(k_strides, Hkv, Sk, d); pp.cs[1] = packed_strides(v_strides, Hkv, Sk, d);
    pp.lengths = lengths; pp.offsets = offsets;
    pp.B = B; pp.Hkv = Hkv; pp.T = T; pp.Sk = Sk; pp.d = d;
    const bool bf16 = dtype == SMHA_BF16;
    const int G = packed_groups(d);
    auto *const put = G == 1   ? (bf16 ? smha_packed_put<1, true> : smha_packed_put<1, false>)
                      : G == 2 ? (bf16 ? smha_packed_put<2, true> : smha_packed_put<2, false>)
                      : G == 3 ? (bf16 ? smha_packed_put<3, true> : smha_packed_put<3, false>)
                               : (bf16 ? smha_packed_put<4, true> : smha_packed_put<4, false>);
    const int64_t rows = (int64_t)B * Hkv * T, at_once = 64 / G;
    hipLaunchKernelGGL(put, dim3((unsigned)((rows + at_once - 1) / at_once)), dim3(256), 0, (hipStream_t)hip_stream, pp);
    return hipGetLastError() == hipSuccess ? SMHA_OK : SMHA_ERR_HIP;
}

extern "C" smha_status_t smha_packed_read(const void *K, const void *V, void *K_out, void *V_out, const int32_t *lengths, const int32_t *offsets, int B, int Hkv, int T, int Sk, int d,
                                          smha_dtype_t out_dtype, const int64_t k_strides[3], const int64_t v_strides[3], const int64_t ko_strides[3], const int64_t vo_strides[3],
                                          void *hip_stream) {
    if (!K || !V || !K_out || !V_out || !lengths || K_out == V_out) return SMHA_ERR_INVALID_ARG;
    const smha_status_t st = packed_sizes(B, Hkv, T, Sk, d);
    if (st != SMHA_OK) return st;
    if (out_dtype != SMHA_F16 && out_dtype != SMHA_BF16 && out_dtype != SMHA_F32) return SMHA_ERR_UNSUPPORTED;
    if (((uintptr_t)K_out | (uintptr_t)V_out) & 15 || ((uintptr_t)K | (uintptr_t)V) & 3) return SMHA_ERR_UNSUPPORTED;
    const int size = out_dtype == SMHA_F32 ? 4 : 2;
    if (!packed_strides_fit(k_strides, Sk, d) || !packed_strides_fit(v_strides, Sk, d) || !value_strides_fit(ko_strides, T, d, size) || !value_strides_fit(vo_strides, T, d, size))
        return SMHA_ERR_UNSUPPORTED;
    if (!apart(ko_strides, B, Hkv, T, d) || !apart(vo_strides, B, Hkv, T, d)) return SMHA_ERR_UNSUPPORTED;
    if (Laid(K_out, ko_strides, B, Hkv, T, (int64_t)d * size, size).meets(Laid(V_out, vo_strides, B, Hkv, T, (int64_t)d * size, size))) return SMHA_ERR_INVALID_ARG;
    UnpackParams up{};
    up.cache[0] = (const uint8_t *)K; up.cache[1] = (const uint8_t *)V;
    up.out[0] = K_out; up.out[1] = V_out;
    up.cs[0] = packed_strides(k_strides, Hkv, Sk, d); up.cs[1] = packed_strides(v_strides, Hkv, Sk, d);
    up.os[0] = value_strides(ko_strides, Hkv, T, d); up.os[1] = value_strides(vo_strides, Hkv, T, d);
    up.lengths = lengths; up.offsets = offsets;
    up.B = B; up.Hkv = Hkv; up.T = T; up.Sk = Sk; up.d = d;
    auto *const get = out_dtype == SMHA_F32 ? smha_packed_get<SMHA_F32> : out_dtype == SMHA_BF16 ? smha_packed_get<SMHA_BF16> : smha_packed_get<SMHA_F16>;
    const int64_t rows = (int64_t)B * Hkv * T, at_once = 256 / (d / 8);
    hipLaunchKernelGGL(get, dim3((unsigned)((rows + at_once - 1) / at_once)), dim3(256), 0, (hipStream_t)hip_stream, up);
    return hipGetLastError() == hipSuccess ? SMHA_OK : SMHA_ERR_HIP;
}

// How a call is taken, and its workspace.
struct PackedForm {
    int rows, row_tiles, slots, most_slots;  // rows of a tile: 16, 32, 64 or 128; slots: 0 where a group is a segment
    size_t stats, parts, total;  // after `info`
};
static size_t packed_up(size_t n) { return (n + 255) & ~(size_t)255; }

static smha_status_t packed_form(PackedForm &f, int B, int H, int Hkv, int T, int Sk, int d, int window, int n_sink) {
    if (H < 1 || window < 0 || n_sink < 0) return SMHA_ERR_INVALID_ARG;
    const smha_status_t st = packed_sizes(B, Hkv, T, Sk, d);
    if (st != SMHA_OK) return st;
    if (H % Hkv) return SMHA_ERR_SHAPE;
    if ((int64_t)B * H > (1 << 24) || (int64_t)B * H * T > (1 << 24)) return SMHA_ERR_UNSUPPORTED;
    const int D = d <= 64 ? 64 : 128, rows = H / Hkv * T;
    f.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
    const bool wide = f.rows >= 64;
    const int KT = wide ? 64 : 32;
    f.row_tiles = (rows + f.rows - 1) / f.rows;
    const int64_t groups = (int64_t)B * Hkv * f.row_tiles;
    // (tiles are counted in 32 bits, and a launch has less than 2^32 threads)
    if (groups * (Sk / KT + 8) > (1 << 30) || groups + 4096 >= 1 << 24) return SMHA_ERR_UNSUPPORTED;
    const int64_t see = window == 0 || window > Sk ? Sk : window;
    const int64_t tiles = std::min<int64_t>((Sk + KT - 1) / KT, (see + std::min(n_sink, Sk) + T) / KT + 3);
    const int slots = 256 * (wide ? (D == 64 ? 3 : 2) : packed_workgroups(D, f.rows / 16));
    // Groups are taken whole, in one launch, where they have few tiles: cutting costs a second launch and the search for a segment, and shares out what one workgroup
    // would read alone (us, whole and cut: 64 groups x 128 of 512 keys 9.3 and 9.8, of 1024 13.8 and 11.4; 256 groups of 1024 14.6 and 18.3); where there are too many to count;
    // and where one sequence has 256 or more, a workgroup for every compute unit, so that lengths hardly matter (2 x 1024 tokens x 32 on 8 x 16384 x 128 548 and 555, x 64 339
    // and 387; 1 x 2048 536 and 544, 331 and 377).  With fewer of them a long sequence among short ones would be read by part of the chip (2 x 512 x 32 on 8 x 8192 x 64, of 10
    // to 100 % of that: 100 and 63; 4 x 512 105 and 97, of full length 172 and 207; 512 x 1 x 32 on 8 x 2048 x 128, of 10 to 100 %, 156 and 168).  The bound does not see that
    // one sequence of 256 groups leaves half of the slots empty at 128 columns and two thirds at 64: 1 x 1024 tokens x 32 on 8 x 16384 x 128 takes 388 us, 294 if it were cut, x 64 280 and 177.
    const bool direct = (int64_t)B * f.row_tiles > kPackedEntries || tiles <= (wide ? 8 : std::min<int64_t>(48, (D == 64 ? 24 : 16) + groups / 8)) ||
                        (int64_t)Hkv * f.row_tiles >= 256;
    f.slots = direct ? 0 : groups < slots ? slots : slots / 2;
    f.most_slots = !direct && !wide && groups < slots ? 2 * slots : f.slots;
    f.stats = f.parts = f.total = 0;
    if (direct) return SMHA_OK;
    // cut groups are longer than a segment, so that there are fewer of them than slots, and their segments no more than that and one each
    const int64_t places = std::min(std::min<int64_t>(2 * f.most_slots, f.most_slots + groups), groups * ((tiles + 3) / 4));
    f.stats = packed_up(groups * sizeof(int2));
    f.parts = f.stats + packed_up((size_t)places * 2 * f.rows * 4);
    f.total = f.parts + (size_t)places * f.rows * D * 4;
    return SMHA_OK;
}

extern "C" smha_status_t smha_packed_workspace(int B, int H, int Hkv, int T, int Sk, int d, int window, int n_sink, size_t *need) {
    if (!need) return SMHA_ERR_INVALID_ARG;
    PackedForm f{};
    const smha_status_t st = packed_form(f, B, H, Hkv, T, Sk, d, window, n_sink);
    if (st == SMHA_OK) *need = f.total;
    return st;
}

template <int D, bool BF16> static hipError_t launch_packed(const PackedParams &pp, const PackedForm &f, hipStream_t stream) {
    const int groups = pp.B * pp.Hkv * pp.row_tiles, segments = groups + pp.most_slots;
    const dim3 grid(8 * ((segments + 7) / 8));
    auto *const part = f.rows == 16 ? smha_packed_part<D, 1, BF16> : f.rows == 32 ? smha_packed_part<D, 2, BF16> : f.rows == 64 ? smha_packed_wide<D, 2, BF16> : smha_packed_wide<D, 1, BF16>;
    hipLaunchKernelGGL(part, grid, dim3(256), 0, stream, pp);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !pp.slots) return e;
    const int rows = pp.B * pp.H * pp.T;
    const bool alone = rows > 512;  // a wave a row (960 rows of 9 segments 16.2 us a call with four, 14.7 so; 64 of 47 segments 35.6 and 40.4)
    auto *const join = f.rows == 16   ? (alone ? smha_packed_join<D, 16, 1, BF16> : smha_packed_join<D, 16, 4, BF16>)
                       : f.rows == 32 ? (alone ? smha_packed_join<D, 32, 1, BF16> : smha_packed_join<D, 32, 4, BF16>)
                       : f.rows == 64 ? (alone ? smha_packed_join<D, 64, 1, BF16> : smha_packed_join<D, 64, 4, BF16>)
                                      : (alone ? smha_packed_join<D, 128, 1, BF16> : smha_packed_join<D, 128, 4, BF16>);
    hipLaunchKernelGGL(join, dim3(alone ? std::min(2048, (rows + 3) / 4) : rows), dim3(256), 0, stream, pp);
    return hipGetLastError();
}

extern "C" smha_status_t smha_packed_forward(const void *Q, const void *K, const void *V, void *O, const int32_t *lengths, int B, int H, int Hkv, int T, int Sk, int d,
                                             smha_dtype_t dtype, const int64_t q_strides[3], const int64_t k_strides[3], const int64_t v_strides[3], const int64_t o_strides[3],
                                             int window, int n_sink, float scale, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!Q || !K || !V || !O || !lengths) return SMHA_ERR_INVALID_ARG;
    PackedForm f{};
    const smha_status_t st = packed_form(f, B, H, Hkv, T, Sk, d, window, n_sink);
    if (st != SMHA_OK) return st;
    if (dtype != SMHA_F16 && dtype != SMHA_BF16) return SMHA_ERR_UNSUPPORTED;
    if (workspace_bytes < f.total || (f.total && !workspace)) return SMHA_ERR_INVALID_ARG;
    if (((uintptr_t)Q | (uintptr_t)O | (uintptr_t)workspace) & 15 || ((uintptr_t)K | (uintptr_t)V) & 3) return SMHA_ERR_UNSUPPORTED;
    if (!value_strides_fit(q_strides, T, d) || !value_strides_fit(o_strides, T, d) || !packed_strides_fit(k_strides, Sk, d) || !packed_strides_fit(v_strides, Sk, d))
        return SMHA_ERR_UNSUPPORTED;
    if (!apart(o_strides, B, H, T, d)) return SMHA_ERR_UNSUPPORTED;
    PackedParams pp{};
    pp.Q = (const uint16_t *)Q; pp.K = (const uint8_t *)K; pp.V = (const uint8_t *)V; pp.O = (uint16_t *)O;
    pp.qs = value_strides(q_strides, H, T, d); pp.os = value_strides(o_strides, H, T, d);
    pp.ks = packed_strides(k_strides, Hkv, Sk, d); pp.vs = packed_strides(v_strides, Hkv, Sk, d);
    pp.lengths = lengths;
    pp.B = B; pp.H = H; pp.Hkv = Hkv; pp.G = H / Hkv; pp.T = T; pp.Sk = Sk; pp.d = d;
    pp.window = window == 0 || window > Sk ? Sk : window;
    pp.n_sink = std::min(n_sink, Sk);
    pp.row_tiles = f.row_tiles;
    pp.slots = f.slots;
    pp.most_slots = f.most_slots;
    pp.c = (scale > 0.f ? scale : 1.0f / std::sqrt((float)d)) * 1.4426950408889634f;
    char *const ws = (char *)workspace;
    pp.info = (int2 *)ws; pp.stats = (float *)(ws + f.stats); pp.parts = (float *)(ws + f.parts);
    const hipStream_t stream = (hipStream_t)hip_stream;
    const bool bf16 = dtype == SMHA_BF16;
    const hipError_t e = d <= 64 ? (bf16 ? launch_packed<64, true>(pp, f, stream) : launch_packed<64, false>(pp, f, stream))
                                 : (bf16 ? launch_packed<128, true>(pp, f, stream) : launch_packed<128, false>(pp, f, stream));
    return e == hipSuccess ? SMHA_OK : SMHA_ERR_HIP;
}
