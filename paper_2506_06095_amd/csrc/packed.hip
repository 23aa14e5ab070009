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
// exceeds max x by less than 15 steps of s, 120 at most, so that every code stands for something finite.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "device_common.hpp"
#include "smha.h"

namespace smha {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr float kPackedMost = 65280.f;

static int packed_groups(int d) { return (d + 31) / 32; }
static int packed_row_bytes(int d) { return 4 * packed_groups(d) + d / 2; }

// What eight codes stand for, as pairs of neighbours; `head`: s in the lower half, m in the upper.  0x6400 + c are the bits of 1024 + c and 0x5400 + 16 c those
// of 64 + c, so that a pair is three instructions and a shared shift: and-or, the bias off (exact), fused multiply and add.
__device__ __forceinline__ u32x4 unpack8(uint32_t word, uint32_t head) {
    const f16x2 h = __builtin_bit_cast(f16x2, head), s = {h[0], h[0]}, m = {h[1], h[1]};
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? word : word >> 8;
        const f16x2 biased = __builtin_bit_cast(f16x2, i & 1 ? (w & 0x00F000F0u) | 0x54005400u : (w & 0x000F000Fu) | 0x64006400u);
        const _Float16 bias = i & 1 ? (_Float16)64.f : (_Float16)1024.f;
        v[i] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(biased - f16x2{bias, bias}, s, m));
    }
    return v;
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
    // Of the codes the one below or the right one by 32 bits, and then the border above it in 64, where it is exact: equal inputs and ties give
    // the same code everywhere.  (These are 4 of 25 instructions a value.)
    const double s64 = s, m64 = sb ? (double)m : (double)__builtin_inff();
    uint32_t word = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float k = truncf(fmaf(f[e] - m, inv, 0.5f - 0x1p-10f));
        const uint32_t c = (uint32_t)(int)k + (fma((double)(k + 0.5f), s64, m64) <= (double)f[e] ? 1 : 0);
        word |= c << (4 * (e / 2) + 16 * (e & 1));
    }
    if (bad != 0.f) {
        sb = 0;
        mb = 0x7E00u;
        word = 0;
    }
    head = sb | mb << 16;
    return word;
}

// A quad of lanes takes a group of a new token's key and of its value.  Memory bounds it: 2 d bytes in and R out for each.
template <int G, bool BF16>
__global__ void __launch_bounds__(256) smha_packed_put(const PackParams p) {
    const int64_t quad = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 2;
    const int at = threadIdx.x & 3, row = (int)(quad / G), g = (int)(quad - (int64_t)row * G), col = 32 * g + 8 * at;
    const int bh = row / p.T, t = row - bh * p.T, b = bh / p.Hkv, hk = bh - b * p.Hkv;
    if (b >= p.B) return;
    const int len = min(max(p.lengths[b], 0), p.Sk);
    const int64_t slot = (p.offsets ? (int64_t)p.offsets[b] : (int64_t)len - p.T) + t;
    const bool kept = slot >= 0 && slot < len, there = col < p.d;
    u32x4 x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[i] = u32x4{0, 0, 0, 0};
        if (kept && there) x[i] = *reinterpret_cast<const u32x4 *>(p.x[i] + b * p.xs[i].b + hk * p.xs[i].h + t * p.xs[i].s + col);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t head;
        const uint32_t word = pack8<BF16>(x[i], there, head);
        if (kept) {
            uint8_t *const to = p.cache[i] + b * p.cs[i].b + hk * p.cs[i].h + slot * p.cs[i].s;
            if (at == 0) *reinterpret_cast<uint32_t *>(to + 4 * g) = head;
            if (there) *reinterpret_cast<uint32_t *>(to + 4 * G + 16 * g + 4 * at) = word;
        }
        if (p.values[i] && there) {
            u32x4 v = unpack8(word, head);
            if (BF16)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = as_bf16(v[e]);
            if (!kept) v = u32x4{0, 0, 0, 0};
            *reinterpret_cast<u32x4 *>(p.values[i] + (int64_t)row * p.d + col) = v;
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

// A lane takes 8 columns of a slot's key and of its value.  Memory bounds it: R bytes in and d values out for each.
template <int OUT>
__global__ void __launch_bounds__(256) smha_packed_get(const UnpackParams p) {
    const int chunks = p.d >> 3, G = (p.d + 31) >> 5;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int row = (int)(id / chunks), chunk = (int)(id - (int64_t)row * chunks);
    const int bh = row / p.T, t = row - bh * p.T, b = bh / p.Hkv, hk = bh - b * p.Hkv;
    if (b >= p.B) return;
    const int len = min(max(p.lengths[b], 0), p.Sk);
    const int64_t slot = (p.offsets ? (int64_t)p.offsets[b] : 0) + t;
    const bool kept = slot >= 0 && slot < len;
    uint32_t head[2] = {0, 0}, word[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (kept) {
            const uint8_t *const from = p.cache[i] + b * p.cs[i].b + hk * p.cs[i].h + slot * p.cs[i].s;
            head[i] = *reinterpret_cast<const uint32_t *>(from + 4 * (chunk >> 2));
            word[i] = *reinterpret_cast<const uint32_t *>(from + 4 * G + 4 * chunk);
        }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        u32x4 v = unpack8(word[i], head[i]);
        const int64_t at = b * p.os[i].b + hk * p.os[i].h + t * p.os[i].s + 8 * chunk;
        if constexpr (OUT == SMHA_F32) {
            float *const to = (float *)p.out[i] + at;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<f32x4 *>(to + 4 * h) = f32x4{widen16<false>(v[2 * h] & 0xFFFFu), widen16<false>(v[2 * h] >> 16), widen16<false>(v[2 * h + 1] & 0xFFFFu),
                                                               widen16<false>(v[2 * h + 1] >> 16)};
        } else {
            if (OUT == SMHA_BF16)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = as_bf16(v[e]);
            *reinterpret_cast<u32x4 *>((uint16_t *)p.out[i] + at) = v;
        }
    }
}

// ---------------------------------------------------------------------------------------
// Attention
// ---------------------------------------------------------------------------------------
struct PackedParams {
    const uint16_t *Q;
    const uint8_t *K, *V;
    uint16_t *O;
    Strides qs, ks, vs, os;
    const int32_t *lengths;
    int B, H, Hkv, G, T, Sk, d;
    int window, n_sink;
    int row_tiles;  // of 16 rows, of a key head's G T
    float c;        // scale * log2(e)
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
    __device__ __forceinline__ int key(int tile) const { return KT * (tile < head ? tile : first + tile - head); }
};

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// A row of queries as the B operand of the scores' product, in binary16: lane (row, u) holds columns (D / 4) u + 8 i ...  bfloat16 rows are brought to
// 2^14 .. 2^15 by a power of two, by which they fit binary16 without loss (but for columns below 2^-31 of the largest, which lose digits); returns what the scores have to be multiplied by.
template <int D, bool BF16> __device__ __forceinline__ float load_query(u32x4 (&qf)[D / 32], const uint16_t *row, bool exists, int d, int u) {
    u32x4 raw[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
        const int col = D / 4 * u + 8 * i;
        raw[i] = u32x4{0, 0, 0, 0};
        if (exists && col < d) raw[i] = *reinterpret_cast<const u32x4 *>(row + col);
    }
    if constexpr (!BF16) {
#pragma unroll
        for (int i = 0; i < D / 32; ++i) qf[i] = raw[i];
        return 1.f;
    } else {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, fmaxf(fabsf(widen16<true>(raw[i][e] & 0xFFFFu)), fabsf(widen16<true>(raw[i][e] >> 16))));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const int e2 = min(15 - __builtin_amdgcn_frexp_expf(top), 100);
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                qf[i][e] = pack2<false>(__builtin_amdgcn_ldexpf(widen16<true>(raw[i][e] & 0xFFFFu), e2), __builtin_amdgcn_ldexpf(widen16<true>(raw[i][e] >> 16), e2));
        return __builtin_amdgcn_ldexpf(1.f, -e2);
    }
}

// Swizzle of a 32-row tile of values: writes of 16 rows at one chunk of 16 bytes, and transposing reads of 8 rows x 2 chunks (half a wave), all over the banks.
template <int D> __device__ __forceinline__ int swz_values(int row) {
    if constexpr (D == 128) return ((row & 7) << 1) | ((row >> 3) & 1);
    else return (((row >> 1) & 3) << 1) | ((row >> 3) & 1);
}

// Four waves take the tiles of 32 keys of a group, 16 rows that read the same keys, in turn, and join in LDS.  A lane unpacks D / 4 columns of two keys: keys are an operand
// as they come out; values go through LDS once, for the transposing reads that make them the other product's.
template <int D, bool BF16>
__global__ void __launch_bounds__(256, 2) smha_packed_part(const PackedParams p) {
    constexpr int NS = D / 32, NW = D / 32, NC = D / 16, TB = 32 * D * 2;  // steps of the first product; words of codes a lane has of a key; tiles of columns; bytes of a tile
    __shared__ __attribute__((aligned(1024))) char all_tiles[4 * TB];
    __shared__ float team[4][2][16];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 15, u = lane >> 4;
    char *const smem = all_tiles + w * TB;
    const float NEG_INF = -__builtin_inff();

    const int group = blockIdx.x, bh = group / p.row_tiles, b = bh / p.Hkv, hk = bh - b * p.Hkv, rows0 = 16 * (group - bh * p.row_tiles);
    const int rows = p.G * p.T;
    const PackedKeys<32> keys(uniform_load(p.lengths + b), p.T, p.Sk, p.window, p.n_sink, rows0 / p.G, (min(rows0 + 16, rows) - 1) / p.G);
    const int row = rows0 + j, t = row / p.G, g = row - t * p.G, pos = row < rows ? keys.len - p.T + t : -1;  // below 0: no such query
    u32x4 qf[NS];
    const float c = fmaxf(p.c * load_query<D, BF16>(qf, p.Q + b * p.qs.b + (hk * p.G + g) * p.qs.h + t * p.qs.s, pos >= 0, p.d, u), 0x1p-126f);  // (never 0: -inf times it)

    // keys from `end` on are past the buffers and read as zeros
    const int groups = (p.d + 31) >> 5, row_bytes = 4 * groups + (p.d >> 1);
    const __amdgpu_buffer_rsrc_t rK = make_rsrc(p.K + b * p.ks.b + hk * p.ks.h, keys.end > 0 ? (int64_t)(keys.end - 1) * p.ks.s + row_bytes : 0);
    const __amdgpu_buffer_rsrc_t rV = make_rsrc(p.V + b * p.vs.b + hk * p.vs.h, keys.end > 0 ? (int64_t)(keys.end - 1) * p.vs.s + row_bytes : 0);
    const int my_group = D == 128 ? u : u >> 1, codes_at = 4 * groups + D / 8 * u;
    struct Raw {
        uint32_t head[2], code[2][NW];
    };
    auto load = [&](__amdgpu_buffer_rsrc_t r, int pitch, int key) __attribute__((always_inline)) {
        Raw x;
#pragma unroll
        for (int a = 0; a < 2; ++a) {
            const int k = key + 16 * a + j, at = k * pitch;
            // keys between the sinks and the window read as zeros, and so do the columns that the head does not have
            const bool read = (k < keys.gap0 || k >= keys.gap1) && my_group < groups;
            x.head[a] = __builtin_amdgcn_raw_buffer_load_b32(r, read ? at + 4 * my_group : (int)kPast, 0, 0);
            if constexpr (NW == 4) {
                const u32x4 v = __builtin_amdgcn_raw_buffer_load_b128(r, at + codes_at, 0, 0);
#pragma unroll
                for (int i = 0; i < 4; ++i) x.code[a][i] = v[i];
            } else {
                const u32x2 v = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, at + codes_at, 0, 0));
                x.code[a][0] = v[0];
                x.code[a][1] = v[1];
            }
        }
        return x;
    };

    float m_run = NEG_INF, l_run = 0.f;
    const float thr = raised_over(c);
    f32x4 o[NC];
#pragma unroll
    for (int ct = 0; ct < NC; ++ct) o[ct] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int tr_row = 4 * u + (j >> 2);
    Raw k_raw, v_raw;
    if (w < keys.n) {
        k_raw = load(rK, (int)p.ks.s, keys.key(w));
        v_raw = load(rV, (int)p.vs.s, keys.key(w));
    }
    for (int tile = w; tile < keys.n; tile += 4) {
        const int key = keys.key(tile);
        const Raw k_now = k_raw, v_now = v_raw;
        if (tile + 4 < keys.n) {
            k_raw = load(rK, (int)p.ks.s, keys.key(tile + 4));
            v_raw = load(rV, (int)p.vs.s, keys.key(tile + 4));
        }
        // acc[a][r]: the score of query j and key 16 a + 4 u + r
        f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int a = 0; a < 2; ++a) acc[a] = mfma16(unpack8(k_now.code[a][i], k_now.head[a]), qf[i], acc[a]);
        // values go to LDS under that product
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int i = 0; i < NW; ++i)
                *reinterpret_cast<u32x4 *>(smem + (16 * a + j) * D * 2 + (((D / 32 * u + i) ^ swz_values<D>(j)) * 16)) = unpack8(v_now.code[a][i], v_now.head[a]);
        const uint32_t word = pos >= 0 ? low_bits32(pos - key + 1) & (~low_bits32(pos - p.window + 1 - key) | low_bits32(p.n_sink - key)) : 0;
        if (__builtin_amdgcn_ballot_w64(word != ~0u) != 0) {
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[a][r] = (word >> (16 * a + 4 * u + r)) & 1 ? acc[a][r] : NEG_INF;
        }
        float mt = NEG_INF;
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int r = 0; r < 4; ++r) mt = fmaxf(mt, acc[a][r]);
        if (__builtin_amdgcn_ballot_w64(mt > m_run + thr) != 0) {
            mt = fmaxf(mt, __shfl_xor(mt, 16));
            mt = fmaxf(mt, __shfl_xor(mt, 32));
            const float m_new = fmaxf(m_run, mt), alpha = fast_exp2((m_run - (m_new == NEG_INF ? 0.f : m_new)) * c);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int ct = 0; ct < NC; ++ct) o[ct] *= alpha;
        }
        const float mc = (m_run == NEG_INF ? 0.f : m_run) * c;
        // Probabilities, relative to about the largest, are rounded to binary16 for the second product, whatever the inputs' type.
        u32x4 pf;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float e0 = fast_exp2(fmaf(acc[q >> 1][2 * (q & 1)], c, -mc)), e1 = fast_exp2(fmaf(acc[q >> 1][2 * (q & 1) + 1], c, -mc));
            pf[q] = pack2<false>(e0, e1);
            l_run += e0 + e1;
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int ct = 0; ct < NC; ++ct) {
            const int chunk = 2 * ct + ((j & 3) >> 1), at = tr_row * D * 2 + ((chunk ^ swz_values<D>(tr_row)) * 16) + (j & 1) * 8;
            const u32x2 lo = lds_read_tr(reinterpret_cast<const uint16_t *>(smem + at)), hi = lds_read_tr(reinterpret_cast<const uint16_t *>(smem + at + 16 * D * 2));
            o[ct] = mfma16(u32x4{lo[0], lo[1], hi[0], hi[1]}, pf, o[ct]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the tile is read
    }

    // The team joins: every wave leaves its accumulators in its own tile's place and takes a quarter of the columns of all four.
    constexpr int NQ = NC / 4;
    float l = l_run + __shfl_xor(l_run, 16);
    l += __shfl_xor(l, 32);
#pragma unroll
    for (int ct = 0; ct < NC; ++ct) *reinterpret_cast<f32x4 *>(smem + (ct * 64 + lane) * 16) = o[ct];
    if (u == 0) {
        team[w][0][j] = m_run * c;
        team[w][1][j] = l;
    }
    __syncthreads();
    float mu[4], m_all = NEG_INF, l_all = 0.f;
    f32x4 out[NQ];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        mu[x] = team[x][0][j];
        m_all = fmaxf(m_all, mu[x]);
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i) out[i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const float share = mu[x] != NEG_INF ? fast_exp2(mu[x] - m_all) : 0.f;
        l_all = fmaf(share, team[x][1][j], l_all);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const f32x4 v = *reinterpret_cast<const f32x4 *>(all_tiles + x * TB + ((w * NQ + i) * 64 + lane) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) out[i][e] = fmaf(share, v[e], out[i][e]);
        }
    }
    if (row < rows) {
        const float inv = l_all != 0.f ? 1.0f / l_all : 0.f;
        uint16_t *const to = p.O + b * p.os.b + (hk * p.G + g) * p.os.h + t * p.os.s;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const int col = 16 * (w * NQ + i) + 4 * u;
            if (col < p.d) store4<BF16 ? SMHA_BF16 : SMHA_F16>(to, col, out[i][0] * inv, out[i][1] * inv, out[i][2] * inv, out[i][3] * inv);
        }
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

// What all entry points refuse.
static smha_status_t packed_sizes(int B, int Hkv, int T, int Sk, int d) {
    if (B < 1 || Hkv < 1 || T < 1 || Sk < 1) return SMHA_ERR_INVALID_ARG;
    if (d < 8 || d > 128 || d % 8 || T >= kRowsEnd || Sk >= kRowsEnd) return SMHA_ERR_UNSUPPORTED;
    // (rows are counted in 32 bits, and a launch has less than 2^32 threads)
    if ((int64_t)B * Hkv > (1 << 24) || (int64_t)B * Hkv * T > (1 << 27)) return SMHA_ERR_UNSUPPORTED;
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
    const int64_t quads = (int64_t)B * Hkv * T * G;
    hipLaunchKernelGGL(put, dim3((unsigned)((quads + 63) / 64)), dim3(256), 0, (hipStream_t)hip_stream, pp);
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
    UnpackParams up{};
    up.cache[0] = (const uint8_t *)K; up.cache[1] = (const uint8_t *)V;
    up.out[0] = K_out; up.out[1] = V_out;
    up.cs[0] = packed_strides(k_strides, Hkv, Sk, d); up.cs[1] = packed_strides(v_strides, Hkv, Sk, d);
    up.os[0] = value_strides(ko_strides, Hkv, T, d); up.os[1] = value_strides(vo_strides, Hkv, T, d);
    up.lengths = lengths; up.offsets = offsets;
    up.B = B; up.Hkv = Hkv; up.T = T; up.Sk = Sk; up.d = d;
    auto *const get = out_dtype == SMHA_F32 ? smha_packed_get<SMHA_F32> : out_dtype == SMHA_BF16 ? smha_packed_get<SMHA_BF16> : smha_packed_get<SMHA_F16>;
    const int64_t lanes = (int64_t)B * Hkv * T * (d / 8);
    hipLaunchKernelGGL(get, dim3((unsigned)((lanes + 255) / 256)), dim3(256), 0, (hipStream_t)hip_stream, up);
    return hipGetLastError() == hipSuccess ? SMHA_OK : SMHA_ERR_HIP;
}

static smha_status_t packed_attention_sizes(int B, int H, int Hkv, int T, int Sk, int d, int window, int n_sink) {
    if (H < 1 || window < 0 || n_sink < 0) return SMHA_ERR_INVALID_ARG;
    const smha_status_t st = packed_sizes(B, Hkv, T, Sk, d);
    if (st != SMHA_OK) return st;
    if (H % Hkv) return SMHA_ERR_SHAPE;
    if ((int64_t)B * H > (1 << 24) || (int64_t)B * H * T > (1 << 24)) return SMHA_ERR_UNSUPPORTED;
    return SMHA_OK;
}

extern "C" smha_status_t smha_packed_workspace(int B, int H, int Hkv, int T, int Sk, int d, int window, int n_sink, size_t *need) {
    if (!need) return SMHA_ERR_INVALID_ARG;
    const smha_status_t st = packed_attention_sizes(B, H, Hkv, T, Sk, d, window, n_sink);
    if (st != SMHA_OK) return st;
    *need = 0;
    return SMHA_OK;
}

extern "C" smha_status_t smha_packed_forward(const void *Q, const void *K, const void *V, void *O, const int32_t *lengths, int B, int H, int Hkv, int T, int Sk, int d,
                                             smha_dtype_t dtype, const int64_t q_strides[3], const int64_t k_strides[3], const int64_t v_strides[3], const int64_t o_strides[3],
                                             int window, int n_sink, float scale, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!Q || !K || !V || !O || !lengths) return SMHA_ERR_INVALID_ARG;
    const smha_status_t st = packed_attention_sizes(B, H, Hkv, T, Sk, d, window, n_sink);
    if (st != SMHA_OK) return st;
    if (dtype != SMHA_F16 && dtype != SMHA_BF16) return SMHA_ERR_UNSUPPORTED;
    if (((uintptr_t)Q | (uintptr_t)O | (uintptr_t)workspace) & 15 || ((uintptr_t)K | (uintptr_t)V) & 3) return SMHA_ERR_UNSUPPORTED;
    if (!value_strides_fit(q_strides, T, d) || !value_strides_fit(o_strides, T, d) || !packed_strides_fit(k_strides, Sk, d) || !packed_strides_fit(v_strides, Sk, d))
        return SMHA_ERR_UNSUPPORTED;
    if (!apart(o_strides, B, H, T, d)) return SMHA_ERR_UNSUPPORTED;
    (void)workspace_bytes;
    PackedParams pp{};
    pp.Q = (const uint16_t *)Q; pp.K = (const uint8_t *)K; pp.V = (const uint8_t *)V; pp.O = (uint16_t *)O;
    pp.qs = value_strides(q_strides, H, T, d); pp.os = value_strides(o_strides, H, T, d);
    pp.ks = packed_strides(k_strides, Hkv, Sk, d); pp.vs = packed_strides(v_strides, Hkv, Sk, d);
    pp.lengths = lengths;
    pp.B = B; pp.H = H; pp.Hkv = Hkv; pp.G = H / Hkv; pp.T = T; pp.Sk = Sk; pp.d = d;
    pp.window = window == 0 || window > Sk ? Sk : window;
    pp.n_sink = std::min(n_sink, Sk);
    pp.row_tiles = (pp.G * T + 15) / 16;
    pp.c = (scale > 0.f ? scale : 1.0f / std::sqrt((float)d)) * 1.4426950408889634f;
    const bool bf16 = dtype == SMHA_BF16;
    auto *const part = d <= 64 ? (bf16 ? smha_packed_part<64, true> : smha_packed_part<64, false>) : (bf16 ? smha_packed_part<128, true> : smha_packed_part<128, false>);
    hipLaunchKernelGGL(part, dim3((unsigned)(B * Hkv * pp.row_tiles)), dim3(256), 0, (hipStream_t)hip_stream, pp);
    return hipGetLastError() == hipSuccess ? SMHA_OK : SMHA_ERR_HIP;
}
