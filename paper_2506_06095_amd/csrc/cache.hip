// Attention of a few new tokens on a cache, with a window and sinks, with a prefix that all sequences share, with an account of what
// attention each key received; and the eviction of keys by that account.
//
// Attention.  Query t of sequence b stands at position len_b - T + t of the sequence's own keys.  The rows that read the same keys, G = H / Hkv
// query heads times T tokens of one sequence (own keys) or of all sequences (prefix keys), are taken 32 at a time; the keys are
// read in tiles of 32 by waves that share nothing while they read.  What bounds such a call is memory (a key's 4 d bytes meet
// 4 d G T operations), so what matters is that every compute unit reads, and all of them about as much: the tiles of all
// sequences are counted on the device and cut into as many segments, of about the same length, as workgroups fit the chip
// (segments()); lengths are never needed on the host.  A workgroup's four waves take a segment's tiles in turn and join in LDS; segments
// of the same rows are joined by a second kernel, in a fixed order, which also adds up the keys' accounts from the scores
// that the first left in memory: 8 G T bytes a key, written and read, where reading the key once more would take 2 d (less for up to d / 4 rows on a key
// head, more beyond).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "device_common.hpp"
#include "smha.h"

namespace smha {

struct CacheParams {
    const uint16_t *Q, *K, *V, *PK, *PV;
    uint16_t *O;
    float *weights;
    Strides qs, ks, vs, os;
    int64_t pk_h, pk_s, pv_h, pv_s, w_b, w_h;
    const int32_t *lengths;
    int B, H, Hkv, G, T, Sk, P, d;
    int window, n_sink;
    float c;
    int slots;       // segments wanted
    int own_tiles, prefix_tiles;  // 32-row tiles of G T rows; tiles of B G T rows (0 without a prefix), of
    int wide;                     // 128 rows and 64 keys (prefix_wide), else of 32 and 32
    int direct;                   // a workgroup a group (see CacheForm)
    int prefix_segs, segs;        // segments there is room for: of the prefix, in all
    int score_pitch; // keys per row of `scores`
    // A segment's results are places of 32 rows: one, or four of a wide one.  The prefix's segments come first.
    int2 *info;      // [prefix groups, own groups]: first place, segments
    float *stats;    // [place][2][32]: reference (log2 units), sum
    float *parts;    // [place][32][D]
    float *scores;   // [B][Hkv][G T][score_pitch], log2 units
};

// What one sequence's own keys are to its queries: the tiles of the sinks, then those of the window.
struct OwnKeys {
    int len, head, t0, n, gap0, gap1;
    __device__ __forceinline__ int key(int t) const { return 32 * (t < head ? t : t0 + t - head); }
};
__device__ __forceinline__ OwnKeys own_keys(int length, int T, int Sk, int window, int n_sink) {
    OwnKeys k;
    k.len = min(max(length, 0), Sk);
    const int from = max(0, max(k.len - T, 0) - window + 1);  // the first key in the first query's window
    k.head = (min(n_sink, from) + 31) / 32;
    k.t0 = max(from / 32, k.head);
    k.n = k.len > 0 ? k.head + (k.len - 1) / 32 + 1 - k.t0 : 0;
    k.gap0 = n_sink < from ? n_sink : 0;
    k.gap1 = n_sink < from ? from : 0;
    return k;
}

struct Segment {
    int place;           // of its results; -1: no segment
    int b, hk, rows0;    // rows0: first of its rows; b = -1: prefix
    int part, parts, n;  // of the group's n tiles
    int group, length;   // length: lengths[b]
};

// The reference that a row's segment leaves: -inf says that it has no keys.  (A row of NaN has no largest score either, and must not be passed over.)
__device__ __forceinline__ float reference_of(float m, float l) { return l == l ? m : 0.f; }

__device__ __forceinline__ int wave_sum(int v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    return v;
}

// The segment of a workgroup.  Every wave of the launch computes the same cut: c tiles a segment at most, so many (in fours, a team's turn) that
// all tiles make `slots` segments.  Groups shorter than that are a segment each, and then there are more: what does not fit at first
// starts as others end.  (A wide tile counts like one of the others, though it lasts longer: each of a wide segment's 128 rows leaves a result to
// join, and more and shorter segments cost more than they even out.  64 x 32 on 8 heads, 8192 shared keys and 280 of their own, counted
// as 1, 2, 3, 4: 38.1, 42.3, 44.4, 46.7 us.)
__device__ __forceinline__ Segment segment_of(const CacheParams &p, int lane) {
    const int prefix_groups = p.Hkv * p.prefix_tiles, per_b = p.Hkv * p.own_tiles;
    const int prefix_n = !p.prefix_tiles ? 0 : p.wide ? (p.P + 63) / 64 : (p.P + 31) / 32;
    auto tiles_at = [&](int length) __attribute__((always_inline)) { return own_keys(length, p.T, p.Sk, p.window, p.n_sink).n; };
    auto tiles = [&](int b) __attribute__((always_inline)) { return b < p.B ? tiles_at(p.lengths[b]) : 0; };
    const int length64 = lane < p.B ? p.lengths[lane] : 0, first64 = lane < p.B ? tiles_at(length64) : 0;
    int sum = first64;
    for (int b = 64 + lane; b - lane < p.B; b += 64) sum += tiles(b);
    const int total = prefix_groups * prefix_n + per_b * wave_sum(sum);
    const int c = __builtin_amdgcn_readfirstlane(max(4, ((total + p.slots - 1) / p.slots + 3) & ~3));
    sum = (first64 + c - 1) / c;
    for (int b = 64 + lane; b - lane < p.B; b += 64) sum += (tiles(b) + c - 1) / c;
    const int own_segs = __builtin_amdgcn_readfirstlane(per_b * wave_sum(sum)), prefix_parts = (prefix_n + c - 1) / c, prefix_segs = prefix_groups * prefix_parts;
    // an XCD takes a run of the prefix's segments, which are the longest, and then one of the others: those that read the same keys are neighbours
    const int xcd = (int)blockIdx.x & 7, slot = (int)blockIdx.x >> 3, prefix_run = (prefix_segs + 7) / 8, own_run = (own_segs + 7) / 8;
    Segment s{-1, -1, 0, 0, 0, 1, 0, 0, 0};
    if (slot < prefix_run) {
        const int at = xcd * prefix_run + slot;
        if (at >= prefix_segs) return s;
        s.place = p.wide ? 4 * at : at;
        s.parts = prefix_parts;
        s.group = at / s.parts;
        s.part = at - s.group * s.parts;
        s.hk = s.group / p.prefix_tiles;
        s.rows0 = (p.wide ? 128 : 32) * (s.group - s.hk * p.prefix_tiles);
        s.n = prefix_n;
        return s;
    }
    int at = xcd * own_run + slot - prefix_run;
    if (slot - prefix_run >= own_run || at >= own_segs) return s;
    s.place = (p.wide ? 4 : 1) * p.prefix_segs + at;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int length = b0 == 0 ? length64 : b0 + lane < p.B ? p.lengths[b0 + lane] : 0;
        const int n = b0 == 0 ? first64 : b0 + lane < p.B ? tiles_at(length) : 0, mine = per_b * ((n + c - 1) / c);
        int upto = mine;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int below = __shfl_up(upto, m);
            if (lane >= m) upto += below;
        }
        const uint64_t past = __builtin_amdgcn_ballot_w64(upto > at);
        if (past) {
            const int who = __builtin_ctzll(past);
            const int rest = at - (__builtin_amdgcn_readlane(upto, who) - __builtin_amdgcn_readlane(mine, who));
            s.n = __builtin_amdgcn_readlane(n, who);
            s.length = __builtin_amdgcn_readlane(length, who);
            s.parts = (s.n + c - 1) / c;
            s.b = b0 + who;
            const int in_b = rest / s.parts;
            s.part = rest - in_b * s.parts;
            s.hk = in_b / p.own_tiles;
            s.rows0 = 32 * (in_b - s.hk * p.own_tiles);
            s.group = prefix_groups + s.b * per_b + in_b;
            return s;
        }
        at -= __builtin_amdgcn_readlane(upto, 63);
    }
    s.place = -1;  // (not reached: the segments counted are those found)
    return s;
}

// A segment of a prefix that many rows read: four waves of 32 rows share 64-key tiles, two of each in LDS, as in smha_sink_fwd, but every key is
// visible.  (By the waves on their own, 32 rows and 32 keys at a time, K and V come from L2 four times as often, and its path into LDS sets the
// pace: 64 x 32 on 8 heads, 8192 shared keys and 280 of their own 42 us.)
template <int D, bool BF16>
__device__ __forceinline__ void prefix_wide(const CacheParams &p, const Segment &s, char *smem, const u32x4 (&qf)[D / 16], int lane, int w) {
    constexpr int NS = D / 16, NDT = D / 32, TB = 64 * D * 2, PF = D == 128 ? 8 : 4;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)smem;
    const int j = lane & 31, hh = lane >> 5;
    const float NEG_INF = -__builtin_inff();
    const int ksb = (int)p.pk_s * 2, vsb = (int)p.pv_s * 2;
    const u32x4 rK = make_rsrc4(p.PK + s.hk * p.pk_h, ((int64_t)(p.P - 1) * p.pk_s + p.d) * 2), rV = make_rsrc4(p.PV + s.hk * p.pv_h, ((int64_t)(p.P - 1) * p.pv_s + p.d) * 2);
    const TileLoad<D> loadK(w, lane, ksb, p.d), loadV(w, lane, vsb, p.d);
    const int begin = (int)((int64_t)s.n * s.part / s.parts), end = (int)((int64_t)s.n * (s.part + 1) / s.parts);
    loadK(rK, lds0, w, 64 * begin, ksb, 0, 0);
    loadV(rV, lds0 + 2 * TB, w, 64 * begin, vsb, 0, 0);
    const int rd = j * D * 2 + ((hh ^ swz_both<D>(j)) * 16);
    const int tr_row = 4 * hh + ((lane & 15) >> 2);
    const int tr = tr_row * D * 2 + ((swz_both<D>(tr_row) ^ (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1))) * 16) + (lane & 1) * 8;
    float m_run = NEG_INF, l_run = 0.f;
    const float thr = raised_over(p.c);
    f32x16 o[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) o[dt] = zeros16();
    tiles_landed();
    for (int t = begin; t < end; ++t) {
        const int par = (t - begin) & 1;
        if (t + 1 < end) {
            loadK(rK, lds0 + (par ^ 1) * TB, w, 64 * (t + 1), ksb, 0, 0);
            loadV(rV, lds0 + (2 + (par ^ 1)) * TB, w, 64 * (t + 1), vsb, 0, 0);
        }
        const char *const Kt = smem + par * TB, *const Vt = smem + (2 + par) * TB;
        f32x16 acc[2] = {zeros16(), zeros16()};
        auto k_frag = [&](int i) __attribute__((always_inline)) { return *reinterpret_cast<const u32x4 *>(Kt + ((rd ^ (32 * (i >> 1))) + 64 * (i & 1) * D)); };
        u32x4 kf[PF];
#pragma unroll
        for (int i = 0; i < PF; ++i) kf[i] = k_frag(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2 * NS; ++i) {
            acc[i & 1] = mfma32<BF16>(kf[i % PF], qf[i >> 1], acc[i & 1]);
            if (i + PF < 2 * NS) kf[i % PF] = k_frag(i + PF);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(1);
        if (64 * t + 64 > p.P) {
            const uint64_t word = low_bits(p.P - 64 * t);
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const u32x16 keep = keep_of((uint32_t)(word >> (32 * kt)) >> (4 * hh)), sc = __builtin_bit_cast(u32x16, acc[kt]);
                acc[kt] = __builtin_bit_cast(f32x16, (sc & keep) | (~keep & 0xFF800000u));
            }
        }
        float mt = NEG_INF;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int r = 0; r < 16; ++r) mt = fmaxf(mt, acc[kt][r]);
        if (__builtin_amdgcn_ballot_w64(mt > m_run + thr) != 0) {
            mt = fmaxf(mt, __shfl_xor(mt, 32));
            const float m_new = fmaxf(m_run, mt), alpha = fast_exp2((m_run - (m_new == NEG_INF ? 0.f : m_new)) * p.c);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) o[dt] *= alpha;
        }
        const float mc = (m_run == NEG_INF ? 0.f : m_run) * p.c;
        u32x4 pf[4];
        auto p_pair = [&](int cu, int q) __attribute__((always_inline)) {
            const float e0 = fast_exp2(fmaf(acc[cu >> 1][8 * (cu & 1) + 2 * q], p.c, -mc)), e1 = fast_exp2(fmaf(acc[cu >> 1][8 * (cu & 1) + 2 * q + 1], p.c, -mc));
            pf[cu][q] = pack2<BF16>(e0, e1);
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
        for (int i = 0; i < 4 * NDT; ++i) {
            const int cu = i / NDT, dt = i % NDT;
            o[dt] = mfma32<BF16>(vf[i % PF], pf[cu], o[dt]);
            if (i + PF < 4 * NDT) vf[i % PF] = v_frag(i + PF);
            if (cu < 3) {
#pragma unroll
                for (int q = (4 * dt + NDT - 1) / NDT; q < (4 * dt + NDT + 3) / NDT; ++q) p_pair(cu + 1, q);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        tiles_landed();
    }
    const float l = l_run + __shfl_xor(l_run, 32);
    if (s.part == 0 && threadIdx.x == 0) p.info[s.group] = int2{s.place, s.parts};
    if (s.rows0 + 32 * w + j < p.B * p.G * p.T) {
        const int64_t place = s.place + w;
        if (hh == 0) {
            p.stats[place * 64 + j] = reference_of(m_run * p.c, l);
            p.stats[place * 64 + 32 + j] = l;
        }
        float *const part = p.parts + (place * 32 + j) * D + 4 * hh;
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
            *reinterpret_cast<f32x4 *>(part + 8 * i) = f32x4{o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]};
    }
}

// K, V: one buffer of 32 keys each a wave, refilled as soon as its fragments are read: K of the next tile lands under this tile's softmax
// and second product, V of the next under the next tile's scores.  Eight waves a compute unit at 128 columns, 16 at 64.
// 32 x 32 on 8 x 16384 x 128, window 2048: 52 us, 5.1 TB/s; 8 x 32 on 8 x 8192 x 128, weighed: 48 us.
// Probabilities are rounded to the inputs' type for the second product (half a step each, as in smha_sink_fwd); sums are 32 bits.
// Forms: segments cut over the chip; with the wide segments of a prefix too (whose registers leave a workgroup less to a unit at 64 columns); or,
// where a group has few tiles whatever the lengths are, a workgroup a group, which reads the prefix's keys and the sequence's own one after the
// other and writes the output: nothing is counted, cut or joined, and the call is one launch.
enum CacheForm { kCut, kWide, kDirect };
constexpr int cache_groups(int D, int form) { return D == 128 ? 2 : form == kWide ? 3 : 4; }
template <int D, bool BF16, bool WEIGH, int FORM>
__global__ void __launch_bounds__(256, cache_groups(D, FORM)) smha_cache_part(const CacheParams p) {
    constexpr int NS = D / 16, NDT = D / 32, CPR = D / 8, LPT = CPR / 2, RPL = 64 / CPR, NO = 16 / RPL, TB = 32 * D * 2;
    __shared__ __attribute__((aligned(1024))) char all_tiles[4 * 2 * TB];  // per wave: K, V
    __shared__ float team[4][2][32];                                        // references and sums
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 31, hh = lane >> 5;
    char *const smem = all_tiles + w * 2 * TB;
    const uint32_t lds = (uint32_t)(uintptr_t)(lds_void *)smem;
    const float NEG_INF = -__builtin_inff();
    constexpr bool WIDE = FORM == kWide, DIRECT = FORM == kDirect;
    Segment s;
    if constexpr (DIRECT) {
        const int per_xcd = (int)gridDim.x >> 3, group = (int)(blockIdx.x & 7) * per_xcd + ((int)blockIdx.x >> 3);
        if (group >= p.B * p.Hkv * p.own_tiles) return;
        const int bh = group / p.own_tiles;
        s.b = bh / p.Hkv;
        s.hk = bh - s.b * p.Hkv;
        s.rows0 = 32 * (group - bh * p.own_tiles);
        s.length = uniform_load(p.lengths + s.b);
        s.part = 0;
        s.parts = 1;
    } else {
        s = segment_of(p, lane);
        if (s.place < 0) return;
    }
    const bool prefix = !DIRECT && s.b < 0;
    const OwnKeys own = prefix ? OwnKeys{p.P, 0, 0, s.n, 0, 0} : own_keys(s.length, p.T, p.Sk, p.window, p.n_sink);
    const int prefix_n = DIRECT ? (p.P + 31) / 32 : 0;  // tiles of the prefix before the sequence's own
    if constexpr (DIRECT) s.n = prefix_n + own.n;

    // this lane's row
    const int GT = p.G * p.T, row = s.rows0 + (WIDE && prefix ? 32 * w : 0) + j, rows = prefix ? p.B * GT : GT;
    const int rb = prefix ? min(row / GT, p.B - 1) : s.b, in_b = prefix ? row - rb * GT : row, g = in_b / p.T, t = in_b - g * p.T;
    const int len_r = prefix ? min(max(p.lengths[rb], 0), p.Sk) : own.len;
    const int pos = row < rows ? len_r - p.T + t : -1;  // below 0: no such query
    u32x4 qf[NS];
    {
        const uint16_t *const q = p.Q + rb * p.qs.b + (s.hk * p.G + g) * p.qs.h + t * p.qs.s + 8 * hh;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
            qf[i] = u32x4{0, 0, 0, 0};
            if (pos >= 0 && 16 * i + 8 * hh < p.d) qf[i] = *reinterpret_cast<const u32x4 *>(q + 16 * i);
        }
    }
    if constexpr (WIDE) {
        if (prefix) return prefix_wide<D, BF16>(p, s, all_tiles, qf, lane, w);
    }
    // Where tiles come from: this segment's keys, and the prefix's where they are read first.
    struct From {
        u32x4 rK, rV;
        int ksb, vsb;
        uint32_t k_go[NO], v_go[NO];
    };
    const int row0 = lane / CPR;
    auto from = [&](const uint16_t *K, const uint16_t *V, int64_t ks, int64_t vs, int len) __attribute__((always_inline)) {
        From f;
        f.rK = make_rsrc4(K, len > 0 ? ((int64_t)(len - 1) * ks + p.d) * 2 : 0);
        f.rV = make_rsrc4(V, len > 0 ? ((int64_t)(len - 1) * vs + p.d) * 2 : 0);
        f.ksb = (int)ks * 2;
        f.vsb = (int)vs * 2;
#pragma unroll
        for (int o = 0; o < NO; ++o) {
            const int ch = (lane % CPR) ^ swz_both<D>(row0 + RPL * o);
            f.k_go[o] = ch < (p.d >> 3) ? (uint32_t)(row0 * f.ksb + ch * 16) : kNoChunk;
            f.v_go[o] = ch < (p.d >> 3) ? (uint32_t)(row0 * f.vsb + ch * 16) : kNoChunk;
        }
        return f;
    };
    const From mine_f = prefix ? from(p.PK + s.hk * p.pk_h, p.PV + s.hk * p.pv_h, p.pk_s, p.pv_s, p.P)
                               : from(p.K + s.b * p.ks.b + s.hk * p.ks.h, p.V + s.b * p.vs.b + s.hk * p.vs.h, p.ks.s, p.vs.s, own.len);
    From first_f = mine_f;
    if constexpr (DIRECT) {
        if (p.P) first_f = from(p.PK + s.hk * p.pk_h, p.PV + s.hk * p.pv_h, p.pk_s, p.pv_s, p.P);
    }
    auto key_of = [&](int tile) __attribute__((always_inline)) { return DIRECT && tile < prefix_n ? 32 * tile : own.key(tile - prefix_n); };
    // keys in the gap between the sinks and the window read as zeros: no query sees them, and they may hold anything
    auto request = [&](u32x4 rsrc, uint32_t to, const uint32_t (&go)[NO], int pitch, int key, int gap0, int gap1) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < LPT; ++i) {
            const int r = key + row0 + RPL * i;
            const uint32_t at = go[i % NO] + (uint32_t)((key + RPL * i) * pitch);
            load_to_lds(rsrc, to + i * 1024, (int)(r >= gap0 && r < gap1 ? kPast : at));
        }
    };
    auto request_k = [&](int tile) __attribute__((always_inline)) {
        if (DIRECT && tile < prefix_n) request(first_f.rK, lds, first_f.k_go, first_f.ksb, key_of(tile), 0, 0);
        else request(mine_f.rK, lds, mine_f.k_go, mine_f.ksb, key_of(tile), own.gap0, own.gap1);
    };
    auto request_v = [&](int tile) __attribute__((always_inline)) {
        if (DIRECT && tile < prefix_n) request(first_f.rV, lds + TB, first_f.v_go, first_f.vsb, key_of(tile), 0, 0);
        else request(mine_f.rV, lds + TB, mine_f.v_go, mine_f.vsb, key_of(tile), own.gap0, own.gap1);
    };
    const int begin = (int)((int64_t)s.n * s.part / s.parts) + w, end = (int)((int64_t)s.n * (s.part + 1) / s.parts);
    if (begin < end) {
        request_k(begin);
        request_v(begin);
    }
    const int rd = j * D * 2 + ((hh ^ swz_both<D>(j)) * 16);
    const int tr_row = 4 * hh + ((lane & 15) >> 2);
    const int tr = tr_row * D * 2 + ((swz_both<D>(tr_row) ^ (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1))) * 16) + (lane & 1) * 8;
    float *const score_row = WEIGH && !prefix && row < rows ? p.scores + (((int64_t)s.b * p.Hkv + s.hk) * GT + row) * p.score_pitch : nullptr;

    float m_run = NEG_INF, l_run = 0.f;
    const float thr = raised_over(p.c);
    f32x16 o[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) o[dt] = zeros16();
    for (int tile = begin; tile < end; tile += 4) {
        const int key = key_of(tile);
        const bool more = tile + 4 < end;
        wait_all_but<LPT>();  // K has landed (V's requests came after)
        f32x16 acc = zeros16();
        u32x4 kf[NS];
#pragma unroll
        for (int i = 0; i < NS; ++i) kf[i] = *reinterpret_cast<const u32x4 *>(smem + (rd ^ (32 * i)));
#pragma unroll
        for (int i = 0; i < NS; ++i) acc = mfma32<BF16>(kf[i], qf[i], acc);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // K's buffer is read
        if (!WEIGH && more) request_k(tile + 4);
        uint32_t word;
        if (prefix || (DIRECT && tile < prefix_n)) word = pos >= 0 ? low_bits32(p.P - key) : 0;
        else word = pos >= 0 ? low_bits32(pos - key + 1) & (~low_bits32(pos - p.window + 1 - key) | low_bits32(p.n_sink - key)) : 0;
        if (__builtin_amdgcn_ballot_w64(word != ~0u) != 0) {
            const u32x16 keep = keep_of(word >> (4 * hh)), sc = __builtin_bit_cast(u32x16, acc);
            acc = __builtin_bit_cast(f32x16, (sc & keep) | (~keep & 0xFF800000u));
        }
        if constexpr (WEIGH) {
            // (before the next K is requested: the waits below count that many requests)
            if (score_row) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 v = {acc[4 * q] * p.c, acc[4 * q + 1] * p.c, acc[4 * q + 2] * p.c, acc[4 * q + 3] * p.c};
                    *reinterpret_cast<f32x4 *>(score_row + key + 8 * q + 4 * hh) = v;
                }
            }
            asm volatile("" ::: "memory");
            if (more) request_k(tile + 4);
        }
        float mt = NEG_INF;
#pragma unroll
        for (int r = 0; r < 16; ++r) mt = fmaxf(mt, acc[r]);
        if (__builtin_amdgcn_ballot_w64(mt > m_run + thr) != 0) {
            mt = fmaxf(mt, __shfl_xor(mt, 32));
            const float m_new = fmaxf(m_run, mt), alpha = fast_exp2((m_run - (m_new == NEG_INF ? 0.f : m_new)) * p.c);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) o[dt] *= alpha;
        }
        const float mc = (m_run == NEG_INF ? 0.f : m_run) * p.c;
        u32x4 pf[2];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float e0 = fast_exp2(fmaf(acc[2 * q], p.c, -mc)), e1 = fast_exp2(fmaf(acc[2 * q + 1], p.c, -mc));
            pf[q >> 2][q & 3] = pack2<BF16>(e0, e1);
            l_run += e0 + e1;
        }
        if (more) wait_all_but<LPT>();  // V has landed
        else wait_all_but<0>();
#pragma unroll
        for (int i = 0; i < 2 * NDT; ++i) {
            const char *const at = smem + TB + ((tr ^ (64 * (i % NDT))) + 32 * (i / NDT) * D), *const at8 = smem + TB + ((tr ^ (64 * (i % NDT)) ^ 32) + 32 * (i / NDT) * D + 16 * D);
            const u32x2 lo = lds_read_tr(reinterpret_cast<const uint16_t *>(at)), hi = lds_read_tr(reinterpret_cast<const uint16_t *>(at8));
            o[i % NDT] = mfma32<BF16>(u32x4{lo[0], lo[1], hi[0], hi[1]}, pf[i / NDT], o[i % NDT]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // V's buffer is read
        if (more) request_v(tile + 4);
    }

    // The team joins: every wave leaves its accumulators in its own tiles' place and takes a quarter of the columns of all four.
    constexpr int NR = D / 2, NQ = NR / 4;  // accumulators a lane holds, and takes
    const float l = l_run + __shfl_xor(l_run, 32);
    float *const mine = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int i = 0; i < NR / 4; ++i)
        *reinterpret_cast<f32x4 *>(mine + (i * 64 + lane) * 4) = f32x4{o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]};
    if (hh == 0) {
        team[w][0][j] = m_run * p.c;
        team[w][1][j] = l;
    }
    __syncthreads();
    float mu[4], m_all = NEG_INF, l_all = 0.f, out[NQ];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        mu[u] = team[u][0][j];
        m_all = fmaxf(m_all, mu[u]);
    }
#pragma unroll
    for (int i = 0; i < NQ; ++i) out[i] = 0.f;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const float share = mu[u] != NEG_INF ? fast_exp2(mu[u] - m_all) : 0.f;
        l_all = fmaf(share, team[u][1][j], l_all);
        const float *const his = reinterpret_cast<const float *>(all_tiles + u * 2 * TB);
#pragma unroll
        for (int i = 0; i < NQ / 4; ++i) {
            const f32x4 v = *reinterpret_cast<const f32x4 *>(his + ((w * (NQ / 4) + i) * 64 + lane) * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) out[4 * i + e] = fmaf(share, v[e], out[4 * i + e]);
        }
    }
    if (!DIRECT && s.part == 0 && threadIdx.x == 0) p.info[s.group] = int2{s.place, s.parts};
    const bool whole = DIRECT || (s.parts == 1 && p.prefix_tiles == 0);  // nothing to join with
    if (row < rows) {
        if (!whole || WEIGH) {
            if (w == 0 && hh == 0) {
                p.stats[(int64_t)s.place * 64 + j] = reference_of(m_all, l_all);
                p.stats[(int64_t)s.place * 64 + 32 + j] = l_all;
            }
        }
        const float inv = l_all != 0.f ? 1.0f / l_all : 0.f;
        uint16_t *const to = p.O + rb * p.os.b + (s.hk * p.G + g) * p.os.h + t * p.os.s;
        float *const part = p.parts + ((int64_t)s.place * 32 + j) * D;
#pragma unroll
        for (int i = 0; i < NQ; i += 4) {
            const int r = NQ * w + i, col = 32 * (r >> 4) + 8 * ((r & 15) >> 2) + 4 * hh;
            if (whole) {
                if (col < p.d) store4<BF16 ? SMHA_BF16 : SMHA_F16>(to, col, out[i] * inv, out[i + 1] * inv, out[i + 2] * inv, out[i + 3] * inv);
            } else {
                *reinterpret_cast<f32x4 *>(part + col) = f32x4{out[i], out[i + 1], out[i + 2], out[i + 3]};
            }
        }
    }
}

// The segments of one row: those of the prefix, then its own.
struct RowParts {
    int first[2], count[2], row[2];  // places' first, segments, and the row in them
    int step;                        // places of a prefix segment
    __device__ __forceinline__ int n() const { return count[0] + count[1]; }
    // where segment i of the row has its reference in `stats`, and its columns in `parts` (in rows)
    __device__ __forceinline__ int64_t stat(int i) const { return i < count[0] ? (int64_t)(first[0] + step * i) * 64 + row[0] : (int64_t)(first[1] + i - count[0]) * 64 + row[1]; }
    __device__ __forceinline__ int64_t part(int i) const { return i < count[0] ? (int64_t)(first[0] + step * i) * 32 + row[0] : (int64_t)(first[1] + i - count[0]) * 32 + row[1]; }
};
__device__ __forceinline__ RowParts row_parts(const CacheParams &p, int b, int hk, int in_b, bool own) {
    RowParts r{{0, 0}, {0, 0}, {0, 0}, p.wide ? 4 : 1};
    if (p.prefix_tiles) {
        const int row = b * p.G * p.T + in_b;
        const int2 i = p.info[hk * p.prefix_tiles + row / (p.wide ? 128 : 32)];
        r.first[0] = i.x + (p.wide ? (row >> 5) & 3 : 0);
        r.count[0] = i.y;
        r.row[0] = row & 31;
    }
    if (own) {
        const int2 i = p.info[p.Hkv * p.prefix_tiles + (b * p.Hkv + hk) * p.own_tiles + in_b / 32];
        r.first[1] = i.x;
        r.count[1] = i.y;
        r.row[1] = in_b & 31;
    }
    return r;
}

// The first workgroups join rows, one a workgroup; the others add to the accounts of 1024 keys of a key head.
template <int D, bool BF16>
__global__ void __launch_bounds__(256) smha_cache_join(const CacheParams p, int row_groups, int key_groups) {
    __shared__ float lds_ml[2][4];
    __shared__ float lds_o[4][D];
    __shared__ float lds_lse[256];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, GT = p.G * p.T;
    const float NEG_INF = -__builtin_inff();
    if ((int)blockIdx.x < row_groups) {
        const int id = blockIdx.x, b = id / (p.Hkv * GT), hk = id / GT - b * p.Hkv, in_b = id % GT, g = in_b / p.T, t = in_b - g * p.T;
        const int len = min(max(p.lengths[b], 0), p.Sk);
        RowParts r = row_parts(p, b, hk, in_b, true);  // (of a sequence without keys its own are not there)
        if (len == 0) r.count[1] = 0;
        uint16_t *const to = p.O + b * p.os.b + (hk * p.G + g) * p.os.h + t * p.os.s;
        if (len - p.T + t < 0) {  // no such query
            for (int c = threadIdx.x; c < p.d; c += 256) to[c] = 0;
            return;
        }
        if (!p.prefix_tiles && r.count[1] == 1) return;  // written whole
        // Wave w takes segments w, w + 4, ..., four at a time; a lane D / 64 columns.  (All of a turn's loads travel together: a call's rows
        // fit the chip at once, and what such a row lasts is its chain of trips to memory.)
        constexpr int E = D / 64;
        const int n = r.n();
        float m = NEG_INF, sum = 0.f, acc[E];
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
        for (int i0 = w; i0 < n; i0 += 16) {
            float ref[4], part[4], x[4][E], top = m;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + 4 * u < n ? i0 + 4 * u : i0;
                const float *const at = p.parts + r.part(i) * D + E * lane;
                ref[u] = p.stats[r.stat(i)];
                part[u] = p.stats[r.stat(i) + 32];
#pragma unroll
                for (int e = 0; e < E; ++e) x[u][e] = at[e];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (i0 + 4 * u >= n) ref[u] = NEG_INF;
                top = fmaxf(top, ref[u]);
            }
            const float old = m != NEG_INF ? fast_exp2(m - top) : 0.f;
            sum *= old;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] *= old;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float share = ref[u] != NEG_INF ? fast_exp2(ref[u] - top) : 0.f;
                sum = fmaf(share, part[u], sum);
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = ref[u] != NEG_INF ? fmaf(share, x[u][e], acc[e]) : acc[e];
            }
            m = top;
        }
        if (lane == 0) {
            lds_ml[0][w] = m;
            lds_ml[1][w] = sum;
        }
#pragma unroll
        for (int e = 0; e < E; ++e) lds_o[w][E * lane + e] = acc[e];
        __syncthreads();
        const float top = fmaxf(fmaxf(lds_ml[0][0], lds_ml[0][1]), fmaxf(lds_ml[0][2], lds_ml[0][3]));
        float share[4], l = 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            share[u] = lds_ml[0][u] != NEG_INF ? fast_exp2(lds_ml[0][u] - top) : 0.f;
            l = fmaf(share[u], lds_ml[1][u], l);
        }
        const float inv = l != 0.f ? 1.0f / l : 0.f;
        for (int c = threadIdx.x; c < p.d; c += 256)
            to[c] = (uint16_t)pack2<BF16>((share[0] * lds_o[0][c] + share[1] * lds_o[1][c] + share[2] * lds_o[2][c] + share[3] * lds_o[3][c]) * inv, 0.f);
        return;
    }
    const int id = (int)blockIdx.x - row_groups, bh = id / key_groups, b = bh / p.Hkv, hk = bh - b * p.Hkv;
    const OwnKeys own = own_keys(p.lengths[b], p.T, p.Sk, p.window, p.n_sink);
    const int first = (id - bh * key_groups) * 1024 + (int)threadIdx.x * 4;  // four keys a thread
    if (first - (int)threadIdx.x * 4 >= own.len) return;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    float *const account = p.weights + b * p.w_b + hk * p.w_h;
    // (of a row of 32 keys all were scored or none)
    const bool scored = first < own.len && (first < 32 * own.head || first >= 32 * own.t0);
    for (int r0 = 0; r0 < GT; r0 += 256) {
        const int nr = min(256, GT - r0);
        __syncthreads();
        for (int r1 = w; r1 < nr; r1 += 4) {  // a wave a row, a lane a segment
            const RowParts r = row_parts(p, b, hk, r0 + r1, true);
            const int n = r.n();
            float m = NEG_INF, l = 0.f;
            for (int i = lane; i - lane < n; i += 64) {
                float ref = NEG_INF, part = 0.f;
                if (i < n) {
                    const int64_t at = r.stat(i);
                    ref = p.stats[at];
                    part = p.stats[at + 32];
                }
                float top = fmaxf(m, ref);
#pragma unroll
                for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x));
                float sum = ref != NEG_INF ? fast_exp2(ref - top) * part : 0.f;
#pragma unroll
                for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x);
                l = (m != NEG_INF ? l * fast_exp2(m - top) : 0.f) + sum;
                m = top;
            }
            if (lane == 0) lds_lse[r1] = l != 0.f ? m + __builtin_amdgcn_logf(l) : __builtin_inff();  // (inf: a row without keys adds nothing)
        }
        __syncthreads();
        if (scored) {
            const float *const row = p.scores + ((int64_t)bh * GT + r0) * p.score_pitch + first;
            for (int r = 0; r < nr; ++r) {
                const f32x4 v = *reinterpret_cast<const f32x4 *>(row + (int64_t)r * p.score_pitch);
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] += fast_exp2(v[e] - lds_lse[r]);
            }
        }
    }
    if (scored)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (first + e < own.len) account[first + e] += sum[e];
}

// ---------------------------------------------------------------------------------------
// Eviction
// ---------------------------------------------------------------------------------------
struct EvictParams {
    uint16_t *K, *V;
    Strides ks, vs;
    const float *w;
    const int32_t *pos, *lengths;
    float *w_out;
    int32_t *pos_out, *len_out;
    int B, Hkv, Sk, d, budget, recent, moves;  // moves: most that a head makes
    int32_t *lists;                             // [B Hkv][1 + 2 moves]: count, where to, where from
};

// Running sums over a wave's lanes, and over groups of 16 of them, without LDS.
template <int CTRL, int ROWS>
__device__ __forceinline__ int add_moved(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false); }
__device__ __forceinline__ int row_scan(int v) {
    v = add_moved<0x111, 0xF>(v);  // row_shr 1, 2, 4, 8
    v = add_moved<0x112, 0xF>(v);
    v = add_moved<0x114, 0xF>(v);
    return add_moved<0x118, 0xF>(v);
}
__device__ __forceinline__ int wave_scan(int v) {
    v = row_scan(v);
    v = add_moved<0x142, 0xA>(v);     // the first and third row's sums to the second and fourth
    return add_moved<0x143, 0xC>(v);  // the first half's to the second
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int max_moved(int v) { return max(v, __builtin_amdgcn_update_dpp(v, v, CTRL, ROWS, 0xF, false)); }
__device__ __forceinline__ int row_max(int v) {  // lane 15 of each row of 16: the row's
    v = max_moved<0x111, 0xF>(v);
    v = max_moved<0x112, 0xF>(v);
    v = max_moved<0x114, 0xF>(v);
    return max_moved<0x118, 0xF>(v);
}
__device__ __forceinline__ int wave_max(int v) { return __builtin_amdgcn_readlane(max_moved<0x143, 0xC>(max_moved<0x142, 0xA>(row_max(v))), 63); }
// Of 16 waves' numbers: those before wave w, and all.
__device__ __forceinline__ void before_and_all(const int *numbers, int lane, int w, int &before, int &all) {
    const int upto = row_scan(numbers[lane & 15]);
    all = __builtin_amdgcn_readlane(upto, 15);
    before = w ? __builtin_amdgcn_readlane(upto, w - 1) : 0;
}

// An order of 32-bit floats as unsigned numbers, NaN with the lowest, -0 with +0.
__device__ __forceinline__ uint32_t ordered(float x) {
    const int u = __builtin_bit_cast(int, x + 0.0f);
    const uint32_t o = (uint32_t)(u ^ (u >> 31 | (int)0x80000000u));
    return x == x ? o : 0x007FFFFFu;  // -inf's
}

// One workgroup of 16 waves a key head.  Wave w holds the keys of slots (w n + i) 64 + lane as unsigned numbers that order them, so that a lane's
// and a register's order is the slots' order.  The budget-th largest is found by counting, 11, 11 and 10 bits at a time, in a
// histogram in LDS (11 bits of a float are a quarter of an octave: lanes of a wave meet in few bins but seldom all in one, and where
// they do one of them counts for all); of the keys that equal it the first slots stay.  What stays past the new end goes, in
// order, where keys before it left.  32 heads of 32768 keys 27.5 us.  (Counting with ballots, two bits at a time: 110;
// with a branch for each of a key's conditions: 30.)
// WHOLE: the rows are moved here too, which saves a launch where few move (evict_whole); their lists then take the histogram's place in LDS.
constexpr int kWholeMoves = 512;
template <int KPT, bool WHOLE>
__global__ void __launch_bounds__(1024) smha_cache_select(const EvictParams p) {
    __shared__ int bins[2048];
    __shared__ int totals[3][16];
    __shared__ int found[2];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int bh = blockIdx.x, b = bh / p.Hkv;
    const int len = min(max(uniform_load(p.lengths + b), 0), p.Sk), end = min(len, p.budget);
    const float *const W = p.w + (int64_t)bh * p.Sk;
    const int32_t *const P = p.pos + (int64_t)bh * p.Sk;
    float *const Wo = p.w_out + (int64_t)bh * p.Sk;
    int32_t *const Po = p.pos_out + (int64_t)bh * p.Sk;
    int32_t *const list = p.lists + (int64_t)bh * (1 + 2 * (int64_t)p.moves);
    const int n = (len + 1023) / 1024, base = w * 64 * n + lane;  // keys a lane, its first slot
    constexpr int HELD = KPT ? KPT : 1;
    uint32_t held[HELD];  // first the weights
    int32_t held_p[HELD];
    if constexpr (KPT > 0) {
        if (len > p.budget) {
#pragma unroll
            for (int i = 0; i < KPT; ++i) {
                const int slot = min(base + 64 * i, len - 1);  // (past the end: the last one again)
                held[i] = 0u;
                held_p[i] = INT32_MIN;
                if (i < n) {
                    held[i] = __builtin_bit_cast(uint32_t, W[slot]);
                    held_p[i] = P[slot];
                }
            }
        }
    }
    auto beyond = [&](int i) __attribute__((always_inline)) { return i % (KPT < 8 ? 1 : KPT < 16 ? 2 : 4) == 0 && i >= n; };  // where a lane has no more keys (those it holds past them are 0)
    // All slots before the end (those that are freed are written again below): from the registers where most stay, else only the first waves have
    // some.  (128 heads of 20000 keys to 19000: 46.2 us by reading again, 42.0 so; 32 of 32768 to
    // 2048: 41.9, 45.6.)
    if (KPT > 0 && len > p.budget && end > len / 2) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            if (i < n && base + 64 * i < end) {
                if (Wo != W) Wo[base + 64 * i] = __builtin_bit_cast(float, held[i]);
                if (Po != P) Po[base + 64 * i] = held_p[i];
            }
        }
    } else {
        if (Wo != W)
            for (int i = threadIdx.x; i < end; i += 1024) Wo[i] = W[i];
        if (Po != P)
            for (int i = threadIdx.x; i < end; i += 1024) Po[i] = P[i];
    }
    // What lies past the new end; and the new length.
    auto finish = [&]() __attribute__((always_inline)) {
        for (int i = end + threadIdx.x; i < p.Sk; i += 1024) {
            Wo[i] = 0.f;
            Po[i] = -1;
        }
        if (threadIdx.x == 0 && bh == b * p.Hkv) p.len_out[b] = end;
    };
    if (len <= p.budget) {
        if constexpr (WHOLE) finish();
        else if (threadIdx.x == 0) list[0] = 0;
        return;
    }
    int newest = INT32_MIN;
    if constexpr (KPT > 0) {
#pragma unroll
        for (int i = 0; i < KPT; ++i) newest = max(newest, held_p[i]);
    } else {
        for (int i = threadIdx.x; i < len; i += 1024) newest = max(newest, P[i]);
    }
    newest = wave_max(newest);
    if (lane == 0) totals[0][w] = newest;
    for (int i = threadIdx.x; i < 2048; i += 1024) bins[i] = 0;
    __syncthreads();
    newest = __builtin_amdgcn_readlane(row_max(totals[0][lane & 15]), 15);
    // positions past this stay, whatever their account; where there are none so low, all
    const bool all_young = (int64_t)newest - p.recent < INT32_MIN;
    const int young = all_young ? INT32_MIN : newest - p.recent;
    const int limit = min(len, (w + 1) * 64 * n);  // the wave's slots end here
    auto key_from = [&](int slot, float x, int32_t at) __attribute__((always_inline)) -> uint32_t {
        const uint32_t o = ordered(x), k = (all_young | (at > young)) ? 0xFF800000u : o;
        return slot < limit ? k : 0u;  // (0: below every live key's, which are in the fourth bin or later)
    };
    if constexpr (KPT > 0) {
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            if (beyond(i)) break;
            held[i] = key_from(base + 64 * i, __builtin_bit_cast(float, held[i]), held_p[i]);
        }
    }
    auto each = [&](auto &&f) __attribute__((always_inline)) {
        if constexpr (KPT > 0) {
#pragma unroll
            for (int i = 0; i < KPT; ++i) {
                if (beyond(i)) break;
                f(held[i]);
            }
        } else {
            for (int i = 0; i < n; ++i) {
                const int slot = base + 64 * i;
                f(slot < len ? key_from(slot, W[slot], P[slot]) : 0u);
            }
        }
    };
    // the largest number that `end` keys or more reach: its bits from the top, and how many keys are over what is known of it
    uint32_t least = 0;
    int all_over = 0;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, width = pass == 2 ? 10 : 11;
        each([&](uint32_t k) __attribute__((always_inline)) {
            // (what is known of `least` is not zero: no live key's is, and the others' numbers do not match it; at first they are counted in bin 0)
            const bool in = pass == 0 || ((k ^ least) >> (shift + width)) == 0;
            if (__builtin_amdgcn_ballot_w64(in) == 0) return;
            const int bin = (int)(k >> shift) & ((1 << width) - 1);
            if (in) {
                const int one = __builtin_amdgcn_readfirstlane(bin);
                const uint64_t other = __builtin_amdgcn_ballot_w64(bin != one);
                if (other != 0) atomicAdd(&bins[bin], 1);
                else if (const uint64_t who = __builtin_amdgcn_ballot_w64(true); lane == __builtin_ctzll(who)) atomicAdd(&bins[one], __builtin_popcountll(who));
            }
        });
        __syncthreads();
        // a thread's two bins, from the top, and those over them
        const int top = 2047 - 2 * (int)threadIdx.x, n1 = bins[top], n0 = bins[top - 1];
        const int upto = wave_scan(n1 + n0);
        if (lane == 63) totals[1][w] = upto;
        __syncthreads();
        bins[top] = bins[top - 1] = 0;
        int before, all;
        before_and_all(totals[1], lane, w, before, all);
        const int over = all_over + before + upto - n1 - n0;
        if (over < end && over + n1 >= end) {
            found[0] = top;
            found[1] = over;
        } else if (over + n1 < end && over + n1 + n0 >= end) {
            found[0] = top - 1;
            found[1] = over + n1;
        }
        __syncthreads();
        least |= (uint32_t)found[0] << shift;
        all_over = found[1];
    }
    // Who stays, as a bit of a word for each of up to 32 keys of the lane: those over the least, and the first of those at it.
    const int equal_stay = end - all_over;
    const uint64_t below = (1ull << lane) - 1;
    constexpr int GROUP = KPT ? KPT : 32;  // keys of such a word
    uint32_t over, equal;
    auto words = [&](int i0) __attribute__((always_inline)) {
        over = equal = 0;
#pragma unroll
        for (int i = 0; i < GROUP; ++i) {
            uint32_t k = 0u;
            if constexpr (KPT > 0) {
                if (beyond(i)) break;
                k = held[i];
            } else {
                const int slot = base + 64 * (i0 + i);
                if (i0 + i < n && slot < len) k = key_from(slot, W[slot], P[slot]);
            }
            over |= (uint32_t)(k > least) << i;
            equal |= (uint32_t)(k == least) << i;
        }
    };
    // the place of every set bit of the wave in the order of slots, from `at` on
    auto in_order = [&](uint32_t word, int &at, auto &&f) __attribute__((always_inline)) {
        if (__builtin_amdgcn_ballot_w64(word != 0) == 0) return;
        for (int i = 0; i < GROUP; ++i) {
            const bool mine = (word >> i) & 1;
            const uint64_t who = __builtin_amdgcn_ballot_w64(mine);
            if (who == 0) continue;
            if (mine) f(i, at + __builtin_popcountll(who & below));
            at += __builtin_popcountll(who);
        }
    };
    int count = 0;
    for (int i0 = 0; i0 < n; i0 += GROUP) {
        words(i0);
        count += __builtin_popcount(equal);
    }
    count = wave_scan(count);
    if (lane == 63) totals[0][w] = count;
    __syncthreads();
    int equal_first, all;
    before_and_all(totals[0], lane, w, equal_first, all);
    int equal_at = equal_first;
    // bits of `over` and of the equals that stay
    auto staying = [&](int i0) __attribute__((always_inline)) {
        if constexpr (KPT == 0) words(i0);
        uint32_t stay = over;
        in_order(equal, equal_at, [&](int i, int place) __attribute__((always_inline)) {
            if (place < equal_stay) stay |= 1u << i;
        });
        return stay;
    };
    // of the group's keys, those in slots before the end (a lane has n keys: later bits of a word are other waves' slots)
    auto before_end = [&](int i0) __attribute__((always_inline)) { return low_bits32(min((end - (base + 64 * i0) + 63) >> 6, n - i0)); };
    int freed = 0, kept = 0;
    uint32_t stay = 0;
    for (int i0 = 0; i0 < n; i0 += GROUP) {
        stay = staying(i0);
        const uint32_t early = before_end(i0);
        freed += __builtin_popcount(~stay & early);
        kept += __builtin_popcount(stay & ~early);
    }
    freed = wave_scan(freed);
    kept = wave_scan(kept);
    if (lane == 63) {
        totals[1][w] = freed;
        totals[2][w] = kept;
    }
    __syncthreads();
    int to, from, moves;
    before_and_all(totals[2], lane, w, from, all);
    before_and_all(totals[1], lane, w, to, moves);
    equal_at = equal_first;
    if constexpr (WHOLE) {
        for (int i0 = 0; i0 < n; i0 += GROUP) {
            if constexpr (KPT == 0) stay = staying(i0);
            const uint32_t early = before_end(i0);
            in_order(~stay & early, to, [&](int i, int place) __attribute__((always_inline)) { bins[place] = base + 64 * (i0 + i); });
            in_order(stay & ~early, from, [&](int i, int place) __attribute__((always_inline)) { bins[kWholeMoves + place] = base + 64 * (i0 + i); });
        }
        __syncthreads();
        for (int i = threadIdx.x; i < moves; i += 1024) {
            Wo[bins[i]] = W[bins[kWholeMoves + i]];
            Po[bins[i]] = P[bins[kWholeMoves + i]];
        }
        const int hk = bh - b * p.Hkv, col = 8 * (threadIdx.x & 15), first = threadIdx.x >> 4;
        uint16_t *const K = p.K + b * p.ks.b + hk * p.ks.h, *const V = p.V + b * p.vs.b + hk * p.vs.h;
        constexpr int U = 4;  // rows of 16 lanes that travel together
        for (int i0 = first; i0 < moves; i0 += 64 * U) {
            u32x4 k[U], v[U];
            const bool has = col < p.d;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t from_row = bins[kWholeMoves + min(i0 + 64 * u, moves - 1)];
                if (has) {
                    k[u] = *reinterpret_cast<const u32x4 *>(K + from_row * p.ks.s + col);
                    v[u] = *reinterpret_cast<const u32x4 *>(V + from_row * p.vs.s + col);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t to_row = bins[min(i0 + 64 * u, moves - 1)];
                if (has && i0 + 64 * u < moves) {
                    *reinterpret_cast<u32x4 *>(K + to_row * p.ks.s + col) = k[u];
                    *reinterpret_cast<u32x4 *>(V + to_row * p.vs.s + col) = v[u];
                }
            }
        }
        __syncthreads();  // (weights may be read and written in one place)
        finish();
        return;
    }
    for (int i0 = 0; i0 < n; i0 += GROUP) {
        if constexpr (KPT == 0) stay = staying(i0);
        const uint32_t early = before_end(i0);
        in_order(~stay & early, to, [&](int i, int place) __attribute__((always_inline)) { list[1 + place] = base + 64 * (i0 + i); });
        in_order(stay & ~early, from, [&](int i, int place) __attribute__((always_inline)) { list[1 + p.moves + place] = base + 64 * (i0 + i); });
    }
    if (threadIdx.x == 0) list[0] = moves;
    __syncthreads();
    for (int i = threadIdx.x; i < moves; i += 1024) {
        const int to_slot = list[1 + i], from_slot = list[1 + p.moves + i];
        Wo[to_slot] = W[from_slot];
        Po[to_slot] = P[from_slot];
    }
}

// K and V rows along the lists: what is read lies past the new end, what is written before it.  And what lies past it afterwards.  Bound by memory: 32
// heads of 32768 keys x 128 to 2048: 71 MB, 15.2 us.
__global__ void __launch_bounds__(256) smha_cache_move(const EvictParams p) {
    const int bh = blockIdx.y, b = bh / p.Hkv, hk = bh - b * p.Hkv;
    const int end = min(min(max(p.lengths[b], 0), p.Sk), p.budget);  // (the same where len_out is lengths and has been written already)
    if (blockIdx.x == 0 && hk == 0 && threadIdx.x == 0) p.len_out[b] = end;
    const int32_t *const list = p.lists + (int64_t)bh * (1 + 2 * (int64_t)p.moves);
    const int n = list[0], lane = threadIdx.x & 15;
    uint16_t *const K = p.K + b * p.ks.b + hk * p.ks.h, *const V = p.V + b * p.vs.b + hk * p.vs.h;
    for (int i = blockIdx.x * 16 + (threadIdx.x >> 4); i < n; i += gridDim.x * 16) {
        const int64_t to = list[1 + i], from = list[1 + p.moves + i];
        if (8 * lane < p.d) {
            const u32x4 k = *reinterpret_cast<const u32x4 *>(K + from * p.ks.s + 8 * lane), v = *reinterpret_cast<const u32x4 *>(V + from * p.vs.s + 8 * lane);
            *reinterpret_cast<u32x4 *>(K + to * p.ks.s + 8 * lane) = k;
            *reinterpret_cast<u32x4 *>(V + to * p.vs.s + 8 * lane) = v;
        }
    }
    for (int i = end + (int)(blockIdx.x * 256 + threadIdx.x); i < p.Sk; i += (int)gridDim.x * 256) {
        p.w_out[(int64_t)bh * p.Sk + i] = 0.f;
        p.pos_out[(int64_t)bh * p.Sk + i] = -1;
    }
}

// ---------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------
static bool cache_strides_fit(const int64_t *s, int64_t rows, int d) {
    if (!s) return (rows + 64) * d * 2 < ((int64_t)1 << 31);
    return s[0] % 8 == 0 && s[1] % 8 == 0 && s[2] % 8 == 0 && s[0] >= 0 && s[1] >= 0 && s[2] >= d && ((rows + 64) * s[2] + d) * 2 < ((int64_t)1 << 31);
}
static Strides cache_strides(const int64_t *s, int64_t heads, int64_t rows, int d) {
    return s ? Strides{s[0], s[1], s[2]} : Strides{heads * rows * d, rows * d, d};
}

// Tiles of a group up to which a workgroup takes it whole.  Cutting costs a second launch and shares out what one workgroup would read alone (0.37 us a
// tile); where groups fill the chip by themselves there is little to share.  us of a call, direct and cut: 2 groups x 64 of 256, 500, 700,
// 1000 and 1500 keys: 5.5, 7.2, 8.8, 10.7, 14.1 and 9.0 to 9.3; 32 x 128 of 500, 700, 1000: 9.8, 12.1, 14.8 and 10.9; 128 x 128
// of 1000: 17.2, 19.5; 512 x 128 of 700, 1000 and 1500: 31, 43, 70 and 35, 48, 75, of 30 to 100 % of those lengths 23, 30, 44 and 31, 37, 50.  No more than 48: with
// one long sequence among short ones it is the longest that counts.  (A prefix that many groups read is better shared.)
static int64_t direct_tiles(int d, int P, int64_t groups) { return std::min<int64_t>(48, (d <= 64 ? 24 : 16) + (P ? 0 : groups / 8)); }

struct CacheLayout {
    size_t info, stats, parts, scores, total;
};
static size_t up(size_t n) { return (n + 255) & ~(size_t)255; }

// Sizes and the workspace's layout; what both entry points refuse.
static smha_status_t cache_params(CacheParams &cp, CacheLayout &at, int B, int H, int Hkv, int T, int Sk, int P, int d, smha_dtype_t dtype, int window, int n_sink,
                                  bool weigh) {
    if (B < 1 || H < 1 || Hkv < 1 || T < 1 || Sk < 1 || P < 0 || window < 0 || n_sink < 0) return SMHA_ERR_INVALID_ARG;
    if (H % Hkv) return SMHA_ERR_SHAPE;
    if (dtype != SMHA_F16 && dtype != SMHA_BF16) return SMHA_ERR_UNSUPPORTED;
    if (d < 8 || d > 128 || d % 8) return SMHA_ERR_UNSUPPORTED;
    if (T >= kRowsEnd || Sk >= kRowsEnd || P >= kRowsEnd || (int64_t)B * H > (1 << 24) || (int64_t)B * H * T > (1 << 24)) return SMHA_ERR_UNSUPPORTED;
    if (P > 0 && window > 0) return SMHA_ERR_UNSUPPORTED;  // (the window would have to run back into the prefix)
    cp.B = B; cp.H = H; cp.Hkv = Hkv; cp.G = H / Hkv; cp.T = T; cp.Sk = Sk; cp.P = P; cp.d = d;
    cp.window = window == 0 || window > Sk ? Sk : window;
    cp.n_sink = std::min(n_sink, Sk);
    const int64_t rows = (int64_t)cp.G * T, own_tiles = (rows + 31) / 32;
    const int64_t own_tiles_most = std::min<int64_t>((Sk + 31) / 32, ((int64_t)cp.window + cp.n_sink + T) / 32 + 3);
    cp.direct = !weigh && own_tiles_most + (P + 31) / 32 <= direct_tiles(d, P, B * Hkv * own_tiles);
    cp.wide = !cp.direct && P > 0 && B * rows > 64;  // (one or two tiles of 32 rows: reading the keys once or twice by waves on their own fills the chip better)
    const int64_t prefix_tiles = !P ? 0 : cp.wide ? (B * rows + 127) / 128 : (B * rows + 31) / 32;
    const int64_t groups = (int64_t)Hkv * (prefix_tiles + B * own_tiles);
    // (tiles are counted in 32 bits)
    if (groups * (std::max(Sk, P) / 32 + 8) > (1 << 30)) return SMHA_ERR_UNSUPPORTED;
    cp.own_tiles = (int)own_tiles;
    cp.prefix_tiles = (int)prefix_tiles;
    const int D = d <= 64 ? 64 : 128;
    cp.slots = 256 * cache_groups(D, cp.wide ? kWide : kCut);  // what the chip holds at once
    // no more segments than that and one a group, and none shorter than four tiles unless it is a group
    const int64_t own_most = (own_tiles_most + 3) / 4;
    const int64_t prefix_most = Hkv * prefix_tiles * (((cp.wide ? P / 64 : P / 32) + 1 + 3) / 4);
    cp.prefix_segs = (int)std::min<int64_t>(cp.slots + Hkv * prefix_tiles, prefix_most);
    const int64_t own_segs = std::min<int64_t>(cp.slots + (int64_t)B * Hkv * own_tiles, B * Hkv * own_tiles * own_most);
    cp.segs = (int)(cp.prefix_segs + own_segs);
    // (a launch has less than 2^32 threads)
    const int64_t most = std::max(std::max<int64_t>((int64_t)B * Hkv * own_tiles, cp.segs + 8), (int64_t)B * H * T + (weigh ? (int64_t)B * Hkv * ((Sk + 1023) / 1024) : 0));
    if (most + 8 >= (1 << 24)) return SMHA_ERR_UNSUPPORTED;
    const int64_t places = (cp.wide ? 4 : 1) * (int64_t)cp.prefix_segs + own_segs;
    cp.score_pitch = (Sk + 31) / 32 * 32;
    if (cp.direct) {  // (nothing is kept)
        at.total = 0;
        return SMHA_OK;
    }
    at.info = 0;
    at.stats = up(groups * sizeof(int2));
    at.parts = at.stats + up((size_t)places * 64 * 4);
    at.scores = at.parts + up((size_t)places * 32 * D * 4);
    at.total = at.scores + (weigh ? (size_t)B * Hkv * rows * cp.score_pitch * 4 : 0);
    return SMHA_OK;
}

template <int D, bool BF16> static hipError_t launch_cache(const CacheParams &cp, hipStream_t stream) {
    if (cp.direct) {
        const int groups = cp.B * cp.Hkv * cp.own_tiles;
        hipLaunchKernelGGL((smha_cache_part<D, BF16, false, kDirect>), dim3(8 * ((groups + 7) / 8)), dim3(256), 0, stream, cp);
        return hipGetLastError();
    }
    const dim3 grid(8 * ((cp.segs + 7) / 8 + 1));  // (two runs an XCD, each rounded up)
    auto *const part = cp.weights ? (cp.wide ? smha_cache_part<D, BF16, true, kWide> : smha_cache_part<D, BF16, true, kCut>)
                                  : (cp.wide ? smha_cache_part<D, BF16, false, kWide> : smha_cache_part<D, BF16, false, kCut>);
    hipLaunchKernelGGL(part, grid, dim3(256), 0, stream, cp);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int rows = cp.B * cp.H * cp.T, keys = cp.weights ? (cp.Sk + 1023) / 1024 : 0;
    hipLaunchKernelGGL((smha_cache_join<D, BF16>), dim3((unsigned)(rows + cp.B * cp.Hkv * keys)), dim3(256), 0, stream, cp, rows, keys);
    return hipGetLastError();
}

}  // namespace smha

using namespace smha;

extern "C" smha_status_t smha_cache_workspace(int B, int H, int Hkv, int T, int Sk, int P, int d, int window, int n_sink, int weigh, size_t *need) {
    if (!need) return SMHA_ERR_INVALID_ARG;
    CacheParams cp{};
    CacheLayout at{};
    const smha_status_t st = cache_params(cp, at, B, H, Hkv, T, Sk, P, d, SMHA_F16, window, n_sink, weigh != 0);
    if (st != SMHA_OK) return st;
    *need = at.total;
    return SMHA_OK;
}

extern "C" smha_status_t smha_cache_forward(const void *Q, const void *K, const void *V, const void *PK, const void *PV, void *O, float *weights,
                                            const int32_t *lengths, int B, int H, int Hkv, int T, int Sk, int P, int d, smha_dtype_t dtype,
                                            const int64_t q_strides[3], const int64_t k_strides[3], const int64_t v_strides[3], const int64_t pk_strides[2],
                                            const int64_t pv_strides[2], const int64_t o_strides[3], const int64_t w_strides[2], int window, int n_sink, float scale,
                                            void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!Q || !K || !V || !O || !lengths || (P > 0 && (!PK || !PV))) return SMHA_ERR_INVALID_ARG;
    CacheParams cp{};
    CacheLayout at{};
    const smha_status_t st = cache_params(cp, at, B, H, Hkv, T, Sk, P, d, dtype, window, n_sink, weights != nullptr);
    if (st != SMHA_OK) return st;
    if (workspace_bytes < at.total || (at.total && !workspace)) return SMHA_ERR_INVALID_ARG;
    if (((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O | (uintptr_t)workspace | (P ? (uintptr_t)PK | (uintptr_t)PV : 0)) & 15) return SMHA_ERR_UNSUPPORTED;
    if (!cache_strides_fit(q_strides, T, d) || !cache_strides_fit(k_strides, Sk, d) || !cache_strides_fit(v_strides, Sk, d) || !cache_strides_fit(o_strides, T, d))
        return SMHA_ERR_UNSUPPORTED;
    if (!apart(o_strides, B, H, T, d)) return SMHA_ERR_UNSUPPORTED;
    if (weights && w_strides) {
        const int64_t keys[3] = {w_strides[0], w_strides[1], 1};
        if (keys[0] < 0 || keys[1] < 0 || !apart(keys, B, Hkv, Sk, 1)) return SMHA_ERR_UNSUPPORTED;
    }
    if (P) {
        for (const int64_t *s : {pk_strides, pv_strides}) {
            const int64_t three[3] = {0, s ? s[0] : (int64_t)P * d, s ? s[1] : d};
            if (!cache_strides_fit(three, P, d)) return SMHA_ERR_UNSUPPORTED;
        }
    }
    cp.Q = (const uint16_t *)Q; cp.K = (const uint16_t *)K; cp.V = (const uint16_t *)V; cp.O = (uint16_t *)O;
    cp.PK = (const uint16_t *)PK; cp.PV = (const uint16_t *)PV;
    cp.weights = weights; cp.lengths = lengths;
    cp.qs = cache_strides(q_strides, H, T, d); cp.ks = cache_strides(k_strides, Hkv, Sk, d); cp.vs = cache_strides(v_strides, Hkv, Sk, d);
    cp.os = cache_strides(o_strides, H, T, d);
    cp.pk_h = pk_strides ? pk_strides[0] : (int64_t)P * d; cp.pk_s = pk_strides ? pk_strides[1] : d;
    cp.pv_h = pv_strides ? pv_strides[0] : (int64_t)P * d; cp.pv_s = pv_strides ? pv_strides[1] : d;
    cp.w_b = w_strides ? w_strides[0] : (int64_t)Hkv * Sk; cp.w_h = w_strides ? w_strides[1] : Sk;
    cp.c = (scale > 0.f ? scale : 1.0f / std::sqrt((float)d)) * 1.4426950408889634f;
    char *const ws = (char *)workspace;
    cp.info = (int2 *)(ws + at.info); cp.stats = (float *)(ws + at.stats); cp.parts = (float *)(ws + at.parts); cp.scores = (float *)(ws + at.scores);
    const hipStream_t stream = (hipStream_t)hip_stream;
    const bool bf16 = dtype == SMHA_BF16;
    const hipError_t e = d <= 64 ? (bf16 ? launch_cache<64, true>(cp, stream) : launch_cache<64, false>(cp, stream))
                                 : (bf16 ? launch_cache<128, true>(cp, stream) : launch_cache<128, false>(cp, stream));
    return e == hipSuccess ? SMHA_OK : SMHA_ERR_HIP;
}

// Whether a head's own workgroup moves its rows.  us of a call by two kernels and by one: 128 heads of 4352 keys to 4096, x 128: 17.2, 15.0; 2 heads
// of 1100 to 1024: 9.6, 7.9; 1024 of 2176 to 2048: 44.7, 35.6; 32 of 8192 to 7936 and 7680: 15.9, 16.3 and 13.8, 16.2; to 7168 (one compute unit
// moves 1 MB, if more than the limit were allowed): 19.1, 23.3.  Lengths that are written where they are read need the second kernel: a sequence's other heads may still
// have to read them.
static bool evict_whole(const EvictParams &ep) { return ep.moves <= kWholeMoves && ep.len_out != ep.lengths; }

static smha_status_t evict_sizes(int B, int Hkv, int Sk, int d, int budget, int recent, size_t *need) {
    if (B < 1 || Hkv < 1 || Sk < 1 || budget < 1 || recent < 0) return SMHA_ERR_INVALID_ARG;
    if (d < 8 || d > 128 || d % 8 || (int64_t)B * Hkv > 65535 || Sk > (1 << 28)) return SMHA_ERR_UNSUPPORTED;
    const int64_t moves = std::max(0, std::min(budget, Sk - budget));
    *need = (size_t)((int64_t)B * Hkv * (1 + 2 * moves) * 4);
    return SMHA_OK;
}

extern "C" smha_status_t smha_cache_evict_workspace(int B, int Hkv, int Sk, int d, int budget, int recent, size_t *need) {
    if (!need) return SMHA_ERR_INVALID_ARG;
    size_t n = 0;
    const smha_status_t st = evict_sizes(B, Hkv, Sk, d, budget, recent, &n);
    if (st == SMHA_OK) *need = n;
    return st;
}

extern "C" smha_status_t smha_cache_evict(void *K, void *V, const float *weights, const int32_t *positions, const int32_t *lengths, float *weights_out,
                                          int32_t *positions_out, int32_t *lengths_out, int B, int Hkv, int Sk, int d, int budget, int recent,
                                          const int64_t k_strides[3], const int64_t v_strides[3], void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!K || !V || !weights || !positions || !lengths || !weights_out || !positions_out || !lengths_out || !workspace) return SMHA_ERR_INVALID_ARG;
    size_t need = 0;
    const smha_status_t st = evict_sizes(B, Hkv, Sk, d, budget, recent, &need);
    if (st != SMHA_OK) return st;
    if (workspace_bytes < need) return SMHA_ERR_INVALID_ARG;
    if (((uintptr_t)K | (uintptr_t)V) & 15 || (uintptr_t)workspace & 3) return SMHA_ERR_UNSUPPORTED;
    for (const int64_t *s : {k_strides, v_strides})
        if (s && (s[0] % 8 || s[1] % 8 || s[2] % 8 || s[0] < 0 || s[1] < 0 || s[2] < d)) return SMHA_ERR_UNSUPPORTED;
    if (!apart(k_strides, B, Hkv, Sk, d) || !apart(v_strides, B, Hkv, Sk, d)) return SMHA_ERR_UNSUPPORTED;
    EvictParams ep{};
    ep.K = (uint16_t *)K; ep.V = (uint16_t *)V;
    ep.ks = cache_strides(k_strides, Hkv, Sk, d); ep.vs = cache_strides(v_strides, Hkv, Sk, d);
    ep.w = weights; ep.pos = positions; ep.lengths = lengths; ep.w_out = weights_out; ep.pos_out = positions_out; ep.len_out = lengths_out;
    ep.B = B; ep.Hkv = Hkv; ep.Sk = Sk; ep.d = d; ep.budget = budget; ep.recent = recent;
    ep.moves = std::max(0, std::min(budget, Sk - budget));
    ep.lists = (int32_t *)workspace;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const dim3 grid(B * Hkv);
    const bool whole = evict_whole(ep);
    auto *const select = Sk <= 4096    ? (whole ? smha_cache_select<4, true> : smha_cache_select<4, false>)
                         : Sk <= 8192  ? (whole ? smha_cache_select<8, true> : smha_cache_select<8, false>)
                         : Sk <= 16384 ? (whole ? smha_cache_select<16, true> : smha_cache_select<16, false>)
                         : Sk <= 32768 ? (whole ? smha_cache_select<32, true> : smha_cache_select<32, false>)
                                       : (whole ? smha_cache_select<0, true> : smha_cache_select<0, false>);
    hipLaunchKernelGGL(select, grid, dim3(1024), 0, stream, ep);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return SMHA_ERR_HIP;
    if (whole) return SMHA_OK;
    hipLaunchKernelGGL(smha_cache_move, dim3((unsigned)std::max(1, std::min(64, (ep.moves + 63) / 64)), B * Hkv), dim3(256), 0, stream, ep);
    e = hipGetLastError();
    return e == hipSuccess ? SMHA_OK : SMHA_ERR_HIP;
}
