// Attention within a causal window and a few first keys that stay visible (sinks): forward and backward.
//
//   position of query i of sequence b: p = offset_b + i; it exists where 0 <= p < length_b
//   key j is visible to it iff j <= p and (p - j < window or j < n_sink)
//   s = scale q.k,  lse = log sum exp s,  P = exp(s - lse),  O = P V
//   delta = sum_c dO_c O_c,  dP = dO V^T,  dS = P (dP - delta),  dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
//
// G = H / Hkv query heads share a key head (dK and dV are sums over them).  No mask and no plan: what a tile needs is arithmetic on
// positions, and offsets and lengths are read on the device, so that a call neither synchronises nor depends on their values.
//
// All products run on v_mfma_f32_32x32x16 in the orientation in which the accumulators of the scores are the other products'
// B operand as they stand (P and dS never go through LDS), and tiles sit in LDS row-major, chunks of 16 bytes swizzled so that both
// ways of reading them are spread over the banks: rows 16 bytes at a time (A operand of the first products), and transposing reads
// of 4 rows x 16 columns (A operand of the second ones).  See smha_block_fwd for the operand layouts.
// Kernels <D, C> keep rows of D columns in LDS and form products over C of them, 32, 64, 96 or 128, the next above the head size.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "device_common.hpp"
#include "smha.h"

namespace smha {

struct SinkParams {
    const uint16_t *Q, *K, *V, *dO;
    const uint16_t *Oin;  // backward: the forward's output
    uint16_t *O, *rest;   // rest: what O's rounding left out, packed, or null
    uint16_t *dQ, *dK, *dV;
    float *lse;           // [B][H][Sq]
    Strides qs, ks, vs, os, gs, dqs, dks, dvs;
    int B, H, Hkv, G, Sq, Sk, d;
    int window, n_sink;   // 1 .. Sk (a window of Sk keys limits nothing), 0 .. Sk
    const int32_t *offsets, *lengths;
    float c, scale;       // c = scale * log2(e)
    int per, together;    // work items of a key head of a sequence; such heads whose items are taken in turn
    // backward
    float *stats;         // [2][B][H][Sqp]: lse * log2(e) (inf where there is no query), -delta
    int Sqp;
    float *parts;         // partial dK, dV of key tiles that are cut along their queries
    int n_tiles, n_sink_tiles;              // key tiles, those with sinks
    int chunk_sink, chunk_rest, cut_sink, cut_rest;  // steps of a part, parts at most: of a tile with sinks, of another
    int places, rest_at;  // partial sums that a key head of a sequence has room for (tiles in one part need none), and where those of tiles without sinks begin
};

struct Sequence {
    int len, off;  // keys, first query's position
    int qa, qb;    // queries qa .. qb - 1 exist
};
__device__ __forceinline__ Sequence sequence(const SinkParams &p, int b) {
    Sequence s;
    s.len = p.lengths ? min(max(uniform_load(p.lengths + b), 0), p.Sk) : p.Sk;
    s.off = p.offsets ? min(max(uniform_load(p.offsets + b), -p.Sq), p.Sk) : p.Sk - p.Sq;
    s.qa = max(0, -s.off);
    s.qb = min(p.Sq, s.len - s.off);
    return s;
}

// What a workgroup of a launch takes: item `item` of the key head `hk` of sequence `b`.  `together` of these groups go through their items in turn, the
// longest first, so that what starts last is short; a multiple of eight of them keep to an XCD each, whose L2 their workgroups share, and
// no more go together than a few rounds of the chip.  (By group, each XCD a run of them: a backward pass of 8 x 32 on 8 x 4096 x 128, window
// 1024, 4 sinks 2229 us, 1778 so, the sinks' tiles of the last groups began last; 1 x 32 x 4096 x 128, window 2048: 453, 386;
// 4 x 16 x 1024 x 128, window 128: 68, 63.)
struct Turn {
    int b, hk, item;
    __device__ __forceinline__ explicit Turn(const SinkParams &p) {
        const int at = blockIdx.x, n = p.B * p.Hkv, block = at / (p.together * p.per), first = block * p.together, groups = min(p.together, n - first);
        const int rest = at - first * p.per;
        item = rest / groups;
        const int group = first + rest - item * groups;
        b = group / p.Hkv;  // (an XCD has sequences of all lengths: by key head first, 4 x 12 x 1537 x 80 with 60 to 100 % of it had one length each: 94 us a pass for 83)
        hk = group - b * p.Hkv;
    }
};
// `at_once`: workgroups of an XCD that go together, about.  Keys' tiles 256 (2 x 16 x 8192 x 64, backward: 954 us with 128, 918), queries' 128 (the
// same, forward: 304 us, 310 with 256); all of 16 x 32 x 2048 x 128, window 1024: 590 and 1710 us -> 790 and 1963.
static inline int sink_together(int groups, int per, int at_once) { return std::min(groups, 8 * std::max(1, (at_once + per - 1) / per)); }

// A workgroup's 128 queries.  A head's last queries, which have the longest lists, come first.
struct QueryTile {
    int b, hk, h, q0;
    __device__ __forceinline__ explicit QueryTile(const SinkParams &p) {
        const Turn turn(p);
        const int nt = (p.Sq + 127) / 128, down = turn.item / p.G;
        b = turn.b;
        hk = turn.hk;
        h = hk * p.G + turn.item - down * p.G;
        q0 = (nt - 1 - down) * 128;
    }
};

// the keys k0 .. k0 + 63 that a query at position pos sees
__device__ __forceinline__ uint64_t seen_keys(int pos, int k0, int window, int n_sink) {
    return low_bits(pos - k0 + 1) & (~low_bits(pos - window + 1 - k0) | low_bits(n_sink - k0));
}
// whether queries at positions p0 .. p1 see any / all of keys k0 .. k1
__device__ __forceinline__ bool any_seen(int p0, int p1, int k0, int k1, int window, int n_sink) {
    return k0 <= p1 && (p0 - k1 < window || k0 < n_sink);
}
__device__ __forceinline__ bool all_seen(int p0, int p1, int k0, int k1, int window, int n_sink) {
    return k1 <= p0 && (p1 - k0 < window || k1 < n_sink);
}

// What rounding a and b to the pair v left out, rounded.
template <bool BF16> __device__ __forceinline__ uint32_t pack2_left(float a, float b, uint32_t v) {
    return pack2<BF16>(a - widen16<BF16>(v & 0xFFFFu), b - widen16<BF16>(v >> 16));
}
// a and b as a pair of rounded values and another of what that leaves out.  (The first is a register from then on: the compiler would form a product's
// rounding to binary16 a second time for the difference, in one instruction where it takes two for the pair, and at ties get the other neighbour.)
struct Halves {
    uint32_t hi, lo;
};
template <bool BF16> __device__ __forceinline__ Halves halves_of(float a, float b) {
    uint32_t v = pack2<BF16>(a, b);
    if constexpr (!BF16) asm("" : "+v"(v));
    return {v, pack2_left<BF16>(a, b, v)};
}

// A wave's 32 x D accumulators (acc[dt][r] = row j, column 32 dt + 8 (r / 4) + 4 hh + r % 4) to rows row0 .. of a tensor with 16-bit values,
// through 32 rows of LDS so that whole rows are written; rows from `rows` on are left out.
// REST: not the rounded values, but what their rounding left out, by the very values that the call before left in `slab` (formed anew they may differ in
// the last place: a product and its rounding to binary16 are one instruction or two, as the compiler sees fit).
template <int D, int C, bool BF16, bool REST = false>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[C / 32], float factor, char *slab, int lane, uint16_t *base, int64_t pitch, int row0, int rows, int d) {
    constexpr int CPR = D / 8;
    const int j = lane & 31, hh = lane >> 5;
#pragma unroll
    for (int dt = 0; dt < C / 32; ++dt)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = acc[dt][4 * g + e] * factor;
            u32x2 *const at = reinterpret_cast<u32x2 *>(slab + j * D * 2 + (((4 * dt + g) ^ swz_both<D>(j)) * 16) + hh * 8);
            if constexpr (REST) *at = u32x2{pack2_left<BF16>(x[0], x[1], (*at)[0]), pack2_left<BF16>(x[2], x[3], (*at)[1])};
            else *at = u32x2{pack2<BF16>(x[0], x[1]), pack2<BF16>(x[2], x[3])};
        }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < CPR / 2; ++i) {
        const int row = (i * 64 + lane) / CPR, c = (lane % CPR) ^ swz_both<D>(row);
        const u32x4 v = *reinterpret_cast<const u32x4 *>(slab + i * 1024 + lane * 16);
        if (row0 + row < rows && c < (d >> 3)) *reinterpret_cast<u32x4 *>(base + (row0 + row) * pitch + c * 8) = v;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

// A wave's 32 rows as the B operand of products over the columns: lane (j, hh) holds columns 16 s + 8 hh .. of row j.  Rows outside [a, b) are zeros.
template <int C>
__device__ __forceinline__ void load_operand(u32x4 (&f)[C / 16], const uint16_t *base, int64_t pitch, int row0, int a, int b, int d, int lane) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(base, b > 0 ? ((int64_t)(b - 1) * pitch + d) * 2 : 0);
    const int j = lane & 31, hh = lane >> 5, row = row0 + j;
#pragma unroll
    for (int s = 0; s < C / 16; ++s)
        f[s] = buf_load16(r, row >= a && row < b && 16 * s + 8 * hh < d ? (int)(row * pitch * 2) + 32 * s + 16 * hh : (int)kPast);
}

// ---------------------------------------------------------------------------------------
// Forward
// ---------------------------------------------------------------------------------------
// A workgroup is four waves of 32 queries; they share 64-key tiles of K and V, two of each in LDS (the next lands while one is used).
// The tiles are those of the sinks and those of the window of any of the 128 queries; a wave passes over tiles that its own
// queries do not see, and forms masks only on tiles that they see in part.
// P is rounded to the inputs' type for the second product: half a step, 2^-8 (bfloat16) or 2^-11 (binary16) of each weight at most, independent
// from weight to weight, which leaves the output as far off as its own rounding does.  Sums and statistics are 32 bits.
// Bound by power: 1 x 32 on 8 x 8192 x 128, window 4096, 128 sinks: 419 us, matrix pipes busy half of the cycles at 2.0 GHz (55 % in a large library
// product).  Waves in the mixed phase (masks, exponentials, second product) go first.
template <int D, int C, bool BF16>
__global__ void __launch_bounds__(256, D == 64 ? 4 : 2) smha_sink_fwd(const SinkParams p) {
    constexpr int NS = C / 16, NDT = C / 32, TB = 64 * D * 2;
    constexpr int PF = C == 128 ? 8 : 4;  // operands requested ahead
    __shared__ __attribute__((aligned(1024))) char smem[4 * TB];  // K[0], K[1], V[0], V[1]
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)smem;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 31, hh = lane >> 5;
    const float NEG_INF = -__builtin_inff();

    const QueryTile at(p);
    const int q0 = at.q0, b = at.b, h = at.h, hk = at.hk, bh = b * p.H + h;
    const Sequence s = sequence(p, b);
    const int window = p.window, n_sink = p.n_sink;

    // the workgroup's keys: sinks [0, .), then the window's tiles
    const int first = s.off + max(q0, s.qa), last = s.off + min(q0 + 128, s.qb) - 1;  // positions
    int n_head = 0, t0 = 0, n = 0, gap0 = 0, gap1 = 0;
    if (first <= last) {
        const int from = max(0, first - window + 1);
        n_head = (min(n_sink, from) + 63) / 64;
        t0 = max(from / 64, n_head);
        n = n_head + last / 64 + 1 - t0;
        if (n_sink < from) gap0 = n_sink, gap1 = from;  // keys that none of these queries sees
    }
    const int ksb = (int)p.ks.s * 2, vsb = (int)p.vs.s * 2;
    const u32x4 rK = make_rsrc4(p.K + b * p.ks.b + hk * p.ks.h, n ? ((int64_t)last * p.ks.s + p.d) * 2 : 0);
    const u32x4 rV = make_rsrc4(p.V + b * p.vs.b + hk * p.vs.h, n ? ((int64_t)last * p.vs.s + p.d) * 2 : 0);
    const TileLoad<D> loadK(w, lane, ksb, p.d), loadV(w, lane, vsb, p.d);
    auto key_of = [&](int t) __attribute__((always_inline)) { return 64 * (t < n_head ? t : t0 + t - n_head); };

    const int qw = q0 + 32 * w, qpos = s.off + qw + j;
    const bool exists = qw + j >= s.qa && qw + j < s.qb;
    const int wp0 = s.off + max(qw, s.qa), wp1 = s.off + min(qw + 32, s.qb) - 1;  // the wave's positions
    const bool whole = qw >= s.qa && qw + 32 <= s.qb;
    if (n > 0) {
        loadK(rK, lds0, w, key_of(0), ksb, gap0, gap1);
        loadV(rV, lds0 + 2 * TB, w, key_of(0), vsb, gap0, gap1);
    }
    u32x4 qf[NS];
    load_operand<C>(qf, p.Q + b * p.qs.b + h * p.qs.h, p.qs.s, qw, s.qa, s.qb, p.d, lane);

    const int rd = j * D * 2 + ((hh ^ swz_both<D>(j)) * 16);
    const int tr_row = 4 * hh + ((lane & 15) >> 2);
    const int tr = tr_row * D * 2 + ((swz_both<D>(tr_row) ^ (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1))) * 16) + (lane & 1) * 8;
    float m_run = NEG_INF, l_run = 0.f;
    const float thr = raised_over(p.c);
    f32x16 o[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) o[dt] = zeros16();
    tiles_landed();

    for (int t = 0; t < n; ++t) {
        const int par = t & 1, key = key_of(t);
        if (t + 1 < n) {
            loadK(rK, lds0 + (par ^ 1) * TB, w, key_of(t + 1), ksb, gap0, gap1);
            loadV(rV, lds0 + (2 + (par ^ 1)) * TB, w, key_of(t + 1), vsb, gap0, gap1);
        }
        if (wp0 <= wp1 && any_seen(wp0, wp1, key, key + 63, window, n_sink)) {
            const char *const Kt = smem + par * TB, *const Vt = smem + (2 + par) * TB;
            // acc[kt][r] = score of query j and key 32 kt + 8 (r / 4) + 4 hh + r % 4
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
            if (!(whole && all_seen(wp0, wp1, key, key + 63, window, n_sink))) {
                const uint64_t word = exists ? seen_keys(qpos, key, window, n_sink) : 0;
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    const u32x16 keep = keep_of((uint32_t)(word >> (32 * kt)) >> (4 * hh)), sc = __builtin_bit_cast(u32x16, acc[kt]);
                    acc[kt] = __builtin_bit_cast(f32x16, (sc & keep) | (~keep & 0xFF800000u));
                }
            }
            // probabilities are formed against a reference that is raised only where a score is over it by 8 / c: they stay below 2^8
            float mc = (m_run == NEG_INF ? 0.f : m_run) * p.c, mt = NEG_INF;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int r = 0; r < 16; ++r) mt = fmaxf(mt, acc[kt][r]);
            if (__builtin_amdgcn_ballot_w64(mt > m_run + thr) != 0) {
                mt = fmaxf(mt, __shfl_xor(mt, 32));
                const float m_new = fmaxf(m_run, mt), m_use = m_new == NEG_INF ? 0.f : m_new;
                const float alpha = fast_exp2((m_run - m_use) * p.c);
                m_run = m_new;
                mc = m_use * p.c;
                l_run *= alpha;
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) o[dt] *= alpha;
            }
            u32x4 pf[4];
            auto p_pair = [&](int cu, int q) __attribute__((always_inline)) {  // pair q of the 16 keys cu
                const float e0 = fast_exp2(fmaf(acc[cu >> 1][8 * (cu & 1) + 2 * q], p.c, -mc));
                const float e1 = fast_exp2(fmaf(acc[cu >> 1][8 * (cu & 1) + 2 * q + 1], p.c, -mc));
                pf[cu][q] = pack2<BF16>(e0, e1);
                l_run += e0 + e1;
            };
            auto v_frag = [&](int i) __attribute__((always_inline)) {  // i = cu NDT + dt: keys 16 cu + 8 a + 4 hh .., columns 32 dt + j
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
        }
        tiles_landed();
    }
    const float l = l_run + __shfl_xor(l_run, 32);
    if (p.lse && hh == 0 && qw + j < p.Sq)
        p.lse[(int64_t)bh * p.Sq + qw + j] = l != 0.f ? (m_run * p.c + __builtin_amdgcn_logf(l)) * 0.6931471805599453f : NEG_INF;
    const float inv = l != 0.f ? 1.0f / l : 0.f;  // (a sum that is not a number stays one)
    store_rows<D, C, BF16>(o, inv, smem + w * (32 * D * 2), lane, p.O + b * p.os.b + h * p.os.h, p.os.s, qw, p.Sq, p.d);
    if (p.rest) store_rows<D, C, BF16, true>(o, inv, smem + w * (32 * D * 2), lane, p.rest + (int64_t)bh * p.Sq * p.d, p.d, qw, p.Sq, p.d);
}

// ---------------------------------------------------------------------------------------
// Backward
// ---------------------------------------------------------------------------------------
// dQ: four waves of 32 queries over the same key tiles as the forward; a lane owns a query, so lse and delta are its own two registers.  It forms
// delta from the rows of dO that it holds anyway, and leaves both where smha_sink_bwd_kv, which runs after it, reads them; queries that do not
// exist get lse = inf, so that their probabilities are zero.  (A kernel of its own for that: 10 us of 114 for 4 x 12 x 1537 x 80.)
// delta from the rounded output alone is as far off as dS is by its own rounding: dQ and dK 1.52 times as far from 64 bits as an evaluation in
// 32 bits that is rounded once, 1.42 times with what the rounding left out.
// dS is rounded to the inputs' type for the product with K, as P is in the forward; FINE (see fine_ds): its rounding error is multiplied too.
// 563 us for the forward's case above, matrix pipes busy 59 %.
template <int D, int C, bool BF16, bool FINE>
__global__ void __launch_bounds__(256, 2) smha_sink_bwd_q(const SinkParams p) {
    constexpr int NS = C / 16, NDT = C / 32, TB = 64 * D * 2, PF = C == 128 ? 6 : 4;
    __shared__ __attribute__((aligned(1024))) char smem[4 * TB];  // K[0], K[1], V[0], V[1]
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)smem;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 31, hh = lane >> 5;

    const QueryTile at(p);
    const int q0 = at.q0, b = at.b, h = at.h, hk = at.hk, bh = b * p.H + h;
    const Sequence s = sequence(p, b);
    const int window = p.window, n_sink = p.n_sink;
    const int first = s.off + max(q0, s.qa), last = s.off + min(q0 + 128, s.qb) - 1;
    int n_head = 0, t0 = 0, n = 0, gap0 = 0, gap1 = 0;
    if (first <= last) {
        const int from = max(0, first - window + 1);
        n_head = (min(n_sink, from) + 63) / 64;
        t0 = max(from / 64, n_head);
        n = n_head + last / 64 + 1 - t0;
        if (n_sink < from) gap0 = n_sink, gap1 = from;
    }
    const int ksb = (int)p.ks.s * 2, vsb = (int)p.vs.s * 2;
    const u32x4 rK = make_rsrc4(p.K + b * p.ks.b + hk * p.ks.h, n ? ((int64_t)last * p.ks.s + p.d) * 2 : 0);
    const u32x4 rV = make_rsrc4(p.V + b * p.vs.b + hk * p.vs.h, n ? ((int64_t)last * p.vs.s + p.d) * 2 : 0);
    const TileLoad<D> loadK(w, lane, ksb, p.d), loadV(w, lane, vsb, p.d);
    auto key_of = [&](int t) __attribute__((always_inline)) { return 64 * (t < n_head ? t : t0 + t - n_head); };
    const int qw = q0 + 32 * w, qpos = s.off + qw + j;
    const bool exists = qw + j >= s.qa && qw + j < s.qb;
    const int wp0 = s.off + max(qw, s.qa), wp1 = s.off + min(qw + 32, s.qb) - 1;
    const bool whole = qw >= s.qa && qw + 32 <= s.qb;
    if (n > 0) {
        loadK(rK, lds0, w, key_of(0), ksb, gap0, gap1);
        loadV(rV, lds0 + 2 * TB, w, key_of(0), vsb, gap0, gap1);
    }
    u32x4 qf[NS], gf[NS];
    load_operand<C>(qf, p.Q + b * p.qs.b + h * p.qs.h, p.qs.s, qw, s.qa, s.qb, p.d, lane);
    load_operand<C>(gf, p.dO + b * p.gs.b + h * p.gs.h, p.gs.s, qw, s.qa, s.qb, p.d, lane);
    float delta = 0.f;
    {
        u32x4 of[NS], rest[NS];
        load_operand<C>(of, p.Oin + b * p.os.b + h * p.os.h, p.os.s, qw, s.qa, s.qb, p.d, lane);
        if (p.rest) load_operand<C>(rest, p.rest + (int64_t)bh * p.Sq * p.d, p.d, qw, s.qa, s.qb, p.d, lane);
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float lo = widen16<BF16>(of[i][e] & 0xFFFFu), hi = widen16<BF16>(of[i][e] >> 16);
                if (p.rest) lo += widen16<BF16>(rest[i][e] & 0xFFFFu), hi += widen16<BF16>(rest[i][e] >> 16);
                delta = fmaf(lo, widen16<BF16>(gf[i][e] & 0xFFFFu), delta);
                delta = fmaf(hi, widen16<BF16>(gf[i][e] >> 16), delta);
            }
        delta += __shfl_xor(delta, 32);
    }
    const float lse2 = exists ? p.lse[(int64_t)bh * p.Sq + qw + j] * 1.4426950408889634f : __builtin_inff();
    if (hh == 0) {
        const int64_t row = (int64_t)bh * p.Sqp + qw + j;
        p.stats[row] = lse2;
        p.stats[(int64_t)p.B * p.H * p.Sqp + row] = -delta;
    }

    const int rd = j * D * 2 + ((hh ^ swz_both<D>(j)) * 16);
    const int tr_row = 4 * hh + ((lane & 15) >> 2);
    const int tr = tr_row * D * 2 + ((swz_both<D>(tr_row) ^ (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1))) * 16) + (lane & 1) * 8;
    f32x16 dq[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) dq[dt] = zeros16();
    tiles_landed();
    for (int t = 0; t < n; ++t) {
        const int par = t & 1, key = key_of(t);
        if (t + 1 < n) {
            loadK(rK, lds0 + (par ^ 1) * TB, w, key_of(t + 1), ksb, gap0, gap1);
            loadV(rV, lds0 + (2 + (par ^ 1)) * TB, w, key_of(t + 1), vsb, gap0, gap1);
        }
        if (wp0 <= wp1) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
                const int k0 = key + 32 * kt;
                if (!any_seen(wp0, wp1, k0, k0 + 31, window, n_sink)) continue;
                const char *const Kt = smem + par * TB + kt * (TB / 2), *const Vt = smem + (2 + par) * TB + kt * (TB / 2);
                // The left operands of the three products, in their order: K's rows, V's rows, K's columns; requested PF products ahead.
                auto operand = [&](int n) __attribute__((always_inline)) {
                    if (n < 2 * NS) return *reinterpret_cast<const u32x4 *>((n < NS ? Kt : Vt) + (rd ^ (32 * (n % NS))));
                    const int cu = (n - 2 * NS) / NDT, dt = (n - 2 * NS) % NDT;
                    const u32x2 lo = lds_read_tr(reinterpret_cast<const uint16_t *>(Kt + ((tr ^ (64 * dt)) + 32 * cu * D)));
                    const u32x2 hi = lds_read_tr(reinterpret_cast<const uint16_t *>(Kt + ((tr ^ (64 * dt) ^ 32) + 32 * cu * D + 16 * D)));
                    return u32x4{lo[0], lo[1], hi[0], hi[1]};
                };
                constexpr int ALL = 2 * NS + 2 * NDT;
                u32x4 f[PF];
                f32x16 sc = zeros16(), dp = zeros16();
#pragma unroll
                for (int i = 0; i < PF; ++i) f[i] = operand(i);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    sc = mfma32<BF16>(f[i % PF], qf[i], sc);
                    if (i + PF < ALL) f[i % PF] = operand(i + PF);
                    __builtin_amdgcn_sched_barrier(0);
                }
                u32x16 keep;
                const bool part_seen = !(whole && all_seen(wp0, wp1, k0, k0 + 31, window, n_sink));
                if (part_seen) {
                    keep = keep_of((uint32_t)(exists ? seen_keys(qpos, k0, window, n_sink) : 0) >> (4 * hh));
                    const u32x16 raw = __builtin_bit_cast(u32x16, sc);
                    sc = __builtin_bit_cast(f32x16, (raw & keep) | (~keep & 0xFF800000u));
                }
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_setprio(1);
                // dP, and P from the scores
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    dp = mfma32<BF16>(f[(NS + i) % PF], gf[i], dp);
                    if (NS + i + PF < ALL) f[(NS + i) % PF] = operand(NS + i + PF);
#pragma unroll
                    for (int r = 16 * i / NS; r < 16 * (i + 1) / NS; ++r) sc[r] = fast_exp2(fmaf(sc[r], p.c, -lse2));
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (part_seen) {  // (where P is zero dP may be anything)
#pragma unroll
                    for (int r = 0; r < 16; ++r) dp[r] = sc[r] != 0.f ? dp[r] : delta;
                }
                u32x4 pf[2], left[2];
                auto ds_pair = [&](int q) __attribute__((always_inline)) {
                    const float lo = sc[2 * q] * (dp[2 * q] - delta), hi = sc[2 * q + 1] * (dp[2 * q + 1] - delta);
                    if constexpr (FINE) {
                        const Halves x = halves_of<BF16>(lo, hi);
                        pf[q >> 2][q & 3] = x.hi;
                        left[q >> 2][q & 3] = x.lo;
                    } else {
                        pf[q >> 2][q & 3] = pack2<BF16>(lo, hi);
                    }
                };
#pragma unroll
                for (int q = 0; q < 4; ++q) ds_pair(q);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 2 * NDT; ++i) {
                    dq[i % NDT] = mfma32<BF16>(f[(2 * NS + i) % PF], pf[i / NDT], dq[i % NDT]);
                    if constexpr (FINE) dq[i % NDT] = mfma32<BF16>(f[(2 * NS + i) % PF], left[i / NDT], dq[i % NDT]);
                    if (2 * NS + i + PF < ALL) f[(2 * NS + i) % PF] = operand(2 * NS + i + PF);
                    if (i < NDT) {  // the other 16 keys' dS, under these products
#pragma unroll
                        for (int q = 4 + 4 * i / NDT; q < 4 + 4 * (i + 1) / NDT; ++q) ds_pair(q);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_s_setprio(0);
            }
        }
        tiles_landed();
    }
    store_rows<D, C, BF16>(dq, p.scale, smem + w * (32 * D * 2), lane, p.dQ + b * p.dqs.b + h * p.dqs.h, p.dqs.s, qw, p.Sq, p.d);
}

// The queries that see a tile of 128 keys, as steps of 32 queries of one head: qt0 .. qt0 + nq - 1 of each of the G heads.
struct KeyTile {
    int qt0, nq;
};
__device__ __forceinline__ KeyTile key_tile(const SinkParams &p, const Sequence &s, int k0) {
    // the earliest query at or after the first key, the last that has the last key in its window
    const int k1 = min(k0 + 128, s.len) - 1;
    const int qa = max(s.qa, k0 - s.off);
    int qb = s.qb;
    if (k0 >= p.n_sink) qb = min(qb, k1 + p.window - s.off);
    if (k0 >= s.len || qa >= qb) return {0, 0};
    return {qa / 32, (qb - 1) / 32 - qa / 32 + 1};
}

// Parts of `chunk` steps at most, all alike.
__device__ __forceinline__ int parts_of(int steps, int cut, int chunk) { return max(1, min(cut, (steps + chunk - 1) / chunk)); }

// dK and dV: four waves of 32 keys each over 32-query tiles of Q and dO (and their lse and delta) in LDS, two of each.  A lane owns a key.
// At 128 columns a wave holds 128 registers of dK and dV; V's 32 beside them leave room for operands that are requested four products
// ahead, K's do not, and so K stays in LDS (with both in registers every product waited for its operand, and what had spilled was waited for
// with the tile in flight: 1062 us for the case above, 815 so, matrix pipes busy 49 %).  The exponentials run under the product that gives
// dP, the rest of dS under the one that gives dV.
// A tile's steps (its queries, head by head) may be cut into parts that other workgroups take: the sinks' tiles are seen by every
// query, and few key heads would leave most of the chip idle.  Parts go to memory in 32 bits and are added in order by smha_sink_sum.
template <int D, int C, bool BF16, bool FINE>
__global__ void __launch_bounds__(256, D == 64 && !FINE ? 3 : 2) smha_sink_bwd_kv(const SinkParams p) {
    constexpr int NS = C / 16, NDT = C / 32, TB = 32 * D * 2, PF = 4;
    __shared__ __attribute__((aligned(1024))) char smem[4 * TB + 4 * TB];  // K, Q[0], Q[1], dO[0], dO[1]
    __shared__ __attribute__((aligned(1024))) float stats[2][2][64];       // [buffer][lse, delta][query] (32 of 64)
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_void *)smem, stats0 = (uint32_t)(uintptr_t)(lds_void *)stats;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 31, hh = lane >> 5;

    // the sinks' tiles, then the others' last parts (which only the longest have), ..., their first
    const Turn turn(p);
    const int b = turn.b, hk = turn.hk, n_sinks = p.n_sink_tiles * p.cut_sink, n_rest = p.n_tiles - p.n_sink_tiles;
    int tile, part, cut, place;  // place: of its sums
    if (turn.item < n_sinks) {
        cut = p.cut_sink;
        part = turn.item / p.n_sink_tiles;
        tile = turn.item - part * p.n_sink_tiles;
        place = tile * cut + part;
    } else {
        cut = p.cut_rest;
        const int at = turn.item - n_sinks, turns = at / n_rest;
        part = cut - 1 - turns;
        place = p.rest_at + (at - turns * n_rest) * cut + part;
        tile = p.n_sink_tiles + at - turns * n_rest;
    }
    const Sequence s = sequence(p, b);
    const int window = p.window, n_sink = p.n_sink, k0 = tile * 128;
    const KeyTile kt = key_tile(p, s, k0);
    const int steps = kt.nq * p.G, parts = parts_of(steps, cut, tile < p.n_sink_tiles ? p.chunk_sink : p.chunk_rest);
    if (part >= parts) return;
    const int begin = (int)((int64_t)steps * part / parts), end = (int)((int64_t)steps * (part + 1) / parts);

    const int kw = k0 + 32 * w;
    const int qsb = (int)p.qs.s * 2, gsb = (int)p.gs.s * 2;
    const TileLoad<D, 32> loadQ(w, lane, qsb, p.d), loadG(w, lane, gsb, p.d);
    const int64_t rows = (int64_t)p.B * p.H * p.Sqp;
    constexpr int Q_AT = 4 * TB, G_AT = 6 * TB;
    auto request = [&](int g, int q, int par) __attribute__((always_inline)) {
        const int h = hk * p.G + g;
        const u32x4 rQ = make_rsrc4(p.Q + b * p.qs.b + h * p.qs.h, ((int64_t)(s.qb - 1) * p.qs.s + p.d) * 2);
        const u32x4 rG = make_rsrc4(p.dO + b * p.gs.b + h * p.gs.h, ((int64_t)(s.qb - 1) * p.gs.s + p.d) * 2);
        loadQ(rQ, lds0 + Q_AT + par * TB, w, q, qsb, 0, s.qa);
        loadG(rG, lds0 + G_AT + par * TB, w, q, gsb, 0, s.qa);
        if (w < 2) {  // (64 queries' worth, of which the first 32 are used)
            const u32x4 rS = make_rsrc4(p.stats + w * rows + ((int64_t)b * p.H + h) * p.Sqp, (int64_t)p.Sqp * 4);
            load_words_to_lds(rS, stats0 + (par * 2 + w) * 256, (uint32_t)((q + lane) * 4));
        }
    };
    int g = 0, qt = 0;
    u32x4 vf[NS];
    load_operand<C>(vf, p.V + b * p.vs.b + hk * p.vs.h, p.vs.s, kw, 0, s.len, p.d, lane);
    if (begin < end) {
        const int ksb = (int)p.ks.s * 2;
        const TileLoad<D, 128> loadK(w, lane, ksb, p.d);
        loadK(make_rsrc4(p.K + b * p.ks.b + hk * p.ks.h, ((int64_t)(s.len - 1) * p.ks.s + p.d) * 2), lds0, w, k0, ksb, 0, 0);
        g = begin / kt.nq;
        qt = begin - g * kt.nq;
        request(g, 32 * (kt.qt0 + qt), 0);
    }
    const int rd_ = j * D * 2 + ((hh ^ swz_both<D>(j)) * 16);
    const int tr_row = 4 * hh + ((lane & 15) >> 2);
    const int tr_ = tr_row * D * 2 + ((swz_both<D>(tr_row) ^ (2 * ((lane >> 4) & 1) + ((lane & 3) >> 1))) * 16) + (lane & 1) * 8;
    f32x16 dk[NDT], dv[NDT];
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) dk[dt] = dv[dt] = zeros16();
    tiles_landed();
    for (int t = begin; t < end; ++t) {
        const int par = (t - begin) & 1, q = 32 * (kt.qt0 + qt);
        if (++qt == kt.nq) qt = 0, ++g;
        if (t + 1 < end) request(g, 32 * (kt.qt0 + qt), par ^ 1);
        const int p0 = s.off + max(q, s.qa), p1 = s.off + min(q + 32, s.qb) - 1;
        if (p0 <= p1 && any_seen(p0, p1, kw, kw + 31, window, n_sink)) {
            int rd = rd_ + par * TB, rdk = rd_ + w * TB, tr = tr_ + par * TB;
            asm volatile("" : "+v"(rd), "+v"(rdk), "+v"(tr));  // (operand addresses are made here, not kept in registers across steps)
            auto row_frag = [&](int base, int at, int i) __attribute__((always_inline)) { return *reinterpret_cast<const u32x4 *>(smem + ((at ^ (32 * i)) + base)); };
            auto col_frag = [&](int base, int i) __attribute__((always_inline)) {  // i = cu NDT + dt: queries 16 cu + 8 a + 4 hh .., columns 32 dt + j
                const int cu = i / NDT, dt = i % NDT;
                const u32x2 lo = lds_read_tr(reinterpret_cast<const uint16_t *>(smem + ((tr ^ (64 * dt)) + (base + 32 * cu * D))));
                const u32x2 hi = lds_read_tr(reinterpret_cast<const uint16_t *>(smem + ((tr ^ (64 * dt) ^ 32) + (base + 32 * cu * D + 16 * D))));
                return u32x4{lo[0], lo[1], hi[0], hi[1]};
            };
            // The left operands of the step's products, in their order: Q's rows, dO's rows, dO's columns, Q's columns.
            auto operand = [&](int n) __attribute__((always_inline)) {
                return n < NS ? row_frag(Q_AT, rd, n) : n < 2 * NS ? row_frag(G_AT, rd, n - NS) : n < 2 * NS + 2 * NDT ? col_frag(G_AT, n - 2 * NS) : col_frag(Q_AT, n - 2 * NS - 2 * NDT);
            };
            constexpr int ALL = 2 * NS + 4 * NDT;
            u32x4 f[PF], fk[PF];
            auto next = [&](int n) __attribute__((always_inline)) {  // product n has its operand: the one PF on is requested
                if (n + PF < ALL) f[n % PF] = operand(n + PF);
            };
            // sc[r] = score of key j and query 8 (r / 4) + 4 hh + r % 4; dp: likewise, dP - delta, whose sum begins at -delta
            f32x16 sc = zeros16(), dp;
#pragma unroll
            for (int i = 0; i < PF; ++i) {
                if (i < NS) fk[i] = row_frag(0, rdk, i);
                f[i] = operand(i);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                sc = mfma32<BF16>(f[i % PF], fk[i % PF], sc);
                if (i + PF < NS) fk[i % PF] = row_frag(0, rdk, i + PF);
                next(i);
                __builtin_amdgcn_sched_barrier(0);
            }
            const float *const lse_at = &stats[par][0][4 * hh], *const delta_at = &stats[par][1][4 * hh];
            f32x4 of[2];  // lse: of[r4 & 1] is that of accumulators 4 r4 .. 4 r4 + 3
            of[0] = *reinterpret_cast<const f32x4 *>(lse_at);
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(delta_at + 8 * r4);
#pragma unroll
                for (int e = 0; e < 4; ++e) dp[4 * r4 + e] = x[e];
            }
            const bool part_seen = !all_seen(s.off + q, s.off + q + 31, kw, kw + 31, window, n_sink) || q < s.qa || q + 32 > s.qb;
            uint32_t word = ~0u;
            if (part_seen) {
                // queries at or after this key (or those that exist), and in whose window it is
                int me;  // (the lane's number, made here: kept across steps it would be one register too many)
                asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(me));
                const int k = kw + (me & 31), at = s.off + q;
                word = (k < n_sink ? ~0u : low_bits32(k + window - at)) & ~low_bits32(max(k - at, s.qa - q)) & low_bits32(s.qb - q);
                const u32x16 keep = keep_of(word >> (4 * hh)), raw = __builtin_bit_cast(u32x16, sc);
                sc = __builtin_bit_cast(f32x16, (raw & keep) | (~keep & 0xFF800000u));
            }
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_setprio(1);
            // dP, and P from the scores
            u32x4 pf[2], left[2];
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                dp = mfma32<BF16>(f[(NS + i) % PF], vf[i], dp);
                next(NS + i);
#pragma unroll
                for (int r = 16 * i / NS; r < 16 * (i + 1) / NS; ++r) {
                    if (r % 4 == 0 && r < 12) of[(r / 4 + 1) & 1] = *reinterpret_cast<const f32x4 *>(lse_at + 2 * r + 8);
                    sc[r] = fast_exp2(fmaf(sc[r], p.c, -of[(r / 4) & 1][r % 4]));
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) pf[i >> 2][i & 3] = pack2<BF16>(sc[2 * i], sc[2 * i + 1]);
            __builtin_amdgcn_sched_barrier(0);
            // dV, and dS from P and dP
#pragma unroll
            for (int i = 0; i < 2 * NDT; ++i) {
                dv[i % NDT] = mfma32<BF16>(f[(2 * NS + i) % PF], pf[i / NDT], dv[i % NDT]);
                next(2 * NS + i);
#pragma unroll
                for (int r = 16 * i / (2 * NDT); r < 16 * (i + 1) / (2 * NDT); ++r) dp[r] *= sc[r];
                __builtin_amdgcn_sched_barrier(0);
            }
            if (part_seen) {  // (where P is zero dP may be anything)
                const u32x16 keep = keep_of(word >> (4 * hh));
                dp = __builtin_bit_cast(f32x16, __builtin_bit_cast(u32x16, dp) & keep);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (FINE) {
                    const Halves x = halves_of<BF16>(dp[2 * i], dp[2 * i + 1]);
                    pf[i >> 2][i & 3] = x.hi;
                    left[i >> 2][i & 3] = x.lo;
                } else {
                    pf[i >> 2][i & 3] = pack2<BF16>(dp[2 * i], dp[2 * i + 1]);
                }
            }
#pragma unroll
            for (int i = 0; i < 2 * NDT; ++i) {
                dk[i % NDT] = mfma32<BF16>(f[(2 * NS + 2 * NDT + i) % PF], pf[i / NDT], dk[i % NDT]);
                if constexpr (FINE) dk[i % NDT] = mfma32<BF16>(f[(2 * NS + 2 * NDT + i) % PF], left[i / NDT], dk[i % NDT]);
                next(2 * NS + 2 * NDT + i);
                __builtin_amdgcn_sched_barrier(0);
            }
            __builtin_amdgcn_s_setprio(0);
        }
        tiles_landed();
    }
    if (parts == 1) {
        char *const slab = smem + w * TB;
        store_rows<D, C, BF16>(dv, 1.f, slab, lane, p.dV + b * p.dvs.b + hk * p.dvs.h, p.dvs.s, kw, p.Sk, p.d);
        store_rows<D, C, BF16>(dk, p.scale, slab, lane, p.dK + b * p.dks.b + hk * p.dks.h, p.dks.s, kw, p.Sk, p.d);
        return;
    }
    // [place][dV, dK][wave][4 accumulators][lane][4]
    float *const mine = p.parts + (((int64_t)(hk * p.B + b) * p.places + place) * 2 * 4 + w) * (C / 8) * 256 + lane * 4;
#pragma unroll
    for (int i = 0; i < C / 8; ++i) {
        *reinterpret_cast<f32x4 *>(mine + i * 256) = f32x4{dv[i / 4][4 * (i % 4)], dv[i / 4][4 * (i % 4) + 1], dv[i / 4][4 * (i % 4) + 2], dv[i / 4][4 * (i % 4) + 3]};
        *reinterpret_cast<f32x4 *>(mine + 4 * (C / 8) * 256 + i * 256) = f32x4{dk[i / 4][4 * (i % 4)], dk[i / 4][4 * (i % 4) + 1], dk[i / 4][4 * (i % 4) + 2], dk[i / 4][4 * (i % 4) + 3]};
    }
}

// The parts of a key tile that was cut, added in order, four on the way at once.  A workgroup takes one wave's 32 keys of dK or dV.  Where only
// tiles with sinks are cut it is launched for those alone.
template <int C, bool BF16>
__global__ void __launch_bounds__(256) smha_sink_sum(const SinkParams p) {
    const int tile_at = (int)blockIdx.x >> 3, w = (int)blockIdx.x & 3, is_k = ((int)blockIdx.x >> 2) & 1;
    const int tiles = p.cut_rest > 1 ? p.n_tiles : p.n_sink_tiles;
    const int bh = tile_at / tiles, tile = tile_at - bh * tiles, b = bh / p.Hkv, hk = bh - b * p.Hkv;
    const bool sink = tile < p.n_sink_tiles;
    const int cut = sink ? p.cut_sink : p.cut_rest;
    const int place = sink ? tile * cut : p.rest_at + (tile - p.n_sink_tiles) * cut;
    const Sequence s = sequence(p, b);
    const int parts = parts_of(key_tile(p, s, tile * 128).nq * p.G, cut, sink ? p.chunk_sink : p.chunk_rest);
    if (parts == 1) return;  // it was written whole
    uint16_t *const out = is_k ? p.dK + b * p.dks.b + hk * p.dks.h : p.dV + b * p.dvs.b + hk * p.dvs.h;
    const int64_t pitch = is_k ? p.dks.s : p.dvs.s;
    const float factor = is_k ? p.scale : 1.f;
    const float *const from = p.parts + (((int64_t)(hk * p.B + b) * p.places + place) * 8 + is_k * 4 + w) * (C / 8) * 256;
    for (int i = threadIdx.x; i < C / 8 * 64; i += 256) {
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        for (int c0 = 0; c0 < parts; c0 += 4) {
            f32x4 x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = *reinterpret_cast<const f32x4 *>(from + (int64_t)min(c0 + u, parts - 1) * 8 * (C / 8) * 256 + i * 4);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (c0 + u < parts) sum += x[u];
        }
        const int quad = i >> 6, lane = i & 63, key = tile * 128 + 32 * w + (lane & 31), col = 8 * quad + 4 * (lane >> 5);
        if (key < p.Sk && col < p.d)
            *reinterpret_cast<u32x2 *>(out + key * pitch + col) = u32x2{pack2<BF16>(sum[0] * factor, sum[1] * factor), pack2<BF16>(sum[2] * factor, sum[3] * factor)};
    }
}

// ---------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------
static bool strides_fit(const int64_t *s, int64_t rows, int d) {
    if (!s) return rows * d * 2 < ((int64_t)1 << 31);
    // (a head is addressed through 32-bit offsets; batch and head strides may be zero where a tensor is only read)
    return s[0] % 8 == 0 && s[1] % 8 == 0 && s[2] % 8 == 0 && s[0] >= 0 && s[1] >= 0 && s[2] >= d && (rows * s[2] + d) * 2 < ((int64_t)1 << 31);
}

static Strides strides_of(const int64_t *s, int64_t heads, int64_t rows, int d) {
    return s ? Strides{s[0], s[1], s[2]} : Strides{heads * rows * d, rows * d, d};
}

// A launch has less than 2^32 threads; workgroups are 256, in a multiple of eight.
static bool grid_fits(int64_t groups) { return groups + 8 < (1 << 24); }

// What both directions check and fill in.
static smha_status_t sink_params(SinkParams &sp, int B, int H, int Hkv, int Sq, int Sk, int d, smha_dtype_t dtype, const int32_t *offsets, const int32_t *lengths,
                                 int window, int n_sink, float scale) {
    if (B < 1 || H < 1 || Hkv < 1 || Sq < 1 || Sk < 1 || window < 0 || n_sink < 0) return SMHA_ERR_INVALID_ARG;
    if (H % Hkv) return SMHA_ERR_SHAPE;
    if (dtype != SMHA_F16 && dtype != SMHA_BF16) return SMHA_ERR_UNSUPPORTED;
    if (d < 8 || d > 128 || d % 8) return SMHA_ERR_UNSUPPORTED;
    if (Sq >= kRowsEnd || Sk >= kRowsEnd) return SMHA_ERR_UNSUPPORTED;
    // (work items are numbered in 32 bits)
    if ((int64_t)B * H > (1 << 24) || (int64_t)B * H * (std::max(Sq, Sk) / 64 + 2) > (1 << 28)) return SMHA_ERR_UNSUPPORTED;
    if (!grid_fits((int64_t)B * H * ((Sq + 127) / 128))) return SMHA_ERR_UNSUPPORTED;
    sp.B = B; sp.H = H; sp.Hkv = Hkv; sp.G = H / Hkv; sp.Sq = Sq; sp.Sk = Sk; sp.d = d;
    sp.window = window == 0 || window > Sk ? Sk : window;
    sp.n_sink = std::min(n_sink, Sk);
    sp.offsets = offsets; sp.lengths = lengths;
    sp.scale = scale > 0.f ? scale : 1.0f / std::sqrt((float)d);
    sp.c = sp.scale * 1.4426950408889634f;
    sp.Sqp = (Sq + 127) / 128 * 128;
    return SMHA_OK;
}

// How dK and dV are cut.  512 workgroups fit the chip, and a part costs 8 D 128 bytes of traffic: parts of a little more than a 512th of all steps
// even out the load, longer ones leave units idle, shorter ones are slower again.  `all` counts every tile of a window as a whole one; without a
// window tiles differ more and may be longer, since the longest begin first.  A tile with sinks is its queries' only in one or two of its
// waves, whose steps are short: its parts are a little longer.  us of a backward pass, parts of 0.7, 1, 1.25, 1.5 and 2 of a 512th of the true steps at most: 2 x 16 on
// 4 x 4096 x 128, window 1024: 273, 282, 258, 264, 294; 1 x 32 on 8 x 4096 x 64, window 512: 121, 119, 118, 126, 124; 1 x 8 on 1 x 8192 x 128, window 1024: 177, 188, 160,
// 163, 174 (359 whole); all before: 1 x 20 on 4 x 6000 x 128: 650, 713, 633, 654, 725 (1130 whole); 2 x 32 on 8 x 4096 x 128: 931, 989, 953, 948, 1002; 3 x
// 10 on 5 x 3000 x 128: 296, 309, 296, 288, 307; 7 x 12 x 1000 x 64: 89, 86, 85, 72, 72.
static void sink_cuts(SinkParams &sp) {
    const int64_t nq = (sp.Sq + 31) / 32;
    const int64_t near = std::min<int64_t>(nq, (sp.window + 127 + 31) / 32 + 1);
    sp.n_tiles = (sp.Sk + 127) / 128;
    sp.n_sink_tiles = sp.window < sp.Sk ? (sp.n_sink + 127) / 128 : 0;
    const int64_t all = (int64_t)sp.B * sp.Hkv * sp.G * (sp.n_sink_tiles * nq + (sp.n_tiles - sp.n_sink_tiles) * (sp.window < sp.Sk ? near : (nq + 1) / 2));
    const int64_t parts = sp.window < sp.Sk ? 448 : 341;
    sp.chunk_rest = (int)std::max<int64_t>(8, (all + parts - 1) / parts);
    sp.chunk_sink = (int)std::max<int64_t>(12, (all + 399) / 400);
    sp.cut_sink = (int)((nq * sp.G + sp.chunk_sink - 1) / sp.chunk_sink);
    sp.cut_rest = (int)((near * sp.G + sp.chunk_rest - 1) / sp.chunk_rest);
    if (sp.n_sink_tiles == 0) sp.cut_sink = 1;
    // (with a few sinks theirs is often the only tile that is cut: 1 x 32 x 131072 x 128, window 1024, would keep 4 GiB for 8 MiB of sums)
    sp.rest_at = sp.cut_sink > 1 ? (int)((int64_t)sp.n_sink_tiles * sp.cut_sink) : 0;
    sp.places = (int)(sp.rest_at + (sp.cut_rest > 1 ? (int64_t)(sp.n_tiles - sp.n_sink_tiles) * sp.cut_rest : 0));
}

static int64_t sink_stats_bytes(const SinkParams &sp) { return (int64_t)2 * sp.B * sp.H * sp.Sqp * 4; }
static int64_t sink_items(const SinkParams &sp) {
    return (int64_t)sp.B * sp.Hkv * ((int64_t)sp.n_sink_tiles * sp.cut_sink + (int64_t)(sp.n_tiles - sp.n_sink_tiles) * sp.cut_rest);
}
static bool sink_grids_fit(const SinkParams &sp) {
    return grid_fits(sink_items(sp)) && ((sp.cut_sink == 1 && sp.cut_rest == 1) || grid_fits((int64_t)8 * sp.B * sp.Hkv * sp.n_tiles));
}

// Whether dS goes into dQ and dK with what its rounding leaves out.  dQ and dK of rounded dS are 1.44 times as far from 64 bits as their own
// rounding on average; of few queries, where a few large rows make most of the norm, up to 1.50 (2 x 12 x 68 x 64).  There both halves are
// multiplied, a product more of three and of four: 1.05 (1.10 where windows are shortest).  us of a backward pass without and with them: 2 x 4 x 128 x 64, window 16: 15.6,
// 16.4; 1 x 8 x 1024 x 64, window 256: 28.1, 30.3; 1 x 8 x 700 x 128: 47.8, 52.4; 1 x 2 x 1400 x 128: 68.7, 76.7 (most of which the host's 65 us
// for a pass hide).  Of more queries errors average out, and products are what such a call lasts.
static bool fine_ds(const SinkParams &sp) { const int64_t queries = (int64_t)sp.B * sp.H * sp.Sq;
    return queries <= 8192 && queries * std::min<int64_t>(sp.Sk, (int64_t)sp.window + sp.n_sink) <= 1 << 22; }

static int sink_width(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 96 ? 96 : 128; }

template <int D, int C, bool BF16> static hipError_t launch_sink_fwd(SinkParams &sp, hipStream_t stream) {
    sp.per = sp.G * ((sp.Sq + 127) / 128);
    sp.together = sink_together(sp.B * sp.Hkv, sp.per, 128);
    hipLaunchKernelGGL((smha_sink_fwd<D, C, BF16>), dim3((unsigned)(sp.B * sp.Hkv * sp.per)), dim3(256), 0, stream, sp);
    return hipGetLastError();
}

template <int D, int C, bool BF16, bool FINE> static hipError_t launch_sink_bwd(SinkParams &sp, hipStream_t stream) {
    sp.per = sp.G * ((sp.Sq + 127) / 128);
    sp.together = sink_together(sp.B * sp.Hkv, sp.per, 128);
    hipLaunchKernelGGL((smha_sink_bwd_q<D, C, BF16, FINE>), dim3((unsigned)(sp.B * sp.Hkv * sp.per)), dim3(256), 0, stream, sp);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    sp.per = (int)(sink_items(sp) / (sp.B * sp.Hkv));
    sp.together = sink_together(sp.B * sp.Hkv, sp.per, 256);
    hipLaunchKernelGGL((smha_sink_bwd_kv<D, C, BF16, FINE>), dim3((unsigned)(sp.B * sp.Hkv * sp.per)), dim3(256), 0, stream, sp);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if (sp.cut_sink > 1 || sp.cut_rest > 1) hipLaunchKernelGGL((smha_sink_sum<C, BF16>), dim3((unsigned)(8 * sp.B * sp.Hkv * (sp.cut_rest > 1 ? sp.n_tiles : sp.n_sink_tiles))), dim3(256), 0, stream, sp);
    return hipGetLastError();
}

}  // namespace smha

using namespace smha;

extern "C" smha_status_t smha_sink_forward(const void *Q, const void *K, const void *V, void *O, float *lse, void *O_rest, int B, int H, int Hkv, int Sq, int Sk, int d,
                                           smha_dtype_t dtype, const int64_t q_strides[3], const int64_t k_strides[3], const int64_t v_strides[3],
                                           const int64_t o_strides[3], const int32_t *offsets, const int32_t *lengths, int window, int n_sink, float scale,
                                           void *hip_stream) {
    if (!Q || !K || !V || !O) return SMHA_ERR_INVALID_ARG;
    SinkParams sp{};
    const smha_status_t st = sink_params(sp, B, H, Hkv, Sq, Sk, d, dtype, offsets, lengths, window, n_sink, scale);
    if (st != SMHA_OK) return st;
    if (((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O | (uintptr_t)O_rest) & 15) return SMHA_ERR_UNSUPPORTED;
    if (!strides_fit(q_strides, Sq + 128, d) || !strides_fit(k_strides, (int64_t)Sk + 128, d) || !strides_fit(v_strides, (int64_t)Sk + 128, d) || !strides_fit(o_strides, Sq + 128, d) ||
        !apart(o_strides, B, H, Sq, d))
        return SMHA_ERR_UNSUPPORTED;
    sp.Q = (const uint16_t *)Q; sp.K = (const uint16_t *)K; sp.V = (const uint16_t *)V; sp.O = (uint16_t *)O; sp.lse = lse; sp.rest = (uint16_t *)O_rest;
    sp.qs = strides_of(q_strides, H, Sq, d); sp.ks = strides_of(k_strides, Hkv, Sk, d); sp.vs = strides_of(v_strides, Hkv, Sk, d); sp.os = strides_of(o_strides, H, Sq, d);
    const hipStream_t stream = (hipStream_t)hip_stream;
    auto go = [&](auto bf16) {
        constexpr bool BF = decltype(bf16)::value;
        switch (sink_width(d)) {
            case 32: return launch_sink_fwd<64, 32, BF>(sp, stream);
            case 64: return launch_sink_fwd<64, 64, BF>(sp, stream);
            case 96: return launch_sink_fwd<128, 96, BF>(sp, stream);
            default: return launch_sink_fwd<128, 128, BF>(sp, stream);
        }
    };
    const hipError_t e = dtype == SMHA_BF16 ? go(std::true_type()) : go(std::false_type());
    return e == hipSuccess ? SMHA_OK : SMHA_ERR_HIP;
}

extern "C" smha_status_t smha_sink_workspace(int B, int H, int Hkv, int Sq, int Sk, int d, int window, int n_sink, size_t *need) {
    if (!need) return SMHA_ERR_INVALID_ARG;
    SinkParams sp{};
    const smha_status_t st = sink_params(sp, B, H, Hkv, Sq, Sk, d, SMHA_F16, nullptr, nullptr, window, n_sink, 0.f);
    if (st != SMHA_OK) return st;
    sink_cuts(sp);
    if (!sink_grids_fit(sp)) return SMHA_ERR_UNSUPPORTED;
    *need = (size_t)(sink_stats_bytes(sp) + (int64_t)B * Hkv * sp.places * 2 * 128 * sink_width(d) * 4);
    return SMHA_OK;
}

extern "C" smha_status_t smha_sink_backward(const void *Q, const void *K, const void *V, const void *O, const void *O_rest, const float *lse, const void *dO, void *dQ, void *dK, void *dV,
                                            int B, int H, int Hkv, int Sq, int Sk, int d, smha_dtype_t dtype, const int64_t q_strides[3],
                                            const int64_t k_strides[3], const int64_t v_strides[3], const int64_t o_strides[3], const int64_t do_strides[3],
                                            const int64_t dq_strides[3], const int64_t dk_strides[3], const int64_t dv_strides[3], const int32_t *offsets,
                                            const int32_t *lengths, int window, int n_sink, float scale, void *workspace, size_t workspace_bytes,
                                            void *hip_stream) {
    if (!Q || !K || !V || !O || !lse || !dO || !dQ || !dK || !dV || !workspace) return SMHA_ERR_INVALID_ARG;
    SinkParams sp{};
    const smha_status_t st = sink_params(sp, B, H, Hkv, Sq, Sk, d, dtype, offsets, lengths, window, n_sink, scale);
    if (st != SMHA_OK) return st;
    size_t need = 0;
    const smha_status_t fits = smha_sink_workspace(B, H, Hkv, Sq, Sk, d, window, n_sink, &need);
    if (fits != SMHA_OK) return fits;
    if (workspace_bytes < need) return SMHA_ERR_INVALID_ARG;
    if (((uintptr_t)Q | (uintptr_t)K | (uintptr_t)V | (uintptr_t)O | (uintptr_t)O_rest | (uintptr_t)dO | (uintptr_t)dQ | (uintptr_t)dK | (uintptr_t)dV | (uintptr_t)workspace) & 15)
        return SMHA_ERR_UNSUPPORTED;
    for (const int64_t *s : {q_strides, o_strides, do_strides, dq_strides})
        if (!strides_fit(s, Sq + 128, d)) return SMHA_ERR_UNSUPPORTED;
    for (const int64_t *s : {k_strides, v_strides, dk_strides, dv_strides})
        if (!strides_fit(s, (int64_t)Sk + 128, d)) return SMHA_ERR_UNSUPPORTED;
    if (!apart(dq_strides, B, H, Sq, d) || !apart(dk_strides, B, Hkv, Sk, d) || !apart(dv_strides, B, Hkv, Sk, d)) return SMHA_ERR_UNSUPPORTED;
    sink_cuts(sp);
    sp.Q = (const uint16_t *)Q; sp.K = (const uint16_t *)K; sp.V = (const uint16_t *)V; sp.Oin = (const uint16_t *)O; sp.rest = (uint16_t *)const_cast<void *>(O_rest); sp.dO = (const uint16_t *)dO;
    sp.dQ = (uint16_t *)dQ; sp.dK = (uint16_t *)dK; sp.dV = (uint16_t *)dV; sp.lse = const_cast<float *>(lse);
    sp.qs = strides_of(q_strides, H, Sq, d); sp.ks = strides_of(k_strides, Hkv, Sk, d); sp.vs = strides_of(v_strides, Hkv, Sk, d);
    sp.os = strides_of(o_strides, H, Sq, d); sp.gs = strides_of(do_strides, H, Sq, d);
    sp.dqs = strides_of(dq_strides, H, Sq, d); sp.dks = strides_of(dk_strides, Hkv, Sk, d); sp.dvs = strides_of(dv_strides, Hkv, Sk, d);
    sp.stats = (float *)workspace;
    sp.parts = (float *)((char *)workspace + sink_stats_bytes(sp));
    const hipStream_t stream = (hipStream_t)hip_stream;
    auto go = [&](auto bf16, auto fine) {
        constexpr bool BF = decltype(bf16)::value, FINE = decltype(fine)::value;
        switch (sink_width(d)) {
            case 32: return launch_sink_bwd<64, 32, BF, FINE>(sp, stream);
            case 64: return launch_sink_bwd<64, 64, BF, FINE>(sp, stream);
            case 96: return launch_sink_bwd<128, 96, BF, FINE>(sp, stream);
            default: return launch_sink_bwd<128, 128, BF, FINE>(sp, stream);
        }
    };
    auto by_type = [&](auto fine) { return dtype == SMHA_BF16 ? go(std::true_type(), fine) : go(std::false_type(), fine); };
    const hipError_t e = fine_ds(sp) ? by_type(std::true_type()) : by_type(std::false_type());
    return e == hipSuccess ? SMHA_OK : SMHA_ERR_HIP;
}
