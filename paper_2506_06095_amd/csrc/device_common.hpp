// Device code that the kernel files share: vector types, matrix instructions, conversions, loads into LDS and the swizzles of
// the tiles there.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "smha.h"

namespace smha {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct Strides {
    int64_t b, h, s;
};

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

template <bool BF16>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c) {
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                       __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                      __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// two fp32 -> one dword of two 16-bit floats (round to nearest even), lo = a
template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    if constexpr (BF16) {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        bf2 v = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, v);
    } else {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        h2 v = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, v);
    }
}

template <bool BF16>
__device__ __forceinline__ float widen16(uint32_t bits16) {
    if constexpr (BF16) {
        return __builtin_bit_cast(float, bits16 << 16);
    } else {
        return (float)__builtin_bit_cast(_Float16, (uint16_t)bits16);
    }
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t make_rsrc(const void *base, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, 0x00020000);
}
__device__ __forceinline__ u32x4 buf_load16(__amdgpu_buffer_rsrc_t r, int byte_off) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, byte_off, 0, 0);  // out of range -> zeros
}
// (rows of 256 bytes or more: a row's chunks are permuted inside each aligned group of 16)
// Rows of an odd number of 64-byte groups (32, 96 and 160 columns) spread by themselves: four consecutive rows start in
// the four groups of a 256-byte window, so V needs no swizzle, and for K the chunks of each aligned group of four are permuted
// by which of four such row quadruples the row is in.  (Bank conflicts per LDS cycle: first form at 96 columns 0.03, wave form 0.2 to 0.3
// at 96, third form 0.33 at 160; at 64 and 128 columns 0.01 to 0.09.)
template <int D> constexpr bool kOddRows = D % 64 == 32;
template <int D> __device__ __forceinline__ int swz_k(int row) {
    if constexpr (kOddRows<D>) return (row >> 2) & 3;
    else if constexpr (D >= 128) return row & 15;
    else return (row / (128 / D)) & (D / 8 - 1);
}
template <int D> __device__ __forceinline__ int swz_v(int row) {
    if constexpr (kOddRows<D>) return 0;
    else if constexpr (D >= 128) return (row & 3) << 2;
    else return ((row / (128 / D)) & (D / 32 - 1)) << 2;
}
// A swizzled row's chunk pair 2 s (+ lane part) and its 64-byte group g, from the byte address of pair / group 0.
template <int D> __device__ __forceinline__ int at_pair(int base, int s) {
    if constexpr (kOddRows<D>) return (base ^ (32 * (s & 1))) + 64 * (s >> 1);
    else return base ^ (32 * s);
}
template <int D> __device__ __forceinline__ int at_group(int base, int g) {
    if constexpr (kOddRows<D>) return base + 64 * g;
    else return base ^ (64 * g);
}
typedef __attribute__((address_space(3))) void lds_void;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Buffer descriptor as four dwords (base, no stride, size in bytes, raw 32-bit data format) for the
// loads below; out-of-range offsets return zeros.
__device__ __forceinline__ u32x4 make_rsrc4(const void *base, int64_t bytes) {
    const uint64_t a = (uint64_t)base;
    return u32x4{(uint32_t)a, (uint32_t)(a >> 32) & 0xFFFFu, (uint32_t)bytes, 0x00020000u};
}
// 64 lanes x 16 bytes from per-lane global offsets into 1 KiB of LDS at byte address `lds`
// (lane l -> lds + 16 l), bypassing registers.  Written as an instruction: the compiler's own
// form makes it track which LDS object each load in flight may write, which forces the two
// buffers of a pair to be compile-time objects (a loop body per buffer) and adds full waits
// wherever it cannot tell; here every wait for these loads is an explicit s_waitcnt in the
// kernel (memory operations retire in order, so the compiler's own vmcnt waits stay safe).
// M0 is written here without being listed as clobbered: the compiler reserves it, sets it right
// before each use of its own and rejects it on a clobber list with a warning.
__device__ __forceinline__ void load_to_lds(u32x4 rsrc, uint32_t lds, int byte_off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(byte_off), "s"(rsrc) : "memory");
}
template <int LOADS>
__device__ __forceinline__ void wait_all_but() {  // every memory operation of the wave but the last LOADS has finished
    asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LOADS) : "memory");
}
// 64 lanes x 4 bytes from per-lane global offsets into 256 bytes of LDS (see load_to_lds)
__device__ __forceinline__ void load_words_to_lds(u32x4 rsrc, uint32_t lds, uint32_t byte_off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(byte_off), "s"(rsrc) : "memory");
}
// transposing LDS read: see the kernel comment; returns this lane's 4 keys of one column
__device__ __forceinline__ u32x2 lds_read_tr(const uint16_t *src) {
    s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)src);
    return __builtin_bit_cast(u32x2, v);
}

// Read-only plan data at a wave-uniform address: through the constant address space, so the
// load is a scalar one (a vector load would have to drain the wave's outstanding tile loads and
// output stores before its value could be used).
template <typename T>
__device__ __forceinline__ T uniform_load(const T *ptr) {
    static_assert(sizeof(T) == 4 || sizeof(T) == 8 || sizeof(T) == 16, "one, two or four dwords");
    if constexpr (sizeof(T) == 4) {
        typedef const uint32_t __attribute__((address_space(4))) *const_ptr;
        return __builtin_bit_cast(T, *(const_ptr)(uintptr_t)ptr);
    } else if constexpr (sizeof(T) == 8) {
        typedef const u32x2 __attribute__((address_space(4))) *const_ptr;
        return __builtin_bit_cast(T, *(const_ptr)(uintptr_t)ptr);
    } else {
        typedef const u32x4 __attribute__((address_space(4))) *const_ptr;
        return __builtin_bit_cast(T, *(const_ptr)(uintptr_t)ptr);
    }
}

template <int OUT>  // smha_dtype_t of the output
__device__ __forceinline__ void store4(void *O, int64_t elem_off, float a, float b, float c, float d) {
    if constexpr (OUT == SMHA_F32) {
        f32x4 v = {a, b, c, d};
        *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(O) + elem_off) = v;
    } else {
        u32x2 v = {pack2<OUT == SMHA_BF16>(a, b), pack2<OUT == SMHA_BF16>(c, d)};
        *reinterpret_cast<u32x2 *>(reinterpret_cast<uint16_t *>(O) + elem_off) = v;
    }
}

// --- for kernels whose masks are arithmetic on positions
// How far over the running reference a score may be before that is raised: 2^8 in the probabilities.  (Finite for every scale: with a reference
// of -inf the comparison has to hold.)
__device__ __forceinline__ float raised_over(float c) { return fminf(8.0f / c, 3e38f); }
constexpr uint32_t kNoChunk = 0x80000000u;  // a column that the head does not have: past every buffer, with any row's offset added
constexpr uint32_t kPast = 0x7FFFFF00u;     // a row that is not to be read

// Both of a tile's reading orders: 16 rows at one chunk (16-byte reads), and 4 rows x 4 chunks (transposing reads).  The two low bits
// of the row choose the aligned group of four chunks, the next two the place in it.
template <int D> __device__ __forceinline__ int swz_both(int row) {
    if constexpr (D == 128) return ((row & 3) << 2) | ((row >> 2) & 3);
    else return ((row & 2) << 1) | ((row >> 2) & 3);
}

// bits 0 .. n - 1
__device__ __forceinline__ uint64_t low_bits(int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }
__device__ __forceinline__ uint32_t low_bits32(int n) { return n <= 0 ? 0 : n >= 32 ? ~0u : (1u << n) - 1; }
typedef uint32_t u32x16 __attribute__((ext_vector_type(16)));
// all ones where accumulator r of the lane (8 (r / 4) + r % 4 of the lane's half) has its bit set
__device__ __forceinline__ u32x16 keep_of(uint32_t bits) {
    u32x16 keep;
#pragma unroll
    for (int r = 0; r < 16; ++r) keep[r] = (uint32_t)__builtin_amdgcn_sbfe((int)bits, 8 * (r / 4) + (r % 4), 1);
    return keep;
}
__device__ __forceinline__ f32x16 zeros16() { return f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}; }

// A tile of ROWS rows into LDS by a workgroup's four waves: wave w brings the 1 KiB blocks w, w + 4, ...
template <int D, int ROWS = 64> struct TileLoad {
    static constexpr int CPR = D / 8, LPW = CPR * ROWS / 256, RSTEP = 4 * 64 / CPR;  // chunks a row, loads a wave, rows between two of its loads
    uint32_t go;  // the lane's offset in the wave's first block
    int row;
    __device__ __forceinline__ TileLoad(int w, int lane, int row_bytes, int d) {
        row = (w * 64 + lane) / CPR;
        const int c = (lane % CPR) ^ swz_both<D>(row);
        go = c < (d >> 3) ? (uint32_t)(row * row_bytes + c * 16) : kNoChunk;
    }
    // rows r0 ..; those in [gap0, gap1) read as zeros, as do those past the buffer
    __device__ __forceinline__ void operator()(u32x4 rsrc, uint32_t lds, int w, int r0, int row_bytes, int gap0, int gap1) const {
#pragma unroll
        for (int i = 0; i < LPW; ++i) {
            const int r = r0 + row + i * RSTEP;
            const uint32_t at = go + (uint32_t)((r0 + i * RSTEP) * row_bytes);
            load_to_lds(rsrc, lds + (w + 4 * i) * 1024, (int)(r >= gap0 && r < gap1 ? kPast : at));
        }
    }
};

// The next tile is in LDS and this one may be overwritten, for every wave.  (The last line keeps reads of LDS where they are: for the
// compiler the barrier touches no memory.)
__device__ __forceinline__ void tiles_landed() {
    __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// --- what their entry points check (strides {batch, head, token}, null: packed)
// Rows of a head: 2^31 bytes hold fewer than this.  (With it, products of sizes fit their integers.)
constexpr int kRowsEnd = 1 << 27;
// Rows that are written must not share memory: from the closest rows outwards, each dimension steps over all that those before it span.
inline bool apart(const int64_t *s, int64_t B, int64_t H, int64_t rows, int64_t d) {
    if (!s) return true;
    struct {
        int64_t n, step;
    } dims[3] = {{B, s[0]}, {H, s[1]}, {rows, s[2]}};
    std::sort(dims, dims + 3, [](const auto &x, const auto &y) { return x.step < y.step; });
    __int128 span = d;
    for (const auto &dim : dims)
        if (dim.n > 1) {
            if (dim.step < span) return false;
            span += (__int128)dim.step * (dim.n - 1);
        }
    return true;
}

}  // namespace smha
