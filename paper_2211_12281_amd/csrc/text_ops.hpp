// Shared by the kernels of the text side (embed.hip, quantize.hip, matmul_quantized.hip): groups of eight elements of a row, and the dropout
// generator.
#pragma once
#include "kge_internal.h"

typedef uint32_t kge_u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t kge_u32x4 __attribute__((ext_vector_type(4)));
typedef float kge_f32x4 __attribute__((ext_vector_type(4)));

// A thread's share of a row is a group of eight consecutive columns.  Rows may start anywhere (odd widths, odd strides): vector memory
// instructions of gfx950 take any byte address, so the types below only promise the element's own alignment and there is one
// path for all rows; a group that the row's end cuts goes element by element.
typedef uint32_t kge_u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t kge_u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t kge_u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef float kge_f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));

template <bool BF16> __device__ __forceinline__ void kge_load8(const void *row, int64_t col, int n, float (&v)[8]) {
    if (n >= 8) {
        if constexpr (BF16) {
            const kge_u32x4 r = *(const kge_u32x4_a2 *)((const uint16_t *)row + col);
#pragma unroll
            for (int u = 0; u < 4; ++u) { v[2 * u] = __uint_as_float(r[u] << 16); v[2 * u + 1] = __uint_as_float(r[u] & 0xffff0000u); }
        } else {
            const kge_f32x4 a = *(const kge_f32x4_a4 *)((const float *)row + col), b = *(const kge_f32x4_a4 *)((const float *)row + col + 4);
#pragma unroll
            for (int u = 0; u < 4; ++u) { v[u] = a[u]; v[4 + u] = b[u]; }
        }
    } else {
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            v[u] = 0.f;
            if (u < n) v[u] = BF16 ? __uint_as_float((uint32_t)((const uint16_t *)row)[col + u] << 16) : ((const float *)row)[col + u];
        }
    }
}

// The same in two steps, for loads that stay in flight: a whole group's words, and its values.
template <bool BF16> struct KgeRaw8 { kge_u32x4 w[BF16 ? 1 : 2]; };
template <bool BF16> __device__ __forceinline__ KgeRaw8<BF16> kge_raw8(const void *row, int64_t col) {
    KgeRaw8<BF16> r;
    if constexpr (BF16) r.w[0] = *(const kge_u32x4_a2 *)((const uint16_t *)row + col);
    else {
        r.w[0] = *(const kge_u32x4_a4 *)((const uint32_t *)row + col);
        r.w[1] = *(const kge_u32x4_a4 *)((const uint32_t *)row + col + 4);
    }
    return r;
}
template <bool BF16> __device__ __forceinline__ void kge_values8(const KgeRaw8<BF16> &r, float (&v)[8]) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if constexpr (BF16) { v[2 * u] = __uint_as_float(r.w[0][u] << 16); v[2 * u + 1] = __uint_as_float(r.w[0][u] & 0xffff0000u); }
        else { v[u] = __uint_as_float(r.w[0][u]); v[4 + u] = __uint_as_float(r.w[1][u]); }
    }
}

// STREAM: past the caches, for results that are larger than they are
template <bool BF16, bool STREAM = false> __device__ __forceinline__ void kge_store8(void *row, int64_t col, int n, const float (&v)[8]) {
    if (n >= 8) {
        if constexpr (BF16) {
            typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf2;
            kge_u32x4 r;
#pragma unroll
            for (int u = 0; u < 4; ++u) r[u] = __builtin_bit_cast(uint32_t, bf2{(__bf16)v[2 * u], (__bf16)v[2 * u + 1]});
            if constexpr (STREAM) __builtin_nontemporal_store(r, (kge_u32x4_a2 *)((uint16_t *)row + col));
            else *(kge_u32x4_a2 *)((uint16_t *)row + col) = r;
        } else {
            const kge_f32x4 x = {v[0], v[1], v[2], v[3]}, y = {v[4], v[5], v[6], v[7]};
            if constexpr (STREAM) {
                __builtin_nontemporal_store(x, (kge_f32x4_a4 *)((float *)row + col));
                __builtin_nontemporal_store(y, (kge_f32x4_a4 *)((float *)row + col + 4));
            } else { *(kge_f32x4_a4 *)((float *)row + col) = x; *(kge_f32x4_a4 *)((float *)row + col + 4) = y; }
        }
    } else {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (u < n) {
                if constexpr (BF16) ((__bf16 *)row)[col + u] = (__bf16)v[u];
                else ((float *)row)[col + u] = v[u];
            }
    }
}

// Dropout: element (row, column) is kept iff its 16 bits of Philox4x32-10 (key = seed, counter (row, column / 8, step, tag); word
// (column % 8) / 2, the low half for even columns) are >= thr, and is then scaled by 2^16 / (2^16 - thr).  The mask is a function of these
// alone, so the backward pass makes it again and nothing is stored.  Sixteen bits an element and not a word: a block costs ten
// rounds of two wide products, which at four elements a block is as much time as a bf16 element takes to copy.
struct KgeDropDev {
    uint32_t k0, k1, step, tag, thr; float scale; const uint64_t *step_counter;
};

__device__ __forceinline__ uint32_t kge_drop_step(const KgeDropDev &d) { return d.step + (d.step_counter ? (uint32_t)*d.step_counter : 0u); }

__device__ __forceinline__ uint32_t kge_xor3(uint32_t a, uint32_t b, uint32_t c) { return (uint32_t)__builtin_amdgcn_bitop3_b32((int)a, (int)b, (int)c, 0x96); }

__device__ __forceinline__ void kge_drop8(const KgeDropDev &d, uint32_t step, uint32_t row, uint32_t group, float (&v)[8]) {
    uint32_t c0 = row, c1 = group, c2 = step, c3 = d.tag, k0 = d.k0, k1 = d.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
        c0 = kge_xor3((uint32_t)(p1 >> 32), c1, k0); c1 = (uint32_t)p1;
        c2 = kge_xor3((uint32_t)(p0 >> 32), c3, k1); c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    const uint32_t w[4] = {c0, c1, c2, c3};
#pragma unroll
    for (int u = 0; u < 4; ++u) {                              // (a select, not a product: what is dropped may be infinite)
        v[2 * u] = (w[u] & 0xffffu) >= d.thr ? v[2 * u] * d.scale : 0.f;
        v[2 * u + 1] = (w[u] >> 16) >= d.thr ? v[2 * u + 1] * d.scale : 0.f;
    }
}

// The kernels' form of a caller's dropout; nullptr and p that rounds to nothing drop nothing (thr = 0).  KGE_E_INVALID_ARG: p outside [0, 1) or
// a step that is no 32-bit word.
int kge_drop_dev(const kge_dropout_t *drop, KgeDropDev *out);

// Item -> (row, group of the row) without a division: the quotient n / d of n, d < 2^16 from one product.
struct KgeFastDiv { uint32_t d; uint64_t magic; };
inline KgeFastDiv kge_fast_div(uint32_t d) { return KgeFastDiv{d, ((1ull << 32) + d - 1) / d}; }
__device__ __forceinline__ uint32_t kge_div(uint32_t n, const KgeFastDiv &f) { return (uint32_t)((n * f.magic) >> 32); }

// Workgroups of a launch: a grid is limited to 2^32 threads, beyond 2^22 workgroups they take turns
inline dim3 kge_grid_of(int64_t n, int64_t per) { const int64_t b = (n + per - 1) / per; return dim3((unsigned)(b < (1 << 22) ? b : 1 << 22)); }

inline bool kge_bad_type(int32_t dtype) { return dtype != KGE_F32 && dtype != KGE_BF16; }
// rows of a matrix: a stride below the width would make them overlap, and the addresses have to be whole elements
inline bool kge_bad_rows(const void *p, int32_t dtype, int64_t ld, int64_t cols) {
    return !p || ld < cols || ((uintptr_t)p & (dtype == KGE_BF16 ? 1 : 3)) != 0;
}
constexpr int64_t KGE_MAX_ROWS = (1ll << 31) - 1, KGE_MAX_LD = 1ll << 31;
constexpr int KGE_MAX_DIM = 65536;
// From this size on results are stored past the caches (the L2s hold 32 MB in all).  Dropout with residual, past them and through them, fresh matrices in
// turn: 128 MB 76.6 and 82.4 us, 64 MB 40.5 and 44.7, 32 MB 22.3 and 24.6, 24 MB 19.2 and 20.7, 8 MB 10.8 and 11.7; followed by a reader of the result
// 128 MB 128 and 141, 64 MB 69.1 and 72.4, 24 MB 32.4 and 33.3, 8 MB 16.5 and 16.5.  (The same matrices again and again come from the last
// cache: 128 MB 64.7 and 81.9.)
constexpr int64_t KGE_STREAM_BYTES = 32ll << 20;
