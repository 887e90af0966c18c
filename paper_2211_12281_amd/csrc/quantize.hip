// Quantisation to 8-bit floating point with a power-of-two scale for each block of 128 consecutive elements of a row.
//
//   amax = 1.f x 2^E over the block's finite elements;  e = E - EMAX + (1.f > 1.75): the smallest exponent with amax <= 1.75 x 2^(EMAX + e)
//   (EMAX 8 for e4m3, 15 for e5m2);  scale byte = clamp(e + 127, 0, 254);  code = RNE(x 2^(127 - byte)) on the format's grid
//
// The scale is a power of two because the matrix instructions take it as an exponent byte and apply it for nothing; a scale of any other
// value would cost one multiply-add per accumulator and 128 elements of the contraction, and a block of a floating-point format gains less than one
// bit of range by it and no precision.  Memory bounds the kernels: 2 or 4 bytes read, one (or one for each layout) written per element.  Measured:
// 24,576 x 768 bf16 in both layouts 15.7 us (76 MB, 4.8 TB/s); by rows 131,072 x 1,024 bf16 81 us (5.0 TB/s), fp32 115 (5.9); 1,000 x 1,111 fp32 by
// rows 3.6 us, of which a launch is 2.
#include "text_ops.hpp"

namespace {

constexpr int NT = 256, BLOCK = 128;

template <int FMT> struct Fmt;
template <> struct Fmt<KGE_E4M3> { static constexpr int EMAX = 8; };
template <> struct Fmt<KGE_E5M2> { static constexpr int EMAX = 15; };

// amax: bits of a magnitude.  A mantissa above 1.75 carries into the exponent; zero and subnormal numbers end below byte 0.
template <int FMT> __device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    return (uint32_t)max((int)((amax + 0x1fffffu) >> 23) - Fmt<FMT>::EMAX, 0);
}
__device__ __forceinline__ float inv_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }   // byte <= 247: a normal number

// Codes of two values.  No finite value outgrows the format; the conversion keeps NaN, and an infinity where the format has one (e4m3: NaN).
template <int FMT> __device__ __forceinline__ uint32_t encode2(float a, float b, float inva, float invb) {
    return (uint32_t)(FMT == KGE_E4M3 ? __builtin_amdgcn_cvt_pk_fp8_f32(a * inva, b * invb, 0, false) : __builtin_amdgcn_cvt_pk_bf8_f32(a * inva, b * invb, 0, false)) & 0xffffu;
}

// Eight elements as they lie in memory, and what the kernels ask of them.  Magnitudes are compared as integers (two bf16 ones at once): what is not
// finite is larger than everything that is, and is left out in a second look (FINITE) where the first one meets it.
constexpr uint32_t INF32 = 0x7f800000u;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max16(uint32_t a, uint32_t b) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
template <bool IN16> struct Group {
    static constexpr int W = IN16 ? 4 : 8;
    uint32_t w[W];
    __device__ __forceinline__ void load(const void *row, int64_t col, int n) {
        if (n >= 8) {
            const KgeRaw8<IN16> r = kge_raw8<IN16>(row, col);
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = r.w[i >> 2][i & 3];
        } else {
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = 0u;
            if (n > 0) {                                      // (the last element's again for those behind it: one branch for all)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t at = col + min(e, n - 1);
                    const uint32_t u = IN16 ? (uint32_t)((const uint16_t *)row)[at] : ((const uint32_t *)row)[at];
                    w[IN16 ? e >> 1 : e] |= e < n ? (IN16 ? u << (16 * (e & 1)) : u) : 0u;
                }
            }
        }
    }
    __device__ __forceinline__ float value(int e) const {
        if constexpr (IN16) return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
        else return __uint_as_float(w[e]);
    }
    // magnitudes of word i (bf16: of two elements)
    template <bool FINITE> __device__ __forceinline__ uint32_t mag(int i) const {
        if constexpr (IN16) {
            uint32_t m = w[i] & 0x7fff7fffu;
            if (FINITE) { m = (m & 0xffffu) >= 0x7f80u ? m & 0xffff0000u : m; m = m >= INF32 ? m & 0xffffu : m; }
            return m;
        } else {
            const uint32_t m = w[i] & 0x7fffffffu;
            return FINITE && m >= INF32 ? 0u : m;
        }
    }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return IN16 ? max16(a, b) : max(a, b); }
    template <bool FINITE> __device__ __forceinline__ uint32_t amax() const {             // bits of the largest magnitude
        uint32_t m = mag<FINITE>(0);
#pragma unroll
        for (int i = 1; i < W; ++i) m = larger(m, mag<FINITE>(i));
        return IN16 ? max(m << 16, m & 0xffff0000u) : m;
    }
    template <int FMT> __device__ __forceinline__ kge_u32x2 encode(float inv) const {
        return kge_u32x2{encode2<FMT>(value(0), value(1), inv, inv) | encode2<FMT>(value(2), value(3), inv, inv) << 16,
                         encode2<FMT>(value(4), value(5), inv, inv) | encode2<FMT>(value(6), value(7), inv, inv) << 16};
    }
};

// largest of sixteen neighbouring lanes
__device__ __forceinline__ uint32_t max_of_16(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, true));      // lane ^ 1
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, true));      // lane ^ 2
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xf, 0xf, true));     // 7 - lane
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xf, 0xf, true));  // 15 - lane
}
template <bool IN16> __device__ __forceinline__ uint32_t block_amax(const Group<IN16> &g) {
    uint32_t m = max_of_16(g.template amax<false>());
    if (__any(m >= INF32)) m = max_of_16(g.template amax<true>());
    return m;
}

struct QuantArgs {
    const void *x; int64_t ld, rows, cols;
    uint8_t *rc, *rs; int64_t rc_ld, rs_ld;      // by rows
    uint8_t *cc, *cs; int64_t cc_ld, cs_ld;      // by columns (of the transposed matrix)
};

// Rows alone: sixteen lanes hold a block, eight elements each.  (The whole wave goes round together: its lanes look at each other's values.)
template <bool IN16, int FMT>
__global__ __launch_bounds__(NT) void quantize_rows_kernel(const QuantArgs a) {
    const int64_t nb = (a.cols + BLOCK - 1) / BLOCK, total = a.rows * nb;
    const int l16 = threadIdx.x & 15;
    for (int64_t b0 = (int64_t)blockIdx.x * (NT / 16); b0 < total; b0 += (int64_t)gridDim.x * (NT / 16)) {
        const int64_t b = b0 + (threadIdx.x >> 4), row = b / nb, kb = b - row * nb, col = kb * BLOCK + 8 * l16, left = a.cols - col;
        const bool in = b < total;
        Group<IN16> g;
        g.load((const char *)a.x + (in ? row : 0) * a.ld * (IN16 ? 2 : 4), col, in ? (left > 8 ? 8 : (int)left) : 0);
        const uint32_t s = scale_byte<FMT>(block_amax(g));
        if (!in) continue;
        *(kge_u32x2 *)(a.rc + row * a.rc_ld + col) = g.template encode<FMT>(inv_scale(s));
        if (l16 == 0) a.rs[row * a.rs_ld + kb] = (uint8_t)s;
        if (kb == nb - 1 && nb + l16 < (nb + 3) / 4 * 4) a.rs[row * a.rs_ld + nb + l16] = 0;
    }
}

// Tiles of 128 x 128, for the columns and, where both layouts are asked for, for the rows too: x is read once.  Thread (rg, cg) holds rows
// 4 rg .. + 3 and 64 + 4 rg .. + 3 of columns 8 cg .. + 7: a row's block is sixteen neighbouring lanes, a column's is eight registers of
// each of sixteen threads, and four rows of a column make one word of the transposed tile.
struct TileLds {
    uint32_t top[NT / 64][16][9];
    uint32_t tile[BLOCK][BLOCK / 4 + 1];                         // (one word more per column: a wave's words fall into different banks)
};
// INSIDE: the whole tile lies inside the matrix, nothing is asked about rows and columns
template <bool IN16, int FMT, bool ROWS, bool INSIDE>
__device__ __forceinline__ void quantize_tile(const QuantArgs &a, TileLds &l, int64_t tr, int64_t tc, int64_t nb, int64_t rb) {
    using G = Group<IN16>;
    constexpr int W = G::W;
    const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t row0 = tr * BLOCK, col0 = tc * BLOCK;
    const int rows = INSIDE ? BLOCK : (int)min((int64_t)BLOCK, a.rows - row0), cols = INSIDE ? BLOCK : (int)min((int64_t)BLOCK, a.cols - col0);
    const int n = INSIDE ? 8 : cols - 8 * cg;
    const char *x0 = (const char *)a.x + ((row0 + 4 * rg) * a.ld + col0) * (IN16 ? 2 : 4);
    G v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int d = 64 * (i >> 2) + (i & 3);
        v[i].load(x0 + d * a.ld * (IN16 ? 2 : 4), 8 * cg, INSIDE || 4 * rg + d < rows ? n : 0);
    }
    uint32_t cm[W];
    bool odd = false;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        cm[w] = v[0].template mag<false>(w);
#pragma unroll
        for (int i = 1; i < 8; ++i) cm[w] = G::larger(cm[w], v[i].template mag<false>(w));
        odd = odd || (IN16 ? (cm[w] & 0xffffu) >= 0x7f80u || cm[w] >= INF32 : cm[w] >= INF32);
    }
    if (__any(odd)) {
#pragma unroll
        for (int w = 0; w < W; ++w) {
            cm[w] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) cm[w] = G::larger(cm[w], v[i].template mag<true>(w));
        }
    }
#pragma unroll
    for (int w = 0; w < W; ++w) {
        cm[w] = G::larger(cm[w], (uint32_t)__shfl_xor((int)cm[w], 16));
        cm[w] = G::larger(cm[w], (uint32_t)__shfl_xor((int)cm[w], 32));
    }
    if (lane < 16) {
#pragma unroll
        for (int w = 0; w < W; ++w) l.top[wave][cg][w] = cm[w];
    }
    if constexpr (ROWS) {
        uint32_t m[8];
        odd = false;
#pragma unroll
        for (int i = 0; i < 8; ++i) { m[i] = max_of_16(v[i].template amax<false>()); odd = odd || m[i] >= INF32; }
        if (__any(odd)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) m[i] = max_of_16(v[i].template amax<true>());
        }
        uint8_t *codes = a.rc + (row0 + 4 * rg) * a.rc_ld + col0 + 8 * cg, *scales = a.rs + (row0 + 4 * rg) * a.rs_ld + tc;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int d = 64 * (i >> 2) + (i & 3);
            const uint32_t s = scale_byte<FMT>(m[i]);
            const kge_u32x2 c = v[i].template encode<FMT>(inv_scale(s));
            m[i] = s;
            if (INSIDE || 4 * rg + d < rows) *(kge_u32x2 *)(codes + d * a.rc_ld) = c;
        }
        const int pad = tc == nb - 1 ? (int)((nb + 3) / 4 * 4 - nb) : 0;                   // bytes behind a row's last scale
        if (cg <= pad) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int d = 64 * (i >> 2) + (i & 3);
                if (INSIDE || 4 * rg + d < rows) scales[d * a.rs_ld + cg] = cg == 0 ? (uint8_t)m[i] : 0;
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) cm[w] = G::larger(G::larger(l.top[0][cg][w], l.top[1][cg][w]), G::larger(l.top[2][cg][w], l.top[3][cg][w]));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = 8 * cg + e;
        const uint32_t s = scale_byte<FMT>(IN16 ? (e & 1 ? cm[e >> 1] & 0xffff0000u : cm[e >> 1] << 16) : cm[e]);
        const float inv = inv_scale(s);
        l.tile[c][rg] = encode2<FMT>(v[0].value(e), v[1].value(e), inv, inv) | encode2<FMT>(v[2].value(e), v[3].value(e), inv, inv) << 16;
        l.tile[c][16 + rg] = encode2<FMT>(v[4].value(e), v[5].value(e), inv, inv) | encode2<FMT>(v[6].value(e), v[7].value(e), inv, inv) << 16;
        const int pad = tr == rb - 1 ? (int)((rb + 3) / 4 * 4 - rb) : 0;
        if (rg <= pad && (INSIDE || e < n)) a.cs[(col0 + c) * a.cs_ld + tr + rg] = rg == 0 ? (uint8_t)s : 0;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < BLOCK * 8 / NT; ++j) {
        const int q = threadIdx.x + j * NT, c = q >> 3, w = q & 7;
        if (INSIDE || c < cols)
            *(kge_u32x4 *)(a.cc + (col0 + c) * a.cc_ld + row0 + 16 * w) = kge_u32x4{l.tile[c][4 * w], l.tile[c][4 * w + 1], l.tile[c][4 * w + 2], l.tile[c][4 * w + 3]};
    }
}
template <bool IN16, int FMT, bool ROWS>
__global__ __launch_bounds__(NT, IN16 ? 4 : 3) void quantize_tiles_kernel(const QuantArgs a) {
    __shared__ TileLds l;
    const int64_t nb = (a.cols + BLOCK - 1) / BLOCK, rb = (a.rows + BLOCK - 1) / BLOCK;
    // (one tile per workgroup: in a loop over tiles the strides' multiples are kept in registers that spill)
    const int64_t tr = blockIdx.x / (uint32_t)nb, tc = blockIdx.x - tr * nb;
    if ((tr + 1) * BLOCK <= a.rows && (tc + 1) * BLOCK <= a.cols) quantize_tile<IN16, FMT, ROWS, true>(a, l, tr, tc, nb, rb);
    else quantize_tile<IN16, FMT, ROWS, false>(a, l, tr, tc, nb, rb);
}

template <bool IN16, int FMT> void launch(const QuantArgs &a, hipStream_t st) {
    const int64_t nb = (a.cols + BLOCK - 1) / BLOCK, rb = (a.rows + BLOCK - 1) / BLOCK;
    const dim3 tiles((unsigned)(nb * rb));
    if (!a.cc) hipLaunchKernelGGL((quantize_rows_kernel<IN16, FMT>), kge_grid_of(a.rows * nb, NT / 16), dim3(NT), 0, st, a);
    else if (a.rc) hipLaunchKernelGGL((quantize_tiles_kernel<IN16, FMT, true>), tiles, dim3(NT), 0, st, a);
    else hipLaunchKernelGGL((quantize_tiles_kernel<IN16, FMT, false>), tiles, dim3(NT), 0, st, a);
}

}  // namespace

// Layout rules of a quantised matrix that every call checks: whole blocks in a row of codes, whole words in a row of scales
int kge_check_quantized(const kge_quantized_t *q) {
    if (!q || (q->format != KGE_E4M3 && q->format != KGE_E5M2) || q->reserved != 0 || q->rows < 0 || q->cols < 0 || q->rows >= (1ll << 31) ||
        q->cols >= (1ll << 31)) return KGE_E_INVALID_ARG;
    const int64_t nb = (q->cols + BLOCK - 1) / BLOCK;
    if (q->ld < nb * BLOCK || q->ld % 16 != 0 || q->ld >= (1ll << 32) || q->scales_ld < (nb + 3) / 4 * 4 || q->scales_ld % 4 != 0 ||
        q->scales_ld >= (1ll << 32)) return KGE_E_INVALID_ARG;
    if (q->rows > 0 && q->cols > 0 && (!q->codes || !q->scales || ((uintptr_t)q->codes & 15) != 0 || ((uintptr_t)q->scales & 3) != 0))
        return KGE_E_INVALID_ARG;
    return KGE_OK;
}

extern "C" int kge_quantize(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, const kge_quantized_t *by_row,
                            const kge_quantized_t *by_col, void *hip_stream) {
    if ((dtype != KGE_F32 && dtype != KGE_BF16) || rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31) || ld >= (1ll << 31) || (!by_row && !by_col))
        return KGE_E_INVALID_ARG;
    if (by_row && (kge_check_quantized(by_row) != KGE_OK || by_row->rows != rows || by_row->cols != cols)) return KGE_E_INVALID_ARG;
    if (by_col && (kge_check_quantized(by_col) != KGE_OK || by_col->rows != cols || by_col->cols != rows)) return KGE_E_INVALID_ARG;
    if (by_row && by_col && by_row->format != by_col->format) return KGE_E_INVALID_ARG;
    if (rows == 0 || cols == 0) return KGE_OK;
    if (!x || ld < cols || ((uintptr_t)x & (dtype == KGE_BF16 ? 1 : 3)) != 0) return KGE_E_INVALID_ARG;
    if (by_col && ((rows + BLOCK - 1) / BLOCK) * ((cols + BLOCK - 1) / BLOCK) >= (1ll << 24)) return KGE_E_UNSUPPORTED;   // (a grid's limit)
    QuantArgs a = {};
    a.x = x; a.ld = ld; a.rows = rows; a.cols = cols;
    if (by_row) { a.rc = by_row->codes; a.rs = by_row->scales; a.rc_ld = by_row->ld; a.rs_ld = by_row->scales_ld; }
    if (by_col) { a.cc = by_col->codes; a.cs = by_col->scales; a.cc_ld = by_col->ld; a.cs_ld = by_col->scales_ld; }
    hipStream_t st = (hipStream_t)hip_stream;
    const bool e4 = (by_row ? by_row : by_col)->format == KGE_E4M3;
    if (dtype == KGE_BF16) { if (e4) launch<true, KGE_E4M3>(a, st); else launch<true, KGE_E5M2>(a, st); }
    else { if (e4) launch<false, KGE_E4M3>(a, st); else launch<false, KGE_E5M2>(a, st); }
    return kge_launch_status();
}
