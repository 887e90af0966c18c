// Quantisation to 8-bit floating point with a power-of-two scale for each block of 128 consecutive elements of a row.
//
//   amax = 1.f x 2^E over the block's finite elements;  e = E - EMAX + (1.f > 1.75): the smallest exponent with amax <= 1.75 x 2^(EMAX + e)
//   (EMAX 8 for e4m3, 15 for e5m2);  scale byte = clamp(e + 127, 0, 254);  code = RNE(x 2^(127 - byte)) on the format's grid
//
// The scale is a power of two because the matrix instructions take it as an exponent byte and apply it for nothing; a scale of any other
// value would cost one multiply-add per accumulator and 128 elements of the contraction, and a block of a floating-point format gains less than one
// bit of range by it and no precision.  Memory bounds the kernels: 2 or 4 bytes read, one (or one for each layout) written per element.
#include "text_ops.hpp"

namespace {

constexpr int NT = 256, BLOCK = 128;

template <int FMT> struct Fmt;
template <> struct Fmt<KGE_E4M3> { static constexpr int EMAX = 8; };
template <> struct Fmt<KGE_E5M2> { static constexpr int EMAX = 15; };

// magnitude bits of x where it is finite, else 0: unsigned comparison orders them
__device__ __forceinline__ uint32_t finite_bits(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}
template <int FMT> __device__ __forceinline__ uint32_t scale_byte(uint32_t amax) {
    if (amax == 0u) return 0u;
    // (a subnormal amax has E <= -127 here and in truth: its byte is 0 either way)
    const int s = (int)(amax >> 23) - Fmt<FMT>::EMAX + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);
    return s < 0 ? 0u : (uint32_t)s;
}
__device__ __forceinline__ float inv_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }   // byte <= 247: a normal number

// codes of two values; what is not finite keeps its meaning where the format has it (e4m3 has no infinity)
template <int FMT> __device__ __forceinline__ uint32_t encode2(float a, float b, float inv) {
    const float x = a * inv, y = b * inv;
    uint32_t c = FMT == KGE_E4M3 ? (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false) : (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(x, y, 0, false);
    c &= 0xffffu;
    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
    if (__builtin_expect((ua & 0x7f800000u) == 0x7f800000u, 0))
        c = (c & 0xff00u) | (ua >> 31 << 7) | (FMT == KGE_E5M2 && (ua & 0x7fffffu) == 0u ? 0x7cu : 0x7fu);
    if (__builtin_expect((ub & 0x7f800000u) == 0x7f800000u, 0))
        c = (c & 0x00ffu) | (ub >> 31 << 15) | (FMT == KGE_E5M2 && (ub & 0x7fffffu) == 0u ? 0x7c00u : 0x7f00u);
    return c;
}

struct QuantArgs {
    const void *x; int64_t ld, rows, cols;
    uint8_t *rc, *rs; int64_t rc_ld, rs_ld;      // by rows
    uint8_t *cc, *cs; int64_t cc_ld, cs_ld;      // by columns (of the transposed matrix)
};

// Rows alone: sixteen lanes hold a block, eight elements each.
template <bool IN16, int FMT>
__global__ __launch_bounds__(NT) void quantize_rows_kernel(const QuantArgs a) {
    const int64_t nb = (a.cols + BLOCK - 1) / BLOCK, total = a.rows * nb;
    const int l16 = threadIdx.x & 15;
    for (int64_t b = (int64_t)blockIdx.x * (NT / 16) + (threadIdx.x >> 4); b < total; b += (int64_t)gridDim.x * (NT / 16)) {
        const int64_t row = b / nb, kb = b - row * nb, col = kb * BLOCK + 8 * l16;
        const int64_t left = a.cols - col;
        float v[8];
        kge_load8<IN16>((const char *)a.x + row * a.ld * (IN16 ? 2 : 4), col, left > 8 ? 8 : (int)left, v);
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, finite_bits(v[e]));
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 16));
        const uint32_t s = scale_byte<FMT>(m);
        const float inv = inv_scale(s);
        const kge_u32x2 c = {encode2<FMT>(v[0], v[1], inv) | encode2<FMT>(v[2], v[3], inv) << 16,
                             encode2<FMT>(v[4], v[5], inv) | encode2<FMT>(v[6], v[7], inv) << 16};
        *(kge_u32x2 *)(a.rc + row * a.rc_ld + col) = c;
        if (l16 == 0) a.rs[row * a.rs_ld + kb] = (uint8_t)s;
        if (kb == nb - 1 && nb + l16 < (nb + 3) / 4 * 4) a.rs[row * a.rs_ld + nb + l16] = 0;
    }
}

// Tiles of 128 x 128, for the columns and, where both layouts are asked for, for the rows too: x is read once.  Thread (rg, cg) holds rows
// 4 rg .. + 3 and 64 + 4 rg .. + 3 of columns 8 cg .. + 7: a row's block is sixteen neighbouring lanes, a column's is eight registers of
// each of sixteen threads, and four rows of a column make one word of the transposed tile.
template <bool IN16, int FMT, bool ROWS>
__global__ __launch_bounds__(NT) void quantize_tiles_kernel(const QuantArgs a) {
    __shared__ uint32_t top[NT / 64][BLOCK];
    __shared__ uint32_t tile[BLOCK][BLOCK / 4 + 1];              // (one word more per column: a wave's words fall into different banks)
    const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t nb = (a.cols + BLOCK - 1) / BLOCK, rb = (a.rows + BLOCK - 1) / BLOCK;
    for (int64_t t = blockIdx.x; t < nb * rb; t += gridDim.x) {
        const int64_t tr = t / nb, tc = t - tr * nb, row0 = tr * BLOCK, col = tc * BLOCK + 8 * cg, left = a.cols - col;
        float v[8][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t row = row0 + 64 * (i >> 2) + 4 * rg + (i & 3);
            kge_load8<IN16>((const char *)a.x + (row < a.rows ? row : 0) * a.ld * (IN16 ? 2 : 4), col, row < a.rows ? (left > 8 ? 8 : (int)left) : 0, v[i]);
        }
        if constexpr (ROWS) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t row = row0 + 64 * (i >> 2) + 4 * rg + (i & 3);
                uint32_t m = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) m = max(m, finite_bits(v[i][e]));
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o, 16));
                const uint32_t s = scale_byte<FMT>(m);
                const float inv = inv_scale(s);
                const kge_u32x2 c = {encode2<FMT>(v[i][0], v[i][1], inv) | encode2<FMT>(v[i][2], v[i][3], inv) << 16,
                                     encode2<FMT>(v[i][4], v[i][5], inv) | encode2<FMT>(v[i][6], v[i][7], inv) << 16};
                if (row < a.rows) {
                    *(kge_u32x2 *)(a.rc + row * a.rc_ld + col) = c;
                    if (cg == 0) a.rs[row * a.rs_ld + tc] = (uint8_t)s;
                    if (tc == nb - 1 && nb + cg < (nb + 3) / 4 * 4) a.rs[row * a.rs_ld + nb + cg] = 0;
                }
            }
        }
        uint32_t cm[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            cm[e] = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) cm[e] = max(cm[e], finite_bits(v[i][e]));
            cm[e] = max(cm[e], (uint32_t)__shfl_xor((int)cm[e], 16));
            cm[e] = max(cm[e], (uint32_t)__shfl_xor((int)cm[e], 32));
        }
        if (lane < 16) {
#pragma unroll
            for (int e = 0; e < 8; ++e) top[wave][8 * cg + e] = cm[e];
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = 8 * cg + e;
            const uint32_t m = max(max(top[0][c], top[1][c]), max(top[2][c], top[3][c]));
            const uint32_t s = scale_byte<FMT>(m);
            const float inv = inv_scale(s);
            tile[c][rg] = encode2<FMT>(v[0][e], v[1][e], inv) | encode2<FMT>(v[2][e], v[3][e], inv) << 16;
            tile[c][16 + rg] = encode2<FMT>(v[4][e], v[5][e], inv) | encode2<FMT>(v[6][e], v[7][e], inv) << 16;
            if (rg == 0 && col + e < a.cols) {
                a.cs[(col + e) * a.cs_ld + tr] = (uint8_t)s;
                if (tr == rb - 1)
                    for (int64_t p = rb; p < (rb + 3) / 4 * 4; ++p) a.cs[(col + e) * a.cs_ld + p] = 0;
            }
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < BLOCK * 8 / NT; ++j) {
            const int q = threadIdx.x + j * NT, c = q >> 3, w = q & 7;
            if (tc * BLOCK + c < a.cols)
                *(kge_u32x4 *)(a.cc + (tc * BLOCK + c) * a.cc_ld + row0 + 16 * w) =
                    kge_u32x4{tile[c][4 * w], tile[c][4 * w + 1], tile[c][4 * w + 2], tile[c][4 * w + 3]};
        }
        __syncthreads();
    }
}

template <bool IN16, int FMT> void launch(const QuantArgs &a, hipStream_t st) {
    const int64_t nb = (a.cols + BLOCK - 1) / BLOCK, rb = (a.rows + BLOCK - 1) / BLOCK;
    auto grid = [](int64_t n) { return dim3((unsigned)(n < (1 << 23) ? n : 1 << 23)); };
    if (!a.cc) hipLaunchKernelGGL((quantize_rows_kernel<IN16, FMT>), grid((a.rows * nb + NT / 16 - 1) / (NT / 16)), dim3(NT), 0, st, a);
    else if (a.rc) hipLaunchKernelGGL((quantize_tiles_kernel<IN16, FMT, true>), grid(nb * rb), dim3(NT), 0, st, a);
    else hipLaunchKernelGGL((quantize_tiles_kernel<IN16, FMT, false>), grid(nb * rb), dim3(NT), 0, st, a);
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
