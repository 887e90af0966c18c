// Quantisation to 8-bit integers with one scale per row, by rows and of the transposed matrix.
//
//   a = max(largest magnitude of the row, 2^-100),   scale = a / 127,   code = RNE(x * (127 / a)),  every operation rounded to fp32
//   (2^-100: below it 127 / a would leave fp32's range.)  A row with a NaN or an infinity: scale NaN, codes 0.
//
// Memory bounds it.  By rows a row of up to 32,768 elements stays in its threads' registers between the search for the largest magnitude and the
// codes, so x is read once.  By columns the largest magnitudes come first (partial ones for each run of rows, in the workspace), then tiles of 128 x 128 are
// turned in the LDS: x is read twice.  For both layouts (up to 4,096 columns) the search finds the rows' magnitudes too, and a tile writes both.
// Up to 512 rows a strip of columns stays in registers and one launch does it.  Measured: by rows 65,536 x 1,024 bf16 35.3 us (201 MB, 5.7 TB/s); by columns 30,000 x 2,048 bf16 63
// (search 24, scales 4.6, tiles 34); both, 9,999 x 1,001 fp32 24 (27 under the profiler: 9.9, 3.4, 13.4); 30 x 768 by columns 7.5, a launch and the chain from load to store.
#include "text_ops.hpp"

namespace {

constexpr int NT = 256, BLOCK = 128, MAX_RUNS = 128;
constexpr uint32_t INF32 = 0x7f800000u;
constexpr int64_t MAX_COLS = 131071, MAX_GROUPS = 1 << 21;       // (workgroups of a launch: a grid has fewer than 2^32 threads)

int check_rowwise(const kge_rowwise_t *q) {
    if (!q || q->rows < 0 || q->cols < 0 || q->rows >= (1ll << 31) || q->cols >= (1ll << 31)) return KGE_E_INVALID_ARG;
    if (q->ld < kge_round_up(q->cols, BLOCK) || q->ld % 16 != 0 || q->ld >= (1ll << 32)) return KGE_E_INVALID_ARG;
    if (q->rows > 0 && (!q->scales || ((uintptr_t)q->scales & 3) != 0 || (q->cols > 0 && (!q->codes || ((uintptr_t)q->codes & 15) != 0)))) return KGE_E_INVALID_ARG;
    return q->cols > MAX_COLS ? KGE_E_UNSUPPORTED : KGE_OK;
}

// scale and its inverse of a row whose largest magnitude has these bits (which compare like the numbers; what is not finite is largest)
struct Scale { float scale, inv; };
__device__ __forceinline__ Scale scale_of(uint32_t amax) {
    const float a = fmaxf(__uint_as_float(amax), 0x1p-100f);
    return amax >= INF32 ? Scale{__uint_as_float(0x7fc00000u), 0.f} : Scale{a / 127.f, 127.f / a};
}
__device__ __forceinline__ uint32_t code(float x, float inv) {           // (inv 0: whatever x is)
    const float q = rintf(x * inv);
    return (uint32_t)(int)(inv > 0.f ? q : 0.f) & 255u;
}
__device__ __forceinline__ int64_t padded(int64_t n) { return (n + BLOCK - 1) / BLOCK * BLOCK; }
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ kge_u32x2 codes8(const float (&v)[8], float inv) {
    kge_u32x2 r = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e >> 2] |= code(v[e], inv) << (8 * (e & 3));
    return r;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, true));      // lane ^ 1
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, true));      // lane ^ 2
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xf, 0xf, true));     // 7 - lane
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xf, 0xf, true));     // 15 - lane
    return max(max((uint32_t)__builtin_amdgcn_readlane((int)m, 0), (uint32_t)__builtin_amdgcn_readlane((int)m, 16)),
               max((uint32_t)__builtin_amdgcn_readlane((int)m, 32), (uint32_t)__builtin_amdgcn_readlane((int)m, 48)));
}

struct Args {
    const void *x; int64_t ld, rows, cols;
    int8_t *rc; float *rs; int64_t rc_ld;                         // by rows
    int8_t *cc; float *cs; int64_t cc_ld;                         // by columns
    uint32_t *part; int64_t part_ld, run; int runs;               // largest magnitudes of the columns in runs of rows: [run][part_ld]
    uint32_t *row_part; int64_t row_ld;                           // and of the rows in blocks of 128 columns: [block][row_ld]
    float *col_inv, *row_inv;                                     // inverses of the scales
};

// A row per team of waves (one wave: four rows per workgroup), NG groups of eight columns per thread; longer rows (LONG) are read twice.
template <bool B16, int NG, int WAVES, bool LONG>
__global__ __launch_bounds__(WAVES == 1 ? NT : 64 * WAVES) void rows_kernel(const Args a) {
    constexpr int T = 64 * WAVES, TEAMS = WAVES == 1 ? NT / 64 : 1, SPAN = 8 * T * NG;
    __shared__ uint32_t top[WAVES];
    const int lane = (int)threadIdx.x % T, team = (int)threadIdx.x / T;
    const int64_t wide = padded(a.cols);
    for (int64_t row = (int64_t)blockIdx.x * TEAMS + team; row < a.rows; row += (int64_t)gridDim.x * TEAMS) {
        const char *x = (const char *)a.x + row * a.ld * (B16 ? 2 : 4);
        float v[NG][8];
        uint32_t m = 0;
        for (int64_t c0 = 0; c0 < wide; c0 += SPAN) {
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                const int64_t col = c0 + 8 * (lane + k * T), left = a.cols - col;
                kge_load8<B16>(x, col, left > 8 ? 8 : (int)left, v[k]);
            }
#pragma unroll
            for (int k = 0; k < NG; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) m = max(m, mag(v[k][e]));
            if (!LONG) break;
        }
        m = wave_max(m);
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = m;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < WAVES; ++w) m = max(m, top[w]);
        }
        const Scale s = scale_of(m);
        for (int64_t c0 = 0; c0 < wide; c0 += SPAN) {
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                const int64_t col = c0 + 8 * (lane + k * T), left = a.cols - col;
                if (LONG) kge_load8<B16>(x, col, left > 8 ? 8 : (int)left, v[k]);
                if (col < wide) *(kge_u32x2 *)(a.rc + row * a.rc_ld + col) = codes8(v[k], s.inv);
            }
            if (!LONG) break;
        }
        if (lane == 0) a.rs[row] = s.scale;
        if constexpr (WAVES > 1) __syncthreads();                     // (of the next row's largest magnitudes)
    }
}

// largest of sixteen neighbouring lanes
__device__ __forceinline__ uint32_t max_of_16(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, true));      // lane ^ 1
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, true));      // lane ^ 2
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xf, 0xf, true));     // 7 - lane
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xf, 0xf, true));  // 15 - lane
}
// Largest magnitudes of 128 columns in a run of rows: a thread takes eight columns of every sixteenth row.  BOTH: those of the rows' 128 columns too.
template <bool B16, bool BOTH> __global__ __launch_bounds__(NT) void column_max_kernel(const Args a) {
    __shared__ uint32_t top[16][16][9];
    const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4;
    const int64_t col = (int64_t)blockIdx.x * BLOCK + 8 * cg, left = a.cols - col;
    const int64_t r0 = (int64_t)blockIdx.y * a.run, r1 = min(r0 + a.run, a.rows);
    uint32_t m[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (BOTH || left > 0)                                         // (the lanes of a row go round together)
#pragma unroll 8
        for (int64_t r = r0 + rg; r < r1; r += 16) {
            float v[8];
            kge_load8<B16>((const char *)a.x + r * a.ld * (B16 ? 2 : 4), col, left > 8 ? 8 : (int)left, v);
            uint32_t row = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                m[e] = max(m[e], mag(v[e]));
                if (BOTH) row = max(row, mag(v[e]));
            }
            if constexpr (BOTH) {
                row = max_of_16(row);
                if (cg == 0) a.row_part[(int64_t)blockIdx.x * a.row_ld + r] = row;
            }
        }
#pragma unroll
    for (int e = 0; e < 8; ++e) top[rg][cg][e] = m[e];
    __syncthreads();
    if (threadIdx.x >= BLOCK) return;
    uint32_t t = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) t = max(t, top[i][threadIdx.x >> 3][threadIdx.x & 7]);
    a.part[blockIdx.y * a.part_ld + (int64_t)blockIdx.x * BLOCK + threadIdx.x] = t;
}

// Scales of the columns (128 of them per workgroup, 32 slices of the runs) and, behind those workgroups, of the rows (one per thread), and their inverses, which the
// tiles take: from the partial magnitudes every tile would read 64 KB, twice its own share of x in bf16.
__global__ __launch_bounds__(1024) void scales_kernel(const Args a) {
    const int64_t blocks = a.part_ld / BLOCK;
    if (blockIdx.x >= blocks) {
        const int64_t row = (int64_t)(blockIdx.x - blocks) * 1024 + threadIdx.x;
        if (row >= a.rows) return;
        uint32_t m = 0;
#pragma unroll 8
        for (int b = 0; b < (int)blocks; ++b) m = max(m, a.row_part[b * a.row_ld + row]);
        const Scale s = scale_of(m);
        a.rs[row] = s.scale;
        a.row_inv[row] = s.inv;
        return;
    }
    __shared__ __attribute__((aligned(16))) uint32_t top[32][BLOCK];
    const int c = 4 * (threadIdx.x & 31), r0 = threadIdx.x >> 5;
    kge_u32x4 m = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < MAX_RUNS / 32; ++i) {
        const int r = r0 + 32 * i;
        m = __builtin_elementwise_max(m, *(const kge_u32x4 *)(a.part + (r < a.runs ? r : 0) * a.part_ld + (int64_t)blockIdx.x * BLOCK + c));
    }
    *(kge_u32x4 *)&top[r0][c] = m;
    __syncthreads();
    const int64_t col = (int64_t)blockIdx.x * BLOCK + threadIdx.x;
    if (threadIdx.x >= BLOCK || col >= a.cols) return;
    uint32_t t = 0;
#pragma unroll
    for (int r = 0; r < 32; ++r) t = max(t, top[r][threadIdx.x]);
    const Scale s = scale_of(t);
    a.cs[col] = s.scale;
    a.col_inv[col] = s.inv;
}

// Tiles of 128 x 128 turned in the LDS.  Thread (rg, cg) holds rows 4 rg .. + 3 and 64 + 4 rg .. + 3 of columns 8 cg .. + 7: four rows of a column make one
// word of the transposed tile.
template <bool B16, bool BOTH> __global__ __launch_bounds__(NT) void columns_kernel(const Args a) {
    __shared__ uint32_t tile[BLOCK][BLOCK / 4 + 1];                // (one word more per column: a wave's words fall into different banks)
    __shared__ float inv[BLOCK];
    __shared__ float row_inv[BOTH ? BLOCK : 1];
    const int64_t nb = (a.cols + BLOCK - 1) / BLOCK, tr = blockIdx.x / (uint32_t)nb, tc = blockIdx.x - tr * nb;
    const int cg = threadIdx.x & 15, rg = threadIdx.x >> 4;
    const int64_t row0 = tr * BLOCK, col0 = tc * BLOCK;
    const int rows = (int)min((int64_t)BLOCK, a.rows - row0), cols = (int)min((int64_t)BLOCK, a.cols - col0), n = cols - 8 * cg;
    float v[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int d = 4 * rg + 64 * (i >> 2) + (i & 3);
        kge_load8<B16>((const char *)a.x + (row0 + (d < rows ? d : 0)) * a.ld * (B16 ? 2 : 4), col0 + 8 * cg, d < rows ? (n > 8 ? 8 : n) : 0, v[i]);
    }
    if (threadIdx.x < BLOCK) inv[threadIdx.x] = (int)threadIdx.x < cols ? a.col_inv[col0 + threadIdx.x] : 0.f;
    else if (BOTH) row_inv[threadIdx.x - BLOCK] = (int)threadIdx.x - BLOCK < rows ? a.row_inv[row0 + threadIdx.x - BLOCK] : 0.f;
    __syncthreads();
    if constexpr (BOTH) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int d = 4 * rg + 64 * (i >> 2) + (i & 3);
            if (d < rows) *(kge_u32x2 *)(a.rc + (row0 + d) * a.rc_ld + col0 + 8 * cg) = codes8(v[i], row_inv[d]);
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = 8 * cg + e;
        const float s = inv[c];
#pragma unroll
        for (int h = 0; h < 2; ++h)
            tile[c][16 * h + rg] = code(v[4 * h][e], s) | code(v[4 * h + 1][e], s) << 8 | code(v[4 * h + 2][e], s) << 16 | code(v[4 * h + 3][e], s) << 24;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < BLOCK * 8 / NT; ++j) {
        const int q = threadIdx.x + j * NT, c = q >> 3, w = q & 7;
        if (c < cols)
            *(kge_u32x4 *)(a.cc + (col0 + c) * a.cc_ld + row0 + 16 * w) = kge_u32x4{tile[c][4 * w], tile[c][4 * w + 1], tile[c][4 * w + 2], tile[c][4 * w + 3]};
    }
}

// A matrix of few rows, by columns in one launch: a workgroup takes 32 columns and all rows (512 at most), which stay in registers between the search and the codes.
// Thread (rg, cg) holds rows 4 rg .. + 3 and 256 + 4 rg .. + 3 of columns 8 cg .. + 7: four rows of a column make one word of the transposed strip.
constexpr int STRIP = 32, STRIP_ROWS = 512;
bool in_strips(int64_t rows, int64_t cols) { return rows <= STRIP_ROWS && cols < 1ll << 28; }                  // (a grid has fewer than 2^32 threads)
template <bool B16> __global__ __launch_bounds__(NT) void strips_kernel(const Args a) {
    __shared__ uint32_t tile[STRIP][STRIP_ROWS / 4 + 1];
    __shared__ uint32_t top[NT / 64][4][9];
    const int cg = threadIdx.x & 3, rg = threadIdx.x >> 2, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int rows = (int)a.rows, halves = rows > STRIP_ROWS / 2 ? 2 : 1;
    const int64_t col0 = (int64_t)blockIdx.x * STRIP;
    const int cols = (int)min((int64_t)STRIP, a.cols - col0), n = cols - 8 * cg;
    float v[8][8];
    uint32_t m[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int d = 4 * rg + 256 * (i >> 2) + (i & 3);
        kge_load8<B16>((const char *)a.x + (int64_t)(d < rows ? d : 0) * a.ld * (B16 ? 2 : 4), col0 + 8 * cg, d < rows ? (n > 8 ? 8 : n) : 0, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) m[e] = max(m[e], mag(v[i][e]));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
        for (int s = 4; s < 64; s *= 2) m[e] = max(m[e], (uint32_t)__shfl_xor((int)m[e], s));
        if (lane < 4) top[wave][cg][e] = m[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int c = 8 * cg + e;
        const Scale s = scale_of(max(max(top[0][cg][e], top[1][cg][e]), max(top[2][cg][e], top[3][cg][e])));
        if (rg == 0 && c < cols) a.cs[col0 + c] = s.scale;
#pragma unroll
        for (int h = 0; h < 2; ++h)
            tile[c][64 * h + rg] = code(v[4 * h][e], s.inv) | code(v[4 * h + 1][e], s.inv) << 8 | code(v[4 * h + 2][e], s.inv) << 16 | code(v[4 * h + 3][e], s.inv) << 24;
    }
    __syncthreads();
    const int pieces = (int)(padded(rows) / 16);                  // of a column
    for (int q = threadIdx.x; q < STRIP * 16 * halves; q += NT) {
        const int c = q / (16 * halves), w = q % (16 * halves);
        if (c < cols && w < pieces)
            *(kge_u32x4 *)(a.cc + (col0 + c) * a.cc_ld + 16 * w) = kge_u32x4{tile[c][4 * w], tile[c][4 * w + 1], tile[c][4 * w + 2], tile[c][4 * w + 3]};
    }
}

// Runs of rows of the search for the columns' largest magnitudes, of a matrix that has any: about 1,024 workgroups, of 32 rows at least
constexpr int64_t WANTED = 1024, MIN_RUN = 32;
void runs_of(int64_t rows, int64_t cols, Args &a) {
    const int64_t across = (cols + BLOCK - 1) / BLOCK;
    int64_t runs = (WANTED + across - 1) / across;
    if (runs > MAX_RUNS) runs = MAX_RUNS;
    if (runs > (rows + MIN_RUN - 1) / MIN_RUN) runs = (rows + MIN_RUN - 1) / MIN_RUN;
    a.run = (rows + runs - 1) / runs; a.runs = (int)runs; a.part_ld = across * BLOCK; a.row_ld = (rows + BLOCK - 1) / BLOCK * BLOCK;
}
// words of the workspace; in both layouts at once (24,576 x 768 bf16: 28 us, one after the other 36) where a row has few blocks
constexpr int64_t MOST_BLOCKS = 32;
bool at_once(int64_t cols) { return cols <= MOST_BLOCKS * BLOCK; }
int64_t words_of(const Args &a, bool both) { return (a.runs + 1) * a.part_ld + (both ? (a.part_ld / BLOCK + 1) * a.row_ld : 0); }

template <bool B16, int NG, int WAVES, bool LONG> void launch_rows(const Args &a, hipStream_t st) {
    const int64_t teams = WAVES == 1 ? NT / 64 : 1, groups = (a.rows + teams - 1) / teams;
    hipLaunchKernelGGL((rows_kernel<B16, NG, WAVES, LONG>), dim3((unsigned)(groups < MAX_GROUPS ? groups : MAX_GROUPS)), dim3(WAVES == 1 ? NT : 64 * WAVES), 0, st, a);
}
template <bool B16> void launch(const Args &a, hipStream_t st) {
    if (a.rc && !a.row_part) {
        if (a.cols <= 512) launch_rows<B16, 1, 1, false>(a, st);
        else if (a.cols <= 1024) launch_rows<B16, 2, 1, false>(a, st);
        else if (a.cols <= 2048) launch_rows<B16, 1, 4, false>(a, st);
        else if (a.cols <= 4096) launch_rows<B16, 2, 4, false>(a, st);
        else if (a.cols <= 8192) launch_rows<B16, 4, 4, false>(a, st);
        else if (a.cols <= 32768) launch_rows<B16, 4, 16, false>(a, st);
        else launch_rows<B16, 4, 16, true>(a, st);
    }
    if (a.cc) {
        const dim3 runs((unsigned)(a.part_ld / BLOCK), (unsigned)a.runs), tiles((unsigned)(((a.cols + BLOCK - 1) / BLOCK) * ((a.rows + BLOCK - 1) / BLOCK)));
        if (in_strips(a.rows, a.cols)) {
            const int64_t strips = (a.cols + STRIP - 1) / STRIP;
            hipLaunchKernelGGL((strips_kernel<B16>), dim3((unsigned)strips), dim3(NT), 0, st, a);
        } else if (a.row_part) {
            hipLaunchKernelGGL((column_max_kernel<B16, true>), runs, dim3(NT), 0, st, a);
            hipLaunchKernelGGL(scales_kernel, dim3((unsigned)(a.part_ld / BLOCK + (a.rows + 1023) / 1024)), dim3(1024), 0, st, a);
            hipLaunchKernelGGL((columns_kernel<B16, true>), tiles, dim3(NT), 0, st, a);
        } else {
            hipLaunchKernelGGL((column_max_kernel<B16, false>), runs, dim3(NT), 0, st, a);
            hipLaunchKernelGGL(scales_kernel, dim3((unsigned)(a.part_ld / BLOCK)), dim3(1024), 0, st, a);
            hipLaunchKernelGGL((columns_kernel<B16, false>), tiles, dim3(NT), 0, st, a);
        }
    }
}

}  // namespace

int kge_check_rowwise(const kge_rowwise_t *q) { return check_rowwise(q); }

extern "C" {

size_t kge_quantize_rowwise_workspace_bytes(int64_t rows, int64_t cols) {
    if (rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31)) return 0;
    if (rows == 0 || cols == 0) return 256;                       // (nothing to search)
    Args a = {};
    runs_of(rows, cols, a);
    return !in_strips(rows, cols) ? (size_t)words_of(a, at_once(cols)) * sizeof(uint32_t) + 256 : 256;
}

int kge_quantize_rowwise(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t ld, const kge_rowwise_t *by_row, const kge_rowwise_t *by_col,
                         void *ws, size_t ws_bytes, void *hip_stream) {
    if (kge_bad_type(dtype) || rows < 0 || cols < 0 || rows >= (1ll << 31) || cols >= (1ll << 31) || ld >= KGE_MAX_LD || (!by_row && !by_col)) return KGE_E_INVALID_ARG;
    int rc = KGE_OK;
    for (const kge_rowwise_t *q : {by_row, by_col})
        if (q) {
            const int c = kge_check_rowwise(q);
            if (c == KGE_E_INVALID_ARG || q->rows != (q == by_row ? rows : cols) || q->cols != (q == by_row ? cols : rows)) return KGE_E_INVALID_ARG;
            if (c != KGE_OK) rc = c;
        }
    if (by_row && by_row == by_col) return KGE_E_INVALID_ARG;
    if (rc != KGE_OK) return rc;
    if (rows > 0 && cols > 0 && kge_bad_rows(x, dtype, ld, cols)) return KGE_E_INVALID_ARG;
    // (a grid has fewer than 2^32 threads: the tiles' of 256 each, the scales' of 1,024 for 128 columns)
    const int64_t down = (rows + BLOCK - 1) / BLOCK, across = (cols + BLOCK - 1) / BLOCK;
    if (by_col && (down * across >= (1ll << 24) || across >= (1ll << 22))) return KGE_E_UNSUPPORTED;
    hipStream_t st = (hipStream_t)hip_stream;
    if (rows == 0 || cols == 0) {                                 // rows of no elements have a scale all the same
        Args e = {};
        const kge_rowwise_t *q = rows ? by_row : by_col;
        e.rows = rows ? rows : cols; e.rs = q ? q->scales : nullptr;
        if (!e.rs || e.rows == 0) return KGE_OK;
        launch_rows<false, 1, 1, false>(e, st);
        return kge_launch_status();
    }
    Args a = {};
    a.x = x; a.ld = ld; a.rows = rows; a.cols = cols;
    if (by_row) { a.rc = by_row->codes; a.rs = by_row->scales; a.rc_ld = by_row->ld; }
    if (by_col) {
        a.cc = by_col->codes; a.cs = by_col->scales; a.cc_ld = by_col->ld;
        runs_of(rows, cols, a);
        const size_t lost = ws ? (256 - ((uintptr_t)ws & 255)) & 255 : 0;
        const bool both = by_row && at_once(cols) && !in_strips(rows, cols);
        if (!in_strips(rows, cols) && (!ws || ws_bytes < lost + (size_t)words_of(a, both) * sizeof(uint32_t))) return KGE_E_WORKSPACE_TOO_SMALL;
        a.part = (uint32_t *)((char *)ws + lost);                  // (few rows: nothing is written there)
        a.col_inv = (float *)(a.part + a.runs * a.part_ld);
        if (both) {
            a.row_inv = a.col_inv + a.part_ld;
            a.row_part = (uint32_t *)a.row_inv + a.row_ld;
        }
    }
    if (dtype == KGE_BF16) launch<true>(a, st);
    else launch<false>(a, st);
    return kge_launch_status();
}

}  // extern "C"
