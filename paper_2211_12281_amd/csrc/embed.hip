// Token embeddings: the scaled lookup, its gradient by sorted tokens, and dropout.
//
//   lookup    out[i, :]  = D_i o (scale table[ids[i], :])
//   gradient  G[r, :]   (+)= scale sum over i with ids[i] = r of D_i o g[i, :]
//   dropout   out        = residual + D o x
//
// All three move every element once and compute next to nothing: memory bounds them.  D is made where it is used (text_ops.hpp).
#include "text_ops.hpp"
#include <math.h>

int kge_sort_pairs(const int32_t *idx, const int32_t *h, const int32_t *t, int64_t part_size, int D, int64_t M,
                   int64_t key_range, void *ws, const uint32_t **sk, const uint32_t **sp, hipStream_t st,
                   const int32_t *r, int64_t n_rel);
size_t kge_sort_ws(int64_t M);

int kge_drop_dev(const kge_dropout_t *drop, KgeDropDev *out) {
    *out = KgeDropDev{0, 0, 0, 0, 0, 1.f, nullptr};
    if (!drop) return KGE_OK;
    if (!(drop->p >= 0.f && drop->p < 1.f) || drop->step >= (1ull << 32)) return KGE_E_INVALID_ARG;
    uint32_t thr = (uint32_t)floor((double)drop->p * 65536.0 + 0.5);
    thr = thr > 65535u ? 65535u : thr;
    *out = KgeDropDev{(uint32_t)drop->seed, (uint32_t)(drop->seed >> 32), (uint32_t)drop->step, drop->tag, thr,
                      65536.f / (float)(65536u - thr), drop->step_counter};
    return KGE_OK;
}

namespace {

constexpr int NT = 256;                      // threads of a workgroup
constexpr int UNROLL = 4;                    // groups of eight columns that a thread has in flight

// Rows of a workgroup: about NT x UNROLL groups, at least one row
// Workgroups of a launch: a grid is limited to 2^32 threads, beyond 2^23 workgroups they take turns
inline dim3 grid_of(int64_t n, int64_t per) { const int64_t b = (n + per - 1) / per; return dim3((unsigned)(b < (1 << 23) ? b : 1 << 23)); }
inline int rows_per_block(int cg) { const int r = NT * UNROLL / cg; return r < 1 ? 1 : r; }

struct RowsArgs {
    const void *x; int64_t x_ld;             // table or input
    const int32_t *ids; int64_t n_rows;      // lookup alone
    const void *res; int64_t res_ld;         // dropout alone (may be null)
    void *out; int64_t out_ld;
    int64_t M; int dim, rows; KgeFastDiv cg;
    float scale; KgeDropDev drop;
};

// The lookup and the dropout in one body: a workgroup takes `rows` rows, a thread up to UNROLL groups of eight columns at a time, so that its loads are in
// flight together (the lookup's row numbers first, then the rows).
template <bool LOOKUP, bool IN16, bool OUT16>
__global__ __launch_bounds__(NT) void rows_kernel(const RowsArgs a) {
    const uint32_t step = a.drop.thr ? kge_drop_step(a.drop) : 0u;
    for (int64_t r0 = (int64_t)blockIdx.x * a.rows; r0 < a.M; r0 += (int64_t)gridDim.x * a.rows) {
    const int nr = (int)(a.M - r0 < a.rows ? a.M - r0 : a.rows), items = nr * (int)a.cg.d;
    for (int it0 = threadIdx.x; it0 < items; it0 += NT * UNROLL) {
        int row[UNROLL], grp[UNROLL], n[UNROLL];
        int64_t src[UNROLL];
        bool in[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int it = it0 + u * NT;
            in[u] = it < items;
            row[u] = in[u] ? (int)kge_div((uint32_t)it, a.cg) : 0;
            grp[u] = in[u] ? it - row[u] * (int)a.cg.d : 0;
            n[u] = a.dim - 8 * grp[u];
            if constexpr (LOOKUP) src[u] = in[u] ? (int64_t)a.ids[r0 + row[u]] : -1;
            else src[u] = r0 + row[u];
        }
        float v[UNROLL][8], z[UNROLL][8];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const bool live = LOOKUP ? src[u] >= 0 && src[u] < a.n_rows : in[u];
            if (live) kge_load8<IN16>((const char *)a.x + src[u] * a.x_ld * (IN16 ? 2 : 4), 8 * grp[u], n[u], v[u]);
            else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[u][e] = 0.f;
            }
            if constexpr (!LOOKUP)
                if (a.res && in[u]) kge_load8<IN16>((const char *)a.res + (r0 + row[u]) * a.res_ld * (IN16 ? 2 : 4), 8 * grp[u], n[u], z[u]);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (!in[u]) continue;
            if constexpr (LOOKUP) {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[u][e] *= a.scale;
            }
            if (a.drop.thr) kge_drop8(a.drop, step, (uint32_t)(r0 + row[u]), (uint32_t)grp[u], v[u]);
            if constexpr (!LOOKUP)
                if (a.res) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[u][e] += z[u][e];
                }
            kge_store8<OUT16>((char *)a.out + (r0 + row[u]) * a.out_ld * (OUT16 ? 2 : 4), 8 * grp[u], n[u], v[u]);
        }
    }
    }
}

// ---------------------------------------------------------------------------------------------
// Gradient of the lookup.
//   1. keys_kernel: ids outside the table become the key n_rows; every row's start is marked empty
//   2. the stable sort of (key, position) that the sparse update uses
//   3. runs_kernel: first and last sorted position of every row's run; the sums of whole chunks of RUN_CHUNK positions inside one run
//   4. row_sums_kernel: every table row is written once: zeros, or the sum over its run (positions up to the next chunk, sums of whole chunks,
//      positions behind them), in a fixed order, in fp32
// A gradient row is read once and a table row written once whatever the distribution; only the sort's lists are moved besides.
// ---------------------------------------------------------------------------------------------
constexpr int RUN_CHUNK = 64;
constexpr uint32_t EMPTY = 0xffffffffu;

__global__ __launch_bounds__(NT) void keys_kernel(const int32_t *ids, int64_t M, int64_t n_rows, int32_t *keys, uint32_t *first) {
    const int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x;
    if (i < M) { const int64_t id = ids[i]; keys[i] = (int32_t)(id >= 0 && id < n_rows ? id : n_rows); }
    if (i < n_rows) first[i] = EMPTY;
}

struct BwdArgs {
    const uint32_t *sk, *sp;                 // sorted keys and their positions
    uint32_t *first, *last;                  // [n_rows] run of each row
    float *part;                             // [ceil(M / RUN_CHUNK)][8 cg] sums of whole chunks
    const void *g; int64_t g_ld; int64_t M;
    void *out; int64_t out_ld; int64_t n_rows;
    int dim, cg, accumulate; float scale; KgeDropDev drop;
};

// adds D_i o g[i, group] of n positions sp[0 .. n) in order
template <bool G16> __device__ __forceinline__ void add_rows(const BwdArgs &a, uint32_t step, const uint32_t *sp, int n, int grp, float (&s)[8]) {
    const int cols = a.dim - 8 * grp;
    int k = 0;
    for (; k + 8 <= n; k += 8) {
        uint32_t p[8];
        float v[8][8];
#pragma unroll
        for (int u = 0; u < 8; ++u) p[u] = sp[k + u];
#pragma unroll
        for (int u = 0; u < 8; ++u) kge_load8<G16>((const char *)a.g + (int64_t)p[u] * a.g_ld * (G16 ? 2 : 4), 8 * grp, cols, v[u]);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (a.drop.thr) kge_drop8(a.drop, step, p[u], (uint32_t)grp, v[u]);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += v[u][e];
        }
    }
    for (; k < n; ++k) {
        const uint32_t p = sp[k];
        float v[8];
        kge_load8<G16>((const char *)a.g + (int64_t)p * a.g_ld * (G16 ? 2 : 4), 8 * grp, cols, v);
        if (a.drop.thr) kge_drop8(a.drop, step, p, (uint32_t)grp, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += v[e];
    }
}

// One workgroup per chunk of RUN_CHUNK sorted positions.
template <bool G16>
__global__ __launch_bounds__(NT) void runs_kernel(const BwdArgs a) {
    const uint32_t step = a.drop.thr ? kge_drop_step(a.drop) : 0u;
    for (int64_t c0 = (int64_t)blockIdx.x * RUN_CHUNK; c0 < a.M; c0 += (int64_t)gridDim.x * RUN_CHUNK) {
    if (threadIdx.x < RUN_CHUNK) {
        const int64_t k = c0 + threadIdx.x;
        if (k < a.M) {
            const uint32_t key = a.sk[k];
            if (key < a.n_rows) {
                if (k == 0 || a.sk[k - 1] != key) a.first[key] = (uint32_t)k;
                if (k == a.M - 1 || a.sk[k + 1] != key) a.last[key] = (uint32_t)(k + 1);
            }
        }
    }
    if (c0 + RUN_CHUNK > a.M) break;
    const uint32_t key = a.sk[c0];
    if (key >= a.n_rows || key != a.sk[c0 + RUN_CHUNK - 1]) continue;   // (equal keys lie together: equal ends, equal chunk)
    for (int grp = threadIdx.x; grp < a.cg; grp += NT) {
        float s[8] = {};
        add_rows<G16>(a, step, a.sp + c0, RUN_CHUNK, grp, s);
        float *p = a.part + (c0 / RUN_CHUNK * a.cg + grp) * 8;
        *(kge_f32x4 *)p = kge_f32x4{s[0], s[1], s[2], s[3]};
        *(kge_f32x4 *)(p + 4) = kge_f32x4{s[4], s[5], s[6], s[7]};
    }
    }
}

// 2^lp threads take a row (lp = 6: one wave, which walks the row's groups); 256 >> lp rows per workgroup
template <bool G16, bool OUT16>
__global__ __launch_bounds__(NT) void row_sums_kernel(const BwdArgs a, int lp) {
    const int per = 1 << lp, grp0 = threadIdx.x & (per - 1);
    const uint32_t step = a.drop.thr ? kge_drop_step(a.drop) : 0u;
    for (int64_t r = (int64_t)blockIdx.x * (NT >> lp) + (threadIdx.x >> lp); r < a.n_rows; r += (int64_t)gridDim.x * (NT >> lp)) {
    const uint32_t k0 = a.M ? a.first[r] : EMPTY;
    if (k0 == EMPTY && a.accumulate) continue;
    const uint32_t k1 = k0 == EMPTY ? 0 : a.last[r];
    const uint32_t c0 = (k0 + RUN_CHUNK - 1) / RUN_CHUNK, c1 = k1 / RUN_CHUNK;         // whole chunks [c0, c1)
    char *orow = (char *)a.out + r * a.out_ld * (OUT16 ? 2 : 4);
    for (int grp = grp0; grp < a.cg; grp += per) {
        float s[8] = {};
        if (k0 != EMPTY) {
            if (c0 >= c1) add_rows<G16>(a, step, a.sp + k0, (int)(k1 - k0), grp, s);
            else {
                add_rows<G16>(a, step, a.sp + k0, (int)(c0 * RUN_CHUNK - k0), grp, s);
                for (uint32_t c = c0; c < c1; ++c) {
                    const float *p = a.part + ((int64_t)c * a.cg + grp) * 8;
                    const kge_f32x4 x = *(const kge_f32x4 *)p, y = *(const kge_f32x4 *)(p + 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) { s[e] += x[e]; s[4 + e] += y[e]; }
                }
                add_rows<G16>(a, step, a.sp + c1 * RUN_CHUNK, (int)(k1 - c1 * RUN_CHUNK), grp, s);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] *= a.scale;
        }
        const int n = a.dim - 8 * grp;
        if (a.accumulate) {
            float o[8];
            kge_load8<OUT16>(orow, 8 * grp, n, o);
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += o[e];
        }
        kge_store8<OUT16>(orow, 8 * grp, n, s);
    }
    }
}

struct BwdWs { int32_t *keys; uint32_t *first, *last; float *part; void *sort; };
size_t bwd_carve(int64_t M, int64_t n_rows, int dim, void *ws, BwdWs &w) {
    char *p = (char *)ws;
    size_t off = 0;
    auto take = [&](size_t bytes) { void *q = p ? p + off : nullptr; off += (bytes + 255) / 256 * 256; return q; };
    w.keys = (int32_t *)take((size_t)M * 4);
    w.first = (uint32_t *)take((size_t)n_rows * 4);
    w.last = (uint32_t *)take((size_t)n_rows * 4);
    w.part = (float *)take((size_t)(M / RUN_CHUNK) * ((dim + 7) / 8) * 32);
    w.sort = p ? p + off : nullptr;
    return off + kge_sort_ws(M);
}

bool bad_type(int32_t dtype) { return dtype != KGE_F32 && dtype != KGE_BF16; }
// rows of a matrix: a stride below the width would make them overlap, and the addresses have to be whole elements
bool bad_rows(const void *p, int32_t dtype, int64_t ld, int64_t cols) { return !p || ld < cols || ((uintptr_t)p & (dtype == KGE_BF16 ? 1 : 3)) != 0; }
constexpr int64_t MAX_ROWS = (1ll << 31) - 1, MAX_LD = 1ll << 31;
constexpr int MAX_DIM = 65536;

template <bool LOOKUP> int run_rows(const RowsArgs &a, bool in16, bool out16, hipStream_t st) {
    const dim3 grid = grid_of(a.M, a.rows);
    if (in16 && out16) hipLaunchKernelGGL((rows_kernel<LOOKUP, true, true>), grid, dim3(NT), 0, st, a);
    else if (!in16 && !out16) hipLaunchKernelGGL((rows_kernel<LOOKUP, false, false>), grid, dim3(NT), 0, st, a);
    else if constexpr (LOOKUP) {
        if (in16) hipLaunchKernelGGL((rows_kernel<true, true, false>), grid, dim3(NT), 0, st, a);
        else hipLaunchKernelGGL((rows_kernel<true, false, true>), grid, dim3(NT), 0, st, a);
    }
    return kge_launch_status();
}

}  // namespace

extern "C" {

int kge_embed(const void *table, int32_t table_dtype, int64_t n_rows, int32_t dim, int64_t ld, const int32_t *ids, int64_t M, float scale,
              const kge_dropout_t *drop, void *out, int32_t out_dtype, int64_t out_ld, void *hip_stream) {
    RowsArgs a = {};
    const int rc = kge_drop_dev(drop, &a.drop);
    if (rc != KGE_OK) return rc;
    if (bad_type(table_dtype) || bad_type(out_dtype) || dim < 1 || dim > MAX_DIM || n_rows < 0 || n_rows > MAX_ROWS || M < 0 || M > MAX_ROWS ||
        ld >= MAX_LD || out_ld >= MAX_LD) return KGE_E_INVALID_ARG;
    if (M == 0) return KGE_OK;
    if ((n_rows > 0 && bad_rows(table, table_dtype, ld, dim)) || !ids || bad_rows(out, out_dtype, out_ld, dim)) return KGE_E_INVALID_ARG;
    a.x = table; a.x_ld = ld; a.ids = ids; a.n_rows = n_rows; a.out = out; a.out_ld = out_ld; a.M = M; a.dim = dim;
    a.cg = kge_fast_div((uint32_t)(dim + 7) / 8); a.rows = rows_per_block((int)a.cg.d); a.scale = scale;
    return run_rows<true>(a, table_dtype == KGE_BF16, out_dtype == KGE_BF16, (hipStream_t)hip_stream);
}

int kge_dropout(const void *x, int64_t x_ld, const void *residual, int64_t residual_ld, void *out, int64_t out_ld, int32_t dtype, int64_t rows,
                int32_t cols, const kge_dropout_t *drop, void *hip_stream) {
    RowsArgs a = {};
    const int rc = kge_drop_dev(drop, &a.drop);
    if (rc != KGE_OK) return rc;
    if (!drop || bad_type(dtype) || cols < 0 || cols > MAX_DIM || rows < 0 || rows > MAX_ROWS || x_ld >= MAX_LD || out_ld >= MAX_LD ||
        residual_ld >= MAX_LD) return KGE_E_INVALID_ARG;
    if (rows == 0 || cols == 0) return KGE_OK;
    if (bad_rows(x, dtype, x_ld, cols) || bad_rows(out, dtype, out_ld, cols) || (residual && bad_rows(residual, dtype, residual_ld, cols)))
        return KGE_E_INVALID_ARG;
    a.x = x; a.x_ld = x_ld; a.res = residual; a.res_ld = residual_ld; a.out = out; a.out_ld = out_ld; a.M = rows; a.dim = cols;
    a.cg = kge_fast_div((uint32_t)(cols + 7) / 8); a.rows = rows_per_block((int)a.cg.d); a.scale = 1.f;
    return run_rows<false>(a, dtype == KGE_BF16, dtype == KGE_BF16, (hipStream_t)hip_stream);
}

size_t kge_embed_bwd_workspace_bytes(int64_t M, int64_t n_rows, int32_t dim) {
    if (M < 0 || M > MAX_ROWS || n_rows < 0 || n_rows >= MAX_ROWS || dim < 1 || dim > MAX_DIM) return 0;
    BwdWs w;
    return bwd_carve(M, n_rows, dim, nullptr, w) + 256;
}

int kge_embed_bwd(const void *g, int32_t g_dtype, int64_t g_ld, const int32_t *ids, int64_t M, float scale, const kge_dropout_t *drop,
                  void *g_table, int32_t table_dtype, int64_t n_rows, int32_t dim, int64_t ld, int32_t accumulate, void *ws, size_t ws_bytes,
                  void *hip_stream) {
    BwdArgs a = {};
    int rc = kge_drop_dev(drop, &a.drop);
    if (rc != KGE_OK) return rc;
    // (n_rows itself is a key of the sort: that of the positions without a row)
    if (bad_type(g_dtype) || bad_type(table_dtype) || dim < 1 || dim > MAX_DIM || n_rows < 0 || n_rows >= MAX_ROWS || M < 0 || M > MAX_ROWS ||
        g_ld >= MAX_LD || ld >= MAX_LD || (accumulate != 0 && accumulate != 1)) return KGE_E_INVALID_ARG;
    if (n_rows == 0 || (M == 0 && accumulate)) return KGE_OK;
    if (bad_rows(g_table, table_dtype, ld, dim) || (M > 0 && (!ids || bad_rows(g, g_dtype, g_ld, dim)))) return KGE_E_INVALID_ARG;
    if (!ws) return KGE_E_WORKSPACE_TOO_SMALL;
    const size_t lost = (256 - ((uintptr_t)ws & 255)) & 255;
    BwdWs w;
    if (bwd_carve(M, n_rows, dim, nullptr, w) + lost > ws_bytes) return KGE_E_WORKSPACE_TOO_SMALL;
    bwd_carve(M, n_rows, dim, (char *)ws + lost, w);
    hipStream_t st = (hipStream_t)hip_stream;
    a.first = w.first; a.last = w.last; a.part = w.part; a.g = g; a.g_ld = g_ld; a.M = M; a.out = g_table; a.out_ld = ld; a.n_rows = n_rows;
    a.dim = dim; a.cg = (dim + 7) / 8; a.accumulate = accumulate; a.scale = scale;
    const bool g16 = g_dtype == KGE_BF16, o16 = table_dtype == KGE_BF16;
    if (M > 0) {
        const int64_t n = M > n_rows ? M : n_rows;
        hipLaunchKernelGGL(keys_kernel, dim3((unsigned)((n + NT - 1) / NT)), dim3(NT), 0, st, ids, M, n_rows, w.keys, w.first);
        rc = kge_sort_pairs(w.keys, nullptr, nullptr, 1, 1, M, n_rows + 1, w.sort, &a.sk, &a.sp, st, nullptr, 0);
        if (rc != KGE_OK) return rc;
        const dim3 chunks = grid_of(M, RUN_CHUNK);
        if (g16) hipLaunchKernelGGL(runs_kernel<true>, chunks, dim3(NT), 0, st, a);
        else hipLaunchKernelGGL(runs_kernel<false>, chunks, dim3(NT), 0, st, a);
    }
    int lp = 0;
    while (lp < 6 && (1 << lp) < a.cg) ++lp;
    const dim3 grid = grid_of(n_rows, NT >> lp);
    if (g16 && o16) hipLaunchKernelGGL((row_sums_kernel<true, true>), grid, dim3(NT), 0, st, a, lp);
    else if (g16) hipLaunchKernelGGL((row_sums_kernel<true, false>), grid, dim3(NT), 0, st, a, lp);
    else if (o16) hipLaunchKernelGGL((row_sums_kernel<false, true>), grid, dim3(NT), 0, st, a, lp);
    else hipLaunchKernelGGL((row_sums_kernel<false, false>), grid, dim3(NT), 0, st, a, lp);
    return kge_launch_status();
}

}  // extern "C"
