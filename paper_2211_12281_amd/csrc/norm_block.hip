// Norms before and after a block, fused with its gate and residual scale, forward and backward.
//
//   forward    h = x + s o g o N_post(y),   z = N_pre(h)          N(v) = w o v^ + b,  v^ = (v - mu) r   (rms: mu = 0),  r = 1 / sqrt(var + eps)
//   backward   d  = dh + N_pre'(dz)                               N'(q) = r (t - [mean t] - v^ mean(t o v^)),  t = w o q   ([..]: layer norms)
//              dx = d,   dy = N_post'(s o g o d)
//              with A = sum over rows of g o d o y^ and B = sum of g o d:   ds = w o A + b o B,   dw_post = s o A,   db_post = s o B
//              dg of a group of rows = s o (w o A' + b o B') with A', B' its sums of d o y^ and d;   dw_pre = sum of dz o h^,   db_pre = sum of dz
//
// So the backward pass has four column sums at most, whatever is asked for.  A row's statistics are computed again from h and y, which it has to read
// anyway: nothing is stored between the passes.
//
// Memory bounds both: a row is read once, held in registers by part of a wave (norm_block.hpp), one wave (up to 1,024 columns) or several, and its sums stay there for the run of rows that a
// workgroup takes.  24,576 x 768, layer norms, fp32 stream, bf16 block, gates of 96 rows: forward 42-43 us (227 MB, 5.3 TB/s), backward 76 (340 MB, 4.5 TB/s) and 10 for the launch
// that joins the runs' sums, most of it the wait for what the rows' launch has written (behind small calls it takes 4); one row 3.7 us, a launch and three trips to memory.
// No row is fetched ahead: the registers that it takes are a wave per SIMD (backward with 82, without 77 us; forward 58 and 42).
#include "norm_block.hpp"

namespace {

using namespace kge_norm;

// ---------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------
// A team takes R rows at a time; the vectors stand in the LDS (rows of eight waves: in memory, from where they are read for every turn, more bytes than a row has of its own, so that
// two rows share them and the barriers of their sums: 7,256 x 3,304 86 us and not 114, 5,000 x 4,000 65 and 81, 3,000 x 8,192 88 and 102; with three groups a lane two rows lose,
// 4,000 x 6,000 98 and 82, and where every row has a workgroup they take longer, 10 x 4,096 7.5 and 6.0).
enum { VEC_POST = 0, VEC_POST_BIAS = 1, VEC_SCALE = 2, VEC_PRE = 3, VEC_PRE_BIAS = 4, VECTORS = 5 };
template <bool S16, bool B16, int NG, int SUB, int NT, int OCC, int R>
__global__ __launch_bounds__(NT, OCC) void norm_fwd_kernel(const FwdArgs a) {
    constexpr bool LDS = NT == 256;
    __shared__ float red[2][NT / 64][R];
    extern __shared__ __attribute__((aligned(16))) float vec[];
    const Team<SUB> t(a.waves);
    Reduce<R, NT, SUB> reduce(red, t);
    const Columns<NG> c(a.dim, t.lane, t.size);
    const float inv_dim = 1.f / (float)a.dim;
    const int wide = 4 * t.size * NG;
    const float *const from[VECTORS] = {a.post.w, a.post.b, a.scale, a.pre.w, a.pre.b};
    auto vector = [&](int which, int k) {
        return LDS ? *(const kge_f32x4 *)(vec + which * wide + c.col(k)) : vector4(from[which], c.col(k), a.dim, which == VEC_POST_BIAS || which == VEC_PRE_BIAS ? 0.f : 1.f);
    };
    const int64_t step = (int64_t)gridDim.x * t.teams * R, first = (int64_t)blockIdx.x * t.teams * R;
    Raw<S16> x[R][NG];
    Raw<B16> y[R][NG], g[R][NG];
    auto load = [&](int64_t row0) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = row0 + r;
            const bool in = row < a.rows;
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                x[r][k].load(a.x.row(row), c, k, in && a.x.p);
                y[r][k].load(a.y.row(row), c, k, in && a.y.p);
                g[r][k].load(a.gate.row(a.gate.p && in ? (uint32_t)row / a.gate_rows : 0), c, k, in && a.gate.p);
            }
        }
    };
    load(first + t.team * R);                                     // (under the loads of the vectors; later rows' wait for nobody but their own wave)
    if constexpr (LDS) {
        for (int i = 4 * threadIdx.x; i < wide; i += 4 * NT)
#pragma unroll
            for (int v = 0; v < VECTORS; ++v)
                *(kge_f32x4 *)(vec + v * wide + i) = vector4(from[v], i, a.dim, v == VEC_POST_BIAS || v == VEC_PRE_BIAS ? 0.f : 1.f);
        __syncthreads();
    }
    for (int64_t r0 = first; r0 < a.rows; r0 += step) {           // (every team goes round equally often: the waves of one meet at barriers)
        if constexpr (!LDS) asm volatile("" ::: "memory");        // (the vectors are read for every turn: no registers for them in between)
        const int64_t row0 = r0 + t.team * R;
        bool in[R];
#pragma unroll
        for (int r = 0; r < R; ++r) in[r] = row0 + r < a.rows;
        if (r0 > first) load(row0);
        kge_f32x4 h[R][NG], u[R][NG], f[R][NG];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int k = 0; k < NG; ++k) { h[r][k] = x[r][k].values(); u[r][k] = y[r][k].values(); f[r][k] = g[r][k].values(); }
        if (a.y.p) {
            if (a.post.on) {
                normalise(u, c, a.post, inv_dim, reduce);
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    const kge_f32x4 w = vector(VEC_POST, k), b = vector(VEC_POST_BIAS, k);
#pragma unroll
                    for (int r = 0; r < R; ++r) u[r][k] = fma4(u[r][k], w, b);
                }
            }
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                if (a.scale) {
                    const kge_f32x4 s = vector(VEC_SCALE, k);
#pragma unroll
                    for (int r = 0; r < R; ++r) u[r][k] *= s;
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    h[r][k] = a.gate.p ? fma4(u[r][k], f[r][k], h[r][k]) : u[r][k] + h[r][k];
                    if (a.h.p && in[r] && c.inside(k)) store<S16>(a.h.row(row0 + r), c, k, h[r][k], a.stream);
                }
            }
        }
        if (a.pre.on) {
            normalise(h, c, a.pre, inv_dim, reduce);
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                if (!in[0] || !c.inside(k)) continue;
                const kge_f32x4 w = vector(VEC_PRE, k), b = vector(VEC_PRE_BIAS, k);
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (in[r]) store<B16>(a.z.row(row0 + r), c, k, fma4(h[r][k], w, b), a.stream);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// backward: column sums
// ---------------------------------------------------------------------------------------------
// Sixteen columns (four lanes of four) and 256 slices of the rows per workgroup; the slices' sums are added in a fixed order, two of them at once.
constexpr int JC = 16, JT = 1024, JL = JC / 4, JS = JT / JL;
typedef float JoinLds[2][JS][JC + 1];
__device__ __forceinline__ void add_slices(const kge_f32x4 (&v)[2], float (&sum)[2], JoinLds &lds) {
    const int l = threadIdx.x % JL, s = threadIdx.x / JL, c = threadIdx.x % JC, q = threadIdx.x / JC;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) lds[i][s][4 * l + e] = v[i][e];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) sum[i] = (lds[i][4 * q][c] + lds[i][4 * q + 1][c]) + (lds[i][4 * q + 2][c] + lds[i][4 * q + 3][c]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) lds[i][q][c] = sum[i];
    __syncthreads();
    if (threadIdx.x >= JC) return;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        sum[i] = 0.f;
#pragma unroll
        for (int k = 0; k < JT / JC; ++k) sum[i] += lds[i][k][c];
    }
}

// v[i] += rows r0, r0 + step, ... of p[i]; four of them in flight, at the end too (the last one's again, which do not count)
__device__ __forceinline__ void add_rows(const float *const (&p)[2], kge_f32x4 (&v)[2], int64_t r0, int64_t end, int64_t step, int64_t ld) {
    for (int64_t r = r0; r < end; r += 4 * step) {
        kge_f32x4 x[4][2];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) x[k][i] = *(const kge_f32x4 *)(p[i] + (r + k * step < end ? r + k * step : r) * ld);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[i][e] += r + k * step < end ? x[k][i][e] : 0.f;
    }
}

// Groups whose rows were many runs: their gates' gradients, and their sums times the gates in the place of their first run's.  A lane has four columns; sixteen
// waves share a group's runs.
constexpr int GROUP_SLICES = 16;
template <bool B16> __global__ __launch_bounds__(64 * GROUP_SLICES) void norm_groups_kernel(const BwdArgs a) {
    __shared__ kge_f32x4 lds[GROUP_SLICES][64];
    const int tiles = (int)((a.part_ld + 255) / 256), lane = threadIdx.x & 63, slice = threadIdx.x >> 6;
    const int64_t group = blockIdx.x / (uint32_t)tiles, col = (int64_t)(blockIdx.x - group * tiles) * 256 + 4 * lane;
    kge_f32x4 s[2] = {splat(0.f), splat(0.f)};
    float *const p0 = a.part + group * a.parts * a.part_ld + col;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        if (!(a.want >> w & 1)) continue;
        if (col < a.part_ld) {
            const float *p = p0 + (int64_t)w * a.runs * a.part_ld;
#pragma unroll 8
            for (int r = slice; r < a.parts; r += GROUP_SLICES) s[w] += *(const kge_f32x4 *)(p + r * a.part_ld);
        }
        lds[slice][lane] = s[w];
        __syncthreads();
        s[w] = lds[0][lane];
#pragma unroll
        for (int i = 1; i < GROUP_SLICES; ++i) s[w] += lds[i][lane];
        __syncthreads();
    }
    if (slice > 0) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (col + e >= a.dim) break;
        const float g = load1<B16>(a.gate.row(group), col + e);
        if (a.g_gate.p) {
            const float sc = a.scale ? a.scale[col + e] : 1.f, w = a.post.w ? a.post.w[col + e] : 1.f, b = a.post.b ? a.post.b[col + e] : 0.f;
            store1<B16>(a.g_gate.row(group), col + e, sc * of_sums(w, s[0][e], b, s[1][e], a.post.b));
        }
#pragma unroll
        for (int w = 0; w < 2; ++w)
            if (a.want >> w & 1) p0[(int64_t)w * a.runs * a.part_ld + e] = g * s[w][e];
    }
}

// Sums over all runs, and the gradients of the vectors; where a group is a few runs (each), the gates' gradients too.  FOLDED: norm_groups_kernel has left one
// row of sums for each group.
template <bool B16> __global__ __launch_bounds__(JT) void norm_join_kernel(const BwdArgs a, const bool folded) {
    __shared__ JoinLds lds;
    const int l = threadIdx.x % JL, slice = threadIdx.x / JL;
    const int64_t col = (int64_t)blockIdx.x * JC;
    const bool branch = blockIdx.y == 0, each = branch && a.parts > 0 && !folded;
    const uint32_t want = branch ? a.want : a.want >> 2;
    const float *p[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)                                   // (a sum that is not wanted is not there: the other one's again, for nothing)
        p[i] = a.part + (int64_t)((branch ? 0 : 2) + (want >> i & 1 ? i : 1 - i)) * a.runs * a.part_ld + col + 4 * l;
    kge_f32x4 v[2] = {splat(0.f), splat(0.f)};
    if (each) {
        const kge_f32x4 sc = vector4(a.scale, (int)col + 4 * l, a.dim, 1.f), w = vector4(a.post.w, (int)col + 4 * l, a.dim, 1.f), b = vector4(a.post.b, (int)col + 4 * l, a.dim, 0.f);
        const int64_t groups = a.runs / a.parts;
        for (int64_t g = slice; g < groups; g += JS) {
            kge_f32x4 s[2] = {splat(0.f), splat(0.f)}, gate;
#pragma unroll
            for (int e = 0; e < 4; ++e) gate[e] = col + 4 * l + e < a.dim ? load1<B16>(a.gate.row(g), col + 4 * l + e) : 0.f;
            add_rows(p, s, g * a.parts, (g + 1) * a.parts, 1, a.part_ld);
            if (a.g_gate.p) {
                const kge_f32x4 d = sc * of_sums(w, s[0], b, s[1], a.post.b);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + 4 * l + e < a.dim) store1<B16>(a.g_gate.row(g), col + 4 * l + e, d[e]);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) v[i] = fma4(gate, s[i], v[i]);
        }
    } else {
        const int64_t ld = branch && folded ? a.parts * a.part_ld : a.part_ld, n = branch && folded ? a.runs / a.parts : a.runs;
        if (want & 3) add_rows(p, v, slice, n, JS, ld);
    }
    float s[2];
    add_slices(v, s, lds);
    const int c = threadIdx.x;
    if (c >= JC || col + c >= a.dim) return;
    auto put = [&](float *q, float x) {
        if (q) q[col + c] = a.accumulate ? q[col + c] + x : x;
    };
    if (!branch) { put(a.g_prew, s[0]); put(a.g_preb, s[1]); return; }
    const float sc = a.scale ? a.scale[col + c] : 1.f, w = a.post.w ? a.post.w[col + c] : 1.f, b = a.post.b ? a.post.b[col + c] : 0.f;
    put(a.g_scale, of_sums(w, s[0], b, s[1], a.post.b));
    put(a.g_postw, sc * s[0]);
    put(a.g_postb, sc * s[1]);
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
constexpr int64_t FWD_GROUPS = 2048, PAIRS_FROM = 512, FEW = 2;
constexpr int64_t MANY_PARTS = 16;                              // runs of a group from which on its sums are a launch of their own

bool bad_norm(const kge_norm_t *n) {
    return n && ((n->kind != KGE_NORM_RMS && n->kind != KGE_NORM_LAYER) || !(n->eps > 0.f) || n->eps > 3e38f || ((uintptr_t)n->weight & 3) != 0 ||
                 ((uintptr_t)n->bias & 3) != 0);
}
int check_block(const kge_norm_block_t *b, bool y) {
    if (!b || b->dim < 1 || kge_bad_type(b->stream_dtype) || kge_bad_type(b->block_dtype) || b->reserved != 0 || bad_norm(b->post) || bad_norm(b->pre) ||
        ((uintptr_t)b->scale & 3) != 0) return KGE_E_INVALID_ARG;
    if (!y && (b->post || b->scale || b->gate)) return KGE_E_INVALID_ARG;
    if (!y && !b->pre) return KGE_E_INVALID_ARG;                   // (nothing to do)
    if (b->gate && (b->gate_rows < 1 || kge_bad_rows(b->gate, b->block_dtype, b->gate_ld, b->dim) || b->gate_ld >= KGE_MAX_LD)) return KGE_E_INVALID_ARG;
    return b->dim > MAX_DIM ? KGE_E_UNSUPPORTED : KGE_OK;
}
// a matrix that may be absent
bool bad_matrix(const void *p, int32_t dtype, int64_t ld, int64_t cols) { return p && (kge_bad_rows(p, dtype, ld, cols) || ld >= KGE_MAX_LD); }

Norm norm_of(const kge_norm_t *n) {
    return n ? Norm{true, n->kind == KGE_NORM_LAYER, n->eps, n->weight, n->bias} : Norm{false, false, 1.f, nullptr, nullptr};
}
// Runs of rows of the backward pass: as many as the chip holds at once, of a row for each team at least.  Groups of rows with a gate: whole ones, where every second
// team can have one to itself; else a group is a run or several, so many that the chip's rounds take least.
struct Runs { int64_t run, runs, parts; };
Runs runs_of(const kge_norm_block_t *b, int64_t rows) {
    const int64_t wanted = bwd_runs_of(b->dim), teams = bwd_teams_of(b->dim);
    int64_t run = (rows + wanted - 1) / wanted;
    if (run < teams) run = teams;
    if (b->gate && b->gate_rows > 1) {
        const int64_t len = b->gate_rows < rows ? b->gate_rows : rows, groups = (rows + len - 1) / len;
        if (2 * groups >= wanted * teams) {
            run = (run + len * teams - 1) / (len * teams) * (len * teams);
            return {run, (rows + run - 1) / run, 0};
        }
        int64_t parts = 1, least = 0;
        for (int64_t p = wanted / groups > 1 ? wanted / groups : 1, k = 0; k < 3; ++k, ++p) {
            if (k > 0 && (len + p - 1) / p < teams) break;
            const int64_t cost = (groups * p + wanted - 1) / wanted * ((len + p * teams - 1) / (p * teams) + 2);     // rows of a team and what a run costs besides
            if (k == 0 || cost < least) { least = cost; parts = p; }
        }
        if (parts > (len + teams - 1) / teams) parts = (len + teams - 1) / teams;
        return {(len + parts - 1) / parts, groups * parts, parts};
    }
    if (rows <= FEW * teams) run = rows;                          // (a launch costs more than the longer run)
    return {run, (rows + run - 1) / run, 0};
}
// No call of up to so many rows has more runs: without gates and with whole groups at most `wanted`; else there are fewer than wanted teams / 2 groups, and groups parts runs, parts at
// most wanted / groups + 2 (3 where there are more groups than that): fewer than wanted + 3 wanted teams / 2; and as a run of a whole group has a row, fewer than 2 rows.
int64_t most_runs(const kge_norm_block_t *b, int64_t rows) {
    const int64_t all = bwd_runs_of(b->dim) * (b->gate && b->gate_rows > 1 ? 2 * bwd_teams_of(b->dim) + 3 : 1);
    return 2 * rows < all ? 2 * rows : all;
}
int64_t part_ld_of(int dim) { return (dim + JC - 1) / JC * JC; }

template <bool S16, bool B16> int launch_fwd(const FwdArgs &a, hipStream_t st) {
    const int lanes = fwd_lanes_of(a.dim), teams = lanes < 256 ? 256 / lanes : 1, ng = groups_of(a.dim, lanes);
    const bool pairs = a.waves == 8 && ng != 3 && a.rows > PAIRS_FROM;
    int64_t groups = (a.rows + teams - 1) / teams;
    if (groups > FWD_GROUPS) groups = FWD_GROUPS;
    const dim3 grid((unsigned)groups), blk(lanes * teams);
    const int lds = a.waves <= 2 ? VECTORS * 4 * lanes * ng * (int)sizeof(float) : 0;                   // 60 KB at most
#define KGE_FWD(NG, SUB, NT, OCC, R)                                                                                                    \
    do {                                                                                                                        \
        static KgeLdsLimit limit;                                                                                               \
        const auto kern = norm_fwd_kernel<S16, B16, NG, SUB, NT, OCC, R>;                                                               \
        if (lds > 48 * 1024 && limit.set((const void *)kern, 60 * 1024) != KGE_OK) return KGE_E_HIP;                                     \
        hipLaunchKernelGGL(kern, grid, blk, lds, st, a);                                                                        \
    } while (0)
    if (a.waves == 8) {
        if (ng == 3) KGE_FWD(3, 64, 512, 4, 1);
        else if (ng == 2) { if (pairs) KGE_FWD(2, 64, 512, 4, 2); else KGE_FWD(2, 64, 512, 4, 1); }
        else if (pairs) KGE_FWD(4, 64, 512, 2, 2);
        else KGE_FWD(4, 64, 512, 2, 1);
    } else if (lanes == 16) {
        if (ng == 1) KGE_FWD(1, 16, 256, 8, 1);
        else KGE_FWD(2, 16, 256, 8, 1);
    } else switch (ng) {
    case 1: KGE_FWD(1, 64, 256, 8, 1); break;
    case 2: KGE_FWD(2, 64, 256, 6, 1); break;
    case 3: KGE_FWD(3, 64, 256, 4, 1); break;
    case 4: KGE_FWD(4, 64, 256, 4, 1); break;
    case 5: KGE_FWD(5, 64, 256, 2, 1); break;
    default: KGE_FWD(6, 64, 256, 2, 1);
    }
#undef KGE_FWD
    return kge_launch_status();
}

}  // namespace

extern "C" {

int kge_norm_block(const kge_norm_block_t *blk, const void *x, int64_t x_ld, const void *y, int64_t y_ld, int64_t rows, void *h, int64_t h_ld,
                   void *z, int64_t z_ld, void *hip_stream) {
    if (!blk || rows < 0 || rows > KGE_MAX_ROWS) return KGE_E_INVALID_ARG;
    const bool branch = y || blk->post || blk->scale || blk->gate;
    const int rc = check_block(blk, branch);
    if (rc == KGE_E_INVALID_ARG) return rc;
    if (rows == 0) return rc;
    if ((branch && !y) || (!x && !y) || (!branch && h) || (blk->pre ? !z : z != nullptr) || (!blk->pre && !h) || bad_matrix(x, blk->stream_dtype, x_ld, blk->dim) ||
        bad_matrix(y, blk->block_dtype, y_ld, blk->dim) || bad_matrix(h, blk->stream_dtype, h_ld, blk->dim) ||
        bad_matrix(z, blk->block_dtype, z_ld, blk->dim)) return KGE_E_INVALID_ARG;
    if (rc != KGE_OK) return rc;
    const bool s16 = blk->stream_dtype == KGE_BF16, b16 = blk->block_dtype == KGE_BF16;
    FwdArgs a = {};
    a.dim = blk->dim; a.waves = fwd_waves_of(blk->dim); a.rows = rows;
    a.post = norm_of(blk->post); a.pre = norm_of(blk->pre); a.scale = blk->scale;
    a.gate = matrix((void *)blk->gate, blk->gate_ld, b16); a.gate_rows = (uint32_t)(blk->gate_rows < rows ? blk->gate_rows : rows);
    a.x = matrix((void *)x, x_ld, s16); a.y = matrix((void *)y, y_ld, b16); a.h = matrix(h, h_ld, s16); a.z = matrix(z, z_ld, b16);
    a.stream = rows * blk->dim * ((h ? (s16 ? 2 : 4) : 0) + (z ? (b16 ? 2 : 4) : 0)) >= KGE_STREAM_BYTES;
    hipStream_t st = (hipStream_t)hip_stream;
    if (s16) return b16 ? launch_fwd<true, true>(a, st) : launch_fwd<true, false>(a, st);
    return b16 ? launch_fwd<false, true>(a, st) : launch_fwd<false, false>(a, st);
}

size_t kge_norm_block_bwd_workspace_bytes(const kge_norm_block_t *blk, int64_t rows) {
    if (rows < 0 || rows > KGE_MAX_ROWS || !blk || check_block(blk, blk->post || blk->scale || blk->gate || !blk->pre) != KGE_OK) return 0;
    return (size_t)most_runs(blk, rows) * 4 * part_ld_of(blk->dim) * sizeof(float) + 256;
}

int kge_norm_block_bwd(const kge_norm_block_t *blk, const void *h, int64_t h_ld, const void *y, int64_t y_ld, const void *dh, int64_t dh_ld,
                       const void *dz, int64_t dz_ld, int64_t rows, void *dx, int64_t dx_ld, void *dy, int64_t dy_ld,
                       const kge_norm_block_grads_t *grads, void *ws, size_t ws_bytes, void *hip_stream) {
    if (!blk || rows < 0 || rows > KGE_MAX_ROWS) return KGE_E_INVALID_ARG;
    const bool branch = y || blk->post || blk->scale || blk->gate;
    const int rc = check_block(blk, branch);
    if (rc == KGE_E_INVALID_ARG) return rc;
    kge_norm_block_grads_t none = {};
    const kge_norm_block_grads_t &w = grads ? *grads : none;
    if (w.reserved != 0 || (w.accumulate != 0 && w.accumulate != 1)) return KGE_E_INVALID_ARG;
    for (const float *p : {w.post_weight, w.post_bias, w.pre_weight, w.pre_bias, w.scale})
        if (((uintptr_t)p & 3) != 0) return KGE_E_INVALID_ARG;
    // a gradient of what is not there
    if ((w.post_weight && !(blk->post && blk->post->weight)) || (w.post_bias && !(blk->post && blk->post->bias)) || (w.pre_weight && !(blk->pre && blk->pre->weight)) ||
        (w.pre_bias && !(blk->pre && blk->pre->bias)) || (w.scale && !blk->scale) || (w.gate && !blk->gate)) return KGE_E_INVALID_ARG;
    if (bad_matrix(w.gate, blk->block_dtype, w.gate_ld, blk->dim)) return KGE_E_INVALID_ARG;
    if (rows > 0 && ((branch && !y) || (blk->pre && (!h || !dz)) || (!blk->pre && (dz || !dh)) || (dy && !y) || bad_matrix(h, blk->stream_dtype, h_ld, blk->dim) ||
                     bad_matrix(y, blk->block_dtype, y_ld, blk->dim) || bad_matrix(dh, blk->stream_dtype, dh_ld, blk->dim) ||
                     bad_matrix(dz, blk->block_dtype, dz_ld, blk->dim) || bad_matrix(dx, blk->stream_dtype, dx_ld, blk->dim) ||
                     bad_matrix(dy, blk->block_dtype, dy_ld, blk->dim))) return KGE_E_INVALID_ARG;
    if (rc != KGE_OK) return rc;
    const bool s16 = blk->stream_dtype == KGE_BF16, b16 = blk->block_dtype == KGE_BF16;
    BwdArgs a = {};
    a.dim = blk->dim; a.waves = waves_of(blk->dim); a.rows = rows;
    a.post = norm_of(blk->post); a.pre = norm_of(blk->pre); a.scale = blk->scale;
    a.gate = matrix((void *)blk->gate, blk->gate_ld, b16); a.gate_rows = (uint32_t)(blk->gate_rows < rows ? blk->gate_rows : rows);
    if (blk->gate && blk->gate_rows > 1 && a.gate_rows == 1) a.gate_rows = 2;                 // (one row in a longer group: still a gate of a group)
    a.h = matrix((void *)h, h_ld, s16); a.y = matrix((void *)y, y_ld, b16); a.dh = matrix((void *)dh, dh_ld, s16); a.dz = matrix((void *)dz, dz_ld, b16);
    a.dx = matrix(dx, dx_ld, s16); a.dy = matrix(dy, dy_ld, b16); a.g_gate = matrix(w.gate, w.gate_ld, b16);
    a.g_postw = w.post_weight; a.g_postb = w.post_bias; a.g_prew = w.pre_weight; a.g_preb = w.pre_bias; a.g_scale = w.scale; a.accumulate = w.accumulate;
    a.stream = rows * blk->dim * ((dx ? (s16 ? 2 : 4) : 0) + (dy ? (b16 ? 2 : 4) : 0)) >= KGE_STREAM_BYTES;
    const Runs q = rows > 0 ? runs_of(blk, rows) : Runs{0, 0, 0};
    a.run = q.run; a.runs = q.runs; a.parts = (int)q.parts; a.part_ld = part_ld_of(blk->dim);
    const bool bias = blk->post && blk->post->bias, of_group = w.gate && q.parts > 0;         // (parts: of gates of groups alone)
    if (w.scale || w.post_weight || of_group) a.want |= 1u << SUM_A;
    if (w.post_bias || (bias && (w.scale || of_group))) a.want |= 1u << SUM_B;
    if (w.pre_weight) a.want |= 1u << SUM_C;
    if (w.pre_bias) a.want |= 1u << SUM_D;
    if (a.want && q.runs != 1) {
        const size_t lost = ws ? (256 - ((uintptr_t)ws & 255)) & 255 : 0, need = (size_t)q.runs * 4 * a.part_ld * sizeof(float);
        if (need && (!ws || ws_bytes < lost + need)) return KGE_E_WORKSPACE_TOO_SMALL;
        a.part = (float *)((char *)ws + lost);
    }
    const bool folded = q.parts > MANY_PARTS && q.runs > 1 && (a.want & 3);
    hipStream_t st = (hipStream_t)hip_stream;
    if (rows > 0) {
        if (const int e = s16 ? rows_bwd16(a, b16, st) : rows_bwd32(a, b16, st)) return e;
        if (folded) {
            const dim3 grid((unsigned)(q.runs / q.parts * ((a.part_ld + 255) / 256)));
            if (b16) hipLaunchKernelGGL((norm_groups_kernel<true>), grid, dim3(64 * GROUP_SLICES), 0, st, a);
            else hipLaunchKernelGGL((norm_groups_kernel<false>), grid, dim3(64 * GROUP_SLICES), 0, st, a);
        }
    }
    const bool vectors = w.scale || w.post_weight || w.post_bias || w.pre_weight || w.pre_bias;
    if (q.runs != 1 && (vectors || (of_group && !folded && rows > 0))) {
        const dim3 grid((unsigned)(a.part_ld / JC), a.want >> 2 ? 2 : 1);
        if (b16) hipLaunchKernelGGL(norm_join_kernel<true>, grid, dim3(JT), 0, st, a, folded);
        else hipLaunchKernelGGL(norm_join_kernel<false>, grid, dim3(JT), 0, st, a, folded);
    }
    return rows > 0 || vectors ? kge_launch_status() : KGE_OK;
}

}  // extern "C"
