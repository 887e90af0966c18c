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
#include "norm_block.hpp"

namespace {

using namespace kge_norm;

// ---------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------
template <bool S16, bool B16, int NG, int NT>
__global__ __launch_bounds__(NT) void norm_fwd_kernel(const FwdArgs a) {
    __shared__ float red[2][NT / 64][2];
    const Team t(a.waves);
    Reduce<2, NT> reduce(red, t);
    const float inv_dim = 1.f / (float)a.dim;
    int col[NG], n[NG];
    Vec postw[NG], postb[NG], scale[NG], prew[NG], preb[NG];
#pragma unroll
    for (int k = 0; k < NG; ++k) {
        col[k] = 8 * (t.lane + k * t.size);
        n[k] = a.dim - col[k];
        postw[k].vector(a.post.w, col[k], n[k], 1.f); postb[k].vector(a.post.b, col[k], n[k], 0.f);
        prew[k].vector(a.pre.w, col[k], n[k], 1.f); preb[k].vector(a.pre.b, col[k], n[k], 0.f);
        scale[k].vector(a.scale, col[k], n[k], 1.f);
    }
    const int64_t step = (int64_t)gridDim.x * t.teams, first = (int64_t)blockIdx.x * t.teams;
    Raw<S16> x[NG];
    Raw<B16> y[NG], g[NG];
    auto load = [&](int64_t row) {
        const bool in = row < a.rows;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            const int m = in ? n[k] : 0;
            x[k].load(a.x.row(row), col[k], a.x.p ? m : 0);
            y[k].load(a.y.row(row), col[k], a.y.p ? m : 0);
            g[k].load(a.gate.row(a.gate.p && in ? (uint32_t)row / a.gate_rows : 0), col[k], a.gate.p ? m : 0);
        }
    };
    load(first + t.team);
    for (int64_t r0 = first; r0 < a.rows; r0 += step) {           // (every team goes round equally often: the waves of one meet at barriers)
        const int64_t row = r0 + t.team;
        const bool in = row < a.rows;
        Vec h[NG], u[NG], gv[NG];
#pragma unroll
        for (int k = 0; k < NG; ++k) { x[k].values(h[k]); y[k].values(u[k]); g[k].values(gv[k]); }
        if (r0 + step < a.rows) load(row + step);
        if (a.y.p) {
            if (a.post.on) {
                const Stats s = statistics<NG>(u, n, a.post, inv_dim, reduce);
#pragma unroll
                for (int k = 0; k < NG; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) u[k].v[e] = fmaf((u[k].v[e] - s.mean) * s.r, postw[k].v[e], postb[k].v[e]);
            }
#pragma unroll
            for (int k = 0; k < NG; ++k) {
#pragma unroll
                for (int e = 0; e < 8; ++e) h[k].v[e] = fmaf(u[k].v[e], scale[k].v[e] * (a.gate.p ? gv[k].v[e] : 1.f), h[k].v[e]);
                if (a.h.p && in) kge_store8<S16>(a.h.row(row), col[k], n[k], h[k].v);
            }
        }
        if (a.pre.on) {
            const Stats s = statistics<NG>(h, n, a.pre, inv_dim, reduce);
#pragma unroll
            for (int k = 0; k < NG; ++k) {
#pragma unroll
                for (int e = 0; e < 8; ++e) h[k].v[e] = fmaf((h[k].v[e] - s.mean) * s.r, prew[k].v[e], preb[k].v[e]);
                if (in) kge_store8<B16>(a.z.row(row), col[k], n[k], h[k].v);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// backward: rows
// ---------------------------------------------------------------------------------------------
// A workgroup takes a run of rows, its teams every teams-th row of it, and keeps the run's column sums in registers.  Gates of groups of rows: a run holds
// whole groups (their gradients are written here) or a part of one (the join writes them).
template <bool S16, bool B16, int NG, int NT>
__global__ __launch_bounds__(NT) void norm_bwd_kernel(const BwdArgs a) {
    __shared__ float red[2][NT / 64][4];
    __shared__ __attribute__((aligned(16))) float sums[NT][8];
    const Team t(a.waves);
    Reduce<4, NT> reduce(red, t);
    const float inv_dim = 1.f / (float)a.dim;
    int col[NG], n[NG];
    Vec postw[NG], prew[NG], scale[NG];
    Vec A[NG], B[NG], C[NG], D[NG], ga[NG], gb[NG];
#pragma unroll
    for (int k = 0; k < NG; ++k) {
        col[k] = 8 * (t.lane + k * t.size);
        n[k] = a.dim - col[k];
        postw[k].vector(a.post.w, col[k], n[k], 1.f);
        prew[k].vector(a.pre.w, col[k], n[k], 1.f);
        scale[k].vector(a.scale, col[k], n[k], 1.f);
        A[k].zero(); B[k].zero(); C[k].zero(); D[k].zero(); ga[k].zero(); gb[k].zero();
    }
    // adds the teams' sums; afterwards team 0's are the workgroup's, the others' zeros
    auto join = [&](Vec (&s)[NG]) {
        if (t.teams == 1) return;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            if (t.team > 0) {
                *(kge_f32x4 *)&sums[threadIdx.x][0] = kge_f32x4{s[k].v[0], s[k].v[1], s[k].v[2], s[k].v[3]};
                *(kge_f32x4 *)&sums[threadIdx.x][4] = kge_f32x4{s[k].v[4], s[k].v[5], s[k].v[6], s[k].v[7]};
            }
            __syncthreads();
            if (t.team == 0) {
                for (int i = 1; i < t.teams; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[k].v[e] += sums[threadIdx.x + i * t.size][e];
            } else s[k].zero();
            __syncthreads();
        }
    };
    const bool grouped = a.gate.p && a.gate_rows > 1;
    const int64_t run = blockIdx.x;
    int64_t r0, r1;                                               // rows of the run, and of its first group
    if (a.parts > 1) {                                            // a part of a group
        const int64_t group = run / a.parts, part = run - group * a.parts, g0 = group * a.gate_rows, g1 = min(g0 + a.gate_rows, a.rows);
        r0 = min(g0 + part * a.run, g1); r1 = min(r0 + a.run, g1);
    } else { r0 = run * a.run; r1 = min(r0 + a.run, a.rows); }

    Raw<S16> rh[NG], rd[NG];
    Raw<B16> ry[NG], rz[NG], rg[NG];
    auto load = [&](int64_t row, int64_t end) {
        const bool in = row < end;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            const int m = in ? n[k] : 0;
            rh[k].load(a.h.row(row), col[k], a.pre.on ? m : 0);
            rd[k].load(a.dh.row(row), col[k], a.dh.p ? m : 0);
            rz[k].load(a.dz.row(row), col[k], a.pre.on ? m : 0);
            ry[k].load(a.y.row(row), col[k], a.y.p ? m : 0);
            if (a.gate.p && !grouped) rg[k].load(a.gate.row(row), col[k], m);
        }
    };
    int64_t g0 = r0;                                              // of the group at hand
    do {
        const int64_t g1 = grouped && a.parts <= 1 ? min(g0 + a.gate_rows, r1) : r1;
        Vec gate[NG];
#pragma unroll
        for (int k = 0; k < NG; ++k) {
#pragma unroll
            for (int e = 0; e < 8; ++e) gate[k].v[e] = 1.f;
            if (grouped && g0 < g1) {
                Raw<B16> q;
                q.load(a.gate.row((uint32_t)g0 / a.gate_rows), col[k], n[k]);
                q.values(gate[k]);
                ga[k].zero(); gb[k].zero();
            }
        }
        load(g0 + t.team, g1);
        for (int64_t q0 = g0; q0 < g1; q0 += t.teams) {
            const int64_t row = q0 + t.team;
            const bool in = row < g1;
            Vec h[NG], d[NG], z[NG], y[NG];
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                rh[k].values(h[k]); rd[k].values(d[k]); rz[k].values(z[k]); ry[k].values(y[k]);
                if (a.gate.p && !grouped) rg[k].values(gate[k]);
            }
            if (q0 + t.teams < g1) load(row + t.teams, g1);
            // statistics: of rms norms with the sum of dz's products at once, of layer norms after the means
            float v[4] = {0.f, 0.f, 0.f, 0.f}, rp = 1.f, ry1 = 1.f, c1 = 0.f, c2 = 0.f;
            if (a.pre.layer || a.post.layer) {
#pragma unroll
                for (int k = 0; k < NG; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) { v[0] += h[k].v[e]; v[1] += y[k].v[e]; }
                reduce(v, 2);
                const float mh = a.pre.layer ? v[0] * inv_dim : 0.f, my = a.post.layer ? v[1] * inv_dim : 0.f;
#pragma unroll
                for (int k = 0; k < NG; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        h[k].v[e] = e < n[k] ? h[k].v[e] - mh : 0.f;
                        y[k].v[e] = e < n[k] ? y[k].v[e] - my : 0.f;
                    }
            }
            if (a.pre.on || a.post.on) {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = 0.f;
#pragma unroll
                for (int k = 0; k < NG; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float q = z[k].v[e] * prew[k].v[e];
                        v[0] = fmaf(h[k].v[e], h[k].v[e], v[0]); v[1] = fmaf(y[k].v[e], y[k].v[e], v[1]);
                        v[2] = fmaf(q, h[k].v[e], v[2]); v[3] += q;
                    }
                reduce(v, 4);
                if (a.post.on) ry1 = inv_sqrt(fmaf(v[1], inv_dim, a.post.eps));
                if (a.pre.on) {
                    rp = inv_sqrt(fmaf(v[0], inv_dim, a.pre.eps));
                    c2 = v[2] * rp * inv_dim;
                    c1 = a.pre.layer ? v[3] * inv_dim : 0.f;
                }
            }
            float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                if (a.pre.on) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float hat = h[k].v[e] * rp;
                        C[k].v[e] = fmaf(z[k].v[e], hat, C[k].v[e]);
                        D[k].v[e] += z[k].v[e];
                        d[k].v[e] = fmaf(fmaf(-hat, c2, z[k].v[e] * prew[k].v[e] - c1), rp, d[k].v[e]);
                    }
                }
                if (a.dx.p && in) kge_store8<S16>(a.dx.row(row), col[k], n[k], d[k].v);
                if (!a.y.p) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float hat = y[k].v[e] * ry1, x = e < n[k] ? d[k].v[e] : 0.f;
                    y[k].v[e] = hat;
                    if (grouped) { ga[k].v[e] = fmaf(x, hat, ga[k].v[e]); gb[k].v[e] += x; }
                    else {
                        A[k].v[e] = fmaf(x * gate[k].v[e], hat, A[k].v[e]);
                        B[k].v[e] = fmaf(x, gate[k].v[e], B[k].v[e]);
                    }
                }
                if (a.g_gate.p && !grouped && in) {               // a gate of the row's own: s o d o u
                    Vec q, b;
                    b.vector(a.post.b, col[k], n[k], 0.f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) q.v[e] = d[k].v[e] * scale[k].v[e] * fmaf(y[k].v[e], postw[k].v[e], b.v[e]);
                    kge_store8<B16>(a.g_gate.row(row), col[k], n[k], q.v);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    d[k].v[e] *= scale[k].v[e] * gate[k].v[e] * postw[k].v[e];
                    if (e < n[k]) { s[0] += d[k].v[e]; s[1] = fmaf(d[k].v[e], y[k].v[e], s[1]); }
                }
            }
            if (!a.y.p || !a.dy.p) continue;
            if (a.post.on) {
                reduce(s, 2);
                const float m1 = a.post.layer ? s[0] * inv_dim : 0.f, m2 = s[1] * inv_dim;
#pragma unroll
                for (int k = 0; k < NG; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) d[k].v[e] = (d[k].v[e] - m1 - y[k].v[e] * m2) * ry1;
            }
#pragma unroll
            for (int k = 0; k < NG; ++k)
                if (in) kge_store8<B16>(a.dy.row(row), col[k], n[k], d[k].v);
        }
        if (grouped) {
            join(ga); join(gb);
            if (t.team == 0) {
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    if (a.parts > 1) { A[k] = ga[k]; B[k] = gb[k]; continue; }
                    if (a.g_gate.p && g0 < g1) {
                        Vec q, b;
                        b.vector(a.post.b, col[k], n[k], 0.f);
#pragma unroll
                        for (int e = 0; e < 8; ++e) q.v[e] = scale[k].v[e] * fmaf(postw[k].v[e], ga[k].v[e], b.v[e] * gb[k].v[e]);
                        kge_store8<B16>(a.g_gate.row((uint32_t)g0 / a.gate_rows), col[k], n[k], q.v);
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        A[k].v[e] = fmaf(gate[k].v[e], ga[k].v[e], A[k].v[e]);
                        B[k].v[e] = fmaf(gate[k].v[e], gb[k].v[e], B[k].v[e]);
                    }
                }
            }
        }
        g0 = g1;
    } while (g0 < r1);
    // the run's sums
    auto keep = [&](Vec (&s)[NG], int which, bool joined) {
        if (!(a.want >> which & 1)) return;
        if (!joined) join(s);
        if (t.team == 0)
#pragma unroll
            for (int k = 0; k < NG; ++k)
                if (n[k] > 0) {
                    float *p = a.part + ((int64_t)which * a.runs + run) * a.part_ld + col[k];
                    *(kge_f32x4 *)p = kge_f32x4{s[k].v[0], s[k].v[1], s[k].v[2], s[k].v[3]};
                    *(kge_f32x4 *)(p + 4) = kge_f32x4{s[k].v[4], s[k].v[5], s[k].v[6], s[k].v[7]};
                }
    };
    keep(A, SUM_A, grouped); keep(B, SUM_B, grouped); keep(C, SUM_C, false); keep(D, SUM_D, false);
}

// ---------------------------------------------------------------------------------------------
// backward: column sums
// ---------------------------------------------------------------------------------------------
// 32 columns and 32 slices of the rows per workgroup; the slices are added in order.
constexpr int JC = 32, JS = 32;
__device__ __forceinline__ float column_sum(const float *p, int64_t ld, int64_t n, float (&lds)[JS][JC + 1]) {
    const int c = threadIdx.x & (JC - 1), s = threadIdx.x / JC;
    float v = 0.f;
#pragma unroll 8
    for (int64_t r = s; r < n; r += JS) v += p[r * ld + c];
    lds[s][c] = v;
    __syncthreads();
    float sum = 0.f;
    for (int i = 0; i < JS; ++i) sum += lds[i][c];
    __syncthreads();
    return sum;
}

// Groups whose rows were several runs: their gates' gradients, and their sums times the gates in the place of their first run's
template <bool B16> __global__ __launch_bounds__(JC * JS) void norm_groups_kernel(const BwdArgs a) {
    __shared__ float lds[JS][JC + 1];
    const int tiles = (int)(a.part_ld / JC), c = threadIdx.x & (JC - 1);
    const int64_t group = blockIdx.x / (uint32_t)tiles, col = (int64_t)(blockIdx.x - group * tiles) * JC;
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 2; ++w)
        if (a.want >> w & 1) s[w] = column_sum(a.part + ((int64_t)w * a.runs + group * a.parts) * a.part_ld + col, a.part_ld, a.parts, lds);
    if (threadIdx.x >= JC || col + c >= a.dim) return;
    const float g = load1<B16>(a.gate.row(group), col + c);
    if (a.g_gate.p) {
        const float sc = a.scale ? a.scale[col + c] : 1.f, w = a.post.w ? a.post.w[col + c] : 1.f, b = a.post.b ? a.post.b[col + c] : 0.f;
        store1<B16>(a.g_gate.row(group), col + c, sc * fmaf(w, s[0], b * s[1]));
    }
#pragma unroll
    for (int w = 0; w < 2; ++w)
        if (a.want >> w & 1) a.part[((int64_t)w * a.runs + group * a.parts) * a.part_ld + col + c] = g * s[w];
}

// Sums over all runs, and the gradients of the vectors
__global__ __launch_bounds__(JC * JS) void norm_join_kernel(const BwdArgs a) {
    __shared__ float lds[JS][JC + 1];
    const int c = threadIdx.x & (JC - 1);
    const int64_t col = (int64_t)blockIdx.x * JC;
    const bool branch = blockIdx.y == 0;
    const bool folded = branch && a.parts > 1;                    // (one row of sums for each group)
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int w = branch ? i : 2 + i;
        if (a.want >> w & 1)
            s[i] = column_sum(a.part + (int64_t)w * a.runs * a.part_ld + col, folded ? a.parts * a.part_ld : a.part_ld, folded ? a.runs / a.parts : a.runs, lds);
    }
    if (threadIdx.x >= JC || col + c >= a.dim) return;
    auto put = [&](float *p, float v) {
        if (p) p[col + c] = a.accumulate ? p[col + c] + v : v;
    };
    if (!branch) { put(a.g_prew, s[0]); put(a.g_preb, s[1]); return; }
    const float sc = a.scale ? a.scale[col + c] : 1.f, w = a.post.w ? a.post.w[col + c] : 1.f, b = a.post.b ? a.post.b[col + c] : 0.f;
    put(a.g_scale, fmaf(w, s[0], b * s[1]));
    put(a.g_postw, sc * s[0]);
    put(a.g_postb, sc * s[1]);
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
constexpr int64_t FWD_GROUPS = 2048, BWD_RUNS = 1024;
constexpr int MIN_RUN = 4;

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
// Waves of a row, a power of two: 512 columns each, or 1,024 in rows of more than 4,096.  (Sixteen waves leave a thread 128 registers.)
int waves_of(int dim) {
    int w = 1;
    while (w < 8 && 512 * w < dim) w *= 2;
    return dim > 8192 ? 16 : w;
}

// Runs of rows of the backward pass: about BWD_RUNS of them, of at least MIN_RUN rows for each team, of whole groups of rows where a run holds
// several and of parts of one where it is longer.
struct Runs { int64_t run, runs, parts; };
Runs runs_of(const kge_norm_block_t *b, int64_t rows) {
    const int w = waves_of(b->dim), teams = w < 4 ? 4 / w : 1;
    int64_t run = (rows + BWD_RUNS - 1) / BWD_RUNS;
    if (run < MIN_RUN * teams) run = MIN_RUN * teams;
    Runs q = {run, (rows + run - 1) / run, 1};
    if (b->gate && b->gate_rows > 1) {
        const int64_t len = b->gate_rows < rows ? b->gate_rows : rows;
        if (len > run) {
            q.parts = (len + run - 1) / run;
            q.run = (len + q.parts - 1) / q.parts;
            q.runs = (rows + len - 1) / len * q.parts;
        } else {
            q.run = run / len * len;
            q.runs = (rows + q.run - 1) / q.run;
        }
    }
    return q;
}
// No call of up to so many rows has more runs.  With r rows at least in a run before the groups' ends are looked at: groups of len > r rows are
// ceil(rows / len) ceil(len / r) < rows / r + rows / len + len / r + 1 runs, shorter ones less than 2 rows / r + 1.
int64_t most_runs(const kge_norm_block_t *b, int64_t rows) {
    const int w = waves_of(b->dim), teams = w < 4 ? 4 / w : 1;
    const int64_t short_runs = 3 * (rows / (MIN_RUN * teams) + 1) + 1, all = 3 * BWD_RUNS + 1;
    return rows == 0 ? 0 : short_runs < all ? short_runs : all;
}
int64_t part_ld_of(int dim) { return (dim + JC - 1) / JC * JC; }

template <bool S16, bool B16> void launch_fwd(const FwdArgs &a, hipStream_t st) {
    const int teams = a.waves < 4 ? 4 / a.waves : 1;
    int64_t groups = (a.rows + teams - 1) / teams;
    if (groups > FWD_GROUPS) groups = FWD_GROUPS;
    const dim3 grid((unsigned)groups), blk(64 * a.waves * teams);
    if (a.waves <= 4) hipLaunchKernelGGL((norm_fwd_kernel<S16, B16, 1, 256>), grid, blk, 0, st, a);
    else if (a.dim <= 4096) hipLaunchKernelGGL((norm_fwd_kernel<S16, B16, 1, 512>), grid, blk, 0, st, a);
    else if (a.dim <= 8192) hipLaunchKernelGGL((norm_fwd_kernel<S16, B16, 2, 512>), grid, blk, 0, st, a);
    else hipLaunchKernelGGL((norm_fwd_kernel<S16, B16, 2, 1024>), grid, blk, 0, st, a);
}
template <bool S16, bool B16> void launch_bwd(const BwdArgs &a, hipStream_t st) {
    const int teams = a.waves < 4 ? 4 / a.waves : 1;
    const dim3 grid((unsigned)a.runs), blk(64 * a.waves * teams);
    if (a.waves <= 4) hipLaunchKernelGGL((norm_bwd_kernel<S16, B16, 1, 256>), grid, blk, 0, st, a);
    else if (a.dim <= 4096) hipLaunchKernelGGL((norm_bwd_kernel<S16, B16, 1, 512>), grid, blk, 0, st, a);
    else if (a.dim <= 8192) hipLaunchKernelGGL((norm_bwd_kernel<S16, B16, 2, 512>), grid, blk, 0, st, a);
    else hipLaunchKernelGGL((norm_bwd_kernel<S16, B16, 2, 1024>), grid, blk, 0, st, a);
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
    a.dim = blk->dim; a.waves = waves_of(blk->dim); a.rows = rows;
    a.post = norm_of(blk->post); a.pre = norm_of(blk->pre); a.scale = blk->scale;
    a.gate = matrix((void *)blk->gate, blk->gate_ld, b16); a.gate_rows = (uint32_t)(blk->gate_rows < rows ? blk->gate_rows : rows);
    a.x = matrix((void *)x, x_ld, s16); a.y = matrix((void *)y, y_ld, b16); a.h = matrix(h, h_ld, s16); a.z = matrix(z, z_ld, b16);
    hipStream_t st = (hipStream_t)hip_stream;
    if (s16) b16 ? launch_fwd<true, true>(a, st) : launch_fwd<true, false>(a, st);
    else b16 ? launch_fwd<false, true>(a, st) : launch_fwd<false, false>(a, st);
    return kge_launch_status();
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
    const Runs q = rows > 0 ? runs_of(blk, rows) : Runs{0, 0, 1};
    a.run = q.run; a.runs = q.runs; a.parts = (int)q.parts; a.part_ld = part_ld_of(blk->dim);
    const bool bias = blk->post && blk->post->bias, of_group = w.gate && q.parts > 1;         // (parts: of gates of groups alone)
    if (w.scale || w.post_weight || of_group) a.want |= 1u << SUM_A;
    if (w.post_bias || (bias && (w.scale || of_group))) a.want |= 1u << SUM_B;
    if (w.pre_weight) a.want |= 1u << SUM_C;
    if (w.pre_bias) a.want |= 1u << SUM_D;
    if (a.want) {
        const size_t lost = ws ? (256 - ((uintptr_t)ws & 255)) & 255 : 0, need = (size_t)q.runs * 4 * a.part_ld * sizeof(float);
        if (need && (!ws || ws_bytes < lost + need)) return KGE_E_WORKSPACE_TOO_SMALL;
        a.part = (float *)((char *)ws + lost);
    }
    hipStream_t st = (hipStream_t)hip_stream;
    if (rows > 0) {
        if (s16) b16 ? launch_bwd<true, true>(a, st) : launch_bwd<true, false>(a, st);
        else b16 ? launch_bwd<false, true>(a, st) : launch_bwd<false, false>(a, st);
        if (q.parts > 1 && (a.want & 3)) {
            const dim3 grid((unsigned)(q.runs / q.parts * (a.part_ld / JC)));
            if (b16) hipLaunchKernelGGL((norm_groups_kernel<true>), grid, dim3(JC * JS), 0, st, a);
            else hipLaunchKernelGGL((norm_groups_kernel<false>), grid, dim3(JC * JS), 0, st, a);
        }
    }
    const bool vectors = w.scale || w.post_weight || w.post_bias || w.pre_weight || w.pre_bias;
    if (vectors)
        hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)(a.part_ld / JC), 2), dim3(JC * JS), 0, st, a);
    return rows > 0 || vectors ? kge_launch_status() : KGE_OK;
}

}  // extern "C"
