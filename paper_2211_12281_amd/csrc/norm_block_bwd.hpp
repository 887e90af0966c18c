// Rows of the backward pass of the norms around a block (norm_block.hip); norm_block_bwd16.hip and norm_block_bwd32.hip build it for their type of the stream.
#pragma once
#include "norm_block.hpp"

namespace kge_norm {

// What a run of rows has for gates: none, or one group's, of which the run is a part or the whole (its sums leave the gate out; the join has it); a gate of its
// own for every row; several groups of rows, each of which one team takes from end to end.
enum { GATE_RUN = 0, GATE_ROW = 1, GATE_GROUPS = 2 };
// Vectors in the LDS: w of the pre norm, s o w (GATE_RUN: o g) and s o b of the post norm.  (Kept in registers they leave room for one wave per SIMD less; read from
// memory for every row their loads stand in the queue behind those of the rows.)
enum { VEC_PRE = 0, VEC_F = 1, VEC_SB = 2 };
// GATE_GROUPS: A and B of a team, gates included; in rows of eight waves s o b makes room for them and is read from memory
constexpr int vectors_of(int mode, int nt) { return mode == GATE_RUN || (mode == GATE_GROUPS && nt == 512) ? 2 : 3; }

// A workgroup takes a run of rows, its teams every teams-th row of it (GATE_GROUPS: every teams-th group), and keeps the run's column sums in registers.
template <bool S16, bool B16, int NG, int SUB, int NT, int OCC, int MODE>
__global__ __launch_bounds__(NT, OCC) void norm_bwd_kernel(const BwdArgs a) {
    constexpr bool GROUPS = MODE == GATE_GROUPS, OF_ROW = MODE == GATE_ROW, GATED = GROUPS || OF_ROW, SB = vectors_of(MODE, NT) == 3;
    __shared__ float red[2][NT / 64][4];
    extern __shared__ __attribute__((aligned(16))) float vec[];   // [vector][wide], then [team][wide] where there are teams, [team][A, B][wide] of groups
    const Team<SUB> t(a.waves);
    Reduce<4, NT, SUB> reduce(red, t);
    const Columns<NG> c(a.dim, t.lane, t.size);
    const float inv_dim = 1.f / (float)a.dim;
    const int wide = 4 * t.size * NG;
    float *const of_teams = vec + vectors_of(MODE, NT) * wide;
    kge_f32x4 A[NG], B[NG], C[NG], D[NG];
#pragma unroll
    for (int k = 0; k < NG; ++k) A[k] = B[k] = C[k] = D[k] = splat(0.f);
    const bool sum_b = GROUPS || (a.want >> SUM_B & 1), sum_d = a.want >> SUM_D & 1;
    const int64_t run = blockIdx.x;
    int64_t r0, r1;                                               // rows of the run
    if (a.parts > 0) {                                            // a part of a group
        const int64_t group = run / a.parts, part = run - group * a.parts, first = group * a.gate_rows, end = min(first + a.gate_rows, a.rows);
        r0 = min(first + part * a.run, end); r1 = min(r0 + a.run, end);
    } else { r0 = run * a.run; r1 = min(r0 + a.run, a.rows); }
    auto vector = [&](int which, int k) { return *(const kge_f32x4 *)(vec + which * wide + c.col(k)); };
    auto gate4 = [&](int64_t group, int i) {
        kge_f32x4 g;
#pragma unroll
        for (int e = 0; e < 4; ++e) g[e] = i + e < a.dim ? load1<B16>(a.gate.row(group), i + e) : 0.f;
        return g;
    };
    for (int i = 4 * threadIdx.x; i < wide; i += 4 * NT) {
        auto put = [&](int which, kge_f32x4 x) { *(kge_f32x4 *)(vec + which * wide + i) = x; };
        const kge_f32x4 s = vector4(a.scale, i, a.dim, 1.f), f = s * vector4(a.post.w, i, a.dim, 1.f);
        put(VEC_F, !GATED && a.gate.p && r0 < r1 ? f * gate4((uint32_t)r0 / a.gate_rows, i) : f);
        put(VEC_PRE, vector4(a.pre.w, i, a.dim, 1.f));
        if constexpr (GATED && SB) put(VEC_SB, s * vector4(a.post.b, i, a.dim, 0.f));
    }
    if constexpr (GROUPS)
        for (int i = 4 * threadIdx.x; i < 2 * t.teams * wide; i += 4 * NT) *(kge_f32x4 *)(of_teams + i) = splat(0.f);
    __syncthreads();
    // f(column, four columns' sums over the teams), each by one thread
    auto of_columns = [&](kge_f32x4 (&s)[NG], auto f) {
        if (SUB == 64 && t.teams == 1) {
#pragma unroll
            for (int k = 0; k < NG; ++k)
                if (c.inside(k)) f(c.col(k), s[k]);
            return;
        }
        int teams = t.teams, team = t.team;
        if constexpr (SUB < 64) {                                 // those of a wave first
#pragma unroll
            for (int k = 0; k < NG; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[k][e] = add_32(SUB == 16 ? add_16(s[k][e]) : s[k][e]);
            teams = NT / 64; team = threadIdx.x / 64;
        }
        if (SUB == 64 || (threadIdx.x & 63) < SUB) {
#pragma unroll
            for (int k = 0; k < NG; ++k) *(kge_f32x4 *)(of_teams + team * wide + c.col(k)) = s[k];
        }
        __syncthreads();
        for (int i = 4 * threadIdx.x; i < a.dim; i += 4 * NT) {
            kge_f32x4 x = *(const kge_f32x4 *)(of_teams + i);
            for (int k = 1; k < teams; ++k) x += *(const kge_f32x4 *)(of_teams + k * wide + i);
            f(i, x);
        }
        __syncthreads();
    };

    Raw<S16> rh[NG], rd[NG];
    Raw<B16> ry[NG], rz[NG], rg[GATED ? NG : 1];
    auto load = [&](int64_t row, int64_t group, int64_t end) {
        const bool in = row < end;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            rh[k].load(a.h.row(row), c, k, in && a.pre.on);
            rd[k].load(a.dh.row(row), c, k, in && a.dh.p);
            rz[k].load(a.dz.row(row), c, k, in && a.pre.on);
            ry[k].load(a.y.row(row), c, k, in && a.y.p);
            if constexpr (GATED) rg[k].load(a.gate.row(group), c, k, in);
        }
    };
    // (GROUPS: a team's rows are those of its groups, one behind the other; every team goes round as often, as the waves of one meet at barriers)
    const int64_t len = GROUPS ? a.gate_rows : 1, base = GROUPS ? r0 / len : 0, groups = GROUPS ? (r1 - r0 + len - 1) / len : 0;
    for (int64_t g0 = 0; g0 < (GROUPS ? groups : 1); g0 += t.teams) {
        const int64_t group = base + g0 + t.team, first = GROUPS ? group * len : r0 + t.team, end = GROUPS ? min(first + len, r1) : r1;
        const int64_t rounds = GROUPS ? len : (r1 - r0 + t.teams - 1) / t.teams;
        kge_f32x4 gate[GATED ? NG : 1];
        for (int64_t q = 0; q < rounds; ++q) {
            const int64_t row = GROUPS ? first + q : first + q * t.teams;
            const bool in = row < end;
            load(row, OF_ROW ? row : group, end);
            kge_f32x4 h[NG], d[NG], z[NG], y[NG];
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                h[k] = rh[k].values(); d[k] = rd[k].values(); z[k] = rz[k].values(); y[k] = ry[k].values();
                if constexpr (OF_ROW) gate[k] = rg[k].values();
                if constexpr (GROUPS)
                    if (in) gate[k] = rg[k].values();             // (the group's, whose last row may be beyond the matrix)
            }
            // statistics: of rms norms with the sum of dz's products at once, of layer norms after the means
            float rp = 1.f, rq = 1.f, c1 = 0.f, c2 = 0.f;
            if (a.pre.layer || a.post.layer) {
                float v[2] = {0.f, 0.f};
#pragma unroll
                for (int k = 0; k < NG; ++k) { v[0] = sum4(h[k], v[0]); v[1] = sum4(y[k], v[1]); }
                reduce(v);
                const float mh = a.pre.layer ? v[0] * inv_dim : 0.f, my = a.post.layer ? v[1] * inv_dim : 0.f;
#pragma unroll
                for (int k = 0; k < NG; ++k) { h[k] = c.minus(k, h[k], mh); y[k] = c.minus(k, y[k], my); }
            }
            if (a.pre.on || a.post.on) {
                float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    const kge_f32x4 q = z[k] * vector(VEC_PRE, k);
                    v[0] = dot4(h[k], h[k], v[0]); v[1] = dot4(y[k], y[k], v[1]);
                    v[2] = dot4(q, h[k], v[2]); v[3] = sum4(q, v[3]);
                }
                reduce(v);
                if (a.post.on) rq = inv_sqrt(fmaf(v[1], inv_dim, a.post.eps));
                if (a.pre.on) {
                    rp = inv_sqrt(fmaf(v[0], inv_dim, a.pre.eps));
                    c2 = v[2] * rp * inv_dim;
                    c1 = a.pre.layer ? v[3] * inv_dim : 0.f;
                }
            }
            float s[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                if (a.pre.on) {
                    h[k] *= splat(rp);
                    C[k] = fma4(z[k], h[k], C[k]);
                    if (sum_d) D[k] += z[k];
                    d[k] = fma4(fma4(splat(-c2), h[k], c.minus(k, z[k] * vector(VEC_PRE, k), c1)), splat(rp), d[k]);
                }
                if (a.dx.p && in && c.inside(k)) store<S16>(a.dx.row(row), c, k, d[k], a.stream);
                if (!a.y.p) continue;
                y[k] *= splat(rq);                                // y^, or y itself
                if constexpr (OF_ROW) {
                    if (a.g_gate.p && in && c.inside(k))          // s o d o u
                        store<B16>(a.g_gate.row(row), c, k, d[k] * fma4(y[k], vector(VEC_F, k), vector(VEC_SB, k)), a.stream);
                    d[k] *= gate[k];
                }
                A[k] = fma4(d[k], y[k], A[k]);
                if (sum_b) B[k] += d[k];
                d[k] *= vector(VEC_F, k);
                if constexpr (GROUPS) d[k] *= rg[k].values();     // (zeros where there is no row)
                s[0] = sum4(d[k], s[0]); s[1] = dot4(d[k], y[k], s[1]);
            }
            if (!a.y.p || !a.dy.p) continue;
            if (a.post.on) {
                reduce(s);
                const float m1 = a.post.layer ? s[0] * inv_dim : 0.f, m2 = s[1] * inv_dim;
#pragma unroll
                for (int k = 0; k < NG; ++k) d[k] = fma4(splat(-m2), y[k], d[k] - splat(m1)) * splat(rq);
            }
#pragma unroll
            for (int k = 0; k < NG; ++k)
                if (in && c.inside(k)) store<B16>(a.dy.row(row), c, k, d[k], a.stream);
        }
        if constexpr (GROUPS) {                                   // the group's gate, and its sums times the gate
            if (first < end) {
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    if (!c.inside(k)) continue;
                    if (a.g_gate.p) {
                        const kge_f32x4 sb = SB ? vector(VEC_SB, k) : vector4(a.scale, c.col(k), a.dim, 1.f) * vector4(a.post.b, c.col(k), a.dim, 0.f);
                        store<B16>(a.g_gate.row(group), c, k, of_sums(vector(VEC_F, k), A[k], sb, B[k], a.post.b), false);
                    }
                    float *mine = of_teams + 2 * t.team * wide + c.col(k);
                    *(kge_f32x4 *)mine = fma4(gate[k], A[k], *(const kge_f32x4 *)mine);
                    *(kge_f32x4 *)(mine + wide) = fma4(gate[k], B[k], *(const kge_f32x4 *)(mine + wide));
                }
            }
#pragma unroll
            for (int k = 0; k < NG; ++k) A[k] = B[k] = splat(0.f);
        }
    }
    if constexpr (GROUPS) {                                       // the teams' sums of all groups: A in its place of the first team, B behind it
        __syncthreads();
        for (int i = 4 * threadIdx.x; i < 2 * wide; i += 4 * NT) {
            kge_f32x4 x = *(const kge_f32x4 *)(of_teams + i);
            for (int k = 1; k < t.teams; ++k) x += *(const kge_f32x4 *)(of_teams + 2 * k * wide + i);
            *(kge_f32x4 *)(of_teams + i) = x;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < NG; ++k) {                            // from here on as of a run whose first team has had all rows
            A[k] = t.team ? splat(0.f) : *(const kge_f32x4 *)(of_teams + c.col(k));
            B[k] = t.team ? splat(0.f) : *(const kge_f32x4 *)(of_teams + wide + c.col(k));
        }
        __syncthreads();
    }
    // The only run has everything: the vectors' gradients, and that of the only group's gate, without another launch.
    if (a.runs == 1) {
        auto put = [&](float *q, int i, kge_f32x4 x) {
            if (!q) return;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < a.dim) q[i + e] = a.accumulate ? q[i + e] + x[e] : x[e];
        };
        if (a.y.p) {
            __syncthreads();                                      // (everyone has read the factors, whose place takes B)
            of_columns(B, [&](int i, kge_f32x4 x) { *(kge_f32x4 *)(vec + VEC_F * wide + i) = x; });
            of_columns(A, [&](int i, kge_f32x4 s) {
                kge_f32x4 d = *(const kge_f32x4 *)(vec + VEC_F * wide + i);
                const kge_f32x4 sc = vector4(a.scale, i, a.dim, 1.f), w = vector4(a.post.w, i, a.dim, 1.f), b = vector4(a.post.b, i, a.dim, 0.f);
                if (a.parts > 0) {                                // the gate of the one group
                    const kge_f32x4 v = sc * of_sums(w, s, b, d, a.post.b);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (i + e < a.dim) {
                            const float g = load1<B16>(a.gate.p, i + e);
                            if (a.g_gate.p) store1<B16>(a.g_gate.p, i + e, v[e]);
                            s[e] *= g; d[e] *= g;
                        }
                }
                put(a.g_scale, i, of_sums(w, s, b, d, a.post.b));
                put(a.g_postw, i, sc * s);
                put(a.g_postb, i, sc * d);
            });
        }
        of_columns(C, [&](int i, kge_f32x4 x) { put(a.g_prew, i, x); });
        of_columns(D, [&](int i, kge_f32x4 x) { put(a.g_preb, i, x); });
        return;
    }
    // the run's sums, for the join
    auto keep = [&](kge_f32x4 (&s)[NG], int which) {
        if (!(a.want >> which & 1)) return;
        float *p = a.part + ((int64_t)which * a.runs + run) * a.part_ld;
        of_columns(s, [&](int i, kge_f32x4 x) { *(kge_f32x4 *)(p + i) = x; });
    };
    keep(A, SUM_A); keep(B, SUM_B); keep(C, SUM_C); keep(D, SUM_D);
}

template <bool S16, bool B16, int MODE> int launch_bwd(const BwdArgs &a, hipStream_t st) {
    const int lanes = bwd_lanes_of(a.dim), groups = groups_of(a.dim, lanes), teams = bwd_teams_of(a.dim), nt = lanes * teams;
    const dim3 grid((unsigned)a.runs), blk(nt);
    // 128 KB at most (rows of 8,192 columns with gates of groups)
    const int lds = (vectors_of(MODE, nt) + (MODE == GATE_GROUPS ? 2 * teams : teams > 1 ? teams : 0)) * 4 * lanes * groups * (int)sizeof(float);
#define KGE_BWD(NG, SUB, NT, OCC)                                                                                                    \
    do {                                                                                                                        \
        static KgeLdsLimit limit;                                                                                               \
        const auto kern = norm_bwd_kernel<S16, B16, NG, SUB, NT, OCC, MODE>;                                                         \
        if (lds > 48 * 1024 && limit.set((const void *)kern, 128 * 1024) != KGE_OK) return KGE_E_HIP;                                    \
        hipLaunchKernelGGL(kern, grid, blk, lds, st, a);                                                                        \
    } while (0)
    if (a.waves == 8) {
        if (groups == 2) KGE_BWD(2, 64, 512, 4);
        else if (groups == 3) KGE_BWD(3, 64, 512, 2);
        else KGE_BWD(4, 64, 512, 2);
    } else if (a.waves > 1) {
        if (groups == 2) KGE_BWD(2, 64, 256, 4);
        else KGE_BWD(3, 64, 256, 3);
    } else if (lanes == 16) {
        if (groups == 1) KGE_BWD(1, 16, NARROW_THREADS, 4);
        else KGE_BWD(2, 16, NARROW_THREADS, 4);
    } else if (lanes == 32) KGE_BWD(2, 32, NARROW_THREADS, 4);
    else switch (groups) {
    case 2: KGE_BWD(2, 64, 64 * TEAMS_OF_ONE[0], 4); break;
    case 3: KGE_BWD(3, 64, 64 * TEAMS_OF_ONE[1], 3); break;
    default: KGE_BWD(4, 64, 64 * TEAMS_OF_ONE[2], 2);
    }
#undef KGE_BWD
    return KGE_OK;
}
template <bool S16> int launch_bwd(const BwdArgs &a, bool b16, hipStream_t st) {
    const int mode = !a.gate.p || a.parts > 0 ? GATE_RUN : a.gate_rows == 1 ? GATE_ROW : GATE_GROUPS;
    if (b16) return mode == GATE_RUN ? launch_bwd<S16, true, GATE_RUN>(a, st) : mode == GATE_ROW ? launch_bwd<S16, true, GATE_ROW>(a, st) : launch_bwd<S16, true, GATE_GROUPS>(a, st);
    return mode == GATE_RUN ? launch_bwd<S16, false, GATE_RUN>(a, st) : mode == GATE_ROW ? launch_bwd<S16, false, GATE_ROW>(a, st) : launch_bwd<S16, false, GATE_GROUPS>(a, st);
}

}  // namespace kge_norm
