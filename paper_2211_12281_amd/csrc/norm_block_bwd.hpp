// Rows of the backward pass of the norms around a block (norm_block.hip); norm_block_bwd16.hip and norm_block_bwd32.hip build it for their type of the stream.
#pragma once
#include "norm_block.hpp"

namespace kge_norm {

// What a run of rows has for gates: none, or a part of one group of rows (its sums leave the gate out; the join has it); a gate of its own for every
// row; whole groups of rows, whose gates' gradients are written here, each group's sums being kept apart until its end.
enum { GATE_RUN = 0, GATE_ROW = 1, GATE_GROUPS = 2 };
// vectors in the LDS: of rows of up to 4,096 columns.  (Kept in registers they leave room for one wave per SIMD less; read from memory again and again their
// loads stand in the queue behind those of the next row.)
enum { VEC_PRE = 0, VEC_F = 1, VEC_SCALE = 2, VEC_POST = 3, VEC_BIAS = 4 };
constexpr int vectors_of(int mode) { return mode == GATE_RUN ? 2 : 5; }

// A workgroup takes a run of rows, its teams every teams-th row of it, and keeps the run's column sums in registers.
template <bool S16, bool B16, int NG, int LAST, int NT, int OCC, int MODE>
__global__ __launch_bounds__(NT, OCC) void norm_bwd_kernel(const BwdArgs a) {
    constexpr bool LDS = NT == 256, GROUPS = MODE == GATE_GROUPS, OF_ROW = MODE == GATE_ROW;
    __shared__ float red[2][NT / 64][4];
    __shared__ kge_f32x4 sums[NT];
    extern __shared__ __attribute__((aligned(16))) float vec[];
    const Team t(a.waves);
    Reduce<4, NT> reduce(red, t);
    const Columns<NG, LAST> c(a.dim, t.lane, t.size);
    const float inv_dim = 1.f / (float)a.dim;
    const int wide = 4 * t.size * NG;
    constexpr int KEPT = GROUPS ? NG : 1;
    kge_f32x4 A[NG], B[NG], C[NG], D[NG], ga[KEPT], gb[KEPT];
#pragma unroll
    for (int k = 0; k < NG; ++k) A[k] = B[k] = C[k] = D[k] = splat(0.f);
    const bool sum_b = a.want >> SUM_B & 1, sum_d = a.want >> SUM_D & 1;
    const int64_t run = blockIdx.x;
    int64_t r0, r1;                                               // rows of the run
    if (a.parts > 1) {                                            // a part of a group
        const int64_t group = run / a.parts, part = run - group * a.parts, first = group * a.gate_rows, end = min(first + a.gate_rows, a.rows);
        r0 = min(first + part * a.run, end); r1 = min(r0 + a.run, end);
    } else { r0 = run * a.run; r1 = min(r0 + a.run, a.rows); }
    int64_t g0 = r0;                                              // first row of the group at hand
    auto group_gate = [&](int k) {
        Raw<B16> q;
        q.load(a.gate.row(GROUPS || a.gate.p ? (uint32_t)g0 / a.gate_rows : 0), c, k, true);
        return q.values();
    };
    auto from_memory = [&](int which, int k) {
        switch (which) {
        case VEC_PRE: return vector4(a.pre.w, c.col(k), a.dim, 1.f);
        case VEC_SCALE: return vector4(a.scale, c.col(k), a.dim, 1.f);
        case VEC_POST: return vector4(a.post.w, c.col(k), a.dim, 1.f);
        case VEC_BIAS: return vector4(a.post.b, c.col(k), a.dim, 0.f);
        }
        const kge_f32x4 f = vector4(a.scale, c.col(k), a.dim, 1.f) * vector4(a.post.w, c.col(k), a.dim, 1.f);
        return !OF_ROW && a.gate.p && g0 < r1 ? f * group_gate(k) : f;
    };
    auto vector = [&](int which, int k) { return LDS ? *(const kge_f32x4 *)(vec + which * wide + c.col(k)) : from_memory(which, k); };
    auto fill = [&](bool first) {                                 // (first: all but the factors of a group, which its gate belongs to)
        for (int i = 4 * threadIdx.x; i < wide; i += 4 * NT) {
            auto put = [&](int which, kge_f32x4 x) { *(kge_f32x4 *)(vec + which * wide + i) = x; };
            const kge_f32x4 s = vector4(a.scale, i, a.dim, 1.f), w = vector4(a.post.w, i, a.dim, 1.f);
            if (!GROUPS || !first) {
                kge_f32x4 f = s * w;
                if (!OF_ROW && a.gate.p && g0 < r1)
#pragma unroll
                    for (int e = 0; e < 4; ++e) f[e] *= i + e < a.dim ? load1<B16>(a.gate.row((uint32_t)g0 / a.gate_rows), i + e) : 0.f;
                put(VEC_F, f);
            }
            if (first) {
                put(VEC_PRE, vector4(a.pre.w, i, a.dim, 1.f));
                if (MODE != GATE_RUN) { put(VEC_SCALE, s); put(VEC_POST, w); put(VEC_BIAS, vector4(a.post.b, i, a.dim, 0.f)); }
            }
        }
    };
    // adds the teams' sums; afterwards team 0's are the workgroup's, the others' zeros
    auto join = [&](kge_f32x4 (&s)[NG]) {
        if (t.teams == 1) return;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            if (t.team > 0) sums[threadIdx.x] = s[k];
            __syncthreads();
            if (t.team == 0) {
                for (int i = 1; i < t.teams; ++i) s[k] += sums[threadIdx.x + i * t.size];
            } else s[k] = splat(0.f);
            __syncthreads();
        }
    };

    Raw<S16> rh[NG], rd[NG];
    Raw<B16> ry[NG], rz[NG], rg[OF_ROW ? NG : 1];
    auto load = [&](int64_t row, int64_t end) {
        const bool in = row < end;
#pragma unroll
        for (int k = 0; k < NG; ++k) {
            rh[k].load(a.h.row(row), c, k, in && a.pre.on);
            rd[k].load(a.dh.row(row), c, k, in && a.dh.p);
            rz[k].load(a.dz.row(row), c, k, in && a.pre.on);
            ry[k].load(a.y.row(row), c, k, in && a.y.p);
            if constexpr (OF_ROW) rg[k].load(a.gate.row(row), c, k, in);
        }
    };
    if constexpr (!GROUPS) load(r0 + t.team, r1);                 // (under the loads of the vectors; later rows' wait for nobody but their own wave)
    if constexpr (LDS) {
        fill(true);
        __syncthreads();
    }
    do {
        const int64_t g1 = GROUPS ? min(g0 + a.gate_rows, r1) : r1;
        if constexpr (GROUPS) {
            load(g0 + t.team, g1);
            if constexpr (LDS) {                                  // (everyone has passed the last group's join, if there are teams, and its rows' sums, if not)
                __syncthreads();
                fill(false);
                __syncthreads();
            }
#pragma unroll
            for (int k = 0; k < NG; ++k) ga[k] = gb[k] = splat(0.f);
        }
        for (int64_t q0 = g0; q0 < g1; q0 += t.teams) {
            if constexpr (!LDS) asm volatile("" ::: "memory");    // (the vectors are read for every row: no registers for them in between)
            const int64_t row = q0 + t.team;
            const bool in = row < g1;
            if (q0 > g0) load(row, g1);
            kge_f32x4 h[NG], d[NG], z[NG], y[NG], gate[OF_ROW ? NG : 1];
#pragma unroll
            for (int k = 0; k < NG; ++k) {
                h[k] = rh[k].values(); d[k] = rd[k].values(); z[k] = rz[k].values(); y[k] = ry[k].values();
                if constexpr (OF_ROW) gate[k] = rg[k].values();
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
                if (a.dx.p && in && c.inside(k)) store<S16>(a.dx.row(row), c, k, d[k]);
                if (!a.y.p) continue;
                y[k] *= splat(rq);                                // y^, or y itself
                if constexpr (GROUPS) {
                    ga[k] = fma4(d[k], y[k], ga[k]);
                    gb[k] += d[k];
                }
                if constexpr (OF_ROW) {
                    if (a.g_gate.p && in && c.inside(k))          // s o d o u
                        store<B16>(a.g_gate.row(row), c, k, d[k] * vector(VEC_SCALE, k) * fma4(y[k], vector(VEC_POST, k), vector(VEC_BIAS, k)));
                    d[k] *= gate[k];
                }
                if constexpr (!GROUPS) {
                    A[k] = fma4(d[k], y[k], A[k]);
                    if (sum_b) B[k] += d[k];
                }
                d[k] *= vector(VEC_F, k);
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
                if (in && c.inside(k)) store<B16>(a.dy.row(row), c, k, d[k]);
        }
        if constexpr (GROUPS) {
            join(ga); join(gb);
            if (t.team == 0 && g0 < g1) {
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    if (a.g_gate.p && c.inside(k)) {
                        const kge_f32x4 sum = fma4(vector(VEC_POST, k), ga[k], vector(VEC_BIAS, k) * gb[k]);
                        store<B16>(a.g_gate.row((uint32_t)g0 / a.gate_rows), c, k, vector(VEC_SCALE, k) * sum);
                    }
                    const kge_f32x4 q = group_gate(k);
                    A[k] = fma4(q, ga[k], A[k]);
                    B[k] = fma4(q, gb[k], B[k]);
                }
            }
        }
        g0 = g1;
    } while (g0 < r1);
    // the run's sums
    auto keep = [&](kge_f32x4 (&s)[NG], int which, bool joined) {
        if (!(a.want >> which & 1)) return;
        if (!joined) join(s);
        if (t.team == 0)
#pragma unroll
            for (int k = 0; k < NG; ++k)
                if (c.inside(k)) *(kge_f32x4 *)(a.part + ((int64_t)which * a.runs + run) * a.part_ld + c.col(k)) = s[k];
    };
    keep(A, SUM_A, GROUPS); keep(B, SUM_B, GROUPS); keep(C, SUM_C, false); keep(D, SUM_D, false);
}

template <bool S16, bool B16, int MODE> void launch_bwd(const BwdArgs &a, hipStream_t st) {
    const int teams = a.waves < 4 ? 4 / a.waves : 1, groups = groups_of(a.dim);
    const dim3 grid((unsigned)a.runs), blk(64 * a.waves * teams);
    const int lds = a.waves <= 4 ? vectors_of(MODE) * 256 * a.waves * groups * (int)sizeof(float) : 0;      // 80 KB at most
    // (whole groups of rows keep half as many sums again)
    constexpr int OCC2 = MODE == GATE_GROUPS ? 3 : occ_of(2), OCC3 = MODE == GATE_GROUPS ? 2 : occ_of(3);
#define KGE_BWD(NG, LAST, NT, OCC)                                                                                              \
    do {                                                                                                                        \
        static KgeLdsLimit limit;                                                                                               \
        const auto kern = norm_bwd_kernel<S16, B16, NG, LAST, NT, OCC, MODE>;                                                   \
        if (lds > 48 * 1024 && limit.set((const void *)kern, 80 * 1024) != KGE_OK) return;                                      \
        hipLaunchKernelGGL(kern, grid, blk, lds, st, a);                                                                        \
    } while (0)
    if (a.waves == 16) KGE_BWD(4, 2, 1024, 4);
    else if (a.waves == 8) KGE_BWD(4, 2, 512, 2);
    else switch (groups) {
    case 1: KGE_BWD(1, 1, 256, occ_of(1)); break;
    case 2: KGE_BWD(2, 1, 256, OCC2); break;
    case 3: KGE_BWD(3, 1, 256, OCC3); break;
    default: KGE_BWD(4, 1, 256, occ_of(4));
    }
#undef KGE_BWD
}
template <bool S16> void launch_bwd(const BwdArgs &a, bool b16, hipStream_t st) {
    const int mode = !a.gate.p || a.parts > 1 ? GATE_RUN : a.gate_rows == 1 ? GATE_ROW : GATE_GROUPS;
    if (b16) mode == GATE_RUN ? launch_bwd<S16, true, GATE_RUN>(a, st) : mode == GATE_ROW ? launch_bwd<S16, true, GATE_ROW>(a, st) : launch_bwd<S16, true, GATE_GROUPS>(a, st);
    else mode == GATE_RUN ? launch_bwd<S16, false, GATE_RUN>(a, st) : mode == GATE_ROW ? launch_bwd<S16, false, GATE_ROW>(a, st) : launch_bwd<S16, false, GATE_GROUPS>(a, st);
}

}  // namespace kge_norm
