// Shared by the kernels of norm_block.hip: rows held by teams of waves, their sums, and the arguments of the kernels.
#pragma once
#include "text_ops.hpp"

namespace kge_norm {

constexpr int MAX_DIM = 16384;                                    // 1,024 threads of sixteen columns

// Eight columns of a thread
struct Vec {
    float v[8];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = 0.f;
    }
    // of a vector of parameters, which may be absent; zeros behind the row's end, so that what is scaled by it is zero there and counts in no sum
    __device__ __forceinline__ void vector(const float *p, int col, int n, float otherwise) {
        if (p) kge_load8<false>(p, col, n > 8 ? 8 : n, v);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = e < n ? otherwise : 0.f;
    }
};

// The same of a row as it lies in memory; n: columns left of the row, none or fewer for threads past its end
template <bool B16> struct Raw {
    KgeRaw8<B16> r;
    __device__ __forceinline__ void load(const void *row, int col, int n) {
        if (n >= 8) r = kge_raw8<B16>(row, col);
        else {
#pragma unroll
            for (int i = 0; i < (B16 ? 1 : 2); ++i) r.w[i] = kge_u32x4{0u, 0u, 0u, 0u};
            if (n > 0) {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < n) {
                        if constexpr (B16) r.w[0][e >> 1] |= (uint32_t)((const uint16_t *)row)[col + e] << (16 * (e & 1));
                        else r.w[e >> 2][e & 3] = ((const uint32_t *)row)[col + e];
                    }
            }
        }
    }
    __device__ __forceinline__ void values(Vec &x) const { kge_values8<B16>(r, x.v); }
};
template <bool B16> __device__ __forceinline__ float load1(const void *row, int64_t col) {
    return B16 ? __uint_as_float((uint32_t)((const uint16_t *)row)[col] << 16) : ((const float *)row)[col];
}
template <bool B16> __device__ __forceinline__ void store1(void *row, int64_t col, float v) {
    if constexpr (B16) ((__bf16 *)row)[col] = (__bf16)v;
    else ((float *)row)[col] = v;
}

// A workgroup's waves in teams of `waves`, each of which holds a row
struct Team {
    int waves, size, teams, team, lane;
    __device__ __forceinline__ explicit Team(int w) {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        waves = w; size = 64 * w; teams = max(1, (int)(blockDim.x >> 6) / w);
        team = wave / w; lane = (int)threadIdx.x - team * size;
    }
};

__device__ __forceinline__ float wave_sum(float x) {
    x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0xB1, 0xf, 0xf, true));      // lane ^ 1
    x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x4E, 0xf, 0xf, true));      // lane ^ 2
    x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x141, 0xf, 0xf, true));     // 7 - lane
    x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x140, 0xf, 0xf, true));     // 15 - lane
    const int b = (int)__float_as_uint(x);
    const float s0 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, 0)), s1 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, 16));
    const float s2 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, 32)), s3 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, 48));
    return (s0 + s1) + (s2 + s3);
}

// Sums of up to K values over the threads of a team, for all of them.  Two places in turn: who writes to one again has passed the barrier of the sums in
// between, behind which nobody reads it any more.  (Teams of one wave need no barrier, and go round as they like.)
template <int K, int NT> struct Reduce {
    float (&lds)[2][NT / 64][K];
    const Team &t;
    int place = 0;
    __device__ __forceinline__ Reduce(float (&l)[2][NT / 64][K], const Team &team) : lds(l), t(team) {}
    __device__ __forceinline__ void operator()(float *v, int n) {
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i < n) v[i] = wave_sum(v[i]);
        if (t.waves == 1) return;
        const int wave = (int)threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < K; ++i)
                if (i < n) lds[place][wave][i] = v[i];
        }
        __syncthreads();
        const int w0 = t.team * t.waves;
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i < n) v[i] = lds[place][w0][i];
        for (int w = 1; w < t.waves; ++w)
#pragma unroll
            for (int i = 0; i < K; ++i)
                if (i < n) v[i] += lds[place][w0 + w][i];
        place ^= 1;
    }
};

__device__ __forceinline__ float inv_sqrt(float x) { return 1.f / sqrtf(x); }

struct Norm { bool on, layer; float eps; const float *w, *b; };
struct Stats { float mean, r; };

template <int NG, class R> __device__ __forceinline__ Stats statistics(const Vec (&x)[NG], const int (&n)[NG], const Norm &norm, float inv_dim, R &reduce) {
    Stats s = {0.f, 1.f};
    float v[1] = {0.f};
    if (norm.layer) {
#pragma unroll
        for (int k = 0; k < NG; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[0] += x[k].v[e];
        reduce(v, 1);
        s.mean = v[0] * inv_dim;
        v[0] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < NG; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float q = e < n[k] ? x[k].v[e] - s.mean : 0.f;
            v[0] = fmaf(q, q, v[0]);
        }
    reduce(v, 1);
    s.r = inv_sqrt(fmaf(v[0], inv_dim, norm.eps));
    return s;
}

struct Matrix {
    char *p; int64_t ld;                                          // ld in bytes
    __device__ __forceinline__ char *row(int64_t r) const { return p + r * ld; }
};
inline Matrix matrix(void *p, int64_t ld, bool b16) { return Matrix{(char *)p, ld * (b16 ? 2 : 4)}; }

struct FwdArgs {
    int dim, waves; int64_t rows;
    Norm post, pre; const float *scale;
    Matrix gate; uint32_t gate_rows;
    Matrix x, y, h, z;
};

enum { SUM_A = 0, SUM_B = 1, SUM_C = 2, SUM_D = 3 };
struct BwdArgs {
    int dim, waves; int64_t rows;
    Norm post, pre; const float *scale;
    Matrix gate; uint32_t gate_rows;
    Matrix h, y, dh, dz, dx, dy, g_gate;
    int64_t run, runs, part_ld; int parts;                        // rows of a run, runs, and of a group
    uint32_t want;                                                // sums that are kept
    float *part;                                                  // [sum][run][part_ld]
    float *g_postw, *g_postb, *g_prew, *g_preb, *g_scale; int accumulate;
};

}  // namespace kge_norm
