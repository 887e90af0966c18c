// Shared by the kernels of norm_block.hip: rows held by teams of waves, their sums, and the arguments of the kernels.
#pragma once
#include "text_ops.hpp"

namespace kge_norm {

constexpr int MAX_DIM = 8192;                                     // eight waves of sixteen columns a lane

__device__ __forceinline__ kge_f32x4 splat(float x) { return kge_f32x4{x, x, x, x}; }
__device__ __forceinline__ kge_f32x4 fma4(kge_f32x4 a, kge_f32x4 b, kge_f32x4 c) {
    return kge_f32x4{fmaf(a[0], b[0], c[0]), fmaf(a[1], b[1], c[1]), fmaf(a[2], b[2], c[2]), fmaf(a[3], b[3], c[3])};
}

struct Matrix {
    char *p; int64_t ld;                                          // ld in bytes
    __device__ __forceinline__ char *row(int64_t r) const { return p + r * ld; }
};
inline Matrix matrix(void *p, int64_t ld, bool b16) { return Matrix{(char *)p, ld * (b16 ? 2 : 4)}; }

// Columns i .. i + 3 of a vector of parameters, which may be absent; zeros behind its end
__device__ __forceinline__ kge_f32x4 vector4(const float *p, int i, int dim, float otherwise) {
    kge_f32x4 r = splat(0.f);
    if (i + 4 <= dim) r = p ? *(const kge_f32x4_a4 *)(p + i) : splat(otherwise);
    else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (i + e < dim) r[e] = p ? p[i + e] : otherwise;
    }
    return r;
}

// A thread's share of a row: NG groups of four columns, the team's lanes side by side.  Only the last group may reach past the row's end; `mask` is 1 on
// its columns that are inside and 0 on the others, whose values are kept zero: a mean is subtracted as fma(-mean, mask, x).
template <int NG> struct Columns {
    int dim, lane, size;
    kge_f32x4 mask;
    __device__ __forceinline__ Columns(int d, int l, int s) : dim(d), lane(l), size(s) {
#pragma unroll
        for (int e = 0; e < 4; ++e) mask[e] = col(NG - 1) + e < d ? 1.f : 0.f;
    }
    __device__ __forceinline__ int col(int k) const { return 4 * (lane + size * k); }
    __device__ __forceinline__ int left(int k) const { return dim - col(k); }
    __device__ __forceinline__ bool inside(int k) const { return k < NG - 1 || left(k) > 0; }
    // x - m on the columns that are inside
    __device__ __forceinline__ kge_f32x4 minus(int k, kge_f32x4 x, float m) const {
        return k < NG - 1 ? x - splat(m) : fma4(splat(-m), mask, x);
    }
};

// Four columns as they lie in memory.  Where the row ends inside them, the row's last four are read and moved down: one load for all lanes (rows of fewer
// than four elements take them one by one).
template <bool B16> struct Raw {
    kge_u32x4 w;                                                  // (bf16: two words)
    template <int NG> __device__ __forceinline__ void load(const char *row, const Columns<NG> &c, int k, bool in) {
        w = kge_u32x4{0u, 0u, 0u, 0u};
        const bool whole = k < NG - 1;
        const int n = c.left(k);
        if (!in || (!whole && n <= 0)) return;
        if (whole || c.dim >= 4) {
            const int sh = whole || n >= 4 ? 0 : 4 - n, at = c.col(k) - sh;
            if constexpr (B16) {
                const kge_u32x2 r = *(const kge_u32x2_a2 *)((const uint16_t *)row + at);
                w[0] = r[0]; w[1] = r[1];
            } else w = *(const kge_u32x4_a4 *)((const uint32_t *)row + at);
            if (!whole && (c.dim & 3)) {
                if constexpr (B16) {
                    const uint64_t v = ((uint64_t)w[1] << 32 | w[0]) >> (16 * sh);
                    w[0] = (uint32_t)v; w[1] = (uint32_t)(v >> 32);
                } else {
                    if (sh & 1) w = kge_u32x4{w[1], w[2], w[3], 0u};
                    if (sh & 2) w = kge_u32x4{w[2], w[3], 0u, 0u};
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < n) {
                    if constexpr (B16) w[e >> 1] |= (uint32_t)((const uint16_t *)row)[e] << (16 * (e & 1));
                    else w[e] = ((const uint32_t *)row)[e];
                }
        }
    }
    __device__ __forceinline__ kge_f32x4 values() const {
        if constexpr (B16) return kge_f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
        else return kge_f32x4{__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]), __uint_as_float(w[3])};
    }
};
// stream: past the caches (KGE_STREAM_BYTES)
template <bool B16, int NG> __device__ __forceinline__ void store(char *row, const Columns<NG> &c, int k, kge_f32x4 v, bool stream) {
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf2;
    const int n = k < NG - 1 ? 4 : c.left(k), at = c.col(k);
    if (n >= 4) {
        if constexpr (B16) {
            const kge_u32x2 w = {__builtin_bit_cast(uint32_t, bf2{(__bf16)v[0], (__bf16)v[1]}), __builtin_bit_cast(uint32_t, bf2{(__bf16)v[2], (__bf16)v[3]})};
            if (stream) __builtin_nontemporal_store(w, (kge_u32x2_a2 *)((uint16_t *)row + at));
            else *(kge_u32x2_a2 *)((uint16_t *)row + at) = w;
        } else if (stream) __builtin_nontemporal_store(v, (kge_f32x4_a4 *)((float *)row + at));
        else *(kge_f32x4_a4 *)((float *)row + at) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) {
                if constexpr (B16) ((__bf16 *)row)[at + e] = (__bf16)v[e];
                else ((float *)row)[at + e] = v[e];
            }
    }
}
template <bool B16> __device__ __forceinline__ float load1(const void *row, int64_t col) {
    return B16 ? __uint_as_float((uint32_t)((const uint16_t *)row)[col] << 16) : ((const float *)row)[col];
}
template <bool B16> __device__ __forceinline__ void store1(void *row, int64_t col, float v) {
    if constexpr (B16) ((__bf16 *)row)[col] = (__bf16)v;
    else ((float *)row)[col] = v;
}

// A workgroup's threads in teams, each of which holds a row: of `waves` waves, or (SUB < 64) of SUB lanes of a wave
template <int SUB> struct Team {
    int waves, size, teams, team, lane;
    __device__ __forceinline__ explicit Team(int w) {
        if constexpr (SUB < 64) {
            waves = 1; size = SUB; teams = (int)blockDim.x / SUB;
            team = (int)threadIdx.x / SUB; lane = (int)threadIdx.x % SUB;
            return;
        }
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        waves = w; size = 64 * w; teams = max(1, (int)(blockDim.x >> 6) / w);
        team = wave / w; lane = (int)threadIdx.x - team * size;
    }
};

// x of the lanes 16 (32) further on, or back, added: rows 0 and 1, 2 and 3 of sixteen lanes (halves of the wave) change places
__device__ __forceinline__ float add_16(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float add_32(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// sum over the SUB lanes of a team (64: over the wave), for all of them
template <int SUB> __device__ __forceinline__ float wave_sum(float x) {
    x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0xB1, 0xf, 0xf, true));      // lane ^ 1
    x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x4E, 0xf, 0xf, true));      // lane ^ 2
    x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x141, 0xf, 0xf, true));     // 7 - lane
    x += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), 0x140, 0xf, 0xf, true));     // 15 - lane
    if constexpr (SUB == 16) return x;
    if constexpr (SUB == 32) return add_16(x);
    const int b = (int)__float_as_uint(x);
    const float s0 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, 0)), s1 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, 16));
    const float s2 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, 32)), s3 = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(b, 48));
    return (s0 + s1) + (s2 + s3);
}

// Sums of N values over the threads of a team, for all of them.  Two places in turn: who writes to one again has passed the barrier of the sums in
// between, behind which nobody reads it any more.  (Teams of one wave need no barrier, and go round as they like.)
template <int K, int NT, int SUB> struct Reduce {
    float (&lds)[2][NT / 64][K];
    const Team<SUB> &t;
    int place = 0;
    __device__ __forceinline__ Reduce(float (&l)[2][NT / 64][K], const Team<SUB> &team) : lds(l), t(team) {}
    template <int N> __device__ __forceinline__ void operator()(float (&v)[N]) {
        static_assert(N <= K, "sums at once");
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = wave_sum<SUB>(v[i]);
        if (SUB < 64 || t.waves == 1) return;
        const int wave = (int)threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) lds[place][wave][i] = v[i];
        }
        __syncthreads();
        const int w0 = t.team * t.waves;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lds[place][w0][i];
        for (int w = 1; w < t.waves; ++w)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += lds[place][w0 + w][i];
        place ^= 1;
    }
};

__device__ __forceinline__ float sum4(kge_f32x4 v, float s) { return s + ((v[0] + v[1]) + (v[2] + v[3])); }
__device__ __forceinline__ float dot4(kge_f32x4 a, kge_f32x4 b, float s) { return fmaf(a[3], b[3], fmaf(a[2], b[2], fmaf(a[1], b[1], fmaf(a[0], b[0], s)))); }
__device__ __forceinline__ float inv_sqrt(float x) { return 1.f / sqrtf(x); }

struct Norm { bool on, layer; float eps; const float *w, *b; };

// w A + b B, the sum over rows of what a norm with weight w and bias b has made, from the sums A and B of its parts.  Without a bias B may be infinite, or another sum may stand
// in its place: it does not count.
__device__ __forceinline__ float of_sums(float w, float a, float b, float bias_sum, bool bias) { return bias ? fmaf(w, a, b * bias_sum) : w * a; }
__device__ __forceinline__ kge_f32x4 of_sums(kge_f32x4 w, kge_f32x4 a, kge_f32x4 b, kge_f32x4 bias_sum, bool bias) { return bias ? fma4(w, a, b * bias_sum) : w * a; }

// x -> x^ = (x - mean) / deviation, of R rows at once
template <int NG, int R, class Sums>
__device__ __forceinline__ void normalise(kge_f32x4 (&x)[R][NG], const Columns<NG> &c, const Norm &norm, float inv_dim, Sums &reduce) {
    float v[R];
#pragma unroll
    for (int r = 0; r < R; ++r) v[r] = 0.f;
    if (norm.layer) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int k = 0; k < NG; ++k) v[r] = sum4(x[r][k], v[r]);
        reduce(v);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float mean = v[r] * inv_dim;
#pragma unroll
            for (int k = 0; k < NG; ++k) x[r][k] = c.minus(k, x[r][k], mean);
            v[r] = 0.f;
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int k = 0; k < NG; ++k) v[r] = dot4(x[r][k], x[r][k], v[r]);
    reduce(v);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float s = inv_sqrt(fmaf(v[r], inv_dim, norm.eps));
#pragma unroll
        for (int k = 0; k < NG; ++k) x[r][k] *= splat(s);
    }
}

struct FwdArgs {
    int dim, waves; int64_t rows;
    Norm post, pre; const float *scale;
    Matrix gate; uint32_t gate_rows;
    Matrix x, y, h, z; bool stream;
};

enum { SUM_A = 0, SUM_B = 1, SUM_C = 2, SUM_D = 3 };
struct BwdArgs {
    int dim, waves; int64_t rows;
    Norm post, pre; const float *scale;
    Matrix gate; uint32_t gate_rows;
    Matrix h, y, dh, dz, dx, dy, g_gate; bool stream;
    int64_t run, runs, part_ld; int parts;                        // rows of a run; runs; runs of a group, 0 where a run is not of one group
    uint32_t want;                                                // sums that are kept
    float *part;                                                  // [sum][run][part_ld]
    float *g_postw, *g_postb, *g_prew, *g_preb, *g_scale; int accumulate;
};

// Waves of a row, a power of two: twelve columns a lane at most, sixteen where a row has one wave or eight.  (Backward pass of fp32 / bf16 layer norms: 8,000 x 2,000 with four waves of
// eight columns a lane and with two of sixteen 87 us; 4,000 x 6,000 with twelve columns a lane 152, with sixteen 160.)
inline int waves_of(int dim) {
    if (dim <= 1024) return 1;
    int w = 2;
    while (w < 8 && 768 * w < dim) w *= 2;
    return w;
}
// Forward: two waves hold up to six groups a lane.  (Four waves, whose vectors leave the LDS room for fewer rows at once: 10,000 x 2,048 79 against 61 us, 6,000 x 3,000 76 against 64.  With
// eight groups in two waves 5,000 x 4,000 takes 100 us, with two in eight 81.)
inline int fwd_waves_of(int dim) { return dim <= 1024 ? 1 : dim <= 512 * 6 ? 2 : 8; }
// Lanes of a row: narrow ones share a wave, whose sums over lanes then serve two or four of them.  Layer norms, fp32 / bf16, 25.6M elements, shared and one row per
// wave: forward 64 columns 62 and 167 us, 128 64 and 93 (256 68 and 62: not shared); backward 64 104 and 315, 128 82 and 181, 256 84 and 112.
inline int bwd_lanes_of(int dim) { return dim <= 128 ? 16 : dim <= 256 ? 32 : 64 * waves_of(dim); }
inline int fwd_lanes_of(int dim) { return dim <= 128 ? 16 : 64 * fwd_waves_of(dim); }
// groups of four columns of a lane, the last of which no other group of the row lies behind
inline int groups_of(int dim, int lanes) { return (dim + 4 * lanes - 1) / (4 * lanes); }
// Teams of a workgroup of the backward pass.  Of one wave (no barriers between rows): as many as the registers leave room for on a compute unit, so that there are 256 runs'
// sums to join and not 768 (24,576 x 768: 9.4 MB of sums, 11 us); of more, whose waves meet at barriers, few.
// (Narrow rows have short sums: four workgroups per compute unit.)
constexpr int TEAMS_OF_ONE[3] = {16, 12, 8}, NARROW_THREADS = 256;    // (of two, three, four groups)
inline int bwd_teams_of(int dim) {
    const int w = waves_of(dim), lanes = bwd_lanes_of(dim);
    return lanes < 64 ? NARROW_THREADS / lanes : w == 1 ? TEAMS_OF_ONE[groups_of(dim, lanes) - 2] : w == 2 ? 2 : 1;
}
// workgroups of the backward pass that the chip holds at once
inline int64_t bwd_runs_of(int dim) {
    const int w = waves_of(dim), lanes = bwd_lanes_of(dim), g = groups_of(dim, lanes);
    return 256 * (lanes < 64 ? 4 : w == 1 ? 1 : w == 8 ? (g == 2 ? 2 : 1) : g == 2 ? 4 : 3);
}

// rows of the backward pass, by the stream's type
int rows_bwd16(const BwdArgs &a, bool b16, hipStream_t st);
int rows_bwd32(const BwdArgs &a, bool b16, hipStream_t st);

}  // namespace kge_norm
