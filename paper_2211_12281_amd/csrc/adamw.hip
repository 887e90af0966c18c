// One AdamW step over many dense tensors.
//
//   m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2,   theta <- theta (1 - lr wd) - lr (m c1) / (sqrt(v c2) + eps),   c = 1 / (1 - b^step)
//
// Memory bounds it: 28 bytes an element with fp32 moments and gradients (2 more with a bf16 copy), 14 with 8-bit moments and bf16 gradients.  The tensors are
// cut into chunks of one workgroup each (2,048 elements: 304 us for the tower below, 4,096: 341), which finds its tensor among the launch's by its chunk number; the descriptors are kernel arguments,
// so that nothing has to be copied to the device first and a captured call keeps them.  Measured: 89M elements in 181 tensors with 8-bit moments, bf16 gradients and copies 304 us
// (1.43 GB, 4.7 TB/s; without the generator's rounds 295: the vector pipe is nearly as busy as memory); 25M with fp32 moments 143 (712 MB, 5.0 TB/s); the encoder's two projections 5.4.
//
// 8-bit moments: e4m3 (m) and e5m2 (v) codes with a power of two per 128 elements.  The scale is a power of two, so an element whose value and block stay as they
// are keeps its code exactly, and stochastic rounding adds noise only in proportion to what a step changes.
#include "adam_ops.hpp"
#include "text_ops.hpp"

namespace {

constexpr int NT = 256, GROUPS = 2, CHUNK = NT * 4 * GROUPS;      // a thread takes groups of four elements, NT groups apart
constexpr int MAX_TENSORS = 40;                                   // of a launch: its arguments have to fit 4 KB
constexpr int BLOCK = 128;
constexpr int64_t MAX_CHUNKS = 1 << 23;                           // of a launch: a grid has fewer than 2^32 threads
static_assert(CHUNK % BLOCK == 0, "a block's elements belong to one chunk");

struct Tensor {
    float *p; uint16_t *p16; const void *g; void *m, *v; uint8_t *ms, *vs; int64_t n;
    float keep;                                                   // 1 - lr weight_decay
    uint32_t flags, index;
};
enum { G16 = 1, STATE8 = 2 };
struct Args {
    Tensor t[MAX_TENSORS];
    uint32_t first[MAX_TENSORS];                                  // chunk
    int tensors;
    float lr, b1, b2, omb1, omb2, c1, c2, eps;
    uint32_t k0, k1, tag;
    uint64_t step; const uint64_t *step_counter; const float *grad_scale;
};
static_assert(sizeof(Args) <= 4096, "kernel arguments");

typedef uint16_t u16x4_a2 __attribute__((ext_vector_type(4), aligned(2)));

// four elements at `at`, of which n are inside
__device__ __forceinline__ kge_f32x4 load4(const float *p, int64_t at, int n) {
    if (n >= 4) return *(const kge_f32x4_a4 *)(p + at);
    kge_f32x4 r = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (e < n) r[e] = p[at + e];
    return r;
}
__device__ __forceinline__ kge_f32x4 load4(const uint16_t *p, int64_t at, int n) {
    kge_u32x2 w = {0u, 0u};
    if (n >= 4) w = *(const kge_u32x2_a2 *)(p + at);
    else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) w[e >> 1] |= (uint32_t)p[at + e] << (16 * (e & 1));
    }
    return kge_f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
}
__device__ __forceinline__ void store4(float *p, int64_t at, int n, kge_f32x4 v) {
    if (n >= 4) *(kge_f32x4_a4 *)(p + at) = v;
    else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) p[at + e] = v[e];
    }
}
__device__ __forceinline__ void store4(uint16_t *p, int64_t at, int n, kge_f32x4 v) {
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf2;
    const kge_u32x2 w = {__builtin_bit_cast(uint32_t, bf2{(__bf16)v[0], (__bf16)v[1]}), __builtin_bit_cast(uint32_t, bf2{(__bf16)v[2], (__bf16)v[3]})};
    if (n >= 4) *(kge_u32x2_a2 *)(p + at) = w;
    else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) p[at + e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
    }
}

// ---------------------------------------------------------------------------------------------
// 8-bit moments
// ---------------------------------------------------------------------------------------------
constexpr uint32_t INF32 = 0x7f800000u;
template <int FMT> struct Fmt;
// exponents of the largest and of normal numbers, mantissa bits, largest code, codes of what is not finite
template <> struct Fmt<KGE_E4M3> { static constexpr int EMAX = 8, EMIN = -6, BITS = 3; static constexpr uint32_t TOP = 0x7e, INF = 0x7f, NAN8 = 0x7f; };
template <> struct Fmt<KGE_E5M2> { static constexpr int EMAX = 15, EMIN = -14, BITS = 2; static constexpr uint32_t TOP = 0x7b, INF = 0x7c, NAN8 = 0x7f; };

// 2^(byte - 127)
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte ? byte << 23 : 0x400000u); }

// A value is divided by its block's scale with two factors, 2^a and 2^b, a = floor((127 - byte) / 2), b = 127 - byte - a.  They are the math library's powf, which is 2^-24 low for
// some exponents (2^16 to 2^20 among them), and so is the factor 2^16 of the smallest second moments: a value in units of its spacing comes out up to 2^-19 low.  That is an eighth of what
// the random numbers cut anyway, but it decides the one value in 2^21 that falls on the border exactly, and with these factors it falls where the same steps done
// with elementary operations (power, product, sum, floor) put it, bit for bit: a program that checks its updates against such steps would else find a code in two million off by one, and what follows from
// it the step after.  The price is the table that a workgroup makes and a choice for each number: 304 us
// for the tower above, 291 with exact factors alone.
constexpr int POW0 = 60, POWS = 128;                              // exponents -60 .. 67
__device__ __forceinline__ float two_to(int n) {
    float two = 2.f;
    asm volatile("" : "+v"(two));                                 // (else the call becomes exp2f, which is exact)
    return powf(two, (float)n);
}

template <int FMT> __device__ __forceinline__ kge_f32x4 decode4(uint32_t w, float scale) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    f32x2 a, b;
    if constexpr (FMT == KGE_E4M3) { a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false); b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true); }
    else { a = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false); b = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true); }
    return kge_f32x4{a[0] * scale, a[1] * scale, b[0] * scale, b[1] * scale};
}

// largest of the 32 lanes that hold a block
__device__ __forceinline__ uint32_t max_of_32(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, true));      // lane ^ 1
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, true));      // lane ^ 2
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xf, 0xf, true));     // 7 - lane
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x140, 0xf, 0xf, true));     // 15 - lane
    return max(m, (uint32_t)__shfl_xor((int)m, 16));
}
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// A block's byte: of its finite elements the largest decides (kge_quantize's rule: the smallest power of two that it does not outgrow the format with)
template <int FMT> __device__ __forceinline__ uint32_t block_byte(kge_f32x4 x) {
    uint32_t m = max_of_32(max(max(mag(x[0]), mag(x[1])), max(mag(x[2]), mag(x[3]))));
    if (__any(m >= INF32)) {
        m = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) m = max(m, mag(x[e]) < INF32 ? mag(x[e]) : 0u);
        m = max_of_32(m);
    }
    return (uint32_t)max((int)((m + 0x1fffffu) >> 23) - Fmt<FMT>::EMAX, 0);
}

// x's code: |x| / scale in units of the spacing at its place, q, and floor(q + u), u in [0, 1) a multiple of 2^-16.  The factors take less from q than the
// least u adds; with u = 0 exact powers of two take their place.  So a value on the grid stays, whatever its random number, and no code is below the value's lower neighbour.
struct Inverse { float a, b, least; };                            // of a block's scale; of the spacing of the smallest second moments (that of first moments, 2^9, is exact)
template <int FMT> __device__ __forceinline__ Inverse inverse_of(uint32_t byte, const float *pow) {
    const int n = 127 - (int)byte, a = n >> 1;                        // (byte <= 255 - EMAX: 2^n is a normal number)
    return Inverse{pow[a + POW0], pow[n - a + POW0], pow[Fmt<FMT>::BITS - Fmt<FMT>::EMIN + POW0]};
}
template <int FMT> __device__ __forceinline__ uint32_t encode(float x, const Inverse &inv, uint32_t byte, uint32_t rnd) {
#pragma clang fp contract(off)
    using F = Fmt<FMT>;
    const bool exact = rnd == 0;
    const float t = fabsf(x) * (exact ? __uint_as_float((254u - byte) << 23) : inv.a) * (exact ? 1.f : inv.b);
    const uint32_t eb = max(__float_as_uint(t) >> 23, (uint32_t)(127 + F::EMIN));
    const float q = t * (FMT == KGE_E5M2 && eb == 127 + F::EMIN && !exact ? inv.least : __uint_as_float((uint32_t)(254 + F::BITS - eb) << 23));
    uint32_t code = ((eb - (127 + F::EMIN)) << F::BITS) + (uint32_t)(q + (float)rnd * 0x1p-16f);
    code = min(code, F::TOP);
    if (FMT == KGE_E5M2 && x > 0.f) code = max(code, 1u);
    const uint32_t b = __float_as_uint(x);
    if (mag(x) >= INF32) code = mag(x) == INF32 ? F::INF : F::NAN8;
    return code | (b >> 31 << 7);
}

__device__ __forceinline__ void philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1, uint32_t (&w)[4]) {
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
        c0 = kge_xor3((uint32_t)(p1 >> 32), c1, k0); c1 = (uint32_t)p1;
        c2 = kge_xor3((uint32_t)(p0 >> 32), c3, k1); c3 = (uint32_t)p0;
        k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
    }
    w[0] = c0; w[1] = c1; w[2] = c2; w[3] = c3;
}

// The moments' operations are rounded one by one (no fused multiply-add), so that their codes can be told in advance.
__device__ __forceinline__ void moments(const Args &a, kge_f32x4 g, kge_f32x4 &m, kge_f32x4 &v) {
#pragma clang fp contract(off)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float gm = g[e] * a.omb1, gg = g[e] * g[e];
        m[e] = m[e] * a.b1 + gm;
        v[e] = v[e] * a.b2 + gg * a.omb2;
    }
}

__global__ __launch_bounds__(NT) void adamw_kernel(const Args a) {
    __shared__ float pow[POWS];
    int lo = 0;                                                   // the last tensor whose first chunk is not behind this one
    for (int hi = a.tensors; hi - lo > 1;) {
        const int mid = (lo + hi) >> 1;
        if (a.first[mid] <= blockIdx.x) lo = mid;
        else hi = mid;
    }
    const Tensor &t = a.t[lo];
    const int64_t at0 = (int64_t)(blockIdx.x - a.first[lo]) * CHUNK + 4 * threadIdx.x;
    const bool g16 = t.flags & G16, state8 = t.flags & STATE8;
    kge_f32x4 p[GROUPS], g[GROUPS], m[GROUPS], v[GROUPS];
    uint32_t cm[GROUPS], cv[GROUPS], sm[GROUPS], sv[GROUPS];
    int n[GROUPS];
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
        const int64_t at = at0 + (int64_t)k * 4 * NT, left = t.n - at;
        n[k] = left > 4 ? 4 : left < 0 ? 0 : (int)left;
        p[k] = load4(t.p, at, n[k]);
        g[k] = g16 ? load4((const uint16_t *)t.g, at, n[k]) : load4((const float *)t.g, at, n[k]);
        if (state8) {
            cm[k] = cv[k] = sm[k] = sv[k] = 0;
            if (n[k] > 0) {                                       // (whole words: the codes are padded)
                cm[k] = *(const uint32_t *)((const uint8_t *)t.m + at); cv[k] = *(const uint32_t *)((const uint8_t *)t.v + at);
                sm[k] = t.ms[at / BLOCK]; sv[k] = t.vs[at / BLOCK];
            }
        } else { m[k] = load4((const float *)t.m, at, n[k]); v[k] = load4((const float *)t.v, at, n[k]); }
    }
    if (state8) {
        if (threadIdx.x < POWS) pow[threadIdx.x] = two_to((int)threadIdx.x - POW0);
        __syncthreads();
    }
    float c1 = a.c1, c2 = a.c2;
    uint32_t step = (uint32_t)a.step;
    if (a.step_counter) {
        const uint64_t s = a.step + *a.step_counter;
        c1 = adam_inv_bias(a.b1, s); c2 = adam_inv_bias(a.b2, s);
        step = (uint32_t)s;
    }
    const float gs = a.grad_scale ? *a.grad_scale : 1.f;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) {
        const int64_t at = at0 + (int64_t)k * 4 * NT;
        if (a.grad_scale) {
#pragma unroll
            for (int e = 0; e < 4; ++e) g[k][e] = e < n[k] ? g[k][e] * gs : 0.f;
        }
        if (state8) {
            m[k] = decode4<KGE_E4M3>(cm[k], scale_of(sm[k]));
            v[k] = decode4<KGE_E5M2>(cv[k], scale_of(sv[k]));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e >= n[k]) m[k][e] = v[k][e] = 0.f;
        }
        moments(a, g[k], m[k], v[k]);
        // With 8-bit moments the vector pipe is nearly as busy as memory: root and reciprocal from one instruction each, 2^-23 of themselves off (89M elements
        // 335 -> 304 us), beside a v whose codes carry 0.3 of noise.  (The root of a subnormal number, below 1.1e-19, is 0 there: only beside an eps that it does not change.)
        if (state8 && a.eps >= 1e-12f) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                p[k][e] = p[k][e] * t.keep - a.lr * (m[k][e] * c1) * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v[k][e] * c2) + a.eps);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) p[k][e] = p[k][e] * t.keep - a.lr * (m[k][e] * c1) / (sqrtf(v[k][e] * c2) + a.eps);
        }
        store4(t.p, at, n[k], p[k]);
        if (t.p16) store4(t.p16, at, n[k], p[k]);
        if (!state8) {
            store4((float *)t.m, at, n[k], m[k]);
            store4((float *)t.v, at, n[k], v[k]);
            continue;
        }
        const uint32_t bm = block_byte<KGE_E4M3>(m[k]), bv = block_byte<KGE_E5M2>(v[k]);
        if (at / BLOCK * BLOCK >= t.n) continue;                  // (a whole block behind the end)
        uint32_t w[4], em = 0, ev = 0;
        philox((uint32_t)(at >> 2), t.index, step, a.tag, a.k0, a.k1, w);
        const Inverse im = inverse_of<KGE_E4M3>(bm, pow), iv = inverse_of<KGE_E5M2>(bv, pow);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            em |= encode<KGE_E4M3>(m[k][e], im, bm, w[e] & 0xffffu) << (8 * e);
            ev |= encode<KGE_E5M2>(v[k][e], iv, bv, w[e] >> 16) << (8 * e);
        }
        *(uint32_t *)((uint8_t *)t.m + at) = em;
        *(uint32_t *)((uint8_t *)t.v + at) = ev;
        if ((threadIdx.x & 31) == 0) { t.ms[at / BLOCK] = (uint8_t)bm; t.vs[at / BLOCK] = (uint8_t)bv; }
    }
}

int check_tensor(const kge_adamw_tensor_t &t) {
    if (t.n < 0 || t.n >= (1ll << 34) || kge_bad_type(t.grad_dtype) || (t.state_bits != 32 && t.state_bits != 8) || t.reserved != 0 ||
        !(t.weight_decay >= 0.f) || t.weight_decay > 3e38f) return KGE_E_INVALID_ARG;
    if (t.n == 0) return KGE_OK;
    if (!t.param_f32 || !t.grad || !t.m || !t.v || ((uintptr_t)t.param_f32 & 3) != 0 || ((uintptr_t)t.param_bf16 & 1) != 0 ||
        ((uintptr_t)t.grad & (t.grad_dtype == KGE_BF16 ? 1 : 3)) != 0) return KGE_E_INVALID_ARG;
    if (t.state_bits == 32) return (((uintptr_t)t.m | (uintptr_t)t.v) & 3) != 0 ? KGE_E_INVALID_ARG : KGE_OK;
    return !t.m_scales || !t.v_scales || (((uintptr_t)t.m | (uintptr_t)t.v) & 15) != 0 ? KGE_E_INVALID_ARG : KGE_OK;
}

}  // namespace

extern "C" int kge_adamw(const kge_adamw_tensor_t *tensors, int32_t n_tensors, const kge_adamw_cfg_t *cfg, void *hip_stream) {
    if (n_tensors < 0 || (n_tensors > 0 && !tensors) || !cfg || cfg->reserved != 0 || ((uintptr_t)cfg->adam.step_counter & 7) != 0 || ((uintptr_t)cfg->grad_scale & 3) != 0)
        return KGE_E_INVALID_ARG;
    const kge_adam_cfg_t &c = cfg->adam;
    // (a step of 0 has no bias correction: the division by 1 - b^0 is one by zero)
    if (c.step < (c.step_counter ? 0 : 1) || !(c.beta1 >= 0.f && c.beta1 < 1.f) || !(c.beta2 >= 0.f && c.beta2 < 1.f) || !(c.eps >= 0.f) || !(c.lr == c.lr))
        return KGE_E_INVALID_ARG;
    for (int32_t i = 0; i < n_tensors; ++i)
        if (const int rc = check_tensor(tensors[i])) return rc;
    Args a = {};
    a.lr = c.lr; a.b1 = c.beta1; a.b2 = c.beta2; a.omb1 = 1.f - c.beta1; a.omb2 = 1.f - c.beta2; a.eps = c.eps;
    a.step = (uint64_t)c.step; a.step_counter = c.step_counter; a.grad_scale = cfg->grad_scale;
    if (!c.step_counter) { a.c1 = adam_inv_bias(c.beta1, a.step); a.c2 = adam_inv_bias(c.beta2, a.step); }
    a.k0 = (uint32_t)cfg->seed; a.k1 = (uint32_t)(cfg->seed >> 32); a.tag = cfg->tag;
    hipStream_t st = (hipStream_t)hip_stream;
    int64_t chunks = 0;
    bool any = false;
    auto launch = [&] {
        any = any || a.tensors;
        if (a.tensors) hipLaunchKernelGGL(adamw_kernel, dim3((unsigned)chunks), dim3(NT), 0, st, a);
        a.tensors = 0; chunks = 0;
    };
    for (int32_t i = 0; i < n_tensors; ++i) {
        const kge_adamw_tensor_t &t = tensors[i];
        if (t.n == 0) continue;
        const int64_t more = (t.n + CHUNK - 1) / CHUNK;
        if (a.tensors == MAX_TENSORS || chunks + more > MAX_CHUNKS) launch();
        a.first[a.tensors] = (uint32_t)chunks;
        a.t[a.tensors++] = Tensor{t.param_f32, (uint16_t *)t.param_bf16, t.grad, t.m, t.v, t.m_scales, t.v_scales, t.n,
                                  (float)(1.0 - (double)c.lr * (double)t.weight_decay),
                                  (t.grad_dtype == KGE_BF16 ? G16 : 0u) | (t.state_bits == 8 ? STATE8 : 0u), (uint32_t)i};
        chunks += more;
    }
    launch();
    return any ? kge_launch_status() : KGE_OK;
}
