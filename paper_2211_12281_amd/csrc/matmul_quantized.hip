// Matrix product of two quantised matrices (quantize.hip), both contiguous along the contraction:
//
//   out[i, j] (+)= sum over blocks of 128:  2^(sa[i, kb] + sb[j, kb] - 254)  sum over k in the block of  A[rows[i], k] B[j, k]
//
// The rows of A may be gathered (rows): the projection of the features of a step's slots reads them straight from the entities' table.
//
// Two kinds of products:
//   bf16 output  (unless fp32 sums are asked for) 32 x 32 x 64 matrix instructions on the 8-bit codes themselves, which take the scales as exponent bytes.  They align
//                every eight products to the largest of them and drop what lies 13 bits below it (groups are added in fp32): 1.4e-5 of the
//                result on normal values (2-norm), 1 / 100 of the output's own rounding.  Where products cancel the cut stays: up to 7 x 2^-13 of the largest
//                of each eight.
//   fp32 sums    the codes are widened to bf16 with their scale and multiplied with 32 x 32 x 16 bf16 instructions and fp32 sums: 1e-7, at half
//                the rate.  Widening is exact for every code under scale bytes 3..246 (e4m3) or 10..239 (e5m2); below, what is no multiple of
//                2^-133, bf16's smallest number, is rounded to one, and above, codes of 2^128 and more become infinite.  (The 8-bit
//                instructions add the scales' exponents and know neither end.)
//
// What bounds it: large products the matrix pipe and the clock that it leaves (16,384 x 4,096 x 4,096: bf16 output 230 us, 2.39 PFLOP/s, of
// which first fragments and the last tiles' stores are a tenth, matrix pipe 62 % busy at 1.9 GHz; fp32 output 425 us, 1.29 PFLOP/s, 73 % busy at 1.78 GHz);
// products of a few hundred tiles the trips to memory of a tile's start and end (24,576 gathered rows x 256 x 768, fp32 output: 22 us, of which its bytes are 10);
// one token the weights' bytes or the launch (1 x 2,048 x 2,048 4.1 us, 1 x 4,096 x 16,384 17.4, 3.9 TB/s).
#include "lds_copy.hpp"
#include "text_ops.hpp"
#include <type_traits>

typedef int mq_i32x8 __attribute__((ext_vector_type(8)));
typedef float mq_f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 mq_bf16x8 __attribute__((ext_vector_type(8)));

int kge_check_quantized(const kge_quantized_t *q);

namespace {

constexpr int BLOCK = 128;                                    // elements of a scale's block, and bytes of a row that a stage holds

// acc + u v^t with the scales in byte i of sb and byte j of sa; i and j are known when this is inlined into unrolled loops
template <int FU, int FV, int I, int J> __device__ __forceinline__ mq_f32x16 mq_mma_ij(mq_i32x8 u, mq_i32x8 v, mq_f32x16 acc, int sb, int sa) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(u, v, acc, FU, FV, I, sb, J, sa);
}
template <int FU, int FV> __device__ __forceinline__ mq_f32x16 mq_mma(mq_i32x8 u, mq_i32x8 v, mq_f32x16 acc, int i, int j, int sb, int sa) {
    switch (4 * i + j) {
    case 0: return mq_mma_ij<FU, FV, 0, 0>(u, v, acc, sb, sa);
    case 1: return mq_mma_ij<FU, FV, 0, 1>(u, v, acc, sb, sa);
    case 2: return mq_mma_ij<FU, FV, 0, 2>(u, v, acc, sb, sa);
    case 3: return mq_mma_ij<FU, FV, 0, 3>(u, v, acc, sb, sa);
    case 4: return mq_mma_ij<FU, FV, 1, 0>(u, v, acc, sb, sa);
    case 5: return mq_mma_ij<FU, FV, 1, 1>(u, v, acc, sb, sa);
    case 6: return mq_mma_ij<FU, FV, 1, 2>(u, v, acc, sb, sa);
    default: return mq_mma_ij<FU, FV, 1, 3>(u, v, acc, sb, sa);
    }
}

struct MatmulArgs {
    const uint8_t *a, *as; int64_t a_ld, as_ld; const int32_t *rows; int64_t a_rows;
    const uint8_t *b, *bs; int64_t b_ld, bs_ld;
    int64_t m, n;
    void *out; int64_t out_ld; int out16, accumulate;
    float *part; int64_t part_ld;                             // partial sums [split][m][part_ld] (null: one split)
    int kb, kb_per, splits, tiles_m, tiles_n;
};

// Two codes (low or high half of a word) as two bf16 numbers with their scale 2^(byte - 127), given as a float's bits byte << 23
template <int FMT, bool HI> __device__ __forceinline__ uint32_t mq_widen2(uint32_t w, float scale) {
    if constexpr (FMT == KGE_E4M3) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, HI));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, HI));
}
template <int FMT> __device__ __forceinline__ mq_bf16x8 mq_widen8(uint32_t lo, uint32_t hi, float scale) {
    const kge_u32x4 r = {mq_widen2<FMT, false>(lo, scale), mq_widen2<FMT, true>(lo, scale), mq_widen2<FMT, false>(hi, scale), mq_widen2<FMT, true>(hi, scale)};
    return __builtin_bit_cast(mq_bf16x8, r);
}

// eight (bf16 output) or four (fp32 output, and partial sums) consecutive columns of an output row
template <bool OUT16> __device__ __forceinline__ void mq_store(const MatmulArgs &p, int64_t row, int64_t col, float (&v)[OUT16 ? 8 : 4], bool valid) {
    constexpr int C = OUT16 ? 8 : 4;
    const int n = (int)(p.n - col < C ? p.n - col : C);
    if (n <= 0) return;
#pragma unroll
    for (int e = 0; e < C; ++e) v[e] = valid ? v[e] : 0.f;
    if constexpr (OUT16) {
        uint16_t *q = (uint16_t *)p.out + row * p.out_ld;
        if (p.accumulate) {
            float o[8];
            kge_load8<true>(q, col, n, o);
#pragma unroll
            for (int e = 0; e < C; ++e) v[e] += o[e];
        }
        kge_store8<true>(q, col, n, v);
    } else {
        float *q = (float *)p.out + row * p.out_ld + col;
        if (n == 4) {
            kge_f32x4 r = {v[0], v[1], v[2], v[3]};
            if (p.accumulate) {
                const kge_f32x4 o = *(const kge_f32x4_a4 *)q;
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] += o[e];
            }
            *(kge_f32x4_a4 *)q = r;
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < n) q[e] = p.accumulate ? q[e] + v[e] : v[e];
        }
    }
}
// four columns, whatever the output's type
__device__ __forceinline__ void mq_store4(const MatmulArgs &p, int64_t row, int64_t col, kge_f32x4 s, bool valid) {
    if (!p.out16) {
        float v[4] = {s[0], s[1], s[2], s[3]};
        mq_store<false>(p, row, col, v, valid);
        return;
    }
    const int n = (int)(p.n - col < 4 ? p.n - col : 4);
    uint16_t *q = (uint16_t *)p.out + row * p.out_ld + col;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (p.accumulate && e < n ? __uint_as_float((uint32_t)q[e] << 16) : 0.f) + (valid ? s[e] : 0.f);
    if (n == 4) {
        typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf2;
        *(kge_u32x2_a2 *)q = kge_u32x2{__builtin_bit_cast(uint32_t, bf2{(__bf16)v[0], (__bf16)v[1]}), __builtin_bit_cast(uint32_t, bf2{(__bf16)v[2], (__bf16)v[3]})};
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n) ((__bf16 *)q)[e] = (__bf16)v[e];
    }
}
__device__ __forceinline__ bool mq_row_valid(const MatmulArgs &p, int64_t row) {
    if (!p.rows) return true;
    const int64_t r = p.rows[row];
    return r >= 0 && r < p.a_rows;
}

// Workgroup = WM x WN waves = TM rows of A x TN rows of B, wave = NJ x NI blocks of 32 x 32.  Stages of a block of 128 bytes of every row pass through a
// ring of NST stages in the LDS, filled by asynchronous copies (whole lines: with half of one per row and copy they ran at half the rate, 65 instead
// of 136 GB/s per compute unit from the L2); the words with four blocks' scales of every row come with the first block that needs them, into one of two
// places.  A row's 16-byte pieces lie XOR-swizzled by (row / 2) % 8, so that the fragment reads of sixteen consecutive rows fall into different ones of
// the 64 banks.  Rows beyond the matrices are read from row 0 and
// not stored.  Which bytes of a block a lane half contracts first does not matter as long as both operands agree.
//
// The fragments of the next step are read while this one's are multiplied, across the stages too: the only barrier of a stage stands in front of the
// products of its last step, whose operands are in registers by then, and the stage that it frees is refilled behind it.
//
// FAR: a copy's lanes have 64-bit addresses; else (codes and scales of less than 4 GiB) a base and 32-bit offsets, which the larger wave tile needs for its registers.
template <int WM, int WN, int NJ, int NI, int NST, bool FAR, bool WIDE, int FA, int FB>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(NI * NJ > 8 ? 1 : 2, NI * NJ > 8 ? 1 : 2)))
void matmul_tiles_kernel(const MatmulArgs p) {
    constexpr int NW = WM * WN, TM = 32 * NJ * WM, TN = 32 * NI * WN, ROWS = TM + TN;
    constexpr int CP = ROWS / 8 / NW, SC = (ROWS / 64 + NW - 1) / NW, PER = CP + SC;      // copies of a wave per stage: codes, scales
    constexpr int STAGE = ROWS * BLOCK, WORDS = NW * SC * 256, STEPS = WIDE ? 4 : 2;
    static_assert(ROWS % (8 * NW) == 0 && ROWS % 64 == 0 && TN % 64 == 0 && NST >= 2, "tile");
    static_assert((NST - 1) * PER < 64 && NST * STAGE + 3 * WORDS <= 160 * 1024, "copies in flight, LDS");
    __shared__ __attribute__((aligned(16))) char lds[NST * STAGE + 3 * WORDS];           // (the third place of the words: nothing reads it)
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 31, g = lane >> 5;
    // ids go round-robin to the 8 dies: a die takes a run of tiles, eight tiles of A deep, so that both operands' rows meet in its L2
    const int total = p.tiles_m * p.tiles_n * p.splits, per = (total + 7) >> 3;
    int w = ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);
    if (((int)blockIdx.x >> 3) >= per || w >= total) return;
    const int split = w / (p.tiles_m * p.tiles_n);
    w -= split * p.tiles_m * p.tiles_n;
    const int band = w / (8 * p.tiles_n), deep = min(8, p.tiles_m - 8 * band), in = w - band * 8 * p.tiles_n;
    const int64_t m0 = (int64_t)(8 * band + in % deep) * TM, n0 = (int64_t)(in / deep) * TN;
    const int kb0 = split * p.kb_per, kb1 = min(p.kb, kb0 + p.kb_per);

    // Row r of the stage: B's tile first, then A's.  Copy j of this wave takes rows 8 (CP wave + j) .. + 7
    auto b_row = [&](int r) { const int64_t s = n0 + r; return s < p.n ? s : 0; };
    auto a_row = [&](int r) -> int64_t {
        const int64_t s = m0 + r;
        if (s >= p.m) return 0;
        if (!p.rows) return s;
        const int64_t t = p.rows[s];
        return t >= 0 && t < p.a_rows ? t : 0;
    };
    auto swizzle = [](int r) { return (r >> 1) & 7; };
    static_assert(FAR || (TN % 64 == 0 && SC == 1 && CP == 8), "all rows that a wave copies are of one operand");
    const bool of_b = 64 * wave < TN;                                              // (not FAR)
    const uint8_t *base = of_b ? p.b : p.a, *sbase = of_b ? p.bs : p.as;
    const uint8_t *gc[FAR ? CP : 1], *gs[FAR ? SC : 1];
    uint32_t oc[FAR ? 1 : CP], os = 0;
#pragma unroll
    for (int j = 0; j < CP; ++j) {
        const int r0 = 8 * (CP * wave + j), r = r0 + (lane >> 3), piece = ((lane & 7) ^ swizzle(r)) * 16;
        if constexpr (FAR) gc[j] = (r0 < TN ? p.b + b_row(r) * p.b_ld : p.a + a_row(r - TN) * p.a_ld) + piece + (int64_t)kb0 * BLOCK;   // (a copy's rows are of one operand)
        else oc[j] = (uint32_t)(of_b ? b_row(r) * p.b_ld : a_row(r - TN) * p.a_ld) + piece;
    }
    if constexpr (!FAR) {
        base += (int64_t)kb0 * BLOCK;
        const int r = 64 * wave + lane;
        os = (uint32_t)(of_b ? b_row(r) * p.bs_ld : a_row(r - TN) * p.as_ld);
    } else {
#pragma unroll
        for (int j = 0; j < SC; ++j) {
            const int r = 64 * (SC * wave + j);                                   // (past the last row: row 0 again, to a place that nothing reads)
            gs[j] = r < TN ? p.bs + b_row(r + lane) * p.bs_ld : r < ROWS ? p.as + a_row(r - TN + lane) * p.as_ld : p.bs;
        }
    }
    // (the gathered row numbers have to be there before the loop: a wait of the compiler's inside it would drain the ring)
#pragma unroll
    for (int j = 0; j < CP; ++j) {
        if constexpr (FAR) asm volatile("" : "+v"(gc[j]));
        else asm volatile("" : "+v"(oc[j]));
    }
    if constexpr (FAR) {
#pragma unroll
        for (int j = 0; j < SC; ++j) asm volatile("" : "+v"(gs[j]));
    } else asm volatile("" : "+v"(os));

    int next = kb0;                                                               // block that the next copies fetch, and their addresses'
    auto copy = [&](int slot, int c) {
        if (c >= SC) {
            const uint32_t to = lds0 + (uint32_t)slot * STAGE + (uint32_t)(CP * wave + c - SC) * 1024;
            if constexpr (FAR) kge_copy16(gc[c - SC], to);
            else kge_copy16(base, oc[c - SC], to);
        } else {
            // scales first.  Where the word has been copied before, all lanes take one address and write to the third place: no branch, which would
            // take the products of the step before behind the barrier, and no lines fetched again
            const bool need = (next & 3) == 0 || next == kb0;
            const uint32_t to = lds0 + NST * STAGE + (need ? (uint32_t)(next >> 2 & 1) : 2u) * WORDS + (uint32_t)(SC * wave + c) * 256;
            const int off = (next >> 2) * 4;
            if constexpr (FAR) kge_copy4((need ? gs[c] : p.bs) + off, to);
            else kge_copy4(sbase + off, os & (need ? 0xffffffffu : 0u), to);
        }
    };
    auto advance = [&] {                                                          // past the end: the last block again, harmless
        const int d = next + 1 < kb1 ? 1 : 0;
        next += d;
        if constexpr (FAR) {
#pragma unroll
            for (int j = 0; j < CP; ++j) gc[j] += d * BLOCK;
        } else base += d * BLOCK;
    };
    const int wn = (wave % WN) * 32 * NI, wm = (wave / WN) * 32 * NJ;
    mq_f32x16 acc[NI][NJ];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

    // Fragments of the operands.  Of the codes, the last block of A and all of B have two places each, for this step's and the next one's; the other blocks of A are
    // read again as soon as their last product of the step has been issued.  Widened codes (WIDE) leave their place at once: every block has one; of the
    // widened ones, B and the first block of A have two places (made behind the last products of the step before), the other blocks of A take turns in two.
    constexpr int Q = WIDE ? 1 : 2;                                               // 16-byte pieces of a row that a lane reads per step
    struct Codes { kge_u32x4 b[WIDE ? 1 : 2][NI][Q], a[NJ - 1][Q], l[WIDE ? 1 : 2][Q]; } f;
    struct Wide { mq_bf16x8 b[2][NI][2], a0[2][2], a[2][2]; } v;
    struct Words { uint32_t b[NI], a[NJ]; } words;                                // of the rows, as copied
    uint32_t xb, xa;                                                              // the block's byte of each of the wave's blocks of rows
    constexpr int SLOTS = NI * NJ * (WIDE ? 2 : 1);                               // products per step
    const int swz = swizzle(lr);
    auto read = [&](kge_u32x4 (&to)[Q], int slot, int step, int row) {
        const char *s = lds + slot * STAGE + (row + lr) * BLOCK;
#pragma unroll
        for (int u = 0; u < Q; ++u) to[u] = *(const kge_u32x4 *)(s + (((WIDE ? 2 * step + g : 4 * step + 2 * g + u) ^ swz) << 4));
    };
    auto read_b = [&](int set, int i, int slot, int step) { read(f.b[WIDE ? 0 : set][i], slot, step, wn + 32 * i); };
    auto read_a = [&](int set, int j, int slot, int step) { read(j < NJ - 1 ? f.a[j < NJ - 1 ? j : 0] : f.l[WIDE ? 0 : set], slot, step, TN + wm + 32 * j); };
    auto read_scales = [&](int kb) {                                              // the words; use_scales takes block kb's bytes from them
        const uint32_t *s = (const uint32_t *)(lds + NST * STAGE + (kb >> 2 & 1) * WORDS);
#pragma unroll
        for (int i = 0; i < NI; ++i) words.b[i] = s[wn + 32 * i + lr];
#pragma unroll
        for (int j = 0; j < NJ; ++j) words.a[j] = s[TN + wm + 32 * j + lr];
    };
    auto use_scales = [&](int kb) {
        auto pack = [&](const uint32_t *w, int n) {                               // byte kb % 4 of up to four words
            const uint32_t pick = 0x0c0c0400u + 0x0101u * (kb & 3);               // (of a pair; 0x0c: a zero byte)
            const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], pick);
            return n > 2 ? lo | __builtin_amdgcn_perm(w[n - 1], w[n - 2], pick) << 16 : lo;
        };
        xb = pack(words.b, NI);
        xa = pack(words.a, NJ);
    };
    static_assert(NI == 2 && (NJ == 2 || NJ == 4), "pairs");
    auto widen_b = [&](int set, int i, int h) {
        const kge_u32x4 &q = f.b[0][i][0];
        v.b[set][i][h] = mq_widen8<FB>(q[2 * h], q[2 * h + 1], __uint_as_float((xb >> (8 * i) & 255u) << 23));
    };
    auto widen_a = [&](int set, int j, int h) {
        const kge_u32x4 &q = j < NJ - 1 ? f.a[j < NJ - 1 ? j : 0][0] : f.l[0][0];
        const mq_bf16x8 w = mq_widen8<FA>(q[2 * h], q[2 * h + 1], __uint_as_float((xa >> (8 * j) & 255u) << 23));
        if (j == 0) v.a0[set][h] = w;
        else v.a[j & 1][h] = w;
    };
    // The products of one step and, behind each of them, the reads of the next step's fragments that have their slot there, and whatever `also` does.  (Left to
    // itself the compiler puts all reads in front of all products, and those behind the barrier.)
    auto step = [&](int set, int slot, int st, auto also) {                       // slot, st: of the next step
#pragma unroll
        for (int t = 0; t < SLOTS; ++t) {
            if constexpr (WIDE) {
                const int j = t / (2 * NI), h = t / NI % 2, i = t % NI, u = t % (2 * NI);
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.b[set][i][h], j == 0 ? v.a0[set][h] : v.a[j & 1][h], acc[i][j], 0, 0, 0);
                also(t);
                // the next block of A is widened behind the first products of this one, the next step's B and first block of A behind the step's last
                if (j < NJ - 1 && u < 2) widen_a(set, j + 1, u);
                if (j == NJ - 1) {
                    widen_b(set ^ 1, u / 2, u % 2);
                    if (u < 2) widen_a(set ^ 1, 0, u);
                }
                if (t < NI) read_b(set ^ 1, t, slot, st);
                if (t == NI) read_a(set ^ 1, 0, slot, st);
                if (j < NJ - 1 && u == 3) read_a(set ^ 1, j + 1, slot, st);
            } else {
                const int j = t / NI, i = t % NI;
                auto full = [](const kge_u32x4 (&q)[Q]) {
                    return mq_i32x8{(int)q[0][0], (int)q[0][1], (int)q[0][2], (int)q[0][3], (int)q[Q - 1][0], (int)q[Q - 1][1], (int)q[Q - 1][2], (int)q[Q - 1][3]};
                };
                // (which byte of a scale register counts is part of the instruction)
                acc[i][j] = mq_mma<FB, FA>(full(f.b[set][i]), full(j < NJ - 1 ? f.a[j < NJ - 1 ? j : 0] : f.l[set]), acc[i][j], i, j, (int)xb, (int)xa);
#pragma unroll
                for (int k = 0; k < NI; ++k)
                    if (t == k * NJ / 2) read_b(set ^ 1, k, slot, st);
#pragma unroll
                for (int k = 0; k < NJ - 1; ++k)
                    if (t == NI * (k + 1) - 1) read_a(set ^ 1, k, slot, st);
                if (t == NI * NJ / 2) read_a(set ^ 1, NJ - 1, slot, st);
                also(t);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    if (kb0 < kb1) {
#pragma unroll
        for (int s = 0; s < NST; ++s) {
#pragma unroll
            for (int c = 0; c < PER; ++c) copy(s, c);
            advance();
        }
        kge_wait_vmcnt<(NST - 1) * PER>();
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NI; ++i) read_b(0, i, 0, 0);
#pragma unroll
        for (int j = 0; j < NJ; ++j) read_a(0, j, 0, 0);
        read_scales(kb0);
        use_scales(kb0);
        if constexpr (WIDE) {                                                     // what the step before the first one would have left
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < NI; ++i) widen_b(0, i, h);
                widen_a(0, 0, h);
            }
        }
        // the next block's scales are used behind the step's products, or where its first fragments are widened
        constexpr int READ_SCALES = WIDE ? 1 : SLOTS - 2, USE_SCALES = WIDE ? SLOTS - 2 * NI - 1 : SLOTS - 1;
        int slot = 0;
        for (int kb = kb0; kb < kb1; ++kb) {
            const int after = slot == NST - 1 ? 0 : slot + 1;
#pragma unroll
            for (int st = 0; st < STEPS; ++st) {
                const bool last = st == STEPS - 1;
                if (last) {
                    kge_wait_vmcnt<(NST - 2) * PER>();                             // the next block has landed ...
                    __syncthreads();                                              // ... for everyone, and everyone has read this one, whose stage is refilled
                }
                step(st & 1, last ? after : slot, last ? 0 : st + 1, [&](int t) {
                    if (!last) return;
                    if (t == READ_SCALES) read_scales(kb + 1);
                    if (WIDE && t == USE_SCALES) use_scales(kb + 1);
#pragma unroll
                    for (int c = 0; c < PER; ++c)
                        if (c * SLOTS / PER == t) copy(slot, c);
                });
            }
            if constexpr (!WIDE) use_scales(kb + 1);
            advance();
            slot = after;
        }
        kge_wait_vmcnt<0>();                                                       // no copy may be in flight when the LDS is released
    }

    // Accumulator layout: lane holds row lr of A's block; element e is B's row 8 (e / 4) + 4 g + e % 4.  Stored from there a row gets sixteen bytes at a
    // time, a quarter of the copy rate and up to a third of the call; so 32 rows of the wave at a time go through the LDS, and rows leave in whole lines.
    // (Row stride one piece more than the row: writes and reads of sixteen lanes fall into different banks.)
    constexpr int LD = 32 * NI + 4;
    static_assert(NW * 32 * LD * 4 <= NST * STAGE, "the waves' rows fit the ring");
    float *mine = (float *)lds + wave * (32 * LD);
    __syncthreads();                                                              // everyone is done with the ring
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *(kge_f32x4 *)(mine + lr * LD + 32 * i + 8 * q + 4 * g) = kge_f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        __builtin_amdgcn_wave_barrier();
        const int64_t row0 = m0 + wm + 32 * j, col0 = n0 + wn;
        auto rows = [&](auto wide) {                                              // wide: eight columns per lane, else four
            constexpr int C = decltype(wide)::value ? 8 : 4, LPR = 32 * NI / C, RPI = 64 / LPR;     // lanes per row, rows at a time
            const int c = C * (lane % LPR);
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += RPI) {
                const int r = r0 + lane / LPR;
                const int64_t row = row0 + r;
                float v[C];
#pragma unroll
                for (int e = 0; e < C; e += 4) {
                    const kge_f32x4 x = *(const kge_f32x4 *)(mine + r * LD + c + e);
#pragma unroll
                    for (int u = 0; u < 4; ++u) v[e + u] = x[u];
                }
                if (row >= p.m) continue;
                if constexpr (C == 4)
                    if (p.part) {
                        if (col0 + c < p.part_ld) *(kge_f32x4 *)(p.part + ((int64_t)split * p.m + row) * p.part_ld + col0 + c) = kge_f32x4{v[0], v[1], v[2], v[3]};
                        continue;
                    }
                mq_store<C == 8>(p, row, col0 + c, v, mq_row_valid(p, row));
            }
        };
        if (p.part || !p.out16) rows(std::false_type());
        else rows(std::true_type());
        __builtin_amdgcn_wave_barrier();
    }
}

// Sums the splits' partial results in order.
__global__ __launch_bounds__(256) void matmul_join_kernel(const MatmulArgs p) {
    const int64_t per = p.part_ld / 4, total = p.m * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per, col = (i - row * per) * 4;
        kge_f32x4 s = {0.f, 0.f, 0.f, 0.f};
        for (int k = 0; k < p.splits; ++k) {
            const kge_f32x4 x = *(const kge_f32x4 *)(p.part + ((int64_t)k * p.m + row) * p.part_ld + col);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += x[e];
        }
        mq_store4(p, row, col, s, mq_row_valid(p, row));
    }
}

// Few rows of A (one token, a small batch), and small products of any shape: a workgroup takes sixteen rows of B against 16 MF rows of A, its eight
// waves take the blocks of 128 in turn, straight from memory into fragments, and add up through the LDS in order.  One token reads the weights
// once, which bounds it; a small product is over after one or two trips to memory, where a tile's ring makes one for every two blocks.
constexpr int SKINNY_WAVES = 8;
template <int MF, bool WIDE, int FA, int FB>
__global__ __launch_bounds__(64 * SKINNY_WAVES) void matmul_skinny_kernel(const MatmulArgs p) {
    __shared__ float part[SKINNY_WAVES][MF][16][16 + 4];       // [wave][block][row of A][row of B]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)(blockIdx.x % (uint32_t)p.tiles_n) * 16, m0 = (int64_t)(blockIdx.x / (uint32_t)p.tiles_n) * (16 * MF), rb = n0 + lr < p.n ? n0 + lr : 0;
    const uint8_t *gb = p.b + rb * p.b_ld + 32 * g, *sb = p.bs + rb * p.bs_ld, *ga[MF], *sa[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        const int64_t r = m0 + 16 * f + lr;
        int64_t s = r < p.m ? (p.rows ? (int64_t)p.rows[r] : r) : 0;
        s = s >= 0 && s < p.a_rows ? s : 0;
        ga[f] = p.a + s * p.a_ld + 32 * g; sa[f] = p.as + s * p.as_ld;
    }
    kge_f32x4 acc[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) acc[f] = kge_f32x4{0.f, 0.f, 0.f, 0.f};
    for (int kb = wave; kb < p.kb; kb += SKINNY_WAVES) {
        const kge_u32x4 b0 = *(const kge_u32x4 *)(gb + (int64_t)kb * BLOCK), b1 = *(const kge_u32x4 *)(gb + (int64_t)kb * BLOCK + 16);
        const uint32_t eb = sb[kb];
        kge_u32x4 a0[MF], a1[MF];
        uint32_t ea[MF];
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            a0[f] = *(const kge_u32x4 *)(ga[f] + (int64_t)kb * BLOCK); a1[f] = *(const kge_u32x4 *)(ga[f] + (int64_t)kb * BLOCK + 16);
            ea[f] = sa[f][kb];
        }
        if constexpr (!WIDE) {
            const mq_i32x8 fb = {(int)b0[0], (int)b0[1], (int)b0[2], (int)b0[3], (int)b1[0], (int)b1[1], (int)b1[2], (int)b1[3]};
#pragma unroll
            for (int f = 0; f < MF; ++f) {
                const mq_i32x8 fa = {(int)a0[f][0], (int)a0[f][1], (int)a0[f][2], (int)a0[f][3], (int)a1[f][0], (int)a1[f][1], (int)a1[f][2], (int)a1[f][3]};
                acc[f] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fb, fa, acc[f], FB, FA, 0, (int)eb, 0, (int)ea[f]);
            }
        } else {
            const float xb = __uint_as_float(eb << 23);
            const mq_bf16x8 fb[4] = {mq_widen8<FB>(b0[0], b0[1], xb), mq_widen8<FB>(b0[2], b0[3], xb), mq_widen8<FB>(b1[0], b1[1], xb), mq_widen8<FB>(b1[2], b1[3], xb)};
#pragma unroll
            for (int f = 0; f < MF; ++f) {
                const float xa = __uint_as_float(ea[f] << 23);
                acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[0], mq_widen8<FA>(a0[f][0], a0[f][1], xa), acc[f], 0, 0, 0);
                acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[1], mq_widen8<FA>(a0[f][2], a0[f][3], xa), acc[f], 0, 0, 0);
                acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[2], mq_widen8<FA>(a1[f][0], a1[f][1], xa), acc[f], 0, 0, 0);
                acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[3], mq_widen8<FA>(a1[f][2], a1[f][3], xa), acc[f], 0, 0, 0);
            }
        }
    }
    // lane holds A's row lr; element e is B's row 4 g + e
#pragma unroll
    for (int f = 0; f < MF; ++f) *(kge_f32x4 *)&part[wave][f][lr][4 * g] = acc[f];
    __syncthreads();
    for (int i = tid; i < MF * 64; i += 64 * SKINNY_WAVES) {
        const int f = i >> 6, row = (i >> 2) & 15, c = (i & 3) * 4;
        kge_f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < SKINNY_WAVES; ++k) {
            const kge_f32x4 x = *(const kge_f32x4 *)&part[k][f][row][c];
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] += x[e];
        }
        const int64_t r = m0 + 16 * f + row;
        if (r >= p.m) continue;
        mq_store4(p, r, n0 + c, s, mq_row_valid(p, r));
    }
}

// ---------------------------------------------------------------------------------------------
// Which kernel (times of bf16 output, microseconds, rows of A x rows of B x contraction; those of fp32 output lie the same way):
//   few rows, or little work   up to 512 workgroups of matmul_skinny_kernel whose waves take at most 12 blocks' worth of rows of A each (blocks in
//                              turn x sixteens of rows), or up to 16 rows of A against any number of B's with at most four blocks in turn.
//                              Within: 1 x 4,096 x 4,096 6.7 against 15.6 in tiles, 300 x 256 x 3,000 10.3 against 11.8, 1 x 50,000 x 768
//                              9.2 against 11.1.  Beyond: 64 x 4,096 x 4,096 16.3 against 13.9, 3,000 x 256 x 768 9.3 against 8.0.
//   tiles of 256 x 256         from 192 of them on, unless one row of tiles of 128 x 128 holds either side: 3,584 x 3,584 x 4,096 (196 tiles) 61.9 against
//                              75.7 in tiles of 128 x 128, 160 x 65,536 x 768 20.8 against 25.3; but 32,768 x 256 x 768 (128 tiles) 18.9 against
//                              14.7 and 128 x 50,000 x 4,096 57.2 against 38.2.
//   a split contraction        up to 128 tiles, into parts of at least eight blocks and 512 workgroups in all: 200 x 4,096 x 4,096 20.0, with
//                              parts of four 22.7; 2,000 x 2,000 x 2,000 (256 tiles) 28 split and 16 whole; 768 x 768 x 24,576
//                              at 256, 512 and 1,024 workgroups 41, 38 and 50.
constexpr int SKINNY_GROUPS = 512, SKINNY_WORK = 12, SKINNY_LONG = 4;
constexpr int BIG_TILES = 192;
constexpr int64_t WANTED = 512;
constexpr int SPLIT_BLOCKS = 8;
constexpr int64_t MAX_TILES = 1 << 22;                         // of a launch: a grid has fewer than 2^32 threads

// Tiles of a workgroup: waves and blocks of a wave, in rows of A and of B; stages; whether matrices may be 4 GiB and more
// (2,816 x 2,816 x 4,096 in tiles of 128 x 128 37.5 us, of 64 x 128 54.8, with three stages, hence one workgroup per compute unit, 43.8.)
struct Tile { int wm, wn, nj, ni, nst; bool far; };
constexpr Tile BIG = {2, 4, 4, 2, 2, false}, MID = {2, 2, 2, 2, 2, true};
constexpr int tile_m(const Tile &t) { return 32 * t.wm * t.nj; }
constexpr int tile_n(const Tile &t) { return 32 * t.wn * t.ni; }

// skinny: sixteens of rows of A that a workgroup of matmul_skinny_kernel takes, 0 for tiles
struct Plan { int skinny, big, tiles_m, tiles_n, splits, kb_per; int64_t part_ld, part_bytes; };

Plan make_plan(int64_t m, int64_t n, int64_t k, size_t room, bool far = false) {
    Plan q = {};
    const int64_t kb = (k + BLOCK - 1) / BLOCK;
    q.splits = 1; q.kb_per = (int)kb;
    const int mf = m <= 16 ? 1 : m <= 32 ? 2 : 4;
    const int64_t gm = (m + 16 * mf - 1) / (16 * mf), gn = (n + 15) / 16, rounds = (kb + SKINNY_WAVES - 1) / SKINNY_WAVES;
    if (gm * gn <= SKINNY_GROUPS ? rounds * mf <= SKINNY_WORK : m <= 16 && gn <= MAX_TILES && rounds <= SKINNY_LONG) {
        q.skinny = mf; q.tiles_m = (int)gm; q.tiles_n = (int)gn;
        return q;
    }
    const auto tiles_of = [&](const Tile &t, int64_t &tm, int64_t &tn) { tm = (m + tile_m(t) - 1) / tile_m(t); tn = (n + tile_n(t) - 1) / tile_n(t); return tm * tn; };
    int64_t tm, tn, tiles = tiles_of(BIG, tm, tn);
    q.big = tiles >= BIG_TILES && m > tile_m(MID) && n > tile_n(MID) && !far;
    if (!q.big) tiles = tiles_of(MID, tm, tn);
    q.tiles_m = (int)tm; q.tiles_n = (int)tn;
    q.part_ld = (n + 3) / 4 * 4;
    if (!q.big && tiles * 4 <= WANTED && kb >= 2 * SPLIT_BLOCKS) {
        int64_t s = WANTED / tiles;
        if (s > kb / SPLIT_BLOCKS) s = kb / SPLIT_BLOCKS;
        const int64_t one = m * q.part_ld * 4;
        if (s * one > (int64_t)room) s = (int64_t)room / one;
        if (s > 1) {
            q.kb_per = (int)((kb + s - 1) / s);
            q.splits = (int)((kb + q.kb_per - 1) / q.kb_per);
            q.part_bytes = q.splits * one;
        }
    }
    return q;
}

template <bool WIDE, int FA, int FB> void launch(const MatmulArgs &p, const Plan &q, hipStream_t st) {
    if (q.skinny) {
        const dim3 grid((unsigned)(p.tiles_m * p.tiles_n)), blk(64 * SKINNY_WAVES);
        if (q.skinny == 1) hipLaunchKernelGGL((matmul_skinny_kernel<1, WIDE, FA, FB>), grid, blk, 0, st, p);
        else if (q.skinny == 2) hipLaunchKernelGGL((matmul_skinny_kernel<2, WIDE, FA, FB>), grid, blk, 0, st, p);
        else hipLaunchKernelGGL((matmul_skinny_kernel<4, WIDE, FA, FB>), grid, blk, 0, st, p);
        return;
    }
    const dim3 grid((unsigned)((p.tiles_m * p.tiles_n * p.splits + 7) / 8 * 8));
    if (q.big) hipLaunchKernelGGL((matmul_tiles_kernel<BIG.wm, BIG.wn, BIG.nj, BIG.ni, BIG.nst, BIG.far, WIDE, FA, FB>), grid, dim3(64 * BIG.wm * BIG.wn), 0, st, p);
    else hipLaunchKernelGGL((matmul_tiles_kernel<MID.wm, MID.wn, MID.nj, MID.ni, MID.nst, MID.far, WIDE, FA, FB>), grid, dim3(64 * MID.wm * MID.wn), 0, st, p);
    if (p.part) {
        const int64_t blocks = (p.m * (p.part_ld / 4) + 255) / 256;
        hipLaunchKernelGGL(matmul_join_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st, p);
    }
}

}  // namespace

extern "C" {

size_t kge_matmul_quantized_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (m < 0 || n < 0 || k < 0 || m >= (1ll << 31) || n >= (1ll << 31) || k >= (1ll << 31)) return 0;
    if (m == 0 || n == 0) return 256;                             // (nothing to do, which has no plan)
    return (size_t)make_plan(m, n, k, ~0ull >> 1).part_bytes + 256;
}

int kge_matmul_quantized(const kge_quantized_t *a, const int32_t *rows, int64_t m, const kge_quantized_t *b, int32_t accumulate, void *out,
                         int32_t out_dtype, int64_t out_ld, void *ws, size_t ws_bytes, void *hip_stream) {
    if (kge_check_quantized(a) != KGE_OK || kge_check_quantized(b) != KGE_OK || a->cols != b->cols || m < 0 || m >= (1ll << 31) ||
        (!rows && m != 0 && m != a->rows) || ((uintptr_t)rows & 3) != 0 || (accumulate != 0 && accumulate != 1)) return KGE_E_INVALID_ARG;
    const bool wide = out_dtype != KGE_BF16;
    if (out_dtype == (KGE_BF16 | KGE_FP32_SUMS)) out_dtype = KGE_BF16;
    if (out_dtype != KGE_F32 && out_dtype != KGE_BF16) return KGE_E_INVALID_ARG;
    if (m == 0 || b->rows == 0) return KGE_OK;
    if (!out || out_ld < b->rows || out_ld >= (1ll << 31) || ((uintptr_t)out & (out_dtype == KGE_BF16 ? 1 : 3)) != 0) return KGE_E_INVALID_ARG;
    MatmulArgs p = {};
    p.a = a->codes; p.as = a->scales; p.a_ld = a->ld; p.as_ld = a->scales_ld; p.rows = rows; p.a_rows = a->rows;
    p.b = b->codes; p.bs = b->scales; p.b_ld = b->ld; p.bs_ld = b->scales_ld;
    p.m = m; p.n = b->rows; p.out = out; p.out_ld = out_ld; p.out16 = out_dtype == KGE_BF16; p.accumulate = accumulate;
    const int64_t k = a->rows > 0 ? a->cols : 0;               // (a table without rows: nothing may be read, every row of the result is zeros)
    const size_t lost = ws ? (256 - ((uintptr_t)ws & 255)) & 255 : 0;
    bool far = false;
    for (const kge_quantized_t *q : {a, b}) far = far || q->rows * q->ld >= (1ll << 32) || q->rows * q->scales_ld >= (1ll << 32);
    const Plan q = make_plan(m, p.n, k, ws && ws_bytes > lost ? ws_bytes - lost : 0, far);
    if ((int64_t)q.tiles_m * q.tiles_n > MAX_TILES) return KGE_E_UNSUPPORTED;
    p.kb = (int)((k + BLOCK - 1) / BLOCK); p.kb_per = q.kb_per; p.splits = q.splits; p.tiles_m = q.tiles_m; p.tiles_n = q.tiles_n;
    p.part_ld = q.part_ld;
    if (q.splits > 1) p.part = (float *)((char *)ws + lost);
    hipStream_t st = (hipStream_t)hip_stream;
    const bool a4 = a->format == KGE_E4M3, b4 = b->format == KGE_E4M3;
#define KGE_MQ(W)                                                                                                                        \
    (a4 ? (b4 ? launch<W, KGE_E4M3, KGE_E4M3>(p, q, st) : launch<W, KGE_E4M3, KGE_E5M2>(p, q, st))                                      \
        : (b4 ? launch<W, KGE_E5M2, KGE_E4M3>(p, q, st) : launch<W, KGE_E5M2, KGE_E5M2>(p, q, st)))
    if (wide) KGE_MQ(true);
    else KGE_MQ(false);
#undef KGE_MQ
    return kge_launch_status();
}

}  // extern "C"
