// Product of two matrices in 8-bit integers with one scale per row (quantize_rowwise.hip), both contiguous along the contraction:
//
//   out[i, j] (+)= sa[rows[i]] sb[j]  sum over k of A[rows[i], k] B[j, k]
//
// The sums are exact: 8-bit matrix instructions with 32-bit integer accumulators (k <= 131,071 keeps them below 2^31), partial sums of a split contraction too, so the
// result does not depend on tiles or splits.  The scales are applied once, as the sums leave the accumulators.
//
// What bounds it: large products the matrix pipe under the clock that operands which toggle bits leave it (16,384 x 4,096 x 4,096 243 us, 2.26 PFLOP/s; on zeros 200; 4,096 more of k 220 and 162);
// products of a few hundred tiles the trips to memory of a tile's start and end (24,576 gathered rows x 256 x 768, fp32 output: 18.0 us, of which its bytes are 9); a split contraction the
// reads from the L2 (768 x 1,024 x 24,576 in five parts: 32.4 us, of them 5 for the launch that adds the parts); one token the weights' bytes or the launch (1 x 4,096 x 1,024 3.4 us).
#include "lds_copy.hpp"
#include "text_ops.hpp"
#include <type_traits>

typedef int mi_i32x4 __attribute__((ext_vector_type(4)));
typedef int mi_i32x16 __attribute__((ext_vector_type(16)));

int kge_check_rowwise(const kge_rowwise_t *q);

namespace {

constexpr int BLOCK = 128;                                    // bytes of a row that a stage holds

struct MatmulArgs {
    const int8_t *a, *b; const float *as, *bs; int64_t a_ld, b_ld; const int32_t *rows; int64_t a_rows;
    int64_t m, n;
    void *out; int64_t out_ld; int out16, accumulate;
    int32_t *part; int64_t part_ld;                           // partial sums [split][m][part_ld] (null: one split)
    int kb, kb_per, splits, tiles_m, tiles_n;
};

// eight (bf16 output) or four (fp32 output) consecutive columns of an output row, of which n are inside
template <int C> __device__ __forceinline__ void put(const MatmulArgs &p, int64_t row, int64_t col, float (&v)[C]) {
    const int n = (int)(p.n - col < C ? p.n - col : C);
    if (n <= 0) return;
    if (p.out16) {
        uint16_t *q = (uint16_t *)p.out + row * p.out_ld + col;
        if (p.accumulate) {
#pragma unroll
            for (int e = 0; e < C; ++e)
                if (e < n) v[e] += __uint_as_float((uint32_t)q[e] << 16);
        }
        if constexpr (C == 8) kge_store8<true>(q, 0, n, v);
        else if (n == 4) {
            typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf2;
            *(kge_u32x2_a2 *)q = kge_u32x2{__builtin_bit_cast(uint32_t, bf2{(__bf16)v[0], (__bf16)v[1]}), __builtin_bit_cast(uint32_t, bf2{(__bf16)v[2], (__bf16)v[3]})};
        } else {
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (e < n) ((__bf16 *)q)[e] = (__bf16)v[e];
        }
    } else {
        float *q = (float *)p.out + row * p.out_ld + col;
        if (n == C) {
#pragma unroll
            for (int e = 0; e < C; e += 4) {
                kge_f32x4 r = {v[e], v[e + 1], v[e + 2], v[e + 3]};
                if (p.accumulate) {
                    const kge_f32x4 o = *(const kge_f32x4_a4 *)(q + e);
#pragma unroll
                    for (int u = 0; u < 4; ++u) r[u] += o[u];
                }
                *(kge_f32x4_a4 *)(q + e) = r;
            }
        } else {
#pragma unroll
            for (int e = 0; e < C - 1; ++e)
                if (e < n) q[e] = p.accumulate ? q[e] + v[e] : v[e];
        }
    }
}
// row of A of an output row, -1: a row of zeros
__device__ __forceinline__ int64_t source(const MatmulArgs &p, int64_t row) {
    if (!p.rows) return row;
    const int64_t r = p.rows[row];
    return r >= 0 && r < p.a_rows ? r : -1;
}
// four columns' scales; columns beyond the matrix take the last one's
__device__ __forceinline__ kge_f32x4 scales4(const MatmulArgs &p, int64_t col) {
    kge_f32x4 r;
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = p.bs[min(col + e, p.n - 1)];
    return r;
}

// Workgroup = WM x WN waves = TM rows of A x TN rows of B, wave = NJ x NI blocks of 32 x 32.  Stages of 128 bytes of every row pass through two places in the
// LDS, filled by asynchronous copies of whole lines.  A row's 16-byte pieces lie XOR-swizzled by (row / 2) % 8, so that the
// fragment reads of sixteen consecutive rows fall into different ones of the 64 banks.  Rows beyond the matrices are read from row 0 and not
// stored.  Which bytes a lane half contracts first does not matter as long as both operands agree.
//
// A stage is four steps of 32 bytes.  Its fragments are all in registers before its products begin: those of the next stage are read during the second half of this
// one, into the registers of the steps that are over (the last step's have two places in turn).  So a place of the LDS is read in half a stage and
// free for a stage and a half, which is what the copies from the L2 have to arrive in: with reads one step ahead it was one stage, and half of the time went by waiting
// (16,384 x 4,096 x 4,096: 268 us).  The copies are issued over half a stage, as fast as the address unit takes them.
//
// FAR: a copy's lanes have 64-bit addresses; else (codes of less than 4 GiB) a base and 32-bit offsets.
template <int WM, int WN, int NJ, int NI, int NST, int OCC, bool FAR, bool GATHERED>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(OCC, OCC)))
void matmul_tiles_kernel(const MatmulArgs p) {
    constexpr int NW = WM * WN, TM = 32 * NJ * WM, TN = 32 * NI * WN, ROWS = TM + TN, CP = ROWS / 8 / NW;      // copies of a wave per stage
    constexpr int STAGE = ROWS * BLOCK, SLOTS = NI * NJ, FRAGS = NI + NJ;
    static_assert(ROWS % (8 * NW) == 0 && NST * CP < 64 && (NST & (NST - 1)) == 0 && NST * STAGE <= 160 * 1024, "tile");
    __shared__ __attribute__((aligned(16))) char lds[NST * STAGE];
    const uint32_t lds0 = (uint32_t)(uintptr_t)lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 31, g = lane >> 5;
    // ids go round-robin to the 8 dies: a die takes a run of tiles, eight tiles of A deep, so that both operands' rows meet in its L2
    const int total = p.tiles_m * p.tiles_n * p.splits, per = (total + 7) >> 3;
    int w = ((int)blockIdx.x & 7) * per + ((int)blockIdx.x >> 3);
    if (((int)blockIdx.x >> 3) >= per || w >= total) return;
    const int split = __builtin_amdgcn_readfirstlane(w / (p.tiles_m * p.tiles_n));
    w -= split * p.tiles_m * p.tiles_n;
    const int band = w / (8 * p.tiles_n), deep = min(8, p.tiles_m - 8 * band), in = w - band * 8 * p.tiles_n;
    const int64_t m0 = (int64_t)(8 * band + in % deep) * TM, n0 = (int64_t)(in / deep) * TN;
    const int kb0 = split * p.kb_per, kb1 = min(p.kb, kb0 + p.kb_per);

    // Row r of the stage: B's tile first, then A's.  Copy j of this wave takes rows 8 (CP wave + j) .. + 7
    auto b_row = [&](int r) { const int64_t s = n0 + r; return s < p.n ? s : 0; };
    auto a_row = [&](int r) -> int64_t {
        const int64_t s = m0 + r, t = s < p.m ? (GATHERED ? source(p, s) : s) : 0;
        return t < 0 ? 0 : t;
    };
    auto swizzle = [](int r) { return (r >> 1) & 7; };
    static_assert(FAR || TN % (8 * CP) == 0, "all rows that a wave copies are of one operand");
    const bool of_b = 8 * CP * wave < TN;                                          // (not FAR)
    const uint8_t *base = (const uint8_t *)(of_b ? p.b : p.a), *gc[FAR ? CP : 1];
    uint32_t oc[FAR ? 1 : CP];
#pragma unroll
    for (int j = 0; j < CP; ++j) {
        const int r0 = 8 * (CP * wave + j), r = r0 + (lane >> 3), piece = ((lane & 7) ^ swizzle(r)) * 16;
        if constexpr (FAR) gc[j] = (const uint8_t *)(r0 < TN ? p.b + b_row(r) * p.b_ld : p.a + a_row(r - TN) * p.a_ld) + piece + (int64_t)kb0 * BLOCK;   // (a copy's rows are of one operand)
        else oc[j] = (uint32_t)(of_b ? b_row(r) * p.b_ld : a_row(r - TN) * p.a_ld) + piece;
    }
    if constexpr (!FAR) base += (int64_t)kb0 * BLOCK;
    // (the gathered row numbers have to be there before the loop: a wait of the compiler's inside it would drain the ring)
#pragma unroll
    for (int j = 0; j < CP; ++j) {
        if constexpr (FAR) asm volatile("" : "+v"(gc[j]));
        else asm volatile("" : "+v"(oc[j]));
    }
    int next = kb0;                                                               // block that the next copies fetch, and their addresses'
    auto copy = [&](int slot, int c) {
        const uint32_t to = lds0 + (uint32_t)slot * STAGE + (uint32_t)(CP * wave + c) * 1024;
        if constexpr (FAR) kge_copy16(gc[c], to);
        else kge_copy16(base, oc[c], to);
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
    mi_i32x16 acc[NI][NJ];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;

    mi_i32x4 f[4][FRAGS];                                                         // of the steps: of B, then of A
    const int swz = swizzle(lr);
    auto read = [&](int slot, int r) {                                            // fragment r of a stage in the order of the steps
        const int st = r / FRAGS, k = r % FRAGS, row = k < NI ? wn + 32 * k : TN + wm + 32 * (k - NI);
        f[st][k] = *(const mi_i32x4 *)(lds + slot * STAGE + (row + lr) * BLOCK + (((2 * st + g) ^ swz) << 4));
    };
    // products of a stage: in whose shadow the last step's fragments are read; between two copies; copies in front of the second half
    constexpr int FREE = SLOTS, GAP = SLOTS >= CP ? 2 : 1, ISSUED = SLOTS / GAP < CP ? SLOTS / GAP : CP;
    constexpr int READS = (2 * FRAGS + SLOTS - 1) / SLOTS;                        // reads behind a product
    static_assert(READS * SLOTS >= 2 * FRAGS && FREE + GAP * (CP - 1) < 4 * SLOTS, "slots");
    // What stands behind each product keeps its place (the compiler would put all reads in front of all products).
    auto stage = [&](int P) {
        const int Q = (P + 1) & (NST - 1);
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int i = 0; i < NI; ++i) {
                    const int t = st * SLOTS + j * NI + i, set = st;
                    if (t == FREE) {
                        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                        __syncthreads();                                          // everyone has this stage's fragments: its place takes the stage after the next
                    }
                    if (t == 2 * SLOTS) {
                        kge_wait_vmcnt<ISSUED + (NST - 2) * CP>();
                        __syncthreads();                                          // the next stage has landed for everyone
                    }
                    acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(f[set][i], f[set][NI + j], acc[i][j], 0, 0, 0);
                    if (t >= FREE && (t - FREE) % GAP == 0 && (t - FREE) / GAP < CP) copy(P, (t - FREE) / GAP);
#pragma unroll
                    for (int u = 0; u < READS; ++u) {
                        const int r = READS * (t % SLOTS) + u;
                        if (st == 0 && r < FRAGS) read(P, 3 * FRAGS + r);
                        if (st == 2 && r < 2 * FRAGS) read(Q, r);                 // (the fragments of steps that are over)
                        if (st == 3 && r < FRAGS) read(Q, 2 * FRAGS + r);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
        advance();
    };

    if (kb0 < kb1) {
#pragma unroll
        for (int s = 0; s < NST; ++s) {
#pragma unroll
            for (int c = 0; c < CP; ++c) copy(s, c);
            advance();
        }
        kge_wait_vmcnt<(NST - 1) * CP>();
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 3 * FRAGS; ++r) read(0, r);
        for (int kb = kb0; kb < kb1; ++kb) stage((kb - kb0) & (NST - 1));
        kge_wait_vmcnt<0>();                                                      // no copy may be in flight when the LDS is released
    }

    // Accumulator layout: lane holds row lr of A's block; element e is B's row 8 (e / 4) + 4 g + e % 4.  Stored from there a row gets eight or sixteen bytes at a
    // time; so 32 rows of the wave at a time go through the LDS, with their scales applied and rounded where nothing is added to them, and rows leave in whole
    // lines.  (Row stride one piece more than the row: writes and reads of sixteen lanes fall into different banks.)
    const int64_t col0 = n0 + wn;
    float sa[NJ];
    bool there[NJ];
    kge_f32x4 sb[NI][4];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int64_t row = m0 + wm + 32 * j + lr, from = row < p.m && !p.part ? (GATHERED ? source(p, row) : row) : -1;
        there[j] = from >= 0;
        sa[j] = from < 0 ? 0.f : p.as[from];
    }
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) sb[i][q] = scales4(p, col0 + 32 * i + 8 * q + 4 * g);
    auto scaled = [&](int i, int j, int q) {
        kge_f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = (float)acc[i][j][4 * q + e] * sa[j] * sb[i][q][e];
            if (GATHERED) v[e] = there[j] ? v[e] : 0.f;
        }
        return v;
    };
    constexpr int LD = 32 * NI + 4;                                               // in words; of 16-bit results half of it and a piece
    static_assert(NW * 32 * LD * 4 <= NST * STAGE, "the waves' rows fit the ring");
    uint32_t *mine = (uint32_t *)lds + wave * (32 * LD);
    __syncthreads();                                                              // everyone is done with the ring
    if (p.out16 && !p.part && !p.accumulate) {
        typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf2;
        constexpr int LPR = 4 * NI, RPI = 64 / LPR, LD16 = 16 * NI + 4;           // lanes per row, rows at a time
        const int c = 8 * (lane % LPR);
        const int n = (int)(p.n - col0 - c < 8 ? p.n - col0 - c : 8);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
#pragma unroll
            for (int i = 0; i < NI; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const kge_f32x4 v = scaled(i, j, q);
                    *(kge_u32x2 *)(mine + lr * LD16 + 16 * i + 4 * q + 2 * g) =
                        kge_u32x2{__builtin_bit_cast(uint32_t, bf2{(__bf16)v[0], (__bf16)v[1]}), __builtin_bit_cast(uint32_t, bf2{(__bf16)v[2], (__bf16)v[3]})};
                }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += RPI) {
                const int r = r0 + lane / LPR;
                const int64_t row = m0 + wm + 32 * j + r;
                const kge_u32x4 x = *(const kge_u32x4 *)(mine + r * LD16 + c / 2);
                if (row >= p.m || n <= 0) continue;
                uint16_t *q = (uint16_t *)p.out + row * p.out_ld + col0 + c;
                if (n == 8) *(kge_u32x4_a2 *)q = x;
                else {
#pragma unroll
                    for (int e = 0; e < 7; ++e)
                        if (e < n) q[e] = (uint16_t)(x[e >> 1] >> (16 * (e & 1)));
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        return;
    }
    constexpr int LPR = 8 * NI, RPI = 64 / LPR;
    const int c = 4 * (lane % LPR);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
#pragma unroll
        for (int i = 0; i < NI; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                mi_i32x4 x = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
                if (!p.part) x = __builtin_bit_cast(mi_i32x4, scaled(i, j, q));
                *(mi_i32x4 *)(mine + lr * LD + 32 * i + 8 * q + 4 * g) = x;
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll 4
        for (int r0 = 0; r0 < 32; r0 += RPI) {
            const int r = r0 + lane / LPR;
            const int64_t row = m0 + wm + 32 * j + r;
            const mi_i32x4 x = *(const mi_i32x4 *)(mine + r * LD + c);
            if (row >= p.m) continue;
            if (p.part) {
                if (col0 + c < p.part_ld) *(mi_i32x4 *)(p.part + ((int64_t)split * p.m + row) * p.part_ld + col0 + c) = x;
                continue;
            }
            const kge_f32x4 y = __builtin_bit_cast(kge_f32x4, x);
            float v[4] = {y[0], y[1], y[2], y[3]};
            put<4>(p, row, col0 + c, v);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Sums the splits' partial results.
__global__ __launch_bounds__(256) void matmul_join_kernel(const MatmulArgs p) {
    const int64_t per = p.part_ld / 4, total = p.m * per;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t row = i / per, col = (i - row * per) * 4;
        mi_i32x4 s = {0, 0, 0, 0};
        for (int k = 0; k < p.splits; ++k) s += *(const mi_i32x4 *)(p.part + ((int64_t)k * p.m + row) * p.part_ld + col);
        const int64_t from = source(p, row);
        const kge_f32x4 sb = scales4(p, col);
        const float sa = from < 0 ? 0.f : p.as[from];
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = from < 0 ? 0.f : (float)s[e] * sa * sb[e];
        put<4>(p, row, col, v);
    }
}

// Few rows of A (one token, a small batch), and small products of any shape: a workgroup takes sixteen rows of B against 16 MF rows of A, its eight
// waves take the blocks of 128 in turn, straight from memory into fragments, and add up through the LDS.
constexpr int SKINNY_WAVES = 8;
template <int MF> __global__ __launch_bounds__(64 * SKINNY_WAVES) void matmul_skinny_kernel(const MatmulArgs p) {
    __shared__ int32_t part[SKINNY_WAVES][MF][16][16 + 4];     // [wave][block][row of A][row of B]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 15, g = lane >> 4;
    const int64_t n0 = (int64_t)(blockIdx.x % (uint32_t)p.tiles_n) * 16, m0 = (int64_t)(blockIdx.x / (uint32_t)p.tiles_n) * (16 * MF), rb = n0 + lr < p.n ? n0 + lr : 0;
    const int8_t *gb = p.b + rb * p.b_ld + 32 * g, *ga[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) {
        const int64_t r = m0 + 16 * f + lr, s = r < p.m ? source(p, r) : 0;
        ga[f] = p.a + (s < 0 ? 0 : s) * p.a_ld + 32 * g;
    }
    mi_i32x4 acc[MF];
#pragma unroll
    for (int f = 0; f < MF; ++f) acc[f] = mi_i32x4{0, 0, 0, 0};
    for (int kb = wave; kb < p.kb; kb += SKINNY_WAVES) {
        const mi_i32x4 b0 = *(const mi_i32x4 *)(gb + (int64_t)kb * BLOCK), b1 = *(const mi_i32x4 *)(gb + (int64_t)kb * BLOCK + 16);
        mi_i32x4 a0[MF], a1[MF];
#pragma unroll
        for (int f = 0; f < MF; ++f) { a0[f] = *(const mi_i32x4 *)(ga[f] + (int64_t)kb * BLOCK); a1[f] = *(const mi_i32x4 *)(ga[f] + (int64_t)kb * BLOCK + 16); }
#pragma unroll
        for (int f = 0; f < MF; ++f) {
            acc[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b0, a0[f], acc[f], 0, 0, 0);
            acc[f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(b1, a1[f], acc[f], 0, 0, 0);
        }
    }
    // lane holds A's row lr; element e is B's row 4 g + e
#pragma unroll
    for (int f = 0; f < MF; ++f) *(mi_i32x4 *)&part[wave][f][lr][4 * g] = acc[f];
    __syncthreads();
    for (int i = tid; i < MF * 64; i += 64 * SKINNY_WAVES) {
        const int f = i >> 6, row = (i >> 2) & 15, c = (i & 3) * 4;
        mi_i32x4 s = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < SKINNY_WAVES; ++k) s += *(const mi_i32x4 *)&part[k][f][row][c];
        const int64_t r = m0 + 16 * f + row;
        if (r >= p.m) continue;
        const int64_t from = source(p, r);
        const kge_f32x4 sb = scales4(p, n0 + c);
        const float sa = from < 0 ? 0.f : p.as[from];
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = from < 0 ? 0.f : (float)s[e] * sa * sb[e];
        put<4>(p, r, n0 + c, v);
    }
}

// ---------------------------------------------------------------------------------------------
// Which kernel (bf16 output, replayed from a graph, us):
// sixteen rows of B against 16 of A per workgroup, 32 or 64 if those would be more workgroups than compute units (300 x 300 x 3,000 6.9 us with 32 and 9.8 with 64, 64 x 1,024 x 4,096 5.8 with 16 and 11.0 with 64,
//   but 64 x 4,096 x 4,096 15.3 with 16), where there are few such pairs (SKINNY_GROUPS) and each has little to do (SKINNY_WORK: blocks of k per wave times sixteens of rows):
//   64 x 4,096 x 4,096 12.5 against 15.2 in split tiles and 18.5 in whole ones, 1 x 4,096 x 16,384 16.4 / 23.1 / 54.3, 100 x 1,000 x 6,000 10.7 / 13.5 / 23.8; more work per pair loses
//   (64 x 4,096 x 8,192 21.6 / 16.8, 100 x 1,000 x 12,000 18.1 / 16.8, 1 x 1,000 x 32,768 26.8 / 19.0); and at up to 16 rows with a short k for any number of pairs (1 x 50,000 x 768 10.2 and 10.9 in tiles; 16 rows 12.6 and 11.7);
// tiles of 256 x 256 from BIG_TILES of them on: 196 52.9 and 66.2 in tiles of 128 x 128, 121 47.7 and 43.4 (3,584 and 2,816 squared x 4,096).  Eight waves of 128 x 64 each; four of 128 x 128,
//   which read a quarter less from the LDS, take k = 1,024 105 and not 91, 4,096 254 and not 243, 8,192 449 and not 445 (16,384 x 4,096);
// tiles of 128 x 256, one per compute unit, where those of 128 x 128 would be more than one: 2,200 x 2,200 x 4,096 29.7 and 33.1, 20,000 x 256 x 768 11.4 and 13.2, 8,200 x 512 x 2,048 17.7 and 19.5,
//   2,816 x 2,816 x 4,096 39.5 and 40.0; where both are at most one they lose (1,800 x 1,800 x 4,096 26.4 and 21.8, 16,000 x 256 x 768 10.9 and 9.8);
// tiles of 128 x 128 otherwise, split along k into as many workgroups as there are compute units: 768 x 1,024 x 24,576 32.4 in 5 parts, 51.5 in 2, 34.8 in 10, two per compute unit; 1,000 x 1,000 x 32,768
//   45.3 in 4, 46.5 in 8.  A split takes blocks of k off a workgroup (0.42 us each) and costs a launch (SPLIT_LAUNCH blocks) and its parts' bytes (SPLIT_MB blocks per MB): 200 x 4,096 x 4,096 20.8
//   against 18.9 whole, x 6,144 22.2 / 25.9, 300 x 256 x 4,096 11.6 / 15.3, 1,000 x 1,000 x 4,096 21.5 / 19.4.  The launch that adds the parts reads
//   them one behind the other, so of few tiles a long k has at most sqrt(1.4 k / BLOCK) parts: 100 x 300 x 65,536 24.5 in 24 or 32, 27.5 in 48, 31.8 in 64; 256 x 256 x 24,576 18.5 in 16, 20.4 in 24.
// A workgroup that has its compute unit to itself takes a ring of four stages from DEEP_BLOCKS blocks on: 1,500 x 1,500 x 16,384 53.4 against 61.1 with two, 1,000 x 1,000 x 4,096 17.3 / 19.4, 768 x 1,024 x 24,576
//   33.1 / 33.5 (a workgroup per compute unit reads 12 TB/s from the L2s by then); 100 x 1,000 x 6,000 in eight blocks each 13.7 / 13.4, 2,000 x 2,000 x 256 7.5 / 7.0.
constexpr int SKINNY_GROUPS = 512, SKINNY_WORK = 16, SKINNY_LONG = 4;
constexpr int BIG_TILES = 192;
constexpr int64_t CUS = 256;
constexpr int SPLIT_LAUNCH = 12, SPLIT_MB = 1;
constexpr int DEEP_BLOCKS = 16;
constexpr int64_t MAX_TILES = 1 << 22;                         // of a launch: a grid has fewer than 2^32 threads

// Tiles of a workgroup: waves and blocks of a wave, in rows of A and of B; waves per SIMD; whether matrices may be 4 GiB and more
struct Tile { int wm, wn, nj, ni, stages, occ; bool far; };
constexpr Tile BIG = {2, 4, 4, 2, 2, 2, false}, WIDE = {2, 4, 2, 2, 2, 2, true}, MID = {2, 2, 2, 2, 2, 2, true}, DEEP = {2, 2, 2, 2, 4, 1, true};
constexpr int tile_m(const Tile &t) { return 32 * t.wm * t.nj; }
constexpr int tile_n(const Tile &t) { return 32 * t.wn * t.ni; }

// skinny: sixteens of rows of A that a workgroup of matmul_skinny_kernel takes, 0 for tiles
enum { TILES_MID, TILES_WIDE, TILES_BIG };
struct Plan { int skinny, kind, tiles_m, tiles_n, splits, kb_per; int64_t part_ld, part_bytes; };

Plan make_plan(int64_t m, int64_t n, int64_t k, size_t room, bool far = false) {
    Plan q = {};
    const int64_t kb = (k + BLOCK - 1) / BLOCK;
    q.splits = 1; q.kb_per = (int)kb;
    const int64_t gn = (n + 15) / 16;
    int mf = 1;
    while (mf < 4 && 16 * mf < m && (m + 16 * mf - 1) / (16 * mf) * gn > CUS) mf *= 2;
    const int64_t gm = (m + 16 * mf - 1) / (16 * mf), rounds = (kb + SKINNY_WAVES - 1) / SKINNY_WAVES;
    if (gm * gn <= SKINNY_GROUPS ? rounds * mf <= SKINNY_WORK : m <= 16 && gn <= MAX_TILES && rounds <= SKINNY_LONG) {
        q.skinny = mf; q.tiles_m = (int)gm; q.tiles_n = (int)gn;
        return q;
    }
    const auto tiles_of = [&](const Tile &t, int64_t &tm, int64_t &tn) { tm = (m + tile_m(t) - 1) / tile_m(t); tn = (n + tile_n(t) - 1) / tile_n(t); return tm * tn; };
    int64_t tm, tn;
    if (tiles_of(BIG, tm, tn) >= BIG_TILES && m > tile_m(MID) && n > tile_n(MID) && !far) q.kind = TILES_BIG;
    else if (tiles_of(MID, tm, tn) > CUS && tiles_of(WIDE, tm, tn) <= CUS) q.kind = TILES_WIDE;
    const int64_t tiles = tiles_of(q.kind == TILES_BIG ? BIG : q.kind == TILES_WIDE ? WIDE : MID, tm, tn);
    q.tiles_m = (int)tm; q.tiles_n = (int)tn;
    q.part_ld = (n + 3) / 4 * 4;
    if (q.kind == TILES_MID && tiles * 2 <= CUS) {
        int64_t s = CUS / tiles;
        while (5 * s * s > 7 * kb) s--;
        const int64_t one = m * q.part_ld * 4;
        if (s * one > (int64_t)room) s = (int64_t)room / one;
        if (s > 1 && kb - kb / s > SPLIT_LAUNCH + SPLIT_MB * s * one / 1000000) {
            q.kb_per = (int)((kb + s - 1) / s);
            q.splits = (int)((kb + q.kb_per - 1) / q.kb_per);
            q.part_bytes = q.splits * one;
        }
    }
    return q;
}

void launch(const MatmulArgs &p, const Plan &q, hipStream_t st) {
    if (q.skinny) {
        const dim3 grid((unsigned)(p.tiles_m * p.tiles_n)), blk(64 * SKINNY_WAVES);
        if (q.skinny == 1) hipLaunchKernelGGL((matmul_skinny_kernel<1>), grid, blk, 0, st, p);
        else if (q.skinny == 2) hipLaunchKernelGGL((matmul_skinny_kernel<2>), grid, blk, 0, st, p);
        else hipLaunchKernelGGL((matmul_skinny_kernel<4>), grid, blk, 0, st, p);
        return;
    }
    const dim3 grid((unsigned)((p.tiles_m * p.tiles_n * p.splits + 7) / 8 * 8));
#define KGE_TILES(T, GATHERED) \
    hipLaunchKernelGGL((matmul_tiles_kernel<T.wm, T.wn, T.nj, T.ni, T.stages, T.occ, T.far, GATHERED>), grid, dim3(64 * T.wm * T.wn), 0, st, p)
    if (q.kind == TILES_BIG) { if (p.rows) KGE_TILES(BIG, true); else KGE_TILES(BIG, false); }
    else if (q.kind == TILES_WIDE) { if (p.rows) KGE_TILES(WIDE, true); else KGE_TILES(WIDE, false); }
    else if (p.tiles_m * p.tiles_n * p.splits <= CUS && p.kb_per >= DEEP_BLOCKS) { if (p.rows) KGE_TILES(DEEP, true); else KGE_TILES(DEEP, false); }
    else { if (p.rows) KGE_TILES(MID, true); else KGE_TILES(MID, false); }
#undef KGE_TILES
    if (p.part) {
        const int64_t blocks = (p.m * (p.part_ld / 4) + 255) / 256;
        hipLaunchKernelGGL(matmul_join_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st, p);
    }
}

}  // namespace

extern "C" {

size_t kge_matmul_rowwise_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (m < 0 || n < 0 || k < 0 || m >= (1ll << 31) || n >= (1ll << 31) || k >= (1ll << 31)) return 0;
    if (m == 0 || n == 0) return 256;                             // (nothing to do, which has no plan)
    return (size_t)make_plan(m, n, k, ~0ull >> 1).part_bytes + 256;
}

int kge_matmul_rowwise(const kge_rowwise_t *a, const int32_t *rows, int64_t m, const kge_rowwise_t *b, int32_t accumulate, void *out, int32_t out_dtype,
                       int64_t out_ld, void *ws, size_t ws_bytes, void *hip_stream) {
    const int ca = kge_check_rowwise(a), cb = kge_check_rowwise(b);
    if (ca == KGE_E_INVALID_ARG || cb == KGE_E_INVALID_ARG || a->cols != b->cols || m < 0 || m >= (1ll << 31) || (!rows && m != 0 && m != a->rows) ||
        ((uintptr_t)rows & 3) != 0 || (accumulate != 0 && accumulate != 1) || kge_bad_type(out_dtype)) return KGE_E_INVALID_ARG;
    if (m > 0 && b->rows > 0 && (kge_bad_rows(out, out_dtype, out_ld, b->rows) || out_ld >= KGE_MAX_LD)) return KGE_E_INVALID_ARG;
    if (ca != KGE_OK || cb != KGE_OK) return KGE_E_UNSUPPORTED;
    if (m == 0 || b->rows == 0) return KGE_OK;
    MatmulArgs p = {};
    p.a = a->codes; p.as = a->scales; p.a_ld = a->ld; p.rows = rows; p.a_rows = a->rows;
    p.b = b->codes; p.bs = b->scales; p.b_ld = b->ld;
    p.m = m; p.n = b->rows; p.out = out; p.out_ld = out_ld; p.out16 = out_dtype == KGE_BF16; p.accumulate = accumulate;
    const int64_t k = a->rows > 0 ? a->cols : 0;               // (a table without rows: nothing may be read, every row of the result is zeros)
    const size_t lost = ws ? (256 - ((uintptr_t)ws & 255)) & 255 : 0;
    bool far = false;
    for (const kge_rowwise_t *q : {a, b}) far = far || q->rows * q->ld >= (1ll << 32);
    const Plan q = make_plan(m, p.n, k, ws && ws_bytes > lost ? ws_bytes - lost : 0, far);
    if ((int64_t)q.tiles_m * q.tiles_n > MAX_TILES) return KGE_E_UNSUPPORTED;
    p.kb = (int)((k + BLOCK - 1) / BLOCK); p.kb_per = q.kb_per; p.splits = q.splits; p.tiles_m = q.tiles_m; p.tiles_n = q.tiles_n;
    p.part_ld = q.part_ld;
    if (q.splits > 1) p.part = (int32_t *)((char *)ws + lost);
    launch(p, q, (hipStream_t)hip_stream);
    return kge_launch_status();
}

}  // extern "C"
