// Gradient of the token lookup:  G[r, :] (+)= scale sum over i with ids[i] = r of D_i o g[i, :]
//
//   1. the positions are sorted by row, stable; every row gets the place of its run in the sorted list
//   2. chunks_kernel: sums of the whole chunks (32 or 8 positions) inside one run
//   3. run_rows_kernel: the rows that hold one: sums of their whole chunks, and the positions in front of and behind them; then all other rows
// A gradient row is read once and a table row written once (rows without a position as zeros, or with accumulate not at all), every sum is
// taken in an order that the sorted list alone decides, in fp32, without atomics.
//
// The sort.  Rows are cut into parts of consecutive rows, and one workgroup per part orders the part's list.  Long lists (2^rb rows a part, at
// most 1,024 parts): one launch counts the ids of each part per block of ids, one deals them out stable.  Up to COLLECT_MAX ids the part's workgroup
// (256 of them) reads all ids and collects its own, and these two launches fall away.  Short lists: that workgroup goes on to the sums of its rows,
// and the call is one launch.  Ids outside the table belong to no part and are gone from the list.
//
// What bounds it: at 131,072 positions of 1,024 bf16 columns 167 us in all, where the 431 MB of gradients and touched fp32 rows (20,900) take 97 at a copy's
// rate.  The sort's launches are 36 of them and have nothing to hide behind; the chunks run at 3.9 TB/s, the rows at 2.8 (98 us), as most rows have one
// position and are a chain each: position, gradient row, old row, store.  Short lists in one launch wait for one workgroup's sort and sums in turn
// (1,024 ids 18 us for 2.5 MB), which three launches do no sooner.
//
// The lists are those of text: a handful of rows has most positions, so no step may depend on a row's positions being few (one workgroup per row,
// one lane per digit).  Frequent rows that are neighbours, as in a vocabulary ordered by frequency, fall into one part, whose workgroup then sorts (and in one
// launch sums) most of the list: ids of the same law in order and scattered, 1,024 over 30,000 x 768 95 and 33 us, 2,048 over 50,000 x 256 75 and 22,
// 4,095 over 50,000 x 256 with dropout 37 and 28, 32,768 over 50,000 x 768 163 and 96, 131,072 over 120,000 x 1,024 283 and 171.  The rules below
// were measured on scattered ids.
//
// Rules, both sides measured (microseconds, bf16 gradient, fp32 table of 768 columns and 30,000 rows where nothing else is said; without and with
// dropout, whose bits are the work of a sum):
//   one launch      1,024 ids over 300 rows 18.4 against 23.3 in three launches, 2,048 23.8 against 23.2 (50,000 rows of 256: 21.0 and 24.8), 3,000 over
//                   300 26.2 against 25.3; with dropout 512 27.1 against 32.6, 1,024 35.5 against 32.3 (a frequent row's bits are one workgroup's)
//   collected ids   24,000 51.3 against 63.4 dealt out, 32,768 62.0 against 69.9 (where the bits of a thread's own ids end)
//   chunks of 8     9,000 34.0 against 38.2 in chunks of 32, 24,000 53.5 against 51.4, 50,000 85.7 against 73.3; with dropout 16,384 51.8 against 68.4,
//                   32,768 72.2 against 84.5, 50,000 over 300 rows 69.8 against 68.6
#include "text_ops.hpp"

namespace {

constexpr int NT = 256;
constexpr int SORT_NT = 1024, WAVES = SORT_NT / 64;
constexpr int PARTS_BITS = 10;                                // parts of a long list
static_assert(1 << PARTS_BITS <= SORT_NT, "one thread per part");
constexpr int COLLECT_PARTS = 256;                            // parts of a list that every part reads: one workgroup per compute unit
constexpr int DIGIT_BITS = 8;                                 // of a counting pass inside a part
// Most ids of a call (the rules above): whose parts collect them, of one launch, of chunks of 8; the last two without and with dropout
constexpr int64_t COLLECT_MAX = 32768, WHOLE_MAX = 2048, WHOLE_MAX_DROP = 512, SHORT_MAX = 16384, SHORT_MAX_DROP = 32768;
constexpr int MAX_BLOCKS = 256;                               // blocks of ids of a long list: every one adds up the others' counts
constexpr int CHUNK_BITS = 5, SHORT_CHUNK_BITS = 3;           // a chunk's positions in long and in short lists
// Rows of a slot, whose runs are looked up together: one where the table's rows do not fill the chip (300 rows of 1,024 columns, 5,000 ids with dropout: 28.8 us
// with two rows, 34.6 with four)
constexpr int ROWS = 4;
constexpr int64_t FEW_ROWS = 2048;                            // workgroups of one row per slot
// Of a workgroup of run_rows_kernel that joins long runs: 2^5 groups of columns, so that eight slots share a run, and eight chunks (131,072 x 1,024 with 2^4
// groups 175 us, not 167; 131,072 x 768 with dropout and four chunks 152, not 150; 5,000 x 256 with sixteen 28, not 23).
constexpr int JOIN_LP = 5, JOIN_CHUNKS = 8;
// The table's gradient goes past the caches where it would push the positions' gradient out of them (the last one holds 256 MB) before that is read, and
// only there, as what stays is what the next step reads: 131,072 ids into 30,000 x 768 101 us past and 126 through them, into 120,000 x 1,024 207 and 241; 65,536
// into 30,000 x 768 74.0 and 75.1, 32,768 into 50,000 x 768 70.9 and 67.5, 2,000 into 70,000 x 1,024 75.7 and 63.3.
constexpr int64_t STREAM_READ = 64ll << 20, STREAM_BYTES = 256ll << 20;
constexpr uint32_t EMPTY = 0xffffffffu;

struct SortArgs {
    const int32_t *ids; int64_t M, n_rows;
    uint32_t *ka, *pa, *kb, *pb;                              // (row, position) lists; what is sorted last stands in a or b
    uint32_t *counts;                                         // [blocks][parts]
    uint32_t *base;                                           // [parts + 1] first place of each part's list; the last one: ids in all
    uint32_t *first, *last;                                   // [n_rows] run of each row: places [first, last), first = EMPTY for none
    int64_t part_rows;                                        // of each part; 2^rb where ids are dealt out
    int parts, rb, blocks; int64_t per_block;                 // rb: bits of the numbers below part_rows
};

__device__ __forceinline__ bool in_table(const SortArgs &a, int32_t id) { return (uint32_t)id < (uint64_t)a.n_rows; }

__global__ __launch_bounds__(SORT_NT) void count_kernel(const SortArgs a) {
    __shared__ uint32_t cnt[1 << PARTS_BITS];
    if (threadIdx.x < 1 << PARTS_BITS) cnt[threadIdx.x] = 0;
    __syncthreads();
    const int64_t lo = (int64_t)blockIdx.x * a.per_block, hi = lo + a.per_block < a.M ? lo + a.per_block : a.M;
    for (int64_t i = lo + threadIdx.x; i < hi; i += SORT_NT) {
        const int32_t id = a.ids[i];
        if (in_table(a, id)) atomicAdd(&cnt[(uint32_t)id >> a.rb], 1u);
    }
    __syncthreads();
    if ((int)threadIdx.x < a.parts) a.counts[(int64_t)blockIdx.x * a.parts + threadIdx.x] = cnt[threadIdx.x];
}

// exclusive scan of one value per thread over the workgroup, in thread order
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t *sums, uint32_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t t = (uint32_t)__shfl_up((int)s, o);
        if (lane >= o) s += t;
    }
    if (lane == 63) sums[wave] = s;
    __syncthreads();
    uint32_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { const uint32_t t = sums[w]; before += w < wave ? t : 0u; total += t; }
    __syncthreads();
    return before + s - v;
}

// Lanes whose digit equals this lane's (of the lanes with `valid`).  The lists that take longest are those of a frequent row: nearly all digits are alike, so
// the first two digits that occur are looked for by themselves, and the bits of all only where there are more (eight bits are a hundred instructions).
__device__ __forceinline__ uint64_t peers_of(uint32_t digit, int bits, bool valid) {
    const uint64_t all = __ballot(valid);
    uint64_t left = all, p = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (!left) return p;
        const uint32_t one = (uint32_t)__builtin_amdgcn_readlane((int)digit, __builtin_ctzll(left));
        const uint64_t m = __ballot(valid && digit == one);
        if (digit == one) p = m;
        left &= ~m;
    }
    if (!left) return p;
    p = all;
    for (int b = 0; b < bits; ++b) {
        const uint64_t m = __ballot(valid && (digit >> b & 1u));
        p &= digit >> b & 1u ? m : ~m;
    }
    return p;
}

// Deals a block's ids out to the parts' lists.  A wave owns a run of the block's ids: the waves' counts per part give every wave its places, in which
// it then moves on by itself, 64 ids at a time.
__global__ __launch_bounds__(SORT_NT) void deal_kernel(const SortArgs a) {
    __shared__ uint32_t place[WAVES][1 << PARTS_BITS];
    __shared__ uint32_t sums[WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, p = threadIdx.x;
    uint32_t before = 0, all = 0, total;
    if (p < a.parts) {
        int b = 0;
        for (; b + 8 <= a.blocks; b += 8) {
            uint32_t c[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) c[u] = a.counts[(int64_t)(b + u) * a.parts + p];
#pragma unroll
            for (int u = 0; u < 8; ++u) { before += b + u < (int)blockIdx.x ? c[u] : 0u; all += c[u]; }
        }
        for (; b < a.blocks; ++b) {
            const uint32_t c = a.counts[(int64_t)b * a.parts + p];
            before += b < (int)blockIdx.x ? c : 0u; all += c;
        }
    }
    const uint32_t base = block_scan(all, sums, total);
    if (blockIdx.x == 0) {
        if (p < a.parts) a.base[p] = base;
        if (p == 0) a.base[a.parts] = total;
    }
    const bool counter = p < 1 << PARTS_BITS;                 // threads that have a column of the table of places
    if (counter)
        for (int w = 0; w < WAVES; ++w) place[w][p] = 0;
    __syncthreads();
    const int64_t lo = (int64_t)blockIdx.x * a.per_block, hi = lo + a.per_block < a.M ? lo + a.per_block : a.M;
    const int64_t each = (a.per_block / WAVES + 63) / 64 * 64, w0 = lo + wave * each, w1 = w0 + each < hi ? w0 + each : hi;
    for (int64_t i = w0 + lane; i < w1; i += 64) {
        const int32_t id = a.ids[i];
        if (in_table(a, id)) atomicAdd(&place[wave][(uint32_t)id >> a.rb], 1u);
    }
    __syncthreads();
    if (counter) {
        uint32_t run = base + before;
        for (int w = 0; w < WAVES; ++w) { const uint32_t c = place[w][p]; place[w][p] = run; run += c; }
    }
    __syncthreads();
    volatile uint32_t *mine = place[wave];                    // (one wave's own: its accesses stay in order)
    for (int64_t i0 = w0; i0 < w1; i0 += 64) {
        const int64_t i = i0 + lane;
        const int32_t id = i < w1 ? a.ids[i] : -1;
        const bool valid = in_table(a, id);
        const uint32_t d = (uint32_t)id >> a.rb;
        const uint64_t peers = peers_of(d, PARTS_BITS, valid);
        const int rank = __popcll(peers & ((1ull << lane) - 1ull));
        const uint32_t at = valid ? mine[d] : 0u;
        __builtin_amdgcn_wave_barrier();
        if (valid) {
            a.ka[at + rank] = (uint32_t)id; a.pa[at + rank] = (uint32_t)i;
            if (rank == 0) mine[d] = at + (uint32_t)__popcll(peers);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// Orders the list of the workgroup's part by row, eight bits at a time, and notes the rows' runs.
struct PartLds { uint32_t place[WAVES][1 << DIGIT_BITS]; uint32_t sums[WAVES]; uint32_t found[COLLECT_MAX / (4 * SORT_NT)][WAVES]; };
template <bool COLLECT>
__device__ __forceinline__ void sort_part(const SortArgs &a, PartLds &l) {
    auto &place = l.place;
    uint32_t *sums = l.sums;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t part = blockIdx.x;
    const int64_t row0 = (int64_t)part * a.part_rows, rows = min(a.part_rows, a.n_rows - row0);
    const uint32_t r0 = (uint32_t)row0;
    uint32_t base, n;
    if constexpr (COLLECT) {
        // ids four at a time: element e of thread t in round r is position (r SORT_NT + t) 4 + e
        uint32_t own = 0, lower = 0;                          // own: four bits a round
        const int rounds = (int)((a.M + 4 * SORT_NT - 1) / (4 * SORT_NT));
        for (int r = 0; r < rounds; ++r) {
            const int64_t i = ((int64_t)r * SORT_NT + tid) * 4;
            uint32_t c = 0;
            int32_t four[4];
            if (i + 4 <= a.M) __builtin_memcpy(four, a.ids + i, 16);
            else
#pragma unroll
                for (int e = 0; e < 4; ++e) four[e] = i + e < a.M ? a.ids[i + e] : -1;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t id = (uint32_t)four[e];        // (a negative id is one past every table)
                const bool mine = id - r0 < (uint32_t)rows;
                own |= (mine ? 1u : 0u) << (4 * r + e);
                lower += id < r0 ? 1u : 0u;
                c += (uint32_t)__popcll(__ballot(mine));
            }
            if (lane == 0) l.found[r][wave] = c;
        }
        uint32_t total;
        block_scan(lower, sums, total);                       // (its barriers also publish found)
        base = total;
        uint32_t at = base;
        n = 0;
        for (int r = 0; r < rounds; ++r) {
            uint32_t before = 0, here = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) { const uint32_t t = l.found[r][w]; before += w < wave ? t : 0u; here += t; }
            uint32_t k = at + before;
#pragma unroll
            for (int e = 0; e < 4; ++e) k += (uint32_t)__popcll(__ballot(own >> (4 * r + e) & 1u) & ((1ull << lane) - 1ull));
            const int64_t i = ((int64_t)r * SORT_NT + tid) * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (own >> (4 * r + e) & 1u) { a.ka[k] = (uint32_t)a.ids[i + e]; a.pa[k] = (uint32_t)(i + e); ++k; }
            at += here; n += here;
        }
        if (tid == 0 && part == (uint32_t)a.parts - 1) a.base[a.parts] = base + n;
        __syncthreads();
    } else {
        base = a.base[part];
        n = a.base[part + 1] - base;
    }
    uint32_t *ki = a.ka + base, *pi = a.pa + base, *ko = a.kb + base, *po = a.pb + base;
    const uint32_t each = ((n + WAVES - 1) / WAVES + 63) / 64 * 64, w0 = min(n, wave * each), w1 = min(n, w0 + each);
    for (int shift = 0; shift < a.rb; shift += DIGIT_BITS) {
        const int bits = min(DIGIT_BITS, a.rb - shift);
        const uint32_t mask = (1u << bits) - 1u;
        for (int k = tid; k < WAVES << DIGIT_BITS; k += SORT_NT) (&place[0][0])[k] = 0;
        __syncthreads();
        // (one addition per row and 64 ids: lanes that add to one word take turns)
        constexpr int AHEAD = 4;                              // rounds whose loads are in flight (parts of 131,072 ids: 4 21.3 us, 8 21.9, 16 25.3)
        for (uint32_t i0 = w0; i0 < w1; i0 += 64 * AHEAD) {
            uint32_t key[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) key[u] = ki[min(i0 + 64 * u + lane, w1 - 1)];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (i0 + 64 * u >= w1) break;
                const bool valid = i0 + 64 * u + lane < w1;
                const uint32_t d = (key[u] - r0) >> shift & mask;
                const uint64_t peers = peers_of(d, bits, valid);
                if (valid && __popcll(peers & ((1ull << lane) - 1ull)) == 0) atomicAdd(&place[wave][d], (uint32_t)__popcll(peers));
            }
        }
        __syncthreads();
        uint32_t c = 0, total;
        if (tid < 1 << DIGIT_BITS)
            for (int w = 0; w < WAVES; ++w) c += place[w][tid];
        uint32_t run = block_scan(c, sums, total);
        if (tid < 1 << DIGIT_BITS) {
            if (a.rb <= DIGIT_BITS && tid < rows) {           // one pass: its counts are the runs
                a.first[row0 + tid] = c ? base + run : EMPTY;
                a.last[row0 + tid] = base + run + c;
            }
            for (int w = 0; w < WAVES; ++w) { const uint32_t t = place[w][tid]; place[w][tid] = run; run += t; }
        }
        __syncthreads();
        volatile uint32_t *mine = place[wave];
        for (uint32_t i0 = w0; i0 < w1; i0 += 64 * AHEAD) {
            uint32_t key[AHEAD], pos[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const uint32_t i = min(i0 + 64 * u + lane, w1 - 1);
                key[u] = ki[i]; pos[u] = pi[i];
            }
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (i0 + 64 * u >= w1) break;
                const bool valid = i0 + 64 * u + lane < w1;
                const uint32_t d = (key[u] - r0) >> shift & mask;
                const uint64_t peers = peers_of(d, bits, valid);
                const int rank = __popcll(peers & ((1ull << lane) - 1ull));
                const uint32_t at = mine[d];
                __builtin_amdgcn_wave_barrier();
                if (valid) {
                    ko[at + rank] = key[u]; po[at + rank] = pos[u];
                    if (rank == 0) mine[d] = at + (uint32_t)__popcll(peers);
                }
                __builtin_amdgcn_wave_barrier();
            }
        }
        __syncthreads();
        uint32_t *t = ki; ki = ko; ko = t;
        t = pi; pi = po; po = t;
    }
    if (a.rb > 0 && a.rb <= DIGIT_BITS) return;
    if (a.rb == 0) {                                          // a part is a row
        if (tid == 0) { a.first[row0] = n ? base : EMPTY; a.last[row0] = base + n; }
        return;
    }
    for (int64_t r = tid; r < rows; r += SORT_NT) a.first[row0 + r] = EMPTY;
    __syncthreads();
    for (uint32_t i = tid; i < n; i += SORT_NT) {
        const uint32_t key = ki[i];
        if (i == 0 || ki[i - 1] != key) a.first[key] = base + i;
        if (i == n - 1 || ki[i + 1] != key) a.last[key] = base + i + 1;
    }
}

template <bool COLLECT>
__global__ __launch_bounds__(SORT_NT) void parts_kernel(const SortArgs a) {
    __shared__ PartLds l;
    sort_part<COLLECT>(a, l);
}

// ---------------------------------------------------------------------------------------------
struct SumArgs {
    const uint32_t *sk, *sp, *count;         // sorted rows and positions, their number
    const uint32_t *first, *last;
    float *part;                             // [M >> lc][8 cg] sums of whole chunks of 2^lc positions
    int lc;
    const void *g; int64_t g_ld; int64_t M;
    void *out; int64_t out_ld; int64_t n_rows;
    int dim, cg, accumulate, stream; float scale; KgeDropDev drop;         // stream: the table's rows are stored past the caches
    int64_t chunk_items, row_items;          // chunks; workgroups for the short rows
    int rows;                                // of a slot among the short rows
    int lp, join_lp;                         // 2^lp threads take the groups of a row; of a long run's, 2^join_lp
};

// s += D_i o g[i, group] of the positions sp[0 .. n), in order, 8 (fp32: 4) rows in flight
template <bool G16> __device__ __forceinline__ void add_rows(const SumArgs &a, uint32_t step, const uint32_t *sp, int n, int grp, float (&s)[8]) {
    constexpr int B = G16 ? 8 : 4;
    const int cols = a.dim - 8 * grp;
    const int64_t esz = G16 ? 2 : 4;
    auto add = [&](float (&v)[8], uint32_t p) {
        if (a.drop.thr) kge_drop8(a.drop, step, p, (uint32_t)grp, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += v[e];
    };
    if (cols < 8) {                                            // the row's last columns
        for (int k = 0; k < n; ++k) {
            float v[8];
            kge_load8<G16>((const char *)a.g + (int64_t)sp[k] * a.g_ld * esz, 8 * grp, cols, v);
            add(v, sp[k]);
        }
        return;
    }
    for (int k = 0; k < n; k += B) {
        uint32_t p[B];
        KgeRaw8<G16> raw[B];
#pragma unroll
        for (int u = 0; u < B; ++u) p[u] = sp[min(k + u, n - 1)];          // (past the end: the last one again, from the cache, not added)
#pragma unroll
        for (int u = 0; u < B; ++u) raw[u] = kge_raw8<G16>((const char *)a.g + (int64_t)p[u] * a.g_ld * esz, 8 * grp);
#pragma unroll
        for (int u = 0; u < B; ++u)
            if (k + u < n) {
                float v[8];
                kge_values8<G16>(raw[u], v);
                add(v, p[u]);
            }
    }
}

template <bool OUT16> __device__ __forceinline__ void finish(const SumArgs &a, int64_t row, int grp, float (&s)[8]) {
    char *orow = (char *)a.out + row * a.out_ld * (OUT16 ? 2 : 4);
    const int n = a.dim - 8 * grp;
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] *= a.scale;
    if (a.accumulate) {
        float o[8];
        kge_load8<OUT16>(orow, 8 * grp, n, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] += o[e];
    }
    if (a.stream) kge_store8<OUT16, true>(orow, 8 * grp, n, s);
    else kge_store8<OUT16>(orow, 8 * grp, n, s);
}

// A row of zeros, sixteen bytes per lane side by side (the groups' own stores leave every other sixteen bytes of an fp32 line to a second one)
template <bool OUT16> __device__ __forceinline__ void zero_row(const SumArgs &a, int64_t row, int lane, int lanes) {
    char *orow = (char *)a.out + row * a.out_ld * (OUT16 ? 2 : 4);
    const int whole = a.dim * (OUT16 ? 2 : 4) / 16;
    const kge_u32x4 z = {0u, 0u, 0u, 0u};
    if (a.stream)
        for (int k = lane; k < whole; k += lanes) __builtin_nontemporal_store(z, (kge_u32x4_a2 *)(orow + 16 * k));
    else
        for (int k = lane; k < whole; k += lanes) *(kge_u32x4_a2 *)(orow + 16 * k) = z;
    if (lane == 0)
        for (int c = whole * (OUT16 ? 8 : 4); c < a.dim; ++c) {
            if constexpr (OUT16) ((uint16_t *)orow)[c] = 0;
            else ((float *)orow)[c] = 0.f;
        }
}

__device__ __forceinline__ bool holds_chunk(uint32_t k0, uint32_t k1, int lc) { return (((k0 + (1u << lc) - 1) >> lc) + 1) << lc <= k1; }

// The workgroup's slots (THREADS / 2^lp groups of threads, lp <= 6) add up their parts of a sum, through the LDS, in slot order; slot 0 has the sum.
template <int THREADS> __device__ __forceinline__ void join_slots(float (*red)[8], int lp, float (&s)[8]) {
    __syncthreads();
    *(kge_f32x4 *)red[threadIdx.x] = kge_f32x4{s[0], s[1], s[2], s[3]};
    *(kge_f32x4 *)(red[threadIdx.x] + 4) = kge_f32x4{s[4], s[5], s[6], s[7]};
    __syncthreads();
    if ((int)threadIdx.x < 1 << lp)
        for (int t = threadIdx.x + (1 << lp); t < THREADS; t += 1 << lp)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] += red[t][e];
}

// Short lists: the part's workgroup sorts and adds up.  A slot takes the rows with a FEW positions, ROWS of them at a time; the others are
// shared by all slots one after the other.
constexpr int FEW = 16;
template <bool G16, bool OUT16>
__global__ __launch_bounds__(SORT_NT) void whole_kernel(const SortArgs so, const SumArgs a) {
    __shared__ union { PartLds sort; float red[SORT_NT][8]; } l;
    __shared__ uint32_t many[WHOLE_MAX / FEW][3], n_many;
    if (threadIdx.x == 0) n_many = 0;
    sort_part<true>(so, l.sort);
    __syncthreads();
    const uint32_t step = a.drop.thr ? kge_drop_step(a.drop) : 0u;
    const int per = 1 << a.lp, sub = threadIdx.x >> a.lp, subs = SORT_NT >> a.lp, grp0 = threadIdx.x & (per - 1);
    const int64_t first_row = (int64_t)blockIdx.x * so.part_rows, end = min(first_row + so.part_rows, a.n_rows);
    for (int64_t row0 = first_row + sub * ROWS; row0 < end; row0 += subs * ROWS) {
        uint32_t k0[ROWS], k1[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const bool in = row0 + r < end;
            k0[r] = in ? a.first[row0 + r] : EMPTY; k1[r] = in ? a.last[row0 + r] : EMPTY;
        }
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (row0 + r >= end) break;
            if (k0[r] == EMPTY) {
                if (!a.accumulate) zero_row<OUT16>(a, row0 + r, grp0, per);
                continue;
            }
            if (k1[r] - k0[r] > FEW) {
                if (grp0 == 0) {
                    const uint32_t f = atomicAdd(&n_many, 1u);
                    many[f][0] = (uint32_t)(row0 + r); many[f][1] = k0[r]; many[f][2] = k1[r];
                }
                continue;
            }
            for (int grp = grp0; grp < a.cg; grp += per) {
                float s[8] = {};
                add_rows<G16>(a, step, a.sp + k0[r], (int)(k1[r] - k0[r]), grp, s);
                finish<OUT16>(a, row0 + r, grp, s);
            }
        }
    }
    __syncthreads();
    const uint32_t n = n_many;
    for (uint32_t f = 0; f < n; ++f) {
        const uint32_t row = many[f][0], b0 = many[f][1], len = many[f][2] - b0, each = (len + subs - 1) / subs, lo = min(len, sub * each),
                       hi = min(len, lo + each);
        for (int g0 = 0; g0 < a.cg; g0 += per) {
            const int grp = g0 + grp0;
            float s[8] = {};
            if (grp < a.cg) add_rows<G16>(a, step, a.sp + b0 + lo, (int)(hi - lo), grp, s);
            join_slots<SORT_NT>(l.red, a.lp, s);
            if (sub == 0 && grp < a.cg) finish<OUT16>(a, row, grp, s);
        }
    }
}

// A chunk per workgroup, if it lies inside one run: the slots take its positions in turn.
template <bool G16>
__global__ __launch_bounds__(NT) void chunks_kernel(const SumArgs a) {
    __shared__ float red[NT][8];
    const uint32_t step = a.drop.thr ? kge_drop_step(a.drop) : 0u;
    const int per = 1 << a.lp, sub = threadIdx.x >> a.lp, subs = NT >> a.lp, grp0 = threadIdx.x & (per - 1);
    for (int64_t w = blockIdx.x; w < a.chunk_items; w += gridDim.x) {
        const int chunk = 1 << a.lc;
        const int64_t c0 = w << a.lc;
        if (c0 + chunk > *a.count || a.sk[c0] != a.sk[c0 + chunk - 1]) continue;      // (equal ends, equal chunk)
        const int each = chunk / min(subs, chunk);
        for (int g0 = 0; g0 < a.cg; g0 += per) {
            const int grp = g0 + grp0;
            float s[8] = {};
            if (grp < a.cg && sub * each < chunk) add_rows<G16>(a, step, a.sp + c0 + sub * each, each, grp, s);
            join_slots<NT>(red, a.lp, s);
            if (sub == 0 && grp < a.cg) {
                float *p = a.part + (w * a.cg + grp) * 8;
                *(kge_f32x4 *)p = kge_f32x4{s[0], s[1], s[2], s[3]};
                *(kge_f32x4 *)(p + 4) = kge_f32x4{s[4], s[5], s[6], s[7]};
            }
        }
    }
}

// a.rows rows per slot: rows without a position, and those whose runs hold no whole chunk
template <bool G16, bool OUT16> __device__ __forceinline__ void short_rows(const SumArgs &a, uint32_t step, int64_t item) {
    const int per = 1 << a.lp, sub = threadIdx.x >> a.lp, subs = NT >> a.lp, grp0 = threadIdx.x & (per - 1);
    const int64_t row0 = (item * subs + sub) * a.rows;
    uint32_t k0[ROWS], k1[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const bool in = r < a.rows && row0 + r < a.n_rows && a.M;
        k0[r] = in ? a.first[row0 + r] : EMPTY; k1[r] = in ? a.last[row0 + r] : EMPTY;
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (r >= a.rows || row0 + r >= a.n_rows) break;
        if (k0[r] == EMPTY) {
            if (!a.accumulate) zero_row<OUT16>(a, row0 + r, grp0, per);
            continue;
        }
        if (holds_chunk(k0[r], k1[r], a.lc)) continue;
        for (int grp = grp0; grp < a.cg; grp += per) {
            float s[8] = {};
            add_rows<G16>(a, step, a.sp + k0[r], (int)(k1[r] - k0[r]), grp, s);
            finish<OUT16>(a, row0 + r, grp, s);
        }
    }
}

// The rows: first the long runs, one workgroup per JOIN_CHUNKS chunks and 2^join_lp groups of columns: of the chunks that are a run's first whole one, it adds
// up the run.  Behind them, so that their chains of loads are covered, the short rows.
template <bool G16, bool OUT16>
__global__ __launch_bounds__(NT) void run_rows_kernel(const SumArgs a) {
    __shared__ float red[NT][8];
    __shared__ uint32_t found[JOIN_CHUNKS][3];
    const uint32_t step = a.drop.thr ? kge_drop_step(a.drop) : 0u;
    const int per = 1 << a.join_lp, sub = threadIdx.x >> a.join_lp, subs = NT >> a.join_lp, slices = (a.cg + per - 1) >> a.join_lp;
    const int64_t joins = (a.chunk_items + JOIN_CHUNKS - 1) / JOIN_CHUNKS * slices;
    for (int64_t w = blockIdx.x; w < joins + a.row_items; w += gridDim.x) {
        if (w >= joins) {
            short_rows<G16, OUT16>(a, step, w - joins);
            continue;
        }
        const int64_t tile = w / slices;
        bool owner = false;
        uint32_t row = 0, k0 = 0, k1 = 0;
        if (threadIdx.x < JOIN_CHUNKS) {
            const int64_t c = tile * JOIN_CHUNKS + threadIdx.x, c0 = c << a.lc;
            const int chunk = 1 << a.lc;
            if (c < a.chunk_items && c0 + chunk <= *a.count) {
                row = a.sk[c0];
                if (row == a.sk[c0 + chunk - 1]) { k0 = a.first[row]; k1 = a.last[row]; owner = (k0 + chunk - 1) >> a.lc == c; }
            }
            found[threadIdx.x][0] = owner ? row : EMPTY; found[threadIdx.x][1] = k0; found[threadIdx.x][2] = k1;
        }
        if (!__syncthreads_or(owner)) continue;
        const int grp = (int)(w - tile * slices) * per + (threadIdx.x & (per - 1));
        for (int f = 0; f < JOIN_CHUNKS; ++f) {
            const uint32_t r = found[f][0];
            if (r == EMPTY) continue;
            const uint32_t b0 = found[f][1], b1 = found[f][2], e0 = (b0 + (1u << a.lc) - 1) >> a.lc, e1 = b1 >> a.lc;
            float s[8] = {};
            if (grp < a.cg) {
                // slot by slot: a share of the positions in front, of the chunks, of the positions behind
                auto share = [&](uint32_t n, uint32_t &lo) { const uint32_t x = (n + subs - 1) / subs; lo = min(n, sub * x); return min(n, lo + x) - lo; };
                uint32_t lo, n = share((e0 << a.lc) - b0, lo);
                add_rows<G16>(a, step, a.sp + b0 + lo, (int)n, grp, s);
                n = share(e1 - e0, lo);
                const float *p = a.part + ((int64_t)(e0 + lo) * a.cg + grp) * 8;
                for (uint32_t k = 0; k < n; k += 8) {
                    kge_f32x4 x[8][2];
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const float *q = p + (int64_t)min(k + u, n - 1) * a.cg * 8;
                        x[u][0] = *(const kge_f32x4 *)q; x[u][1] = *(const kge_f32x4 *)(q + 4);
                    }
#pragma unroll
                    for (int u = 0; u < 8; ++u)
                        if (k + u < n) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) { s[e] += x[u][0][e]; s[4 + e] += x[u][1][e]; }
                        }
                }
                n = share(b1 - (e1 << a.lc), lo);
                add_rows<G16>(a, step, a.sp + (e1 << a.lc) + lo, (int)n, grp, s);
            }
            join_slots<NT>(red, a.join_lp, s);
            if (sub == 0 && grp < a.cg) finish<OUT16>(a, r, grp, s);
        }
        __syncthreads();                                       // (found is written again)
    }
}

struct Ws { SortArgs s; float *part; int lc; };
int bits_of(int64_t n) {                     // of the numbers below n
    int b = 0;
    while ((1ll << b) < n) ++b;
    return b;
}
size_t carve(int64_t M, int64_t n_rows, int dim, bool drop, void *ws, Ws &w) {
    char *p = (char *)ws;
    size_t off = 0;
    auto take = [&](size_t bytes) { void *q = p ? p + off : nullptr; off += (bytes + 255) / 256 * 256; return (uint32_t *)q; };
    SortArgs &s = w.s;
    s.M = M; s.n_rows = n_rows;
    if (M <= COLLECT_MAX) {
        s.part_rows = (n_rows + COLLECT_PARTS - 1) / COLLECT_PARTS;
        if (s.part_rows < 1) s.part_rows = 1;
        s.rb = bits_of(s.part_rows);
    } else {
        const int bits = bits_of(n_rows);
        s.rb = bits > PARTS_BITS ? bits - PARTS_BITS : 0;
        s.part_rows = 1ll << s.rb;
    }
    s.parts = (int)((n_rows + s.part_rows - 1) / s.part_rows);
    // blocks of 2,048 ids (32 rounds of a wave), larger ones beyond 256 of them
    s.per_block = 2048;
    while (s.per_block * MAX_BLOCKS < M) s.per_block *= 2;
    s.blocks = (int)((M + s.per_block - 1) / s.per_block);
    s.ka = take((size_t)M * 4); s.pa = take((size_t)M * 4); s.kb = take((size_t)M * 4); s.pb = take((size_t)M * 4);
    s.counts = take((size_t)MAX_BLOCKS * (4u << PARTS_BITS));
    s.base = take((4u << PARTS_BITS) + 4);
    s.first = take((size_t)n_rows * 4); s.last = take((size_t)n_rows * 4);
    w.lc = M <= (drop ? SHORT_MAX_DROP : SHORT_MAX) ? SHORT_CHUNK_BITS : CHUNK_BITS;
    // (room for the shorter chunks wherever a dropout asks for them, so that a longer list never needs less)
    const int64_t shorts = (M < SHORT_MAX_DROP ? M : SHORT_MAX_DROP) >> SHORT_CHUNK_BITS, longs = M >> CHUNK_BITS;
    const int64_t chunks = shorts > longs ? shorts : longs;
    w.part = (float *)take((size_t)chunks * ((dim + 7) / 8) * 32);
    return off;
}

}  // namespace

extern "C" {

size_t kge_embed_bwd_workspace_bytes(int64_t M, int64_t n_rows, int32_t dim) {
    if (M < 0 || M > KGE_MAX_ROWS || n_rows < 0 || n_rows > KGE_MAX_ROWS || dim < 1 || dim > KGE_MAX_DIM) return 0;
    Ws w;
    return carve(M, n_rows, dim, false, nullptr, w) + 256;
}

int kge_embed_bwd(const void *g, int32_t g_dtype, int64_t g_ld, const int32_t *ids, int64_t M, float scale, const kge_dropout_t *drop,
                  void *g_table, int32_t table_dtype, int64_t n_rows, int32_t dim, int64_t ld, int32_t accumulate, void *ws, size_t ws_bytes,
                  void *hip_stream) {
    SumArgs a = {};
    const int rc = kge_drop_dev(drop, &a.drop);
    if (rc != KGE_OK) return rc;
    if (kge_bad_type(g_dtype) || kge_bad_type(table_dtype) || dim < 1 || dim > KGE_MAX_DIM || n_rows < 0 || n_rows > KGE_MAX_ROWS || M < 0 ||
        M > KGE_MAX_ROWS || g_ld >= KGE_MAX_LD || ld >= KGE_MAX_LD || (accumulate != 0 && accumulate != 1)) return KGE_E_INVALID_ARG;
    if (n_rows == 0 || (M == 0 && accumulate)) return KGE_OK;
    if (kge_bad_rows(g_table, table_dtype, ld, dim) || (M > 0 && (!ids || ((uintptr_t)ids & 3) != 0 || kge_bad_rows(g, g_dtype, g_ld, dim))))
        return KGE_E_INVALID_ARG;
    if (!ws) return KGE_E_WORKSPACE_TOO_SMALL;
    const size_t lost = (256 - ((uintptr_t)ws & 255)) & 255;
    Ws w = {};
    if (carve(M, n_rows, dim, a.drop.thr != 0, nullptr, w) + lost > ws_bytes) return KGE_E_WORKSPACE_TOO_SMALL;
    carve(M, n_rows, dim, a.drop.thr != 0, (char *)ws + lost, w);
    hipStream_t st = (hipStream_t)hip_stream;
    SortArgs &s = w.s;
    s.ids = ids;
    const bool odd = ((s.rb + DIGIT_BITS - 1) / DIGIT_BITS & 1) != 0;
    a.sk = odd ? s.kb : s.ka; a.sp = odd ? s.pb : s.pa; a.count = s.base + s.parts; a.first = s.first; a.last = s.last; a.part = w.part; a.lc = w.lc;
    a.g = g; a.g_ld = g_ld; a.M = M; a.out = g_table; a.out_ld = ld; a.n_rows = n_rows; a.dim = dim; a.cg = (dim + 7) / 8;
    a.accumulate = accumulate; a.scale = scale;
    const int64_t read = M * dim * (g_dtype == KGE_BF16 ? 2 : 4), written = n_rows * dim * (table_dtype == KGE_BF16 ? 2 : 4);
    a.stream = !accumulate && read >= STREAM_READ && read + written >= STREAM_BYTES;
    a.lp = bits_of(a.cg);
    if (a.lp > 6) a.lp = 6;
    const bool g16 = g_dtype == KGE_BF16, o16 = table_dtype == KGE_BF16;
    if (M > 0 && M <= (a.drop.thr ? WHOLE_MAX_DROP : WHOLE_MAX)) {
        const dim3 grid((unsigned)s.parts);
        if (g16 && o16) hipLaunchKernelGGL((whole_kernel<true, true>), grid, dim3(SORT_NT), 0, st, s, a);
        else if (g16) hipLaunchKernelGGL((whole_kernel<true, false>), grid, dim3(SORT_NT), 0, st, s, a);
        else if (o16) hipLaunchKernelGGL((whole_kernel<false, true>), grid, dim3(SORT_NT), 0, st, s, a);
        else hipLaunchKernelGGL((whole_kernel<false, false>), grid, dim3(SORT_NT), 0, st, s, a);
        return kge_launch_status();
    }
    if (M > COLLECT_MAX) {
        hipLaunchKernelGGL(count_kernel, dim3(s.blocks), dim3(SORT_NT), 0, st, s);
        hipLaunchKernelGGL(deal_kernel, dim3(s.blocks), dim3(SORT_NT), 0, st, s);
        hipLaunchKernelGGL(parts_kernel<false>, dim3(s.parts), dim3(SORT_NT), 0, st, s);
    } else if (M > 0) hipLaunchKernelGGL(parts_kernel<true>, dim3(s.parts), dim3(SORT_NT), 0, st, s);
    const int slots = NT >> a.lp;
    a.join_lp = a.lp < JOIN_LP ? a.lp : JOIN_LP;               // (many slots, few columns each)
    a.chunk_items = M >> a.lc;
    a.rows = n_rows <= FEW_ROWS * slots ? 1 : ROWS;
    a.row_items = (n_rows + slots * a.rows - 1) / (slots * a.rows);
    const int64_t joins = (a.chunk_items + JOIN_CHUNKS - 1) / JOIN_CHUNKS * ((a.cg + (1 << a.join_lp) - 1) >> a.join_lp);
    const dim3 chunks = kge_grid_of(a.chunk_items, 1), rows = kge_grid_of(joins + a.row_items, 1);
#define KGE_BWD(G, O)                                                                                           \
    do {                                                                                                        \
        if (a.chunk_items > 0) hipLaunchKernelGGL(chunks_kernel<G>, chunks, dim3(NT), 0, st, a);                \
        hipLaunchKernelGGL((run_rows_kernel<G, O>), rows, dim3(NT), 0, st, a);                                      \
    } while (0)
    if (g16 && o16) KGE_BWD(true, true);
    else if (g16) KGE_BWD(true, false);
    else if (o16) KGE_BWD(false, true);
    else KGE_BWD(false, false);
#undef KGE_BWD
    return kge_launch_status();
}

}  // extern "C"
