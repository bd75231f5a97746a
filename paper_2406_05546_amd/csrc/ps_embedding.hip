// Rows of a table for given tokens, and the gradient of the table (include/ps_tokens.h).
//
// The gradient is summed over sorted tokens: rows are put in the order of (group, token), those of equal ones staying in the order
// that they have, and so the rows of one sum lie one behind the other.  No atomics: the same order every time.  The table is cleared
// as a whole beside the sorting, and the tokens that are there are written over it.  A few rows take one launch, in which every block
// sorts what belongs to its part of the table.
#include "../../include/ps_tokens.h"
#include "ps_linear.h"
#include "ps_tokens.h"

#include <cmath>
#include <type_traits>

namespace ps {
namespace {

__host__ __device__ inline int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---- forward ---------------------------------------------------------------------------------------------------------

struct LookupArgs {
    const void *table, *tokens;
    void* out;
    int64_t table_row, table_matrix, out_row, token_stride, vocab;
    int32_t rows, dim, pieces, each;  // pieces of a row; rows of a block
    float scale;
    Groups groups;
};

// A block takes `each` rows (up to 64).  Its first two wavefronts find where they come from, one row to a lane, each among the 64 rows from a
// multiple of 64 on that groups are looked for in; then every thread takes pieces of E columns, LOOKUP_AHEAD of them asked for together.  A row's last piece ends with the row, and so covers columns of the one
// before again: no piece is partial (E is 1 for rows shorter than 16 bytes).  Bound by memory: 16384 rows of 2048 in bf16 from eight tables for 64
// groups 22.7 us, 5.9 TB/s.
constexpr int LOOKUP_AHEAD = 4;
constexpr int64_t NO_GROUP = -1, NO_TOKEN = -2;

template <class T, class TOKEN, int E>
__global__ __launch_bounds__(256) void lookup_kernel(LookupArgs a)
{
    __shared__ int64_t source[64];
    for (int64_t first = (int64_t)blockIdx.x * a.each; first < a.rows; first += (int64_t)gridDim.x * a.each) {
        const int each = (int)min((int64_t)a.each, a.rows - first);
        const int64_t look = (first & ~63ll) + scalar(threadIdx.x & ~63);
        if (threadIdx.x < 128 && look < first + each) {
            const int64_t r = look + (threadIdx.x & 63);
            const int64_t token = static_cast<const TOKEN*>(a.tokens)[min(max(r, first), first + each - 1) * a.token_stride];
            const int g = groups_of_rows(a.groups, look);
            int64_t from = NO_GROUP;
            if (g >= 0) from = token >= 0 && token < a.vocab ? group_matrix(a.groups, g) * a.table_matrix + token * a.table_row : NO_TOKEN;
            if (r >= first && r < first + each) source[r - first] = from;
        }
        __syncthreads();
        const int items = each * a.pieces;
        for (int at = threadIdx.x; at < items; at += 256 * LOOKUP_AHEAD) {
            T raw[LOOKUP_AHEAD][E];
            int64_t from[LOOKUP_AHEAD];
            int line[LOOKUP_AHEAD], col[LOOKUP_AHEAD];
#pragma unroll
            for (int i = 0; i < LOOKUP_AHEAD; ++i) {
                const uint32_t item = min(at + i * 256, items - 1);
                line[i] = (int)(item / (uint32_t)a.pieces);
                col[i] = min((int)(item % (uint32_t)a.pieces) * E, a.dim - E);
                from[i] = source[line[i]];
            }
#pragma unroll
            for (int i = 0; i < LOOKUP_AHEAD; ++i) __builtin_memcpy(raw[i], static_cast<const T*>(a.table) + max(from[i], (int64_t)0) + col[i], sizeof(raw[i]));
#pragma unroll
            for (int i = 0; i < LOOKUP_AHEAD; ++i) {
                if (at + i * 256 >= items || from[i] == NO_GROUP) continue;
                float v[E];
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = from[i] == NO_TOKEN ? 0.f : to_float(raw[i][e]) * a.scale;
                store_n(static_cast<T*>(a.out) + (first + line[i]) * a.out_row + col[i], v);
            }
        }
        __syncthreads();  // source is written again
    }
}

// ---- sorting -----------------------------------------------------------------------------------------------------------

struct SortArgs {
    const void* tokens;
    int64_t token_stride, vocab;
    int32_t rows;
    uint32_t none;  // n_groups * vocab: the key of a row without a token or a group
    Groups groups;
};

// The key of row `first` (a multiple of 64) + lane, for a whole wavefront; `behind` for rows past the last.
template <class TOKEN>
__device__ __forceinline__ uint32_t key_of_row(const SortArgs& a, int64_t first, uint32_t behind)
{
    if (first >= a.rows) return behind;
    const int64_t r = first + (threadIdx.x & 63);
    const int64_t t = static_cast<const TOKEN*>(a.tokens)[min(r, (int64_t)a.rows - 1) * a.token_stride];
    const int g = groups_of_rows(a.groups, first);
    if (r >= a.rows) return behind;
    return g < 0 || t < 0 || t >= a.vocab ? a.none : (uint32_t)(g * a.vocab + t);
}

// What is cleared: lines of contiguous bytes, in blocks of CLEAR_BYTES or whole lines.
constexpr int CLEAR_BYTES = 65536;
struct ClearArgs {
    char* base;
    int64_t lines, per_matrix, line_stride, matrix_stride, line_bytes;  // line l: matrix l / per_matrix, row l % per_matrix
    int32_t size, blocks_per_line, lines_per_block;                     // size of an element; one of the two others is 1
    uint32_t blocks;
};

__device__ __forceinline__ void clear_line(char* to, int64_t first, int64_t end, int size, int t, int threads)
{
    for (int64_t at = first + (int64_t)t * 16; at < end; at += (int64_t)threads * 16) {
        if (at + 16 <= end) {
            const uintx4 zero = {0, 0, 0, 0};
            __builtin_memcpy(to + at, &zero, 16);
        } else if (size == 4) {
            for (int64_t i = at; i < end; i += 4) *reinterpret_cast<uint32_t*>(to + i) = 0;
        } else {
            for (int64_t i = at; i < end; i += 2) *reinterpret_cast<uint16_t*>(to + i) = 0;
        }
    }
}
__device__ __forceinline__ void clear_block(const ClearArgs& a, uint32_t block)
{
    auto line_at = [&](int64_t l) { return a.base + l / a.per_matrix * a.matrix_stride + l % a.per_matrix * a.line_stride; };
    if (a.lines_per_block == 1) {
        const int64_t first = (int64_t)(block % a.blocks_per_line) * CLEAR_BYTES;
        clear_line(line_at(block / a.blocks_per_line), first, min(first + CLEAR_BYTES, a.line_bytes), a.size, threadIdx.x, blockDim.x);
        return;
    }
    // short lines: so many threads to a line as it has pieces
    const int pieces = (int)((a.line_bytes + 15) / 16), threads = blockDim.x / pieces * pieces, at = threadIdx.x / pieces, step = blockDim.x / pieces;
    const int64_t first = (int64_t)block * a.lines_per_block, end = min(first + a.lines_per_block, a.lines);
    if (step == 0) {
        for (int64_t l = first; l < end; ++l) clear_line(line_at(l), 0, a.line_bytes, a.size, threadIdx.x, blockDim.x);
    } else if ((int)threadIdx.x < threads) {
        for (int64_t l = first + at; l < end; l += step) clear_line(line_at(l), 0, a.line_bytes, a.size, threadIdx.x % pieces, pieces);
    }
}

// Up to RANK_MOST rows: a row's place is the number of keys below its own, and of equal ones before it, which is counted.  A block compares
// the keys of RANK_ROWS rows, RANK_EACH to a thread, with RANK_KEYS others, which it reads from LDS, four at a time and the same for all
// lanes; two rows to a thread, so that the comparisons and not these reads are what takes time.  K: keys below 2^24 are compared as floats,
// whose difference, taken into 0 .. 1 as it is formed, is what is counted (two instructions; an integer comparison has to wait for its
// result to be added).  16384 rows alone: 27 us with one row and integers, 24 with two, 19 with floats.  Next to them the table is
// cleared, which is bound by memory: with 206 MB of it 34 us.  By ranks, and by the sort below, all of the call with 256 columns and 1000
// tokens in bf16: 8192 rows 27.9 and 37.0 us, 16384 34.7 and 37.9, 24576 47.0 and 39.5.
constexpr int RANK_THREADS = 256, RANK_EACH = 2, RANK_ROWS = RANK_THREADS * RANK_EACH, RANK_KEYS = 512, RANK_MOST = 16384;

__device__ __forceinline__ uint32_t less(uint32_t a, uint32_t b) { return a < b; }
__device__ __forceinline__ float less(float a, float b) { return __builtin_amdgcn_fmed3f(b - a, 0.f, 1.f); }  // whole numbers

template <class TOKEN, class K>
__global__ __launch_bounds__(RANK_THREADS) void rank_and_clear_kernel(SortArgs a, uint32_t rank_blocks, int parts, uint32_t* __restrict__ keys, uint16_t* __restrict__ counts, ClearArgs clear)
{
    if (blockIdx.x >= rank_blocks) {
        clear_block(clear, blockIdx.x - rank_blocks);
        return;
    }
    typedef K Four __attribute__((ext_vector_type(4)));
    __shared__ __attribute__((aligned(16))) K others[RANK_KEYS];
    const int part = blockIdx.x % parts, first = part * RANK_KEYS, lane = threadIdx.x & 63;
    const int row0 = blockIdx.x / parts * RANK_ROWS + scalar(threadIdx.x & ~63);  // of this wavefront's first 64; the next are RANK_THREADS behind
    uint32_t there[RANK_KEYS / RANK_THREADS], key[RANK_EACH];
    K n[RANK_EACH] = {};
#pragma unroll
    for (int i = 0; i < RANK_KEYS / RANK_THREADS; ++i) there[i] = key_of_row<TOKEN>(a, first + i * RANK_THREADS + scalar(threadIdx.x & ~63), ~0u);  // (above every key)
#pragma unroll
    for (int q = 0; q < RANK_EACH; ++q) key[q] = key_of_row<TOKEN>(a, row0 + q * RANK_THREADS, a.none);
#pragma unroll
    for (int i = 0; i < RANK_KEYS / RANK_THREADS; ++i) others[i * RANK_THREADS + threadIdx.x] = (K)there[i];
    __syncthreads();
    if (row0 >= a.rows) return;
    // 64 keys at a time: those of rows before count where they are equal, too, those of rows behind only where they are below, and of the same
    // 64 rows' the equal ones before are added
    const int many = min(RANK_KEYS, a.rows - first);
    for (int k0 = 0; k0 < many; k0 += 64) {
        K below[RANK_EACH];
#pragma unroll
        for (int q = 0; q < RANK_EACH; ++q) below[q] = (K)(key[q] + (first + k0 < row0 + q * RANK_THREADS));
#pragma unroll
        for (int k = 0; k < 64; k += 4) {
            const Four x = *reinterpret_cast<const Four*>(&others[k0 + k]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int q = 0; q < RANK_EACH; ++q) n[q] += less(x[i], below[q]);
        }
#pragma unroll
        for (int q = 0; q < RANK_EACH; ++q) {
            if (first + k0 != row0 + q * RANK_THREADS) continue;
            uint32_t equal = 0;
            for (int k = 0; k < 63; ++k) equal += (uint32_t)__builtin_amdgcn_readlane(key[q], k) == key[q] && k < lane;
            n[q] += (K)equal;
        }
    }
#pragma unroll
    for (int q = 0; q < RANK_EACH; ++q) {
        const int r = row0 + q * RANK_THREADS + lane;
        if (r >= a.rows) continue;
        if (part == 0) keys[r] = key[q];
        counts[(int64_t)part * a.rows + r] = (uint16_t)n[q];
    }
}

// Puts rows in their places.  An eighth of the table is cleared here: that takes as long as this, which mostly waits.
__global__ __launch_bounds__(RANK_THREADS) void rank_place_kernel(int rows, int parts, uint32_t place_blocks, const uint32_t* __restrict__ keys, const uint16_t* __restrict__ counts,
                                                               uint32_t* __restrict__ keys_to, uint32_t* __restrict__ order_to, ClearArgs clear)
{
    if (blockIdx.x >= place_blocks) {
        clear_block(clear, clear.blocks - 1 - (blockIdx.x - place_blocks));
        return;
    }
    const int r = blockIdx.x * RANK_THREADS + threadIdx.x;
    if (r >= rows) return;
    uint32_t n = 0;
#pragma unroll 8
    for (int p = 0; p < parts; ++p) n += counts[(int64_t)p * rows + r];
    keys_to[n] = keys[r];
    order_to[n] = (uint32_t)r;
}

// More rows: a stable radix sort of their keys, 8 bits at a time.  A tile of keys is ranked by a block: every wavefront has 64 at a time,
// finds with eight ballots which of them have the same digit, and counts them in a column of its own, so that equal digits stay in order.
// Bound by latency: 32768 rows 4.7, 4.0 and 5.6 us for the three launches of a pass.
constexpr int DIGITS = 256, TILE_WAVES = 4, TILE_EACH = 4, SORT_TILE = TILE_WAVES * 64 * TILE_EACH;
static_assert(TILE_WAVES * 64 == DIGITS, "a thread for each digit");

struct TileCounts {
    uint32_t at[TILE_WAVES][DIGITS];  // first counts, then where each wavefront's keys of a digit go
    uint32_t wave_sum[DIGITS / 64];
};

// Ranks of this thread's keys among those of the same digit of its wavefront.  Keys i * 64 + lane of a wavefront's TILE_EACH * 64.
__device__ __forceinline__ void rank_keys(TileCounts& c, const uint32_t (&key)[TILE_EACH], int shift, uint32_t (&rank)[TILE_EACH])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = lane; d < DIGITS; d += 64) c.at[wave][d] = 0;
    wave_meets();
    const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < TILE_EACH; ++i) {
        const uint32_t d = key[i] >> shift & (DIGITS - 1);
        unsigned long long same = ~0ull;
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const bool bit = d >> b & 1;
            const unsigned long long set = __ballot(bit);
            same &= bit ? set : ~set;
        }
        const uint32_t before = c.at[wave][d];
        wave_meets();  // all have read before one of them counts on
        if (!(same & below)) c.at[wave][d] = before + __popcll(same);
        wave_meets();
        rank[i] = before + __popcll(same & below);
    }
}

// Sum of v over the block's threads before this one.
__device__ __forceinline__ uint32_t sum_before(TileCounts& c, uint32_t v)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t upto = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t other = __shfl_up(upto, d, 64);
        if (lane >= d) upto += other;
    }
    if (lane == 63) c.wave_sum[wave] = upto;
    __syncthreads();
    uint32_t s = upto - v;
    for (int w = 0; w < DIGITS / 64; ++w)
        if (w < wave) s += c.wave_sum[w];
    return s;
}

// keys null: the first pass, whose keys are made from the tokens.
template <class TOKEN>
__device__ __forceinline__ void tile_keys(const SortArgs& a, const uint32_t* keys, int tile, uint32_t (&key)[TILE_EACH])
{
    const int64_t first = (int64_t)tile * SORT_TILE + scalar(threadIdx.x >> 6) * 64 * TILE_EACH;
#pragma unroll
    for (int i = 0; i < TILE_EACH; ++i) {
        const int64_t r = first + i * 64 + (threadIdx.x & 63);
        if (keys)
            key[i] = r < a.rows ? keys[r] : ~0u;  // behind all others, and the last among equal digits
        else
            key[i] = key_of_row<TOKEN>(a, first + i * 64, ~0u);
    }
}

// Counts of every digit: [digit][tile].  In the first pass the table is cleared beside it.
template <class TOKEN>
__global__ __launch_bounds__(DIGITS) void sort_count_kernel(SortArgs a, int shift, const uint32_t* __restrict__ keys, uint32_t* __restrict__ counts, int tiles, ClearArgs clear)
{
    __shared__ TileCounts c;
    if ((int)blockIdx.x >= tiles) {
        clear_block(clear, blockIdx.x - tiles);
        return;
    }
    uint32_t key[TILE_EACH], rank[TILE_EACH];
    tile_keys<TOKEN>(a, keys, blockIdx.x, key);
    rank_keys(c, key, shift, rank);
    __syncthreads();
    uint32_t total = 0;
    for (int w = 0; w < TILE_WAVES; ++w) total += c.at[w][threadIdx.x];
    counts[(int64_t)threadIdx.x * tiles + blockIdx.x] = total;
}

// A block for each digit: its counts to sums over the tiles before, their total to counts[DIGITS * tiles + digit].
__global__ __launch_bounds__(DIGITS) void sort_scan_kernel(uint32_t* __restrict__ counts, int tiles)
{
    __shared__ TileCounts c;
    uint32_t* mine = counts + (int64_t)blockIdx.x * tiles;
    uint32_t before = 0;
    for (int t0 = 0; t0 < tiles; t0 += DIGITS) {
        const int t = t0 + threadIdx.x;
        const uint32_t n = t < tiles ? mine[t] : 0;
        const uint32_t s = sum_before(c, n);
        if (t < tiles) mine[t] = before + s;
        for (int w = 0; w < DIGITS / 64; ++w) before += c.wave_sum[w];
        __syncthreads();  // wave_sum is written again
    }
    if (threadIdx.x == 0) counts[(int64_t)DIGITS * tiles + blockIdx.x] = before;
}

template <class TOKEN>
__global__ __launch_bounds__(DIGITS) void sort_place_kernel(SortArgs a, int shift, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ order,
                                                            const uint32_t* __restrict__ counts, int tiles, uint32_t* __restrict__ keys_to, uint32_t* __restrict__ order_to)
{
    __shared__ TileCounts c;
    uint32_t key[TILE_EACH], rank[TILE_EACH];
    tile_keys<TOKEN>(a, keys, blockIdx.x, key);
    rank_keys(c, key, shift, rank);
    __syncthreads();
    uint32_t to = sum_before(c, counts[(int64_t)DIGITS * tiles + threadIdx.x]) + counts[(int64_t)threadIdx.x * tiles + blockIdx.x];
    for (int w = 0; w < TILE_WAVES; ++w) {
        const uint32_t n = c.at[w][threadIdx.x];
        c.at[w][threadIdx.x] = to;
        to += n;
    }
    __syncthreads();
    const int wave = threadIdx.x >> 6;
    const int64_t first = (int64_t)blockIdx.x * SORT_TILE + wave * 64 * TILE_EACH + (threadIdx.x & 63);
#pragma unroll
    for (int i = 0; i < TILE_EACH; ++i) {
        const int64_t r = first + i * 64;
        if (r >= a.rows) continue;
        const uint32_t p = c.at[wave][key[i] >> shift & (DIGITS - 1)] + rank[i];
        keys_to[p] = key[i];
        order_to[p] = order ? order[r] : (uint32_t)r;
    }
}

// ---- sums of runs --------------------------------------------------------------------------------------------------------

// Rows of equal keys are a run.  A run is cut into pieces of PIECE rows from its beginning on; the sum of a run's only piece is
// the gradient, those of a longer run go to `partial`, of which each PIECE places in the order have two rows: for the piece, not the
// first of its run, that begins in them, and for the first piece of a run longer than that.  (There cannot be more: two pieces
// of a run begin PIECE places apart.)
// Pieces of 32 rows, and four or sixteen rows ahead, took as long, within 3 %.
constexpr int PIECE = 16, SUM_AHEAD = 8;

struct SumArgs {
    const void* dy;
    void* dtable;
    const uint32_t *keys, *order;
    float* partial;  // [2 * chunks][dim]
    int64_t dy_row, table_row, table_matrix, vocab;
    int32_t rows, dim, chunks, col_blocks;
    uint32_t none;
    float scale;
};

// The first place of `key` among the sorted keys before `end`, where it is itself.  For a whole wavefront: one look at the 64 before, and
// one for every power of 64 of the rest.
__device__ __forceinline__ int first_place(const uint32_t* keys, uint32_t key, int end)
{
    const int near = end - 64 + (int)(threadIdx.x & 63);
    const int same = __popcll(__ballot(near >= 0 && keys[max(near, 0)] == key));
    if (same < 64) return end - same;
    int lo = 0, hi = end - 64;  // keys before lo are below, the one at hi is not
    while (lo < hi) {
        const int step = (hi - lo + 63) >> 6, p = lo + (int)(threadIdx.x & 63) * step;
        const int below = __popcll(__ballot(p < hi && keys[p] < key));  // lanes in order
        if (below == 0) return lo;
        hi = min(hi, lo + below * step);
        lo = lo + (below - 1) * step + 1;
    }
    return lo;
}

template <class T>
__device__ __forceinline__ T* row_of_key(const SumArgs& a, uint32_t key)
{
    const uint32_t g = key / (uint32_t)a.vocab, v = key - g * (uint32_t)a.vocab;
    return static_cast<T*>(a.dtable) + (int64_t)g * a.table_matrix + (int64_t)v * a.table_row;
}

// The product as 32 bits hold it: the compiler would make one instruction of it and the rounding to 16 bits where it finds them together, whose
// results differ now and then.
__device__ __forceinline__ float scaled(float v, float scale)
{
    v *= scale;
    asm("" : "+v"(v));
    return v;
}

// E values as they were read
template <class T, int E>
struct Held {
    uintx4 bits;
    __device__ __forceinline__ float value(int e) const { return element<T>(bits, e); }
};
template <class T>
struct Held<T, 1> {
    T bits;
    __device__ __forceinline__ float value(int) const { return to_float(bits); }
};

// Wavefronts [chunk][64 * E columns]: the pieces that begin in the chunk's PIECE places; they end within PIECE - 1 places behind.  A lane
// whose columns would go past the row's end takes the last E of the row, which others have too (E is 1 for rows shorter than 16 bytes).  Bound by
// memory: SUM_AHEAD rows are asked for while as many are added up, without a branch between them, at which the compiler would wait.
// 16384 rows of 2048 in bf16 over 50257 tokens 24 us, 3.7 TB/s (28 where its rows of the table are not in the caches).
template <class T, int E>
__global__ __launch_bounds__(256) void sum_runs_kernel(SumArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + scalar(threadIdx.x >> 6);
    const int chunk = (int)(w / a.col_blocks), own = (int)(w % a.col_blocks) * 64 * E + lane * E, col = min(own, a.dim - E);
    const bool there = own < a.dim;
    if (chunk >= a.chunks) return;
    const int p0 = chunk * PIECE, p = p0 + lane;
    const uint32_t key = p < a.rows ? a.keys[p] : ~0u;
    const uint32_t before = p0 ? a.keys[p0 - 1] : ~0u;
    const uint32_t row = p < a.rows ? a.order[p] : 0;
    const uint32_t previous = __shfl_up(key, 1, 64);
    const bool differs = lane ? key != previous : p0 == 0 || key != before;
    const unsigned long long begins = __ballot(differs), exist = __ballot(p < a.rows && key < a.none);
    // where the run of this lane's place begins, counted from p0
    const unsigned long long upto = begins & (~0ull >> (63 - lane));
    int run = upto ? 63 - __builtin_clzll(upto) : 0;
    if (!(begins & 1)) {
        const int first = first_place(a.keys, __builtin_amdgcn_readfirstlane(key), p0) - p0;
        if (!upto) run = first;
    }
    const unsigned long long pieces = __ballot((lane - run) % PIECE == 0) & exist;
    const unsigned long long todo = pieces & ((1ull << PIECE) - 1);
    if (!todo) return;
    // places from the first piece's beginning to where a piece that begins behind the chunk, or nothing, follows
    const int from = __builtin_ctzll(todo);
    const unsigned long long behind = pieces >> PIECE << PIECE | ~exist;  // (rows that exist come first)
    const int to = __builtin_ctzll(behind);                               // (at most 2 * PIECE - 1)
    // the last places of pieces; those that are not all of their run
    const unsigned long long ends = (pieces | ~exist) >> 1;
    const unsigned long long goes_on = exist >> 1 & ~(begins >> 1), starts_run = begins & pieces;
    float sum[E] = {};
    Held<T, E> now[SUM_AHEAD], then[SUM_AHEAD];
    auto take = [&](int at, Held<T, E> (&raw)[SUM_AHEAD]) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < SUM_AHEAD; ++u) {
            const int64_t r = (uint32_t)__builtin_amdgcn_readlane(row, min(at + u, to - 1));
            __builtin_memcpy(&raw[u].bits, static_cast<const T*>(a.dy) + r * a.dy_row + col, sizeof(T) * E);
        }
    };
    take(from, now);
    for (int at = from; at < to; at += SUM_AHEAD) {
        if (at + SUM_AHEAD < to) take(at + SUM_AHEAD, then);
#pragma unroll
        for (int u = 0; u < SUM_AHEAD; ++u) {
            const int place = at + u;
            if (place >= to) continue;
            const bool first = pieces >> place & 1;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float x = now[u].value(e);
                sum[e] = first ? x : sum[e] + x;
            }
            if (!(ends >> place & 1) || !there) continue;
            const int start = 63 - __builtin_clzll(pieces & (~0ull >> (63 - place)));
            const bool whole_start = starts_run >> start & 1;
            if (whole_start && !(goes_on >> place & 1)) {
                float v[E];
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = scaled(sum[e], a.scale);
                store_n(row_of_key<T>(a, (uint32_t)__builtin_amdgcn_readlane(key, place)) + col, v);
            } else {
                store_n(a.partial + (2 * (int64_t)chunk + whole_start) * a.dim + col, sum);
            }
        }
#pragma unroll
        for (int u = 0; u < SUM_AHEAD; ++u) now[u] = then[u];
    }
}

// Adds up the pieces of longer runs, 64 * E columns to a block.  Each of its wavefronts looks at a chunk; if a run longer than PIECE begins
// there it adds up its pieces, one behind the other, or, where these are more than JOIN_ALONE (so that two such runs at most begin among the
// block's chunks), leaves them to all wavefronts: a sixteenth to each, and these sums in order.  Bound by trips to memory that wait for each other:
// 16384 rows of 2048 6.9 us (12.3 with up to 32 pieces to a wavefront alone).
constexpr int JOIN_WAVES = 16, JOIN_ALONE = 8;

template <class T, int E>
__global__ __launch_bounds__(JOIN_WAVES * 64) void join_runs_kernel(SumArgs a)
{
    __shared__ float meet[JOIN_WAVES][64][E + 1];
    struct Run {
        uint32_t key;
        int chunk, pieces;
    };
    __shared__ Run long_runs[JOIN_WAVES];  // pieces 0: none
    const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6);
    const int64_t total = up(a.chunks, JOIN_WAVES) * a.col_blocks;
    for (int64_t block = blockIdx.x; block < total; block += gridDim.x) {
        const int64_t chunk = block / a.col_blocks * JOIN_WAVES + wave;
        const int own = (int)(block % a.col_blocks) * 64 * E + lane * E, col = min(own, a.dim - E);
        auto add_up = [&](int64_t of, int first, int end, float (&sum)[E]) __attribute__((always_inline)) {
#pragma unroll 8
            for (int i = first; i < end; ++i) {
                float x[E];
                load_n(a.partial + (2 * (of + i) + (i == 0)) * a.dim + col, x);
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] += x[e];
            }
        };
        auto give = [&](uint32_t key, float (&sum)[E]) __attribute__((always_inline)) {
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] = scaled(sum[e], a.scale);
            if (own < a.dim) store_n(row_of_key<T>(a, key) + col, sum);
        };
        const int64_t p0 = chunk * PIECE, p = p0 + lane;
        const uint32_t key = p < a.rows ? a.keys[p] : ~0u, before = p0 && p0 < a.rows ? a.keys[p0 - 1] : ~0u;
        const uint32_t previous = __shfl_up(key, 1, 64), later = __shfl_down(key, PIECE, 64);
        const bool differs = lane ? key != previous : p0 == 0 || key != before;
        const unsigned long long longer = __ballot(lane < PIECE && differs && p + PIECE < a.rows && key < a.none && key == later);
        Run run{0, (int)chunk, 0};
        if (longer) {
            const int at = __builtin_ctzll(longer);
            run.key = (uint32_t)__builtin_amdgcn_readlane(key, at);
            // its pieces: those whose first place has the key, counted 64 at a time
            for (bool more = true; more; run.pieces += 64) {
                const int64_t q = p0 + at + (int64_t)(run.pieces + lane) * PIECE;
                const unsigned long long same = __ballot(q < a.rows && a.keys[min(q, (int64_t)a.rows - 1)] == run.key);
                more = same == ~0ull;
                if (!more) run.pieces += __popcll(same) - 64;
            }
            if (run.pieces <= JOIN_ALONE) {
                float sum[E] = {};
                add_up(chunk, 0, run.pieces, sum);
                give(run.key, sum);
                run.pieces = 0;
            }
        }
        if (lane == 0) long_runs[wave] = run;
        __syncthreads();
        for (int k = 0; k < JOIN_WAVES; ++k) {
            const Run of = long_runs[k];
            if (!of.pieces) continue;  // (the same in all wavefronts)
            const int each = (of.pieces + JOIN_WAVES - 1) / JOIN_WAVES, first = min(wave * each, of.pieces);
            float sum[E] = {};
            add_up(of.chunk, first, min(first + each, of.pieces), sum);
#pragma unroll
            for (int e = 0; e < E; ++e) meet[wave][lane][e] = sum[e];
            __syncthreads();
            if (wave == k) {
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] = meet[0][lane][e];
                for (int w = 1; w < JOIN_WAVES; ++w)
#pragma unroll
                    for (int e = 0; e < E; ++e) sum[e] += meet[w][lane][e];
                give(of.key, sum);
            }
            __syncthreads();  // what met is written again
        }
        __syncthreads();  // and the list
    }
}

// ---- fewer rows: one launch ----------------------------------------------------------------------------------------------

struct FewArgs {
    const void *dy, *tokens;
    void* dtable;
    int64_t dy_row, table_row, table_matrix, token_stride, vocab;
    int32_t rows, dim, shift, col_blocks;  // a block has every (2^shift)-th row of a group's table
    float scale;
    Groups groups;
};

// A block has rows of one group's table, evenly apart so that frequent tokens, which are often the first ones, are many blocks'; of wide
// rows 64 * E columns.  It asks for all of the group's tokens, one to a thread, clears its rows meanwhile, puts the rows that have its own
// tokens in their order and writes their sums over what it cleared.  Sums are formed in the order that the kernels above have: the same bits.
// Bound by the clearing, and by trips to memory, offsets, tokens, rows, that wait for each other; a token that all rows have, by the
// one block that adds them up, for which there are eight wavefronts and registers for six of them to a SIMD.  us:
//   all rows cleared, or once it is known those that nothing is added to   fp32 512 rows of 512 over 32000 tokens   16, 19.5
//   eight wavefronts, or four                                              bf16 256 equal rows of 1024              32, 41
//   blocks of 64 KB, of 32, of 128                                         bf16 512 rows of 4096 over 30000         51, 54, 51
constexpr int FEW_WAVES = 8, FEW_MOST = FEW_WAVES * 64, FEW_UNITS = 16, FEW_BYTES = 65536, FEW_AHEAD = 8;

template <class TOKEN, class T, int E>
__global__ __launch_bounds__(FEW_WAVES * 64, 6) void few_rows_kernel(FewArgs a)
{
    __shared__ uint16_t order[FEW_MOST];  // rows, counted from the group's first, in the order of their tokens
    __shared__ union {
        uint32_t at[FEW_WAVES][DIGITS];
        float meet[FEW_UNITS][E][64];
    } s;
    __shared__ uint32_t begins[DIGITS + 1], wave_sum[DIGITS / 64];
    const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6);
    const int col_block = blockIdx.x % a.col_blocks, block = blockIdx.x / a.col_blocks, g = block >> a.shift;
    const int64_t others = (1ll << a.shift) - 1, v0 = block & others;
    const int n = (int)((a.vocab - v0 + others) >> a.shift);
    if (n <= 0) return;
    const GroupRows of = group_rows(a.groups, g);
    const int begin = of.begin, end = of.end;
    T* const table = static_cast<T*>(a.dtable) + g * a.table_matrix + v0 * a.table_row;
    const int64_t table_row = a.table_row << a.shift;
    const int row = wave * 64 + lane, rows = end - begin;
    int64_t t = -1;
    if (rows > 0) t = static_cast<const TOKEN*>(a.tokens)[(int64_t)(begin + min(row, rows - 1)) * a.token_stride];
    // Whether offsets ascend: every wavefront sees 64 of them.  (One group: something that is there, not in a branch, where the compiler would wait.)
    const int groups = a.groups.n;
    const int32_t* const some = groups > 1 ? a.groups.offsets + min(lane, groups - 1) : static_cast<const int32_t*>(a.tokens);
    const int one = some[0], next = some[groups > 1];
    for (int i = threadIdx.x; i < FEW_WAVES * DIGITS; i += FEW_WAVES * 64) s.at[0][i] = 0;

    // All of it is cleared: what is added up is written over it, behind a wait.
    constexpr int WIDE = 64 * E * (int)sizeof(T);
    const int64_t from_byte = (int64_t)col_block * WIDE, to_byte = min(from_byte + WIDE, (int64_t)a.dim * (int)sizeof(T));
    const int pieces = (int)((to_byte - from_byte + 15) / 16), together = FEW_WAVES * 64 / pieces;
    if ((int)threadIdx.x < together * pieces)
        for (int i = threadIdx.x / pieces; i < n; i += together)
            clear_line(reinterpret_cast<char*>(table + i * table_row), from_byte, to_byte, sizeof(T), threadIdx.x % pieces, pieces);

    // Rows of this block's tokens, their places among them, and which lanes have the same
    bool in = row < rows && t >= 0 && t < a.vocab && (t & others) == v0;
    if (!__syncthreads_or(in)) return;
    bool disorder = __ballot(one > next) != 0;
    if (groups > 64) {
        for (int i = 64 + threadIdx.x; i < groups; i += 4 * FEW_WAVES * 64) {
            int begins[4], ends[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int32_t* const at = a.groups.offsets + min(i + k * FEW_WAVES * 64, groups - 1);
                begins[k] = at[0], ends[k] = at[1];
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) disorder |= begins[k] > ends[k];
        }
        disorder = __syncthreads_or(disorder);
    }
    if (disorder) {
        // Of rows of several groups those that groups_of_rows gives to this one.
        if (wave * 64 < a.rows) order[wave * 64 + lane] = groups_of_rows(a.groups, wave * 64) == g;
        __syncthreads();
        in = in && order[begin + row];
    }
    const uint32_t d = in ? (uint32_t)(t >> a.shift) : 0;
    unsigned long long same = __ballot(in);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
        const bool bit = d >> b & 1;
        const unsigned long long set = __ballot(bit);
        same &= bit ? set : ~set;
    }
    const uint32_t before = __popcll(same & ((1ull << lane) - 1));
    if (in && !before) s.at[wave][d] = __popcll(same);
    __syncthreads();
    uint32_t total = 0;
    if (threadIdx.x < DIGITS)
        for (int w = 0; w < FEW_WAVES; ++w) total += s.at[w][threadIdx.x];
    uint32_t upto = total;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const uint32_t other = __shfl_up(upto, k, 64);
        if (lane >= k) upto += other;
    }
    if (lane == 63 && wave < DIGITS / 64) wave_sum[wave] = upto;
    __syncthreads();
    if (threadIdx.x < DIGITS) {
        uint32_t to = upto - total;
        for (int w = 0; w < wave; ++w) to += wave_sum[w];
        begins[threadIdx.x] = to;
        if (threadIdx.x == DIGITS - 1) begins[DIGITS] = to + total;
        for (int w = 0; w < FEW_WAVES; ++w) {
            const uint32_t here = s.at[w][threadIdx.x];
            s.at[w][threadIdx.x] = to;
            to += here;
        }
    }
    __syncthreads();
    if (in) order[s.at[wave][d] + before] = (uint16_t)row;
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0): this wavefront has cleared
    __syncthreads();

    const int own = col_block * 64 * E + lane * E, col = min(own, a.dim - E);
    // Rows from .. to of a run that begins at `run`: `sum` of the last piece, `sums` of all of them.
    auto add_up = [&](int run, int from, int to, float (&sum)[E], float (&sums)[E]) __attribute__((always_inline)) {
        auto some_rows = [&](int at, auto ahead) __attribute__((always_inline)) {
            constexpr int AHEAD = ahead;
            Held<T, E> now[AHEAD];
            const int rows = order[min(at + (lane & (AHEAD - 1)), to - 1)];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                __builtin_memcpy(&now[u].bits, static_cast<const T*>(a.dy) + (int64_t)(begin + __builtin_amdgcn_readlane(rows, u)) * a.dy_row + col, sizeof(T) * E);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int place = at + u;
                if (place >= to) continue;
                const bool first = (place - run) % PIECE == 0, last = (place - run) % PIECE == PIECE - 1 || place == to - 1;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float x = now[u].value(e);
                    sum[e] = first ? x : sum[e] + x;
                    if (last) sums[e] += sum[e];
                }
            }
        };
        if (to - from <= 2)
            some_rows(from, std::integral_constant<int, 2>{});
        else
            for (int at = from; at < to; at += FEW_AHEAD) some_rows(at, std::integral_constant<int, FEW_AHEAD>{});
    };
    auto give = [&](int i, float (&sum)[E]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] = scaled(sum[e], a.scale);
        if (own < a.dim) store_n(table + i * table_row + col, sum);
    };
    // Runs of one piece: a wavefront has every FEW_WAVES-th.  Longer ones afterwards, by all of them, as join_runs_kernel adds them up.
    int k = 0;
    unsigned long long longer[DIGITS / 64];
#pragma unroll
    for (int i0 = 0; i0 < DIGITS; i0 += 64) {
        const int many = i0 + lane < n ? (int)(begins[i0 + lane + 1] - begins[i0 + lane]) : 0;
        longer[i0 / 64] = __ballot(many > PIECE);
        for (unsigned long long runs = __ballot(many > 0 && many <= PIECE); runs; runs &= runs - 1, ++k) {
            if (k % FEW_WAVES != wave) continue;
            const int i = i0 + __builtin_ctzll(runs), run = scalar((int)begins[i]);
            float sum[E], sums[E] = {};
            add_up(run, run, scalar((int)begins[i + 1]), sum, sums);
            give(i, sum);
        }
    }
    __syncthreads();  // (nothing else is left in `at`)
    k = 0;
#pragma unroll
    for (int i0 = 0; i0 < DIGITS; i0 += 64)
        for (unsigned long long runs = longer[i0 / 64]; runs; runs &= runs - 1, ++k) {
            const int i = i0 + __builtin_ctzll(runs), run = scalar((int)begins[i]), end_of_run = scalar((int)begins[i + 1]);
            const int count = (int)up(end_of_run - run, PIECE), each = count <= JOIN_ALONE ? 1 : (int)up(count, FEW_UNITS), units = (int)up(count, each);
            for (int u = wave; u < units; u += FEW_WAVES) {
                float sum[E], sums[E] = {};
                add_up(run, run + u * each * PIECE, min(run + (u + 1) * each * PIECE, end_of_run), sum, sums);
#pragma unroll
                for (int e = 0; e < E; ++e) s.meet[u][e][lane] = sums[e];
            }
            __syncthreads();
            if (wave == k % FEW_WAVES) {
                float sum[E];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    sum[e] = s.meet[0][e][lane];
                    for (int u = 1; u < units; ++u) sum[e] += s.meet[u][e][lane];
                }
                give(i, sum);
            }
            __syncthreads();  // what met is written again
        }
}

// ---- entry points --------------------------------------------------------------------------------------------------------

Groups groups_of(const ps_embedding& e) { return Groups{e.offsets_dev, e.table_of_group_dev, e.n_groups, e.n_tables, (int32_t)e.rows}; }

ps_status check_embedding(const char* call, const ps_embedding* e, bool forward)
{
    if (!e) return dense_fail(PS_EINVAL, "%s: no description", call);
    if (e->dtype != PS_F32 && e->dtype != PS_BF16 && e->dtype != PS_F16) return dense_fail(PS_EINVAL, "%s: unknown type", call);
    if (e->rows < 0 || e->rows > PS_DENSE_MAX_ROWS) return dense_fail(PS_EINVAL, "%s: rows outside 0 .. %d", call, PS_DENSE_MAX_ROWS);
    if (e->vocab < 1 || e->vocab > PS_DENSE_MAX_STRIDE || e->dim < 1 || e->dim > PS_DENSE_MAX_STRIDE)
        return dense_fail(PS_EINVAL, "%s: vocab or dim outside 1 .. %d", call, PS_DENSE_MAX_STRIDE);
    if (e->n_groups < 1 || e->n_groups > PS_DENSE_MAX_GROUPS) return dense_fail(PS_EINVAL, "%s: groups outside 1 .. %d", call, PS_DENSE_MAX_GROUPS);
    if (!e->offsets_dev && e->n_groups != 1) return dense_fail(PS_EINVAL, "%s: several groups need offsets", call);
    if (!forward && e->n_groups * e->vocab > INT32_MAX) return dense_fail(PS_EINVAL, "%s: groups times vocab from 2^31 on", call);
    if (forward && (e->n_tables < 1 || (!e->table_of_group_dev && e->n_tables < e->n_groups)))
        return dense_fail(PS_EINVAL, "%s: fewer tables than groups, and no list of which each uses", call);
    if ((reinterpret_cast<uintptr_t>(e->offsets_dev) & 3) || (forward && (reinterpret_cast<uintptr_t>(e->table_of_group_dev) & 3)))
        return dense_fail(PS_EINVAL, "%s: misaligned offsets or list of tables", call);
    if (!std::isfinite(e->scale) || !std::isfinite((float)e->scale)) return dense_fail(PS_EINVAL, "%s: the scale is not finite", call);
    return PS_OK;
}

// One launch up to FEW_MOST rows.  us of one, and of four (tokens spread evenly in their logarithm, or one that all rows have; four results in turn):
//   bf16   16 rows of 64 over 1000 tokens 5.5, 11.0   64 of 512 over 32000 11.7, 19.5   512 of 1024 over 50257 21.7, 34.4   512 of 4096 over 30000 47.9, 60.6
//          one token: 256 of 1024 over 32000 23.6, 26.0   512 of 1024 over 50257 36.6, 34.6   512 of 4096 over 30000 55, 60   1024 of 1024 over 32000 53, 31
//          512 of 64 in 64 groups over 500 12.0, 26.4   500 of 64 in 500 groups over 1000 17.9, 42.6   500 of 16 in 5000 over 300 38, 148
//   fp32   512 of 512 over 32000 15.9, 29.8   256 of 192 in 64 groups over 4096 37.7, 49.5   all in one of them 37.1, 50.7
struct Few {
    uint32_t blocks;  // 0: not so
    int shift, col_blocks;
};
Few few(const ps_embedding& e)
{
    if (!e.rows || e.rows > FEW_MOST) return {};
    const int64_t size = dtype_size(e.dtype);
    Few f{};
    f.col_blocks = (int)up(e.dim, 1024 / size);
    // blocks of 64 KB, or fewer where that leaves less than four of them to a compute unit
    const int64_t most = std::min<int64_t>(DIGITS, FEW_BYTES / std::min<int64_t>(e.dim * size, 1024));
    const int64_t each = std::max<int64_t>(1, std::min(most, e.n_groups * e.vocab * f.col_blocks / (4 * COMPUTE_UNITS)));
    while (e.vocab > each << f.shift) ++f.shift;
    const int64_t blocks = (e.n_groups << f.shift) * f.col_blocks;
    if (blocks < 1 << 22) f.blocks = (uint32_t)blocks;  // (a launch has less than 2^32 threads)
    return f;
}

struct GradientSpace {
    uint64_t keys[2], order[2], counts, partial, total;
    int passes, tiles, chunks, parts;
};

GradientSpace gradient_space(const ps_embedding& e)
{
    GradientSpace g{};
    if (few(e).blocks) return g;
    const uint64_t none = (uint64_t)e.n_groups * e.vocab;
    while (none >> (8 * g.passes)) ++g.passes;
    g.chunks = (int)up(e.rows, PIECE);
    if (e.rows <= RANK_MOST)
        g.parts = (int)up(e.rows, RANK_KEYS);
    else
        g.tiles = (int)up(e.rows, SORT_TILE);
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        g.keys[i] = take((uint64_t)e.rows * 4);
        g.order[i] = take((uint64_t)e.rows * 4);
    }
    g.counts = take(g.tiles ? (uint64_t)DIGITS * (g.tiles + 1) * 4 : (uint64_t)g.parts * e.rows * 2);
    g.partial = take((uint64_t)2 * g.chunks * e.dim * 4);
    g.total = at;
    return g;
}

// Rows that lie one behind the other are one line.
ClearArgs clear_args(const ps_embedding& e, const ps_matrix& m)
{
    const int size = dtype_size(e.dtype);
    ClearArgs c{};
    c.base = static_cast<char*>(m.data_dev);
    c.size = size;
    c.lines = e.n_groups * e.vocab;
    c.per_matrix = e.vocab;
    c.line_stride = m.row * size;
    c.matrix_stride = m.matrix * size;
    c.line_bytes = e.dim * size;
    if (e.vocab == 1 || m.row == e.dim) {
        c.lines = e.n_groups;
        c.per_matrix = 1;
        c.line_bytes *= e.vocab;
        if (e.n_groups == 1 || m.matrix * size == c.line_bytes) {
            c.lines = 1;
            c.line_bytes *= e.n_groups;
        }
    }
    c.blocks_per_line = (int32_t)up(c.line_bytes, CLEAR_BYTES);
    c.lines_per_block = c.blocks_per_line > 1 ? 1 : (int32_t)(CLEAR_BYTES / c.line_bytes);
    c.blocks = (uint32_t)(c.lines_per_block > 1 ? up(c.lines, c.lines_per_block) : c.lines * c.blocks_per_line);
    return c;
}

template <class F>
void with_types(int dtype, int bytes, F f)
{
    auto with_token = [&](auto t) {
        if (bytes == 4)
            f(t, int32_t{});
        else
            f(t, int64_t{});
    };
    if (dtype == PS_F32)
        with_token(float{});
    else if (dtype == PS_BF16)
        with_token(bf16_t{});
    else
        with_token(f16_t{});
}

}  // namespace

ps_status check_tokens(const char* call, const ps_tokens* t, int64_t rows, bool needed)
{
    if (!t || !t->data_dev) return needed && rows ? dense_fail(PS_EINVAL, "%s: no tokens", call) : PS_OK;
    if (t->bytes != 4 && t->bytes != 8) return dense_fail(PS_EINVAL, "%s: tokens have 4 or 8 bytes", call);
    if (reinterpret_cast<uintptr_t>(t->data_dev) & (t->bytes - 1)) return dense_fail(PS_EINVAL, "%s: misaligned tokens", call);
    if (rows > 1 && (t->stride < 0 || t->stride > PS_DENSE_MAX_STRIDE)) return dense_fail(PS_EINVAL, "%s: tokens are too far apart", call);
    return PS_OK;
}

ps_status check_rows(const char* call, const char* name, int dtype, const ps_matrix* m, int64_t rows, int64_t cols, int64_t matrices)
{
    if (!m || !m->data_dev) return rows ? dense_fail(PS_EINVAL, "%s: %s is missing", call, name) : PS_OK;
    if (reinterpret_cast<uintptr_t>(m->data_dev) & (dtype_size(dtype) - 1)) return dense_fail(PS_EINVAL, "%s: %s is not aligned to its elements", call, name);
    if (rows > 1 && (m->row < cols || m->row > PS_DENSE_MAX_STRIDE)) return dense_fail(PS_EINVAL, "%s: %s has rows that overlap or are too far apart", call, name);
    if (matrices > 1 && m->matrix < (rows - 1) * m->row + cols) return dense_fail(PS_EINVAL, "%s: %s has matrices that overlap", call, name);
    return PS_OK;
}

ps_status tokens_launched(const char* call)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PS_OK : dense_fail(PS_EDEVICE, "%s: %s", call, hipGetErrorString(e));
}

}  // namespace ps

extern "C" ps_status ps_embedding_forward(const ps_embedding* e, const ps_tokens* tokens, const ps_matrix* table, const ps_matrix* out, void* hip_stream)
{
    using namespace ps;
    static const char call[] = "ps_embedding_forward";
    ps_status st = check_embedding(call, e, true);
    if (st != PS_OK) return st;
    if ((st = check_tokens(call, tokens, e->rows, true)) != PS_OK) return st;
    if ((st = check_rows(call, "table", e->dtype, table, e->vocab, e->dim, e->n_tables)) != PS_OK) return st;
    if ((st = check_rows(call, "out", e->dtype, out, e->rows, e->dim, 1)) != PS_OK) return st;
    if (!e->rows) return PS_OK;
    LookupArgs a{};
    a.table = table->data_dev;
    a.table_row = table->row;
    a.table_matrix = table->matrix;
    a.out = out->data_dev;
    a.out_row = out->row;
    a.tokens = tokens->data_dev;
    a.token_stride = tokens->stride;
    a.vocab = e->vocab;
    a.rows = (int32_t)e->rows;
    a.dim = (int32_t)e->dim;
    const int wide = 16 / dtype_size(e->dtype);
    a.pieces = (int32_t)(e->dim < wide ? e->dim : up(e->dim, wide));
    // Rows of 32 KB together, or fewer where that leaves less than four blocks to a compute unit.  bf16, us:
    //   64 rows of 4096 one to a block 7.0, 64 34.5   16384 of 2048 in 64 groups eight 22.1, one 31.2, 64 26.4   65536 of 64 64 8.4, one 56.8
    a.each = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(64, 2048 / a.pieces), e->rows / (4 * COMPUTE_UNITS)));
    a.scale = (float)e->scale;
    a.groups = groups_of(*e);
    const int64_t blocks = std::min<int64_t>(up(e->rows, a.each), 1 << 22);
    with_types(e->dtype, tokens->bytes, [&](auto t, auto token) {
        using T = decltype(t);
        const dim3 grid((uint32_t)blocks), block(256);
        if (e->dim < wide)
            hipLaunchKernelGGL((lookup_kernel<T, decltype(token), 1>), grid, block, 0, static_cast<hipStream_t>(hip_stream), a);
        else
            hipLaunchKernelGGL((lookup_kernel<T, decltype(token), 16 / sizeof(T)>), grid, block, 0, static_cast<hipStream_t>(hip_stream), a);
    });
    return tokens_launched(call);
}

extern "C" ps_status ps_embedding_workspace_bytes(const ps_embedding* e, uint64_t* bytes_out)
{
    using namespace ps;
    const ps_status st = check_embedding("ps_embedding_workspace_bytes", e, false);
    if (st != PS_OK) return st;
    if (!bytes_out) return dense_fail(PS_EINVAL, "ps_embedding_workspace_bytes: no place for the result");
    *bytes_out = gradient_space(*e).total;
    return PS_OK;
}

extern "C" ps_status ps_embedding_backward(const ps_embedding* e, const ps_tokens* tokens, const ps_matrix* dy, const ps_matrix* dtable,
                                           void* workspace, uint64_t workspace_bytes, void* hip_stream)
{
    using namespace ps;
    static const char call[] = "ps_embedding_backward";
    ps_status st = check_embedding(call, e, false);
    if (st != PS_OK) return st;
    if ((st = check_tokens(call, tokens, e->rows, true)) != PS_OK) return st;
    if ((st = check_rows(call, "dy", e->dtype, dy, e->rows, e->dim, 1)) != PS_OK) return st;
    if ((st = check_rows(call, "dtable", e->dtype, dtable, e->vocab, e->dim, e->n_groups)) != PS_OK) return st;
    const GradientSpace space = gradient_space(*e);
    if (space.total && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))) return dense_fail(PS_EINVAL, "%s: null or misaligned workspace", call);
    if (workspace_bytes < space.total) return dense_fail(PS_ENOMEM, "%s: workspace too small", call);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    if (const Few one = few(*e); one.blocks) {
        FewArgs f{};
        f.dy = dy->data_dev;
        f.dy_row = dy->row;
        f.dtable = dtable->data_dev;
        f.table_row = dtable->row;
        f.table_matrix = dtable->matrix;
        f.tokens = tokens->data_dev;
        f.token_stride = tokens->stride;
        f.groups = groups_of(*e);
        f.vocab = e->vocab;
        f.rows = (int32_t)e->rows;
        f.dim = (int32_t)e->dim;
        f.shift = one.shift;
        f.col_blocks = one.col_blocks;
        f.scale = (float)e->scale;
        with_types(e->dtype, tokens->bytes, [&](auto t, auto token) {
            using T = decltype(t);
            constexpr int E = 16 / sizeof(T);
            const auto kernel = e->dim < E ? few_rows_kernel<decltype(token), T, 1> : few_rows_kernel<decltype(token), T, E>;
            hipLaunchKernelGGL(kernel, dim3(one.blocks), dim3(FEW_WAVES * 64), 0, s, f);
        });
        return tokens_launched(call);
    }
    char* const base = static_cast<char*>(workspace);
    const uint32_t none = (uint32_t)(e->n_groups * e->vocab);
    const uint32_t* keys = nullptr;
    const uint32_t* order = nullptr;
    SortArgs a{tokens ? tokens->data_dev : nullptr, tokens ? tokens->stride : 0, e->vocab, (int32_t)e->rows, none, groups_of(*e)};
    const ClearArgs clear = clear_args(*e, *dtable);
    auto word = [&](uint64_t at) { return reinterpret_cast<uint32_t*>(base + at); };
    with_types(PS_F32, tokens && tokens->data_dev ? tokens->bytes : 4, [&](auto, auto token) {
        using TOKEN = decltype(token);
        if (!space.tiles) {
            const uint32_t ranks = (uint32_t)(up(e->rows, RANK_ROWS) * space.parts);
            const uint32_t places = (uint32_t)up(e->rows, RANK_THREADS), later = places ? clear.blocks / 8 : 0;
            const auto rank = none < 1 << 24 ? rank_and_clear_kernel<TOKEN, float> : rank_and_clear_kernel<TOKEN, uint32_t>;
            hipLaunchKernelGGL(rank, dim3(ranks + clear.blocks - later), dim3(RANK_THREADS), 0, s, a, ranks, space.parts, word(space.keys[1]),
                               reinterpret_cast<uint16_t*>(base + space.counts), clear);
            keys = word(space.keys[0]);
            order = word(space.order[0]);
            if (places)
                hipLaunchKernelGGL(rank_place_kernel, dim3(places + later), dim3(RANK_THREADS), 0, s, (int)e->rows, space.parts, places, word(space.keys[1]),
                                   reinterpret_cast<const uint16_t*>(base + space.counts), word(space.keys[0]), word(space.order[0]), clear);
            return;
        }
        for (int pass = 0; pass < space.passes; ++pass) {
            uint32_t *keys_to = word(space.keys[pass & 1]), *order_to = word(space.order[pass & 1]);
            hipLaunchKernelGGL(sort_count_kernel<TOKEN>, dim3(space.tiles + (pass ? 0 : clear.blocks)), dim3(DIGITS), 0, s, a, 8 * pass, keys, word(space.counts), space.tiles, clear);
            hipLaunchKernelGGL(sort_scan_kernel, dim3(DIGITS), dim3(DIGITS), 0, s, word(space.counts), space.tiles);
            hipLaunchKernelGGL(sort_place_kernel<TOKEN>, dim3((uint32_t)space.tiles), dim3(DIGITS), 0, s, a, 8 * pass, keys, order, word(space.counts), space.tiles, keys_to, order_to);
            keys = keys_to;
            order = order_to;
        }
    });
    if (!e->rows) return tokens_launched(call);
    SumArgs b{};
    b.dy = dy->data_dev;
    b.dy_row = dy->row;
    b.dtable = dtable->data_dev;
    b.table_row = dtable->row;
    b.table_matrix = dtable->matrix;
    b.keys = keys;
    b.order = order;
    b.partial = reinterpret_cast<float*>(base + space.partial);
    b.vocab = e->vocab;
    b.rows = (int32_t)e->rows;
    b.dim = (int32_t)e->dim;
    b.chunks = space.chunks;
    b.col_blocks = (int32_t)up(e->dim, 64 * 16 / dtype_size(e->dtype));  // (shorter rows: one, of 64 columns)
    b.none = none;
    b.scale = (float)e->scale;
    const int64_t waves = (int64_t)b.chunks * b.col_blocks;  // below 2^26, as a launch needs: 2^24 chunks at most, and 16 KB of dy for each one more
    with_types(e->dtype, 4, [&](auto t, auto) {
        using T = decltype(t);
        auto sum = [&](auto sum_runs, auto join_runs) {
            hipLaunchKernelGGL(sum_runs, dim3((uint32_t)up(waves, 4)), dim3(256), 0, s, b);
            if (e->rows > PIECE) hipLaunchKernelGGL(join_runs, dim3((uint32_t)std::min<int64_t>(up(b.chunks, JOIN_WAVES) * b.col_blocks, 1 << 18)), dim3(JOIN_WAVES * 64), 0, s, b);
        };
        constexpr int E = 16 / sizeof(T);
        if (e->dim < E)
            sum(sum_runs_kernel<T, 1>, join_runs_kernel<T, 1>);
        else
            sum(sum_runs_kernel<T, E>, join_runs_kernel<T, E>);
    });
    return tokens_launched(call);
}
