// Rows of a table for given tokens, and the gradient of the table (include/ps_tokens.h).
//
// The gradient is summed over sorted tokens: rows are put in the order of (group, token), those of equal ones staying in the order
// that they have (a stable radix sort, 8 bits at a time), and so the rows of one sum lie one behind the other.  No atomics: the
// same order every time.
#include "../../include/ps_tokens.h"
#include "ps_linear.h"
#include "ps_tokens.h"

#include <cmath>

namespace ps {
namespace {

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---- forward ---------------------------------------------------------------------------------------------------------

struct LookupArgs {
    const void *table, *tokens;
    void* out;
    int64_t table_row, table_matrix, out_row, token_stride, vocab;
    int32_t rows, dim, pieces;
    float scale;
    Groups groups;
};

// A thread takes 16 bytes of a row, four times; neighbours in a block take neighbouring pieces of the same row or the next one.  Bound
// by memory: the four are asked for together.
constexpr int LOOKUP_AHEAD = 4;

template <class T, class TOKEN>
__global__ __launch_bounds__(256) void lookup_kernel(LookupArgs a)
{
    constexpr int E = 16 / sizeof(T);
    const int64_t total = (int64_t)a.rows * a.pieces;
    for (int64_t first = (int64_t)blockIdx.x * (256 * LOOKUP_AHEAD); first < total; first += (int64_t)gridDim.x * (256 * LOOKUP_AHEAD)) {
        const int64_t row0 = first / a.pieces;
        const uint32_t rem = (uint32_t)(first - row0 * a.pieces);
        int64_t row[LOOKUP_AHEAD], token[LOOKUP_AHEAD];
        int col[LOOKUP_AHEAD], matrix[LOOKUP_AHEAD];
        T raw[LOOKUP_AHEAD][E];
#pragma unroll
        for (int i = 0; i < LOOKUP_AHEAD; ++i) {
            const uint32_t at = rem + i * 256 + threadIdx.x;
            row[i] = row0 + at / (uint32_t)a.pieces;
            col[i] = (int)(at % (uint32_t)a.pieces) * E;
            matrix[i] = -1;
            if (row[i] < a.rows) {
                token[i] = static_cast<const TOKEN*>(a.tokens)[row[i] * a.token_stride];
                const int g = group_of_row(a.groups, row[i]);
                if (g >= 0) matrix[i] = group_matrix(a.groups, g);
            }
        }
#pragma unroll
        for (int i = 0; i < LOOKUP_AHEAD; ++i) {
#pragma unroll
            for (int e = 0; e < E; ++e) raw[i][e] = T{};
            if (matrix[i] < 0 || token[i] < 0 || token[i] >= a.vocab) continue;
            const T* from = static_cast<const T*>(a.table) + matrix[i] * a.table_matrix + token[i] * a.table_row + col[i];
            if (col[i] + E <= a.dim) {
                __builtin_memcpy(raw[i], from, 16);
            } else {
                asm volatile("" : "+v"(from));
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (col[i] + e < a.dim) raw[i][e] = from[e];
            }
        }
#pragma unroll
        for (int i = 0; i < LOOKUP_AHEAD; ++i) {
            if (matrix[i] < 0) continue;
            float v[E];
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = to_float(raw[i][e]) * a.scale;
            if (token[i] < 0 || token[i] >= a.vocab) {  // also where the scale times 0 is not 0
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = 0.f;
            }
            T* to = static_cast<T*>(a.out) + row[i] * a.out_row + col[i];
            if (col[i] + E <= a.dim)
                store_n(to, v);
            else
                store_some(to, a.dim - col[i], v);
        }
    }
}

// ---- sorting -----------------------------------------------------------------------------------------------------------

// A tile of keys is ranked by a block: every wavefront has 64 at a time, finds with eight ballots which of them have the same
// digit, and counts them in a column of its own, so that equal digits stay in order.
constexpr int DIGITS = 256, TILE_WAVES = 16, TILE_EACH = 8, SORT_TILE = TILE_WAVES * 64 * TILE_EACH;

struct SortArgs {
    const void* tokens;
    int64_t token_stride, vocab;
    int32_t rows;
    uint32_t none;  // n_groups * vocab: the key of a row without a token or a group
    Groups groups;
};

template <class TOKEN>
__device__ __forceinline__ uint32_t key_of_row(const SortArgs& a, int r)
{
    const int64_t t = static_cast<const TOKEN*>(a.tokens)[r * a.token_stride];
    if (t < 0 || t >= a.vocab) return a.none;
    const int g = group_of_row(a.groups, r);
    return g < 0 ? a.none : (uint32_t)(g * a.vocab + t);
}

struct TileCounts {
    uint32_t at[TILE_WAVES][DIGITS];  // first counts, then where each wavefront's keys of a digit go
    uint32_t wave_sum[DIGITS / 64];
};

// Ranks of this thread's keys among those of the same digit of its wavefront.  Keys i * 64 + lane of a wavefront's TILE_EACH * 64.
__device__ __forceinline__ void rank_keys(TileCounts& c, const uint32_t (&key)[TILE_EACH], int shift, uint32_t (&rank)[TILE_EACH])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = lane; d < DIGITS; d += 64) c.at[wave][d] = 0;
    __builtin_amdgcn_wave_barrier();
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
        __builtin_amdgcn_wave_barrier();  // LDS serves a wavefront in order: all have read before one of them counts on
        if (!(same & below)) c.at[wave][d] = before + __popcll(same);
        __builtin_amdgcn_wave_barrier();
        rank[i] = before + __popcll(same & below);
    }
}

// Sum of v over the block's threads before this one, of DIGITS threads that call this.
__device__ __forceinline__ uint32_t sum_before(TileCounts& c, uint32_t v)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t upto = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t other = __shfl_up(upto, d, 64);
        if (lane >= d) upto += other;
    }
    if (threadIdx.x < DIGITS && lane == 63) c.wave_sum[wave] = upto;
    __syncthreads();
    uint32_t s = upto - v;
    for (int w = 0; w < DIGITS / 64; ++w)
        if (w < wave) s += c.wave_sum[w];
    return s;
}

// All of it in one block: up to SORT_TILE rows.
template <class TOKEN>
__global__ __launch_bounds__(TILE_WAVES * 64) void sort_one_kernel(SortArgs a, int passes, uint32_t* __restrict__ keys, uint32_t* __restrict__ order)
{
    __shared__ TileCounts counts;
    __shared__ uint32_t key_at[SORT_TILE];
    __shared__ uint16_t row_at[SORT_TILE];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = wave * 64 * TILE_EACH + lane;
    uint32_t key[TILE_EACH], rank[TILE_EACH];
    uint16_t row[TILE_EACH];
#pragma unroll
    for (int i = 0; i < TILE_EACH; ++i) {
        const int r = first + i * 64;
        row[i] = (uint16_t)r;
        key[i] = r < a.rows ? key_of_row<TOKEN>(a, r) : ~0u;  // behind all others, and the last among equal digits
    }
    for (int pass = 0; pass < passes; ++pass) {
        rank_keys(counts, key, 8 * pass, rank);
        __syncthreads();
        uint32_t total = 0;
        if (threadIdx.x < DIGITS)
            for (int w = 0; w < TILE_WAVES; ++w) total += counts.at[w][threadIdx.x];
        uint32_t to = sum_before(counts, total);
        if (threadIdx.x < DIGITS)
            for (int w = 0; w < TILE_WAVES; ++w) {
                const uint32_t n = counts.at[w][threadIdx.x];
                counts.at[w][threadIdx.x] = to;
                to += n;
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TILE_EACH; ++i) {
            const uint32_t p = counts.at[wave][key[i] >> (8 * pass) & (DIGITS - 1)] + rank[i];
            key_at[p] = key[i];
            row_at[p] = row[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TILE_EACH; ++i) {
            key[i] = key_at[first + i * 64];
            row[i] = row_at[first + i * 64];
        }
    }
#pragma unroll
    for (int i = 0; i < TILE_EACH; ++i) {
        if (first + i * 64 >= a.rows) continue;
        keys[first + i * 64] = key[i];
        order[first + i * 64] = row[i];
    }
}

// One pass over more tiles.  keys and order null: the first pass, whose keys are made from the tokens.
template <class TOKEN>
__device__ __forceinline__ void tile_keys(const SortArgs& a, const uint32_t* keys, int tile, uint32_t (&key)[TILE_EACH])
{
    const int64_t first = (int64_t)tile * SORT_TILE + (threadIdx.x >> 6) * 64 * TILE_EACH + (threadIdx.x & 63);
#pragma unroll
    for (int i = 0; i < TILE_EACH; ++i) {
        const int64_t r = first + i * 64;
        key[i] = r >= a.rows ? ~0u : keys ? keys[r] : key_of_row<TOKEN>(a, (int)r);
    }
}

// Counts of every digit: [digit][tile]
template <class TOKEN>
__global__ __launch_bounds__(TILE_WAVES * 64) void sort_count_kernel(SortArgs a, int shift, const uint32_t* __restrict__ keys, uint32_t* __restrict__ counts, int tiles)
{
    __shared__ TileCounts c;
    uint32_t key[TILE_EACH], rank[TILE_EACH];
    tile_keys<TOKEN>(a, keys, blockIdx.x, key);
    rank_keys(c, key, shift, rank);
    __syncthreads();
    if (threadIdx.x >= DIGITS) return;
    uint32_t total = 0;
    for (int w = 0; w < TILE_WAVES; ++w) total += c.at[w][threadIdx.x];
    counts[(int64_t)threadIdx.x * tiles + blockIdx.x] = total;
}

// A block for each digit: its counts to sums over the tiles before, their total to counts[DIGITS * tiles + digit].
__global__ __launch_bounds__(256) void sort_scan_kernel(uint32_t* __restrict__ counts, int tiles)
{
    __shared__ TileCounts c;
    uint32_t* mine = counts + (int64_t)blockIdx.x * tiles;
    uint32_t before = 0;
    for (int t0 = 0; t0 < tiles; t0 += 256) {
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
__global__ __launch_bounds__(TILE_WAVES * 64) void sort_place_kernel(SortArgs a, int shift, const uint32_t* __restrict__ keys, const uint32_t* __restrict__ order,
                                                                     const uint32_t* __restrict__ counts, int tiles, uint32_t* __restrict__ keys_to,
                                                                     uint32_t* __restrict__ order_to)
{
    __shared__ TileCounts c;
    uint32_t key[TILE_EACH], rank[TILE_EACH];
    tile_keys<TOKEN>(a, keys, blockIdx.x, key);
    rank_keys(c, key, shift, rank);
    __syncthreads();
    const uint32_t of_digit = threadIdx.x < DIGITS ? counts[(int64_t)DIGITS * tiles + threadIdx.x] : 0;
    uint32_t to = sum_before(c, of_digit);
    if (threadIdx.x < DIGITS) {
        to += counts[(int64_t)threadIdx.x * tiles + blockIdx.x];
        for (int w = 0; w < TILE_WAVES; ++w) {
            const uint32_t n = c.at[w][threadIdx.x];
            c.at[w][threadIdx.x] = to;
            to += n;
        }
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
constexpr int PIECE = 32, SUM_AHEAD = 8;

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

// The first place of `key` among the sorted keys before `end`, where it is itself.  For a whole wavefront.
__device__ __forceinline__ int first_place(const uint32_t* keys, uint32_t key, int end)
{
    int lo = 0, hi = end;  // keys before lo are below, the one at hi is not
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

// Wavefronts [chunk][64 * E columns]: the pieces that begin in the chunk's PIECE places; they end within PIECE - 1 places behind.
template <class T>
__global__ __launch_bounds__(256) void sum_runs_kernel(SumArgs a)
{
    constexpr int E = 16 / sizeof(T);
    const int lane = threadIdx.x & 63;
    const int64_t w = (int64_t)blockIdx.x * 4 + scalar(threadIdx.x >> 6);
    const int chunk = (int)(w / a.col_blocks), col = (int)(w % a.col_blocks) * 64 * E + lane * E, n = min(E, a.dim - col);
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
    unsigned long long todo = pieces & ((1ull << PIECE) - 1);
    if (!todo) return;
    // places from the first piece's beginning to where a piece that begins behind the chunk, or nothing, follows
    const int from = __builtin_ctzll(todo);
    const unsigned long long behind = pieces >> PIECE << PIECE | ~exist;  // (rows that exist come first)
    const int to = behind ? __builtin_ctzll(behind) : 64;
    float sum[E] = {};
    for (int at = from; at < to; at += SUM_AHEAD) {
        float x[SUM_AHEAD][E];
        T raw[SUM_AHEAD][E];
#pragma unroll
        for (int u = 0; u < SUM_AHEAD; ++u) {
            if (at + u >= to || n <= 0) continue;
            const T* src = static_cast<const T*>(a.dy) + (int64_t)(uint32_t)__builtin_amdgcn_readlane(row, at + u) * a.dy_row + col;
            if (n == E) {
                __builtin_memcpy(raw[u], src, 16);
            } else {
                asm volatile("" : "+v"(src));
#pragma unroll
                for (int e = 0; e < E; ++e) raw[u][e] = e < n ? src[e] : T{};
            }
        }
#pragma unroll
        for (int u = 0; u < SUM_AHEAD; ++u) {
            if (at + u >= to) continue;
            const int place = at + u;
            const bool first = pieces >> place & 1;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[u][e] = n > 0 ? to_float(raw[u][e]) : 0.f;
                sum[e] = first ? x[u][e] : sum[e] + x[u][e];
            }
            // the piece's end: the next place is another piece's first, or none
            if (place + 1 < 64 && !((pieces | ~exist) >> (place + 1) & 1)) continue;
            const uint32_t k = (uint32_t)__builtin_amdgcn_readlane(key, place);
            const unsigned long long starts = pieces & (~0ull >> (63 - place));
            const int start = 63 - __builtin_clzll(starts), run_at = __builtin_amdgcn_readlane(run, start);
            const bool goes_on = place + 1 < 64 && (exist >> (place + 1) & 1) && !(begins >> (place + 1) & 1);
            if (run_at == start && !goes_on) {
                float v[E];
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = sum[e] * a.scale;
                if (n > 0) store_columns(row_of_key<T>(a, k) + col, n, v);
            } else if (n > 0) {
                store_columns(a.partial + (2 * (int64_t)chunk + (run_at == start)) * a.dim + col, n, sum);
            }
        }
    }
}

// Adds up the pieces of longer runs, and clears the rows of tokens that are nowhere.  Wavefronts [chunk][columns] of the
// first `join` blocks: the run longer than PIECE that begins in the chunk; of the others, 64 rows of the tables each.
template <class T>
__global__ __launch_bounds__(256) void join_and_clear_kernel(SumArgs a, uint32_t join)
{
    constexpr int E = 16 / sizeof(T);
    const int lane = threadIdx.x & 63;
    if (blockIdx.x >= join) {
        const uint32_t first = ((blockIdx.x - join) * 4 + scalar(threadIdx.x >> 6)) * 64, key = first + lane;
        if (first >= a.none) return;
        int lo = 0, hi = a.rows;
        while (lo < hi) {
            const int mid = (int)(((uint32_t)lo + (uint32_t)hi) >> 1);
            if (a.keys[mid] < key)
                lo = mid + 1;
            else
                hi = mid;
        }
        const bool absent = key < a.none && (lo >= a.rows || a.keys[lo] != key);
        const float zero[E] = {};
        for (unsigned long long todo = __ballot(absent); todo; todo &= todo - 1) {
            T* to = row_of_key<T>(a, first + __builtin_ctzll(todo));
            for (int col = lane * E; col < a.dim; col += 64 * E) store_columns(to + col, a.dim - col, zero);
        }
        return;
    }
    const int64_t w = (int64_t)blockIdx.x * 4 + scalar(threadIdx.x >> 6);
    const int chunk = (int)(w / a.col_blocks), col = (int)(w % a.col_blocks) * 64 * E + lane * E, n = min(E, a.dim - col);
    if (chunk >= a.chunks) return;
    // the run that begins in the chunk and still goes on PIECE places behind
    const int p0 = chunk * PIECE, p = p0 + lane;
    const uint32_t key = p < a.rows ? a.keys[p] : ~0u, before = p0 ? a.keys[p0 - 1] : ~0u;
    const uint32_t previous = __shfl_up(key, 1, 64), later = __shfl_down(key, PIECE, 64);
    const bool differs = lane ? key != previous : p0 == 0 || key != before;
    const unsigned long long longer = __ballot(lane < PIECE && differs && p + PIECE < a.rows && key < a.none && key == later);
    if (!longer) return;
    const int at = __builtin_ctzll(longer);
    const uint32_t k = (uint32_t)__builtin_amdgcn_readlane(key, at);
    const int last_piece = (a.rows - 1 - (p0 + at)) / PIECE;
    float sum[E] = {}, x[E];
    for (int i = 0; i <= last_piece; ++i) {
        if (i > 1 && a.keys[p0 + at + i * PIECE] != k) break;
        const float* from = a.partial + (2 * (int64_t)(chunk + i) + (i == 0)) * a.dim + col;
        if (n <= 0) continue;
        load_columns<float>(from, 0, n, x);
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += x[e];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] *= a.scale;
    if (n > 0) store_columns(row_of_key<T>(a, k) + col, n, sum);
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
    if (e->n_groups * e->vocab > INT32_MAX) return dense_fail(PS_EINVAL, "%s: groups times vocab from 2^31 on", call);
    if (forward && (e->n_tables < 1 || (!e->table_of_group_dev && e->n_tables < e->n_groups)))
        return dense_fail(PS_EINVAL, "%s: fewer tables than groups, and no list of which each uses", call);
    if ((reinterpret_cast<uintptr_t>(e->offsets_dev) & 3) || (forward && (reinterpret_cast<uintptr_t>(e->table_of_group_dev) & 3)))
        return dense_fail(PS_EINVAL, "%s: misaligned offsets or list of tables", call);
    if (!std::isfinite(e->scale) || !std::isfinite((float)e->scale)) return dense_fail(PS_EINVAL, "%s: the scale is not finite", call);
    return PS_OK;
}

struct GradientSpace {
    uint64_t keys[2], order[2], counts, partial, total;
    int passes, tiles, chunks;
};

GradientSpace gradient_space(const ps_embedding& e)
{
    GradientSpace g{};
    const uint64_t none = (uint64_t)e.n_groups * e.vocab;
    while (none >> (8 * g.passes)) ++g.passes;
    g.tiles = (int)up(e.rows, SORT_TILE);
    g.chunks = (int)up(e.rows, PIECE);
    uint64_t at = 0;
    auto take = [&](uint64_t bytes) {
        const uint64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    for (int i = 0; i < (g.tiles > 1 ? 2 : 1); ++i) {
        g.keys[i] = take((uint64_t)e.rows * 4);
        g.order[i] = take((uint64_t)e.rows * 4);
    }
    g.counts = take(g.tiles > 1 ? (uint64_t)DIGITS * (g.tiles + 1) * 4 : 0);
    g.partial = take((uint64_t)2 * g.chunks * e.dim * 4);
    g.total = at;
    return g;
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
    a.pieces = (int32_t)up(e->dim * dtype_size(e->dtype), 16);
    a.scale = (float)e->scale;
    a.groups = groups_of(*e);
    const int64_t blocks = std::min<int64_t>(up(e->rows * a.pieces, 256 * LOOKUP_AHEAD), 1 << 20);
    with_types(e->dtype, tokens->bytes, [&](auto t, auto token) {
        hipLaunchKernelGGL((lookup_kernel<decltype(t), decltype(token)>), dim3((uint32_t)blocks), dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
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
    char* const base = static_cast<char*>(workspace);
    const uint32_t none = (uint32_t)(e->n_groups * e->vocab);
    const uint32_t* keys = nullptr;
    const uint32_t* order = nullptr;
    if (e->rows) {
        SortArgs a{tokens->data_dev, tokens->stride, e->vocab, (int32_t)e->rows, none, groups_of(*e)};
        auto word = [&](uint64_t at) { return reinterpret_cast<uint32_t*>(base + at); };
        with_types(PS_F32, tokens->bytes, [&](auto, auto token) {
            using TOKEN = decltype(token);
            if (space.tiles == 1) {
                hipLaunchKernelGGL(sort_one_kernel<TOKEN>, dim3(1), dim3(TILE_WAVES * 64), 0, s, a, space.passes, word(space.keys[0]), word(space.order[0]));
                keys = word(space.keys[0]);
                order = word(space.order[0]);
                return;
            }
            for (int pass = 0; pass < space.passes; ++pass) {
                uint32_t *keys_to = word(space.keys[pass & 1]), *order_to = word(space.order[pass & 1]);
                const dim3 grid((uint32_t)space.tiles), block(TILE_WAVES * 64);
                hipLaunchKernelGGL(sort_count_kernel<TOKEN>, grid, block, 0, s, a, 8 * pass, keys, word(space.counts), space.tiles);
                hipLaunchKernelGGL(sort_scan_kernel, dim3(DIGITS), dim3(256), 0, s, word(space.counts), space.tiles);
                hipLaunchKernelGGL(sort_place_kernel<TOKEN>, grid, block, 0, s, a, 8 * pass, keys, order, word(space.counts), space.tiles, keys_to, order_to);
                keys = keys_to;
                order = order_to;
            }
        });
    }
    SumArgs a{};
    a.dy = dy ? dy->data_dev : nullptr;
    a.dy_row = dy ? dy->row : 0;
    a.dtable = dtable->data_dev;
    a.table_row = dtable->row;
    a.table_matrix = dtable->matrix;
    a.keys = keys;
    a.order = order;
    a.partial = reinterpret_cast<float*>(base + space.partial);
    a.vocab = e->vocab;
    a.rows = (int32_t)e->rows;
    a.dim = (int32_t)e->dim;
    a.chunks = space.chunks;
    a.col_blocks = (int32_t)up(e->dim * dtype_size(e->dtype), 1024);
    a.none = none;
    a.scale = (float)e->scale;
    const uint32_t sums = (uint32_t)up((int64_t)a.chunks * a.col_blocks, 4), clear = (uint32_t)up(none, 256);  // (below 2^24: dy fits the memory)
    with_types(e->dtype, 4, [&](auto t, auto) {
        using T = decltype(t);
        if (sums) hipLaunchKernelGGL(sum_runs_kernel<T>, dim3(sums), dim3(256), 0, s, a);
        hipLaunchKernelGGL(join_and_clear_kernel<T>, dim3(sums + clear), dim3(256), 0, s, a, sums);
    });
    return tokens_launched(call);
}
