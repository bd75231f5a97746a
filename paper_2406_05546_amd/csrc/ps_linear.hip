// Entry points of the dense layers (include/ps_dense.h): checks, choice of tiles, workspaces, and the kernels around the
// products of ps_linear.h.
#include "ps_linear.h"

#include <cstdarg>
#include <cstdio>

namespace ps {

namespace {
thread_local char dense_error[256] = "";
}

ps_status dense_fail(ps_status st, const char* format, ...)
{
    va_list args;
    va_start(args, format);
    std::vsnprintf(dense_error, sizeof(dense_error), format, args);
    va_end(args);
    return st;
}

namespace {

// ---- dz = dy act'(z), and the sums over rows that are the bias's gradient ------------------------------------------

struct SlopeArgs {
    const void *dy, *pre;  // pre null: no activation
    void* dz;              // null: only the sums
    int64_t dy_row, pre_row, dz_row;
    int32_t act, cols, parts;
    float* partial;  // [group][part][cols], or null: no sums
    Groups groups;
};

// A block takes 512 columns (a lane eight consecutive ones) of one part of a group's rows, its four wavefronts every
// fourth row each; their sums meet in LDS in order.  Bound by memory, and next to it by the vector ALU (GELU's slope:
// 30 instructions a value): rows are asked for AHEAD at a time, before those that came are worked on (bf16 8192 x 8192 with GELU
// 114 -> 88-104 us, 3.9-4.6 TB/s; 8192 x 512 13.8 -> 9.6).
constexpr int SLOPE_COLS = 512;

template <class T>
__global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a)
{
    constexpr int AHEAD = sizeof(T) == 2 ? 4 : 2;
    __shared__ float meet[3][64][9];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int g = blockIdx.y / a.parts, part = blockIdx.y % a.parts;
    const GroupRows rows = group_rows(a.groups, g);
    const int each = (rows.end - rows.begin + a.parts - 1) / a.parts;
    const int begin = min(rows.begin + part * each, rows.end), end = min(begin + each, rows.end);
    const int col = blockIdx.x * SLOPE_COLS + lane * 8, n = min(8, a.cols - col);
    float sum[8] = {};
    struct Row {
        T dy[8], pre[8];
    };
    auto take = [&](int64_t r, Row& x) __attribute__((always_inline)) {
        __builtin_memcpy(x.dy, static_cast<const T*>(a.dy) + r * a.dy_row + col, sizeof(x.dy));
        if (a.pre) __builtin_memcpy(x.pre, static_cast<const T*>(a.pre) + r * a.pre_row + col, sizeof(x.pre));
    };
    auto give = [&](int64_t r, const Row& x) __attribute__((always_inline)) {
        float d[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = to_float(x.dy[i]);
        if (a.pre) {
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] *= activation_slope(to_float(x.pre[i]), a.act);
        }
        if (a.dz) {
            T* dz = static_cast<T*>(a.dz) + r * a.dz_row + col;
            if (n == 8)
                store_n(dz, d);
            else
                store_some(dz, (int)min(a.dz_row - col, (int64_t)8), d);  // zeros up to the end of its rows
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += d[i];
    };
    if (n == 8) {
        int64_t r = begin + wave;
        const int64_t last = end - 4 * (AHEAD - 1);  // AHEAD rows from a row below this one on
        Row now[AHEAD], then[AHEAD];
        if (r < last) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) take(r + 4 * u, now[u]);
        }
        for (; r < last; r += 4 * AHEAD) {
            const int64_t next = r + 4 * AHEAD;
            if (next < last) {
#pragma unroll
                for (int u = 0; u < AHEAD; ++u) take(next + 4 * u, then[u]);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) give(r + 4 * u, now[u]);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) now[u] = then[u];
        }
        for (; r < end; r += 4) {
            take(r, now[0]);
            give(r, now[0]);
        }
    } else if (n > 0) {
        for (int64_t r = begin + wave; r < end; r += 4) {
            Row x = {};
#pragma unroll
            for (int i = 0; i < 7; ++i) {
                if (i >= n) continue;
                x.dy[i] = static_cast<const T*>(a.dy)[r * a.dy_row + col + i];
                if (a.pre) x.pre[i] = static_cast<const T*>(a.pre)[r * a.pre_row + col + i];
            }
            give(r, x);
        }
    }
    if (!a.partial) return;
    if (wave > 0) {
#pragma unroll
        for (int i = 0; i < 8; ++i) meet[wave - 1][lane][i] = sum[i];
    }
    __syncthreads();
    if (wave == 0 && n > 0) {
#pragma unroll
        for (int w = 0; w < 3; ++w)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += meet[w][lane][i];
        float* to = a.partial + ((int64_t)g * a.parts + part) * a.cols + col;
        if (n == 8)
            store_n(to, sum);
        else
            store_some(to, n, sum);
    }
}

// Adds up the parts: a block takes 32 columns, each sixteenth of its threads a sixteenth of the parts, whose sums meet in order.
constexpr int BIAS_COLS = 32, BIAS_SHARES = 16;
template <class T>
__global__ __launch_bounds__(BIAS_COLS * BIAS_SHARES) void bias_sum_kernel(const float* __restrict__ partial, T* __restrict__ db, int64_t db_matrix, int cols, int parts)
{
    __shared__ float meet[BIAS_SHARES][BIAS_COLS];
    const int i = threadIdx.x % BIAS_COLS, share = threadIdx.x / BIAS_COLS, g = blockIdx.y, c = blockIdx.x * BIAS_COLS + i;
    const int each = (parts + BIAS_SHARES - 1) / BIAS_SHARES, first = share * each, last = min(first + each, parts);
    float s = 0.f;
    if (c < cols) {
#pragma unroll 4
        for (int k = first; k < last; ++k) s += partial[((int64_t)g * parts + k) * cols + c];
    }
    meet[share][i] = s;
    __syncthreads();
    if (share || c >= cols) return;
#pragma unroll
    for (int k = 1; k < BIAS_SHARES; ++k) s += meet[k][i];
    db[g * db_matrix + c] = from_float<T>(s);
}

// Adds up the parts of a contraction, in order, and finishes the sums.  (There are parts only where there is one group.)
template <class T>
__global__ __launch_bounds__(256) void join_parts_kernel(const float* __restrict__ partial, int parts, int rows, int cols, Groups groups, Epilogue epi)
{
    const int per_row = (cols + 7) / 8;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / per_row;
    if (row >= rows) return;
    const int col = (int)(i % per_row) * 8, n = min(8, cols - col);
    float v[8], x[8];
    for (int k = 0; k < parts; ++k) {
        const float* p = partial + ((int64_t)k * rows + row) * cols + col;
        if (n == 8)
            load_n(p, x);
        else
            load_some(p, n, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k ? v[e] + x[e] : x[e];
    }
    float bias[8], residual[8];
    load_bias<T>(epi, group_matrix(groups, 0), col, n, bias);
    load_residual<T>(epi, row, col, n, residual);
    if (epi.residual)
        finish<T, true>(epi, bias, residual, row, col, n, v);
    else
        finish<T, false>(epi, bias, residual, row, col, n, v);
}

// ---- operands of odd sizes ------------------------------------------------------------------------------------------

// Copies rows of `cols` elements to rows of `cols_to` (a multiple of 16 bytes) and matrices of `rows` to `rows_to`, zeros behind: 16 bytes to a thread.
template <class T>
__global__ __launch_bounds__(256) void pad_kernel(const T* __restrict__ from, int64_t row, int64_t matrix, int rows, int cols, T* __restrict__ to, int rows_to, int cols_to, int64_t pieces)
{
    constexpr int E = 16 / sizeof(T);
    const int per_row = cols_to / E;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * 256) {
        const int64_t line = i / per_row, m = line / rows_to;
        const int r = (int)(line - m * rows_to), c = (int)(i - line * per_row) * E;
        T v[E] = {};
        if (r < rows) {
            const T* p = from + m * matrix + r * row + c;
            if (c + E <= cols) {
                __builtin_memcpy(v, p, 16);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (c + e < cols) v[e] = p[e];
            }
        }
        __builtin_memcpy(to + line * cols_to + c, v, 16);
    }
}

// ---- plans ---------------------------------------------------------------------------------------------------------

enum { FORWARD, DX, DW };

struct Plan {
    int few;  // if not 0: forward pass or input gradient for few rows, so many times 16 of a group to a block
    int tile, parts, part_stages;
    int64_t tiles_r, tiles_c;
    uint64_t partial_bytes;
    double us;  // estimated; 0 for few rows
};

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Blocks of 512 threads in a launch, which has less than 2^32 threads.
constexpr int64_t FEW_BLOCKS = 1 << 23;

// Whether the forward pass takes the kernel for few rows, `each` in a group.  Each of its blocks, 16 columns, reads all rows of its
// group over the whole contraction; tiles read them once for 64 columns or more, and cut the contraction of one group into parts.  So it
// is the faster one up to about so many values for each compute unit.  us, this kernel against tiles (bf16 if not said):
//   one group      4096 -> 4096   16 rows 11.5, 16.9   24 14.8, 15.6   32 16.4, 15.9   64 24.0, 16.9   fp32 24 27.5, 28.6   48 37.3, 33.0
//                  1024 -> 16384   1 8.4, 14.9   24 14.3, 15.2   32 16.3, 15.4   64 24.2, 15.5   4096 -> 16384   4 27.6, 30.0   16 36.7, 31.3
//                  1024 -> 1024   64 7.3, 10.6   2048 -> 512   48 9.8, 9.9   64 11.6, 9.9   512 -> 8192   64 9.1, 9.2
//   deep, narrow   16384 -> 512    1 23.3, 19.3   fp32 8192 -> 512   1 35.6, 21.3   8192 -> 2048   1 38.5, 33.7
//   odd rows       1111 -> 2777   48 12.9, 13.6   64 15.6, 13.7   4097 -> 4099   1 20.2, 18.7   4 29.3, 19.4   (32 bits:   12 29.2, 36.8)
//   groups         64 of 2048 -> 1024   8 rows each 61, 70   16 74, 69   64 172, 71   all 4096 rows in one 152, 28   fp32 8 136, 148
//                  16 of them   32 30.5, 29.3   48 37.5, 29.6   2 of 4096 -> 4096   64 45, 51   64 of 512 -> 512   4 11.8, 12.0   16 15.1, 12.4
//                  fp32 63 of 960 -> 4352   2 224, 296
bool few_rows(const ps_linear& l, int64_t each)
{
    if (each > 64) return false;
    if (l.offsets_dev) return each <= 4 || l.rows * l.out_features <= 1 << 19;
    const int size = dtype_size(l.dtype);
    const int64_t values = l.in_features * std::max<int64_t>(l.out_features, 4096) / 4096;  // of one row, to a compute unit
    if (l.out_features < 4096 && l.in_features * size > 16384) return false;
    if (size == 2 && l.in_features % 8) return (each + 16) * values <= 73728;
    return each * values <= 98304;
}

Plan plan_product(const ps_linear& l, int kind, bool direct)
{
    const int64_t rows = kind == DW ? l.out_features : l.rows, cols = kind == FORWARD ? l.out_features : l.in_features;
    const int64_t depth = kind == FORWARD ? l.in_features : kind == DX ? l.out_features : l.rows;
    const bool one = !l.offsets_dev;
    Plan best{};
    const int64_t each = up(l.rows, l.n_groups);
    if (kind == FORWARD && few_rows(l, each)) {
        best.few = (int)std::max<int64_t>(1, up(each, 16));
        best.parts = 1;
        best.tiles_r = up(l.rows, 16 * best.few) + (one ? 0 : l.n_groups);
        best.tiles_c = up(l.out_features, 16);
        if (best.tiles_r * best.tiles_c < FEW_BLOCKS) return best;
        best = Plan{};
    }
    const int size = dtype_size(l.dtype);
    if (kind == DX && each <= 32 && l.in_features * size >= 16) {  // (ps_linear_few.hip says what both sides measured)
        best.few = each <= 16 ? 1 : 2;
        best.tiles_r = up(l.rows, 16 * best.few) + (one ? 0 : l.n_groups);
        best.tiles_c = up(l.in_features, 256 / size);
        // parts as many as make two blocks to a compute unit, of two steps to a wavefront at least
        const int64_t steps = up(depth, FEW_DX_STEP / size), tiles = std::max<int64_t>(1, best.tiles_r * best.tiles_c);
        const int64_t parts = one ? std::max<int64_t>(1, std::min(2 * COMPUTE_UNITS / tiles, steps / 16)) : 1;
        best.part_stages = (int)up(steps, parts);
        best.parts = (int)up(steps, best.part_stages);
        best.partial_bytes = best.parts > 1 ? (uint64_t)best.parts * rows * cols * 4 : 0;
        if (tiles * best.parts < FEW_BLOCKS) return best;
        best = Plan{};
    }
    // The form that should take least, by what its blocks take when one, or as many as there is room for, are on a compute
    // unit.  What that chooses, in us against the other tiles (256, 128, 64; bf16 if not said): 4096^3 256: 110, 133, 194; 8192 rows
    // 1568 -> 512 128: 53, 20, 27; 1024^3 64: 27, 20, 10; 256 rows 4096 -> 4096 128 in parts: 35, 24, 32; weight gradient of
    // 8192 rows 1568 -> 512 128 in parts: 53, 30, 38, in fp32 128 in parts: -, 92, 146.
    const int stages = (int)up(depth, 128 / size);
    const bool wide = l.dtype == PS_F32;
    for (int tile = wide || !direct ? 1 : 2; tile >= 0; --tile) {
        const int side = LINEAR_TILE[tile], room = tile == 2 ? 1 : tile == 1 ? 2 : 4;  // blocks to a compute unit
        // operands through registers, which in 16 bits are turned element by element where they lie along the result
        const double through = direct ? 1 : wide ? (tile ? 1.5 : 1.1) : (tile ? 2 : 1.6) * (kind == FORWARD ? 1 : 2);
        const double alone = (wide ? (tile ? 1.6 : 0.6) : tile == 2 ? 1.6 : tile == 1 ? 0.6 : 0.35) * through;  // us a stage
        const double full = (wide ? (tile ? 2.8 : 2.2) : tile == 2 ? 1.6 : tile == 1 ? 1.0 : 0.75) * through;
        const double around = tile == 2 ? 7 : 3.5;  // us of a block's first loads and its stores
        Plan p{};
        p.tile = tile;
        // groups that are cut up separately have at most one tile more each than all rows together
        p.tiles_r = kind == DW ? up(rows, side) * l.n_groups : up(rows, side) + (one ? 0 : l.n_groups);
        p.tiles_c = up(cols, side);
        const int64_t likely = (kind == DW ? p.tiles_r : up(rows, side) + (one ? 0 : l.n_groups / 2)) * p.tiles_c;  // half a tile more each
        const int of_group = (int)(kind == DW ? std::max<int64_t>(1, stages / l.n_groups) : stages);
        // one part, or as many as all blocks that there is room for at once (or half or a quarter of them) make of it
        const int64_t tiles = std::max<int64_t>(1, p.tiles_r * p.tiles_c), most = one ? std::min<int64_t>(32, stages / 4) : 1;
        for (int fill : {0, 4, 2, 1}) {
            const int parts = fill ? (int)std::min<int64_t>(most, room * COMPUTE_UNITS / fill / tiles) : 1;
            if (fill && parts < 2) continue;
            p.part_stages = (int)up(stages, parts);
            p.parts = (int)up(std::max(stages, 1), std::max(p.part_stages, 1));
            p.partial_bytes = parts > 1 ? (uint64_t)p.parts * rows * cols * 4 : 0;
            const int64_t blocks = likely * p.parts, rounds = up(blocks, (int64_t)room * COMPUTE_UNITS);
            const double on_a_unit = std::min<double>(room, (double)up(blocks, COMPUTE_UNITS));
            const double stage = room > 1 ? alone + (full - alone) * (on_a_unit - 1) / (room - 1) : full;
            p.us = (double)rounds * (around + stage * std::min(of_group, std::max(p.part_stages, 1)));
            if (parts > 1) p.us += 4 + (double)p.partial_bytes * 1.5 / 4e6;  // written, read and joined
            if (!best.tiles_r || p.us < best.us) best = p;
        }
    }
    return best;
}

int slope_parts(const ps_linear& l)
{
    const int64_t blocks = up(l.out_features, SLOPE_COLS) * l.n_groups;
    return (int)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(up(4 * COMPUTE_UNITS, blocks), up(up(l.rows, l.n_groups), 16)), 65535 / std::min<int64_t>(l.n_groups, 65535)));
}

uint64_t up256(uint64_t b) { return (b + 255) / 256 * 256; }

bool direct_possible(const ps_linear& l, int kind)
{
    const int64_t e = 16 / dtype_size(l.dtype);
    return l.in_features % e == 0 && (kind == FORWARD || l.out_features % e == 0);
}

// Where rows are no multiples of 16 bytes, operands come through registers, in 1.5 (fp32) to 4 times the time, or are copied
// first to rows that are; then the copies come straight to LDS.  Copied if the plans differ by more than copying takes: backward of 7335 rows
// 949 -> 4658 with GELU in bf16 1076 -> 285 us, in fp32 1370 -> 1035, forward 168 -> 124 and 576 -> 405; of 3414 rows 1665 -> 605 in bf16 121 -> 63.
// (The kernels for few rows take any alignment.)
struct Padded {
    int64_t in, out;  // features, up to multiples of 16 bytes
    uint64_t x, w, dz;  // bytes of the copies
};
Padded padded(const ps_linear& l)
{
    const int size = dtype_size(l.dtype), e = 16 / size;
    Padded p{up(l.in_features, e) * e, up(l.out_features, e) * e, 0, 0, 0};
    p.x = up256((uint64_t)l.rows * p.in * size);
    p.w = up256((uint64_t)l.n_weights * p.out * p.in * size);
    p.dz = up256((uint64_t)l.rows * p.out * size);
    return p;
}
bool worth_padding(const ps_linear& l, int kind)
{
    if (direct_possible(l, kind)) return false;
    const Padded p = padded(l);
    const bool dz = l.activation == PS_ACT_NONE;  // with an activation it is in such rows already
    const double bytes = 2. * (kind == FORWARD ? p.x + p.w : (kind == DX ? p.w : p.x) + (dz ? p.dz : 0));
    return plan_product(l, kind, false).us > plan_product(l, kind, true).us + bytes / 4e6 + (kind == FORWARD || dz ? 10 : 5);
}

struct BackwardSpace {
    uint64_t dz, bias, partial, x, w, total;
    int64_t dz_row;
    int parts;
    bool pad_dx, pad_dw;
};

BackwardSpace backward_space(const ps_linear& l)
{
    BackwardSpace b{};
    const Padded p = padded(l);
    b.dz_row = p.out;
    b.parts = slope_parts(l);
    b.pad_dx = worth_padding(l, DX);
    b.pad_dw = worth_padding(l, DW);
    const uint64_t dz = l.activation != PS_ACT_NONE || b.pad_dx || b.pad_dw ? p.dz : 0;
    const uint64_t bias = up256((uint64_t)l.n_groups * b.parts * l.out_features * 4);
    uint64_t partial = 0;
    for (int kind : {DX, DW})
        for (bool direct : {true, false}) partial = std::max(partial, plan_product(l, kind, direct).partial_bytes);
    b.dz = 0;
    b.bias = dz;
    b.partial = dz + bias;
    b.x = b.partial + up256(partial);
    b.w = b.x + (b.pad_dw ? p.x : 0);
    b.total = b.w + (b.pad_dx ? p.w : 0);
    return b;
}

struct ForwardSpace {
    uint64_t x, w, total;
    bool pad;
};

ForwardSpace forward_space(const ps_linear& l)
{
    ForwardSpace f{};
    f.pad = worth_padding(l, FORWARD);
    f.x = up256(std::max(plan_product(l, FORWARD, true).partial_bytes, plan_product(l, FORWARD, false).partial_bytes));
    f.w = f.x + (f.pad ? padded(l).x : 0);
    f.total = f.w + (f.pad ? padded(l).w : 0);
    return f;
}

// ---- checks --------------------------------------------------------------------------------------------------------

ps_status check_layer(const char* call, const ps_linear* l)
{
    if (!l) return dense_fail(PS_EINVAL, "%s: no layer", call);
    if (l->dtype != PS_F32 && l->dtype != PS_BF16 && l->dtype != PS_F16) return dense_fail(PS_EINVAL, "%s: unknown type", call);
    if (l->activation < PS_ACT_NONE || l->activation > PS_ACT_SILU) return dense_fail(PS_EINVAL, "%s: unknown activation", call);
    if (l->rows < 0 || l->rows > PS_DENSE_MAX_ROWS) return dense_fail(PS_EINVAL, "%s: rows outside 0 .. %d", call, PS_DENSE_MAX_ROWS);
    if (l->in_features < 1 || l->in_features > PS_DENSE_MAX_STRIDE || l->out_features < 1 || l->out_features > PS_DENSE_MAX_STRIDE)
        return dense_fail(PS_EINVAL, "%s: features outside 1 .. %d", call, PS_DENSE_MAX_STRIDE);
    if (l->n_groups < 1 || l->n_groups > PS_DENSE_MAX_GROUPS) return dense_fail(PS_EINVAL, "%s: groups outside 1 .. %d", call, PS_DENSE_MAX_GROUPS);
    if (!l->offsets_dev && l->n_groups != 1) return dense_fail(PS_EINVAL, "%s: several groups need offsets", call);
    if (l->n_weights < 1 || (!l->weight_of_group_dev && l->n_weights < l->n_groups))
        return dense_fail(PS_EINVAL, "%s: fewer weight matrices than groups, and no list of which each uses", call);
    if ((reinterpret_cast<uintptr_t>(l->offsets_dev) & 3) || (reinterpret_cast<uintptr_t>(l->weight_of_group_dev) & 3))
        return dense_fail(PS_EINVAL, "%s: misaligned offsets or list of weight matrices", call);
    // Grids are counted in 32 bits.  (Results of so many tiles fit no memory, but groups without rows count as well.)
    const int64_t by_r = up(l->rows, 64) + l->n_groups, by_in = up(l->in_features, 64), by_out = up(l->out_features, 64);
    if (std::max({by_r * by_out, by_r * by_in, by_out * by_in * l->n_groups}) > INT32_MAX / 2) return dense_fail(PS_EINVAL, "%s: too many tiles", call);
    return PS_OK;
}

// m may be null if it need not be there.
ps_status check_matrix(const char* call, const char* name, const ps_linear& l, const ps_matrix* m, bool needed, int64_t rows, int64_t cols, int64_t matrices)
{
    if (!m || (!m->data_dev && rows)) return needed && rows ? dense_fail(PS_EINVAL, "%s: %s is missing", call, name) : PS_OK;
    const int size = dtype_size(l.dtype);
    if (reinterpret_cast<uintptr_t>(m->data_dev) & (size - 1)) return dense_fail(PS_EINVAL, "%s: %s is not aligned to its elements", call, name);
    if (rows > 1 && (m->row < cols || m->row > PS_DENSE_MAX_STRIDE)) return dense_fail(PS_EINVAL, "%s: %s has rows that overlap or are too far apart", call, name);
    if (matrices > 1 && m->matrix < (rows - 1) * m->row + cols) return dense_fail(PS_EINVAL, "%s: %s has matrices that overlap", call, name);
    return PS_OK;
}

bool there(const ps_matrix* m) { return m && m->data_dev; }

// Base, rows and matrices at multiples of 16 bytes
bool aligned16(const ps_linear& l, const void* data, int64_t row, int64_t matrix, bool one_row, bool one_matrix)
{
    const int64_t e = 16 / dtype_size(l.dtype);
    return (reinterpret_cast<uintptr_t>(data) & 15) == 0 && (one_row || row % e == 0) && (one_matrix || matrix % e == 0);
}
bool aligned16(const ps_linear& l, const ps_matrix& m, int64_t rows, int64_t matrices)
{
    return aligned16(l, m.data_dev, m.row, m.matrix, rows <= 1, matrices <= 1);
}

Groups groups_of(const ps_linear& l) { return Groups{l.offsets_dev, l.weight_of_group_dev, l.n_groups, l.n_weights, (int32_t)l.rows}; }

template <class F>
void with_type(int dtype, F f)
{
    if (dtype == PS_F32)
        f(float{});
    else if (dtype == PS_BF16)
        f(bf16_t{});
    else
        f(f16_t{});
}

// A copy of [matrices][rows][cols] in rows of a multiple of 16 bytes, zeros behind rows and columns.
ps_matrix pad(const ps_linear& l, const ps_matrix& m, int64_t matrices, int64_t rows, int64_t cols, int64_t rows_to, int64_t cols_to, void* to, hipStream_t s)
{
    const int64_t pieces = matrices * rows_to * cols_to * dtype_size(l.dtype) / 16;
    if (pieces)
        with_type(l.dtype, [&](auto t) {
            using T = decltype(t);
            hipLaunchKernelGGL(pad_kernel<T>, dim3((uint32_t)std::min<int64_t>(up(pieces, 256), 16 * COMPUTE_UNITS)), dim3(256), 0, s, static_cast<const T*>(m.data_dev),
                               m.row, m.matrix, (int)rows, (int)cols, static_cast<T*>(to), (int)rows_to, (int)cols_to, pieces);
        });
    return ps_matrix{to, cols_to, rows_to * cols_to};
}

// copied: both operands are padded copies.
void run_product(const ps_linear& l, int kind, bool direct, bool copied, const ps_matrix& r, const ps_matrix& c, Epilogue epi, float* partial, hipStream_t s)
{
    const Plan plan = plan_product(l, kind, direct);
    const int64_t in = copied ? padded(l).in : l.in_features, out = copied ? padded(l).out : l.out_features;
    Product p{};
    p.r = r.data_dev;
    p.c = c.data_dev;
    // a single row's distance to the next may be anything, but the kernels multiply with it
    p.r_row = l.rows > 1 ? r.row : kind == FORWARD ? in : out;
    p.c_row = (kind == DW ? l.rows : out) > 1 ? c.row : in;
    p.c_matrix = c.matrix;
    p.out_rows = (int32_t)(kind == DW ? l.out_features : l.rows);
    p.out_cols = (int32_t)(kind == FORWARD ? l.out_features : l.in_features);
    p.rows = (int32_t)(kind == DW ? out : l.rows);
    p.cols = (int32_t)(kind == FORWARD ? l.out_features : in);
    p.depth = (int32_t)(kind == FORWARD ? in : kind == DX ? out : l.rows);
    p.tiles_r = (int32_t)plan.tiles_r;
    p.tiles_c = (int32_t)plan.tiles_c;
    p.parts = plan.parts;
    p.part_stages = plan.part_stages;
    p.groups = groups_of(l);
    p.epi = epi;
    if (plan.parts > 1) p.epi.partial = partial;
    if (plan.few)
        (kind == FORWARD ? launch_linear_few : launch_linear_few_dx)(p, l.dtype, plan.few, s);
    else
        (kind == FORWARD ? launch_linear_forward : kind == DX ? launch_linear_dx : launch_linear_dw)(p, l.dtype, direct, plan.tile, s);
    if (plan.parts > 1) {
        const int64_t threads = up(p.out_cols, 8) * p.out_rows;
        with_type(l.dtype, [&](auto t) {
            hipLaunchKernelGGL((join_parts_kernel<decltype(t)>), dim3((uint32_t)up(threads, 256)), dim3(256), 0, s, partial, plan.parts, p.out_rows, p.out_cols, p.groups, epi);
        });
    }
}

ps_status launched(const char* call)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PS_OK : dense_fail(PS_EDEVICE, "%s: %s", call, hipGetErrorString(e));
}

}  // namespace
}  // namespace ps

extern "C" const char* ps_dense_last_error(void) { return ps::dense_error; }

extern "C" ps_status ps_linear_workspace_bytes(const ps_linear* l, int32_t backward, uint64_t* bytes_out)
{
    using namespace ps;
    const ps_status st = check_layer("ps_linear_workspace_bytes", l);
    if (st != PS_OK) return st;
    if (!bytes_out) return dense_fail(PS_EINVAL, "ps_linear_workspace_bytes: no place for the result");
    *bytes_out = backward ? backward_space(*l).total : forward_space(*l).total;
    return PS_OK;
}

extern "C" ps_status ps_linear_forward(const ps_linear* l, const ps_matrix* x, const ps_matrix* w, const ps_matrix* bias, const ps_matrix* residual,
                                       const ps_matrix* y, const ps_matrix* pre, void* workspace, uint64_t workspace_bytes, void* hip_stream)
{
    using namespace ps;
    static const char call[] = "ps_linear_forward";
    ps_status st = check_layer(call, l);
    if (st != PS_OK) return st;
    if ((st = check_matrix(call, "x", *l, x, true, l->rows, l->in_features, 1)) != PS_OK) return st;
    if ((st = check_matrix(call, "w", *l, w, true, l->out_features, l->in_features, l->n_weights)) != PS_OK) return st;
    if ((st = check_matrix(call, "bias", *l, bias, false, 1, l->out_features, l->n_weights)) != PS_OK) return st;
    if ((st = check_matrix(call, "residual", *l, residual, false, l->rows, l->out_features, 1)) != PS_OK) return st;
    if ((st = check_matrix(call, "y", *l, y, true, l->rows, l->out_features, 1)) != PS_OK) return st;
    if ((st = check_matrix(call, "pre", *l, pre, false, l->rows, l->out_features, 1)) != PS_OK) return st;
    if (!l->rows) return PS_OK;
    const ForwardSpace space = forward_space(*l);
    const uint64_t need = space.total;
    if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))) return dense_fail(PS_EINVAL, "%s: null or misaligned workspace", call);
    if (workspace_bytes < need) return dense_fail(PS_ENOMEM, "%s: workspace too small", call);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    Epilogue e{};
    e.out = y->data_dev;
    e.out_row = y->row;
    if (there(bias)) e.bias = bias->data_dev, e.bias_matrix = bias->matrix;
    if (there(residual)) e.residual = residual->data_dev, e.residual_row = residual->row;
    if (there(pre)) e.pre = pre->data_dev, e.pre_row = pre->row;
    e.act = l->activation;
    const bool direct = direct_possible(*l, FORWARD) && aligned16(*l, *x, l->rows, 1) && aligned16(*l, *w, l->out_features, l->n_weights);
    char* const base = static_cast<char*>(workspace);
    if (space.pad) {
        const Padded to = padded(*l);
        const ps_matrix xp = pad(*l, *x, 1, l->rows, l->in_features, l->rows, to.in, base + space.x, s);
        const ps_matrix wp = pad(*l, *w, l->n_weights, l->out_features, l->in_features, to.out, to.in, base + space.w, s);
        run_product(*l, FORWARD, true, true, xp, wp, e, reinterpret_cast<float*>(base), s);
    } else {
        run_product(*l, FORWARD, direct, false, *x, *w, e, reinterpret_cast<float*>(base), s);
    }
    return launched(call);
}

extern "C" ps_status ps_linear_backward(const ps_linear* l, const ps_matrix* dy, const ps_matrix* x, const ps_matrix* w, const ps_matrix* pre,
                                        const ps_matrix* dx, const ps_matrix* dw, const ps_matrix* db, void* workspace, uint64_t workspace_bytes,
                                        void* hip_stream)
{
    using namespace ps;
    static const char call[] = "ps_linear_backward";
    ps_status st = check_layer(call, l);
    if (st != PS_OK) return st;
    const bool act = l->activation != PS_ACT_NONE, want_dx = there(dx), want_dw = there(dw), want_db = there(db);
    if ((st = check_matrix(call, "dy", *l, dy, true, l->rows, l->out_features, 1)) != PS_OK) return st;
    if ((st = check_matrix(call, "x", *l, x, want_dw, l->rows, l->in_features, 1)) != PS_OK) return st;
    if ((st = check_matrix(call, "w", *l, w, want_dx, l->out_features, l->in_features, l->n_weights)) != PS_OK) return st;
    if ((st = check_matrix(call, "pre", *l, pre, act, l->rows, l->out_features, 1)) != PS_OK) return st;
    if ((st = check_matrix(call, "dx", *l, dx, false, l->rows, l->in_features, 1)) != PS_OK) return st;
    if ((st = check_matrix(call, "dw", *l, dw, false, l->out_features, l->in_features, l->n_groups)) != PS_OK) return st;
    if ((st = check_matrix(call, "db", *l, db, false, 1, l->out_features, l->n_groups)) != PS_OK) return st;
    if (!want_dx && !want_dw && !want_db) return PS_OK;
    const BackwardSpace space = backward_space(*l);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return dense_fail(PS_EINVAL, "%s: null or misaligned workspace", call);
    if (workspace_bytes < space.total) return dense_fail(PS_ENOMEM, "%s: workspace too small", call);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    char* const base = static_cast<char*>(workspace);
    const ps_matrix none{nullptr, 0, 0};
    ps_matrix dz = dy ? *dy : none;
    if (act) dz = ps_matrix{base + space.dz, space.dz_row, 0};
    if (act || want_db) {
        SlopeArgs a{};
        a.dy = dy ? dy->data_dev : nullptr;
        a.dy_row = dy ? dy->row : 0;
        if (act && there(pre)) a.pre = pre->data_dev, a.pre_row = pre->row;
        if (act && (want_dx || want_dw)) a.dz = dz.data_dev, a.dz_row = dz.row;
        a.act = l->activation;
        a.cols = (int32_t)l->out_features;
        a.parts = space.parts;
        a.groups = groups_of(*l);
        if (want_db) a.partial = reinterpret_cast<float*>(base + space.bias);
        const int64_t many = (int64_t)l->n_groups * space.parts;
        with_type(l->dtype, [&](auto t) {
            using T = decltype(t);
            hipLaunchKernelGGL(slope_kernel<T>, dim3((uint32_t)up(l->out_features, SLOPE_COLS), (uint32_t)many), dim3(256), 0, s, a);
            if (want_db)
                hipLaunchKernelGGL(bias_sum_kernel<T>, dim3((uint32_t)up(l->out_features, BIAS_COLS), (uint32_t)l->n_groups), dim3(BIAS_COLS * BIAS_SHARES), 0, s, a.partial,
                                   static_cast<T*>(db->data_dev), db->matrix, (int)l->out_features, space.parts);
        });
    }
    float* const partial = reinterpret_cast<float*>(base + space.partial);
    const Padded to = padded(*l);
    const bool pad_dx = want_dx && space.pad_dx, pad_dw = want_dw && space.pad_dw;
    ps_matrix dzp = dz;
    if ((pad_dx || pad_dw) && !act) dzp = pad(*l, dz, 1, l->rows, l->out_features, l->rows, to.out, base + space.dz, s);
    if (want_dx && l->rows) {
        Epilogue e{};
        e.out = dx->data_dev;
        e.out_row = dx->row;
        const bool direct = direct_possible(*l, DX) && aligned16(*l, dz, l->rows, 1) && aligned16(*l, *w, l->out_features, l->n_weights);
        if (pad_dx)
            run_product(*l, DX, true, true, dzp, pad(*l, *w, l->n_weights, l->out_features, l->in_features, to.out, to.in, base + space.w, s), e, partial, s);
        else
            run_product(*l, DX, direct, false, dz, *w, e, partial, s);
    }
    if (want_dw) {
        Epilogue e{};
        e.out = dw->data_dev;
        e.out_row = dw->row;
        e.out_matrix = dw->matrix;
        const ps_matrix xm = x ? *x : none;
        const bool direct = direct_possible(*l, DW) && aligned16(*l, dz, l->rows, 1) && aligned16(*l, xm, l->rows, 1);
        if (pad_dw)
            run_product(*l, DW, true, true, dzp, pad(*l, xm, 1, l->rows, l->in_features, l->rows, to.in, base + space.x, s), e, partial, s);
        else
            run_product(*l, DW, direct, false, dz, xm, e, partial, s);
    }
    return launched(call);
}
