// Forward pass and input gradient for few rows (a token, a few sequences, few rows of each of many groups): bound by reading the weights
// once, so these go straight to registers, and all wavefronts of a block read the same 16 columns' weights, each its share
// of k.  bf16: 64 matrices of 2048 -> 1024 and 96 rows 44 us (6.1 TB/s), one row 4096 -> 4096 7.8 us (4.3 TB/s: in a launch
// this short the trips to memory that wait for each other, bias, residual and the first weights, are a good part).
#include "ps_linear.h"

namespace ps {

namespace {

// A block: 16 columns, 16 * TR rows of a group.  128 bytes of k of each column make a step (a lane 32 bytes of its column, so that
// a load instruction touches half cache lines in pairs, whole ones together), and wavefront w takes every WAVES-th step.  Which
// k a lane's values have does not matter as long as both operands agree.  The wavefronts' sums are added up in order.
template <class T, int TR, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void linear_few_kernel(Product p)
{
    constexpr int E = Mma<T>::E, STEP = 8 * E, AHEAD = TR > 2 ? 2 : 4;
    __shared__ floatx4 meet[WAVES][TR][64];
    const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6), l = lane & 15, q = lane >> 4;
    const int tc = blockIdx.x % p.tiles_c, tr = blockIdx.x / p.tiles_c;
    GroupRows rows;
    int r0;
    if (!find_rows(p.groups, tr, 16 * TR, rows, r0)) return;
    const int matrix = group_matrix(p.groups, rows.g), c0 = tc * 16;

    // Rows and columns past the end read the last ones again; nobody stores them.
    const T* c = static_cast<const T*>(p.c) + matrix * p.c_matrix + (int64_t)min(c0 + l, p.cols - 1) * p.c_row;
    const T* r[TR];
#pragma unroll
    for (int i = 0; i < TR; ++i) r[i] = static_cast<const T*>(p.r) + (int64_t)min(r0 + 16 * i + l, rows.end - 1) * p.r_row;

    // lane (q, l) of wavefront w finishes row l of row tile w, columns 4q .. 4q + 3.  What is added to them is read first, and
    // waited for: it is converted in the branch that loads it.
    const int row = r0 + 16 * wave + l, col = c0 + 4 * q, valid = wave < TR && row < rows.end ? p.cols - col : 0;
    float bias[4], residual[4];
    load_bias<T>(p.epi, matrix, col, valid, bias);
    load_residual<T>(p.epi, row, col, valid, residual);

    floatx4 acc[TR];
#pragma unroll
    for (int i = 0; i < TR; ++i) acc[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    struct Pair {
        uintx4 v[2];
    };
    auto whole = [&](const T* row, int k) __attribute__((always_inline)) {
        Pair x;
        __builtin_memcpy(&x, row + k, 32);
        return x;
    };
    // The last, partial step: zeros past the end of the row.  A row of a step's share of a lane or more is read once more up to its end,
    // and what other lanes have of it is cleared, in both operands (it may be infinite); element by element, the
    // wavefront that has this step took longer than all others for theirs (37 rows of 1111 -> 2777 in fp16: 17.1 us, this way 12.3, with three row tiles 11.0).
    auto some = [&](const T* row, int k) __attribute__((always_inline)) {
        Pair x = {};
        if (p.depth >= 2 * E) {
            const int at = min(k, p.depth - 2 * E), drop = k - at;  // the first `drop` elements are others'
            x = whole(row, at);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t v = x.v[i / 4][i % 4];
                if constexpr (sizeof(T) == 4)
                    x.v[i / 4][i % 4] = i < drop ? 0u : v;
                else
                    x.v[i / 4][i % 4] = 2 * i + 1 < drop ? 0u : 2 * i < drop ? v & 0xffff0000u : v;
            }
            return x;
        }
        T e[2 * E];
        __builtin_memcpy(e, &x, 32);
#pragma unroll
        for (int i = 0; i < 2 * E; ++i)
            if (k + i < p.depth) e[i] = row[k + i];
        __builtin_memcpy(&x, e, 32);
        return x;
    };
    auto multiply = [&](const Pair& a, const Pair (&b)[TR]) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < TR; ++i) Mma<T>::add(a.v[h], b[i].v[h], acc[i]);
    };
    const int steps = p.depth / STEP;  // whole ones
    int s = wave;
    for (; s + (AHEAD - 1) * WAVES < steps; s += AHEAD * WAVES) {
        Pair a[AHEAD], b[AHEAD][TR];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) a[u] = whole(c, (s + u * WAVES) * STEP + q * 2 * E);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int i = 0; i < TR; ++i) b[u][i] = whole(r[i], (s + u * WAVES) * STEP + q * 2 * E);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) multiply(a[u], b[u]);
    }
    for (; s < steps; s += WAVES) {
        Pair b[TR];
        const Pair a = whole(c, s * STEP + q * 2 * E);
#pragma unroll
        for (int i = 0; i < TR; ++i) b[i] = whole(r[i], s * STEP + q * 2 * E);
        multiply(a, b);
    }
    if (s == steps && steps * STEP < p.depth) {
        Pair b[TR];
        const Pair a = some(c, s * STEP + q * 2 * E);
#pragma unroll
        for (int i = 0; i < TR; ++i) b[i] = some(r[i], s * STEP + q * 2 * E);
        multiply(a, b);
    }
#pragma unroll
    for (int i = 0; i < TR; ++i) meet[wave][i][lane] = acc[i];
    __syncthreads();
    if (wave >= TR) return;
    floatx4 sum = meet[0][wave][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) sum += meet[w][wave][lane];
    float v[4] = {sum[0], sum[1], sum[2], sum[3]};
    if (p.epi.residual)
        finish<T, true>(p.epi, bias, residual, row, col, valid, v);
    else
        finish<T, false>(p.epi, bias, residual, row, col, valid, v);
}

// Input gradient for few rows: dx = dz W, bound by reading W once, whose rows lie along the result's columns.  A lane takes E
// columns of E consecutive k straight to registers, 16 bytes of each row, and turns them there; its c-th column is
// column E * lane + c of the block, so that each of E matrix instructions has one column of every lane.  A block: 16 E columns,
// 16 * TR rows of a group, and a part of the contraction, of which wavefront w takes every WAVES-th step.  bf16, against the
// tiles of ps_linear.h: one row 4096 -> 4096 14.1 -> 8.7 us, 16 rows 17.0 -> 10.8, 16 rows 16384 -> 4096 28.5 -> 26.4 (5.1 TB/s),
// 32 groups of 12 rows 192 -> 7424 57 -> 28, 10 of one row 90 -> 4340 88 -> 14; fp32 4096 -> 4096 30 -> 17 and 18.  From 33 rows
// on it gains nothing (four row tiles, 64 rows 4096 -> 4096 15.6 -> 16.3, 64 groups of 60 rows 512 -> 1024 18.7 -> 19.6).
template <class T, int TR, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 4) void linear_few_dx_kernel(Product p)
{
    constexpr int E = Mma<T>::E, COLS = 16 * E, STEP = FEW_DX_STEP / sizeof(T), AHEAD = TR > 1 ? 1 : 2;
    constexpr int PITCH = COLS + 4, EACH = 16 * COLS / (64 * WAVES);  // sums of a row of the block in LDS, and of a thread at the end
    static_assert(STEP == 4 * E && EACH * 64 * WAVES == 16 * COLS && E % EACH == 0, "");
    __shared__ float meet[WAVES][16 * PITCH];
    const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6), l = lane & 15, q = lane >> 4;
    const int tc = blockIdx.x % p.tiles_c, rest = blockIdx.x / p.tiles_c, part = rest % p.parts, tr = rest / p.parts;
    GroupRows rows;
    int r0;
    if (!find_rows(p.groups, tr, 16 * TR, rows, r0)) return;
    const int matrix = group_matrix(p.groups, rows.g), c0 = tc * COLS;
    // Columns past the end: the last E again (there are as many), stored again with the same value.  Rows past the end: the last one again.
    auto first_column = [&](int of) { return min(c0 + of * E, p.cols - E); };
    const T* const c = static_cast<const T*>(p.c) + matrix * p.c_matrix + first_column(l);
    const T* r[TR];
#pragma unroll
    for (int i = 0; i < TR; ++i) r[i] = static_cast<const T*>(p.r) + (int64_t)min(r0 + 16 * i + l, rows.end - 1) * p.r_row;

    floatx4 acc[TR][E];
#pragma unroll
    for (int i = 0; i < TR; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[i][e] = floatx4{0.f, 0.f, 0.f, 0.f};
    struct Piece {
        uintx4 w[E], d[TR];
    };
    auto load = [&](int k, Piece& x) __attribute__((always_inline)) {  // k: of the lane's first
#pragma unroll
        for (int e = 0; e < E; ++e) __builtin_memcpy(&x.w[e], c + (int64_t)(k + e) * p.c_row, 16);
#pragma unroll
        for (int i = 0; i < TR; ++i) __builtin_memcpy(&x.d[i], r[i] + k, 16);
    };
    auto load_last = [&](int k, Piece& x) __attribute__((always_inline)) {  // zeros past the end of the contraction
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x.w[e] = uintx4{0, 0, 0, 0};
            if (k + e < p.depth) __builtin_memcpy(&x.w[e], c + (int64_t)(k + e) * p.c_row, 16);
        }
#pragma unroll
        for (int i = 0; i < TR; ++i) {
            x.d[i] = uintx4{0, 0, 0, 0};
            T d[E];
            __builtin_memcpy(d, &x.d[i], 16);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (k + e < p.depth) d[e] = r[i][k + e];
            __builtin_memcpy(&x.d[i], d, 16);
        }
    };
    auto multiply = [&](const Piece& x) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            uintx4 column;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (sizeof(T) == 4)
                    column[i] = x.w[i][e];
                else
                    column[i] = __builtin_amdgcn_perm(x.w[2 * i + 1][e / 2], x.w[2 * i][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
            }
#pragma unroll
            for (int i = 0; i < TR; ++i) Mma<T>::add(column, x.d[i], acc[i][e]);
        }
    };
    const int all = (p.depth + STEP - 1) / STEP, from = min(part * p.part_stages, all), to = min(from + p.part_stages, all);
    const int whole = min(to, p.depth / STEP);
    int s = from + wave;
    for (; s + (AHEAD - 1) * WAVES < whole; s += AHEAD * WAVES) {
        Piece x[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) load((s + u * WAVES) * STEP + q * E, x[u]);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) multiply(x[u]);
    }
    for (; s < to; s += WAVES) {
        Piece x;
        if (s < whole)
            load(s * STEP + q * E, x);
        else
            load_last(s * STEP + q * E, x);
        multiply(x);
    }
    // Lane (q, l) has row l and E * 4 consecutive columns from 4 q E on: column e of lane 4 q + n in acc[e][n].
#pragma unroll
    for (int i = 0; i < TR; ++i) {
        if (i) __syncthreads();
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int e = 0; e < E; e += 4)
                *reinterpret_cast<floatx4*>(&meet[wave][l * PITCH + (4 * q + n) * E + e]) = floatx4{acc[i][e][n], acc[i][e + 1][n], acc[i][e + 2][n], acc[i][e + 3][n]};
        __syncthreads();
        const int at = threadIdx.x * EACH, row = at / COLS, of = at % COLS, out_row = r0 + 16 * i + row;
        float v[EACH];
#pragma unroll
        for (int e = 0; e < EACH; ++e) v[e] = meet[0][row * PITCH + of + e];
#pragma unroll
        for (int w = 1; w < WAVES; ++w)
#pragma unroll
            for (int e = 0; e < EACH; ++e) v[e] += meet[w][row * PITCH + of + e];
        if (out_row >= rows.end) continue;
        const int col = first_column(of / E) + of % E;
        if (p.epi.partial)
            store_n(p.epi.partial + ((int64_t)part * p.rows + out_row) * p.cols + col, v);
        else
            store_n(static_cast<T*>(p.epi.out) + out_row * p.epi.out_row + col, v);
    }
}

template <class T>
void start_few(const Product& p, int row_tiles, hipStream_t s)
{
    const dim3 grid(p.tiles_r * p.tiles_c);
    // K in eighths: 16 columns of 4096 values are then eight steps of each wavefront.  Three row tiles against four: 37 rows 1111 -> 2777 in
    // fp16 12.3 -> 11.0 us.
    if (row_tiles == 1)
        hipLaunchKernelGGL((linear_few_kernel<T, 1, 8>), grid, dim3(512), 0, s, p);
    else if (row_tiles == 2)
        hipLaunchKernelGGL((linear_few_kernel<T, 2, 8>), grid, dim3(512), 0, s, p);
    else if (row_tiles == 3)
        hipLaunchKernelGGL((linear_few_kernel<T, 3, 8>), grid, dim3(512), 0, s, p);
    else
        hipLaunchKernelGGL((linear_few_kernel<T, 4, 8>), grid, dim3(512), 0, s, p);
}

template <class T>
void start_few_dx(const Product& p, int row_tiles, hipStream_t s)
{
    const dim3 grid(p.tiles_r * p.tiles_c * p.parts);
    if (row_tiles == 1)
        hipLaunchKernelGGL((linear_few_dx_kernel<T, 1, 8>), grid, dim3(512), 0, s, p);
    else
        hipLaunchKernelGGL((linear_few_dx_kernel<T, 2, 8>), grid, dim3(512), 0, s, p);
}

}  // namespace

void launch_linear_few_dx(const Product& p, int dtype, int row_tiles, hipStream_t s)
{
    if (dtype == PS_F32)
        start_few_dx<float>(p, row_tiles, s);
    else if (dtype == PS_BF16)
        start_few_dx<bf16_t>(p, row_tiles, s);
    else
        start_few_dx<f16_t>(p, row_tiles, s);
}

void launch_linear_few(const Product& p, int dtype, int row_tiles, hipStream_t s)
{
    if (dtype == PS_F32)
        start_few<float>(p, row_tiles, s);
    else if (dtype == PS_BF16)
        start_few<bf16_t>(p, row_tiles, s);
    else
        start_few<f16_t>(p, row_tiles, s);
}

}  // namespace ps
