// Activations to 8 bits and back (include/ps_dense.h; ps_checkpoint.h has the arithmetic).
#include "ps_checkpoint_calls.h"

namespace ps {
namespace {

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct CodeArgs {
    void* x;
    uint8_t *codes, *scales;
    int64_t x_row, row, scale_row, rows;
    int32_t cols, cols_to, pieces, each, act;  // pieces of eight columns of a row; rows of a block
    Groups groups;
};

// A block takes `each` rows (up to 64), a thread pieces of eight columns of them.  Bound by memory: CODE_AHEAD pieces are asked for together,
// without a branch between them, at which the compiler would wait; a row's last piece, where it is partial, is read again.
constexpr int CODE_AHEAD = 4;

struct Piece {
    int64_t row;
    int col, n;  // n: columns that exist
};
__device__ __forceinline__ Piece piece_of(const CodeArgs& a, int64_t first, int item)
{
    const int line = (int)((uint32_t)item / (uint32_t)a.pieces), col = (int)((uint32_t)item % (uint32_t)a.pieces) * 8;
    return {first + line, col, min(8, a.cols - col)};
}

template <class T>
__global__ __launch_bounds__(256) void encode_kernel(CodeArgs a)
{
    __shared__ int inside[64];  // whether a row is in a group
    for (int64_t first = (int64_t)blockIdx.x * a.each; first < a.rows; first += (int64_t)gridDim.x * a.each) {
        const int items = (int)min((int64_t)a.each, a.rows - first) * a.pieces;
        if (a.groups.offsets) {
            if (threadIdx.x < 64) inside[threadIdx.x] = groups_of_rows(a.groups, first) >= 0;
            __syncthreads();
        }
        for (int at = threadIdx.x; at - (int)threadIdx.x < items; at += 256 * CODE_AHEAD) {
            T raw[CODE_AHEAD][8];
            Piece p[CODE_AHEAD];
#pragma unroll
            for (int i = 0; i < CODE_AHEAD; ++i) {
                p[i] = piece_of(a, first, min(at + i * 256, items - 1));
                if (a.cols >= 8) __builtin_memcpy(raw[i], static_cast<const T*>(a.x) + p[i].row * a.x_row + min(p[i].col, a.cols - 8), sizeof(raw[i]));
            }
#pragma unroll
            for (int i = 0; i < CODE_AHEAD; ++i) {
                float v[8];
                if (p[i].n < 8) {
                    load_some(static_cast<const T*>(a.x) + p[i].row * a.x_row + p[i].col, p[i].n, v);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = to_float(raw[i][e]);
                }
                // (all four lanes of a block are there or none is: pieces are whole blocks)
                const bool there = at + i * 256 < items && (!a.groups.offsets || inside[p[i].row - first]);
                checkpoint_store(a.codes + p[i].row * a.row, a.scales + p[i].row * a.scale_row, p[i].col, there ? p[i].n : 0, v);
            }
        }
        if (a.groups.offsets) __syncthreads();  // inside is written again
    }
}

template <class T>
__global__ __launch_bounds__(256) void decode_kernel(CodeArgs a)
{
    for (int64_t first = (int64_t)blockIdx.x * a.each; first < a.rows; first += (int64_t)gridDim.x * a.each) {
        const int items = (int)min((int64_t)a.each, a.rows - first) * a.pieces;
        for (int at = threadIdx.x; at < items; at += 256 * CODE_AHEAD) {
            uint32_t code[CODE_AHEAD][2];
            uint8_t scale[CODE_AHEAD];
            Piece p[CODE_AHEAD];
#pragma unroll
            for (int i = 0; i < CODE_AHEAD; ++i) {
                p[i] = piece_of(a, first, min(at + i * 256, items - 1));
                if (a.cols >= 8) __builtin_memcpy(code[i], a.codes + p[i].row * a.row + min(p[i].col, a.cols - 8), 8);
                scale[i] = a.scales[p[i].row * a.scale_row + min(p[i].col, a.cols - 1) / PS_CHECKPOINT_BLOCK];
            }
#pragma unroll
            for (int i = 0; i < CODE_AHEAD; ++i) {
                if (at + i * 256 >= items) continue;
                float v[8];
                if (p[i].n < 8) {
                    load_codes(a.codes + p[i].row * a.row + p[i].col, p[i].n, code[i]);
                    if (p[i].n <= 0) scale[i] = 127;  // behind the columns: 0 whatever is there
                }
                checkpoint_decode(code[i], scale[i], v);
                if (a.act == PS_ACT_RELU) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = activate<PS_ACT_RELU>(v[e]);
                } else if (a.act == PS_ACT_GELU) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = activate<PS_ACT_GELU>(v[e]);
                } else if (a.act == PS_ACT_SILU) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = activate<PS_ACT_SILU>(v[e]);
                }
                store_columns(static_cast<T*>(a.x) + p[i].row * a.x_row + p[i].col, min(8, a.cols_to - p[i].col), v);
            }
        }
    }
}

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

CodeArgs code_args(const Groups& groups, int64_t rows, int64_t cols, const ps_matrix& x, const ps_checkpoint& c)
{
    CodeArgs a{};
    a.x = x.data_dev;
    a.x_row = x.row;
    a.codes = static_cast<uint8_t*>(c.codes_dev);
    a.scales = static_cast<uint8_t*>(c.scales_dev);
    a.row = c.row;
    a.scale_row = c.scale_row;
    a.rows = rows;
    a.cols = a.cols_to = (int32_t)cols;
    a.pieces = (int32_t)up(cols, PS_CHECKPOINT_BLOCK) * CHECKPOINT_LANES;
    a.groups = groups;
    return a;
}

// Rows of 2048 pieces together, or fewer where that leaves less than eight blocks to a compute unit.
dim3 code_grid(CodeArgs& a)
{
    a.each = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(64, 2048 / a.pieces), a.rows / (8 * COMPUTE_UNITS)));
    return dim3((uint32_t)std::min<int64_t>(up(a.rows, a.each), 1 << 22));
}

ps_status check_matrix_of_codes(const char* call, int32_t dtype, int64_t rows, int64_t cols, const ps_matrix* x, const ps_checkpoint* c)
{
    if (dtype != PS_F32 && dtype != PS_BF16 && dtype != PS_F16) return dense_fail(PS_EINVAL, "%s: unknown type", call);
    if (rows < 0 || rows > PS_DENSE_MAX_ROWS) return dense_fail(PS_EINVAL, "%s: rows outside 0 .. %d", call, PS_DENSE_MAX_ROWS);
    if (cols < 1 || cols > PS_DENSE_MAX_STRIDE) return dense_fail(PS_EINVAL, "%s: columns outside 1 .. %d", call, PS_DENSE_MAX_STRIDE);
    if (rows && (!x || !x->data_dev)) return dense_fail(PS_EINVAL, "%s: x is missing", call);
    if (x && (reinterpret_cast<uintptr_t>(x->data_dev) & (dtype_size(dtype) - 1))) return dense_fail(PS_EINVAL, "%s: x is not aligned to its elements", call);
    if (rows > 1 && (x->row < cols || x->row > PS_DENSE_MAX_STRIDE)) return dense_fail(PS_EINVAL, "%s: x has rows that overlap or are too far apart", call);
    return check_checkpoint(call, "the checkpoint", c, rows, cols);
}

ps_status launched(const char* call)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PS_OK : dense_fail(PS_EDEVICE, "%s: %s", call, hipGetErrorString(e));
}

}  // namespace

ps_status check_checkpoint(const char* call, const char* name, const ps_checkpoint* c, int64_t rows, int64_t cols)
{
    if (!c || ((!c->codes_dev || !c->scales_dev) && rows)) return dense_fail(PS_EINVAL, "%s: %s has no codes or scales", call, name);
    if (rows > 1 && (c->row < cols || c->row > PS_DENSE_MAX_STRIDE || c->scale_row < up(cols, PS_CHECKPOINT_BLOCK) || c->scale_row > PS_DENSE_MAX_STRIDE))
        return dense_fail(PS_EINVAL, "%s: %s has rows that overlap or are too far apart", call, name);
    return PS_OK;
}

void launch_checkpoint_encode(int dtype, const Groups& groups, int64_t rows, int64_t cols, const ps_matrix& x, const ps_checkpoint& to, hipStream_t s)
{
    CodeArgs a = code_args(groups, rows, cols, x, to);
    const dim3 grid = code_grid(a);
    with_type(dtype, [&](auto t) { hipLaunchKernelGGL(encode_kernel<decltype(t)>, grid, dim3(256), 0, s, a); });
}

void launch_checkpoint_decode(int dtype, int64_t rows, int64_t cols, const ps_checkpoint& from, int activation, const ps_matrix& x, int64_t cols_to, hipStream_t s)
{
    CodeArgs a = code_args(Groups{}, rows, cols, x, from);
    a.cols_to = (int32_t)cols_to;
    a.pieces = (int32_t)up(cols_to, 8);
    a.act = activation;
    const dim3 grid = code_grid(a);
    with_type(dtype, [&](auto t) { hipLaunchKernelGGL(decode_kernel<decltype(t)>, grid, dim3(256), 0, s, a); });
}

}  // namespace ps

extern "C" ps_status ps_checkpoint_encode(int32_t dtype, int64_t rows, int64_t cols, const ps_matrix* x, const ps_checkpoint* to, void* hip_stream)
{
    using namespace ps;
    static const char call[] = "ps_checkpoint_encode";
    const ps_status st = check_matrix_of_codes(call, dtype, rows, cols, x, to);
    if (st != PS_OK || !rows) return st;
    launch_checkpoint_encode(dtype, Groups{}, rows, cols, *x, *to, static_cast<hipStream_t>(hip_stream));
    return launched(call);
}

extern "C" ps_status ps_checkpoint_decode(int32_t dtype, int64_t rows, int64_t cols, const ps_checkpoint* from, int32_t activation, const ps_matrix* x,
                                          void* hip_stream)
{
    using namespace ps;
    static const char call[] = "ps_checkpoint_decode";
    const ps_status st = check_matrix_of_codes(call, dtype, rows, cols, x, from);
    if (st != PS_OK) return st;
    if (activation < PS_ACT_NONE || activation > PS_ACT_SILU) return dense_fail(PS_EINVAL, "%s: unknown activation", call);
    if (!rows) return PS_OK;
    launch_checkpoint_decode(dtype, rows, cols, *from, activation, *x, cols, static_cast<hipStream_t>(hip_stream));
    return launched(call);
}
