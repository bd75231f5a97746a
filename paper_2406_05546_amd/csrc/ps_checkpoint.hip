// Activations to 8 bits and back (include/ps_dense.h; ps_checkpoint.h has the arithmetic).
#include "ps_checkpoint_calls.h"

namespace ps {
namespace {

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct CodeArgs {
    void* x;
    uint8_t *codes, *scales;
    int64_t x_row, row, scale_row, rows;
    int32_t cols, cols_to, per_row, act;  // per_row: pieces of eight columns
    Groups groups;
};

// A thread takes eight columns of a row, four times; neighbours in a block take neighbouring pieces.  Bound by memory.
constexpr int CODE_AHEAD = 4;

template <class T>
__global__ __launch_bounds__(256) void encode_kernel(CodeArgs a)
{
    const int64_t total = a.rows * a.per_row;
    for (int64_t first = (int64_t)blockIdx.x * (256 * CODE_AHEAD); first < total; first += (int64_t)gridDim.x * (256 * CODE_AHEAD)) {
        const int64_t row0 = first / a.per_row;
        const uint32_t rem = (uint32_t)(first - row0 * a.per_row);
        float v[CODE_AHEAD][8];
        int64_t row[CODE_AHEAD];
        int col[CODE_AHEAD], n[CODE_AHEAD];
#pragma unroll
        for (int i = 0; i < CODE_AHEAD; ++i) {
            const uint32_t at = rem + i * 256 + threadIdx.x;
            row[i] = row0 + at / (uint32_t)a.per_row;
            col[i] = (int)(at % (uint32_t)a.per_row) * 8;
            n[i] = row[i] < a.rows && group_of_row(a.groups, row[i]) >= 0 ? min(8, a.cols - col[i]) : 0;
            const T* from = static_cast<const T*>(a.x) + row[i] * a.x_row + col[i];
            if (n[i] == 8)
                load_n(from, v[i]);
            else
                load_some(from, n[i], v[i]);
        }
#pragma unroll
        for (int i = 0; i < CODE_AHEAD; ++i) checkpoint_store(a.codes + row[i] * a.row, a.scales + row[i] * a.scale_row, col[i], n[i], v[i]);
    }
}

template <class T>
__global__ __launch_bounds__(256) void decode_kernel(CodeArgs a)
{
    const int64_t total = a.rows * a.per_row;
    for (int64_t first = (int64_t)blockIdx.x * (256 * CODE_AHEAD); first < total; first += (int64_t)gridDim.x * (256 * CODE_AHEAD)) {
        const int64_t row0 = first / a.per_row;
        const uint32_t rem = (uint32_t)(first - row0 * a.per_row);
        uint32_t code[CODE_AHEAD][2], scale[CODE_AHEAD];
        int64_t row[CODE_AHEAD];
        int col[CODE_AHEAD], n[CODE_AHEAD];
#pragma unroll
        for (int i = 0; i < CODE_AHEAD; ++i) {
            const uint32_t at = rem + i * 256 + threadIdx.x;
            row[i] = row0 + at / (uint32_t)a.per_row;
            col[i] = (int)(at % (uint32_t)a.per_row) * 8;
            n[i] = row[i] < a.rows ? min(8, a.cols - col[i]) : 0;
            scale[i] = 0;
            if (n[i] > 0) scale[i] = a.scales[row[i] * a.scale_row + col[i] / PS_CHECKPOINT_BLOCK];
            load_codes(a.codes + row[i] * a.row + col[i], n[i], code[i]);
        }
#pragma unroll
        for (int i = 0; i < CODE_AHEAD; ++i) {
            if (row[i] >= a.rows) continue;
            float v[8];
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
            T* to = static_cast<T*>(a.x) + row[i] * a.x_row + col[i];
            const int m = min(8, a.cols_to - col[i]);
            if (m == 8)
                store_n(to, v);
            else
                store_some(to, m, v);
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
    a.per_row = (int32_t)up(cols, PS_CHECKPOINT_BLOCK) * CHECKPOINT_LANES;
    a.groups = groups;
    return a;
}

dim3 code_grid(const CodeArgs& a) { return dim3((uint32_t)std::min<int64_t>(up(a.rows * a.per_row, 256 * CODE_AHEAD), 1 << 20)); }

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
    const CodeArgs a = code_args(groups, rows, cols, x, to);
    with_type(dtype, [&](auto t) { hipLaunchKernelGGL(encode_kernel<decltype(t)>, code_grid(a), dim3(256), 0, s, a); });
}

void launch_checkpoint_decode(int dtype, int64_t rows, int64_t cols, const ps_checkpoint& from, int activation, const ps_matrix& x, int64_t cols_to, hipStream_t s)
{
    CodeArgs a = code_args(Groups{}, rows, cols, x, from);
    a.cols_to = (int32_t)cols_to;
    a.per_row = (int32_t)up(cols_to, 8);
    a.act = activation;
    with_type(dtype, [&](auto t) { hipLaunchKernelGGL(decode_kernel<decltype(t)>, code_grid(a), dim3(256), 0, s, a); });
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
