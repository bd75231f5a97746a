// Activations to 8 bits and back (include/ps_dense.h; ps_checkpoint.h has the arithmetic).
#include "ps_checkpoint_calls.h"

namespace ps {
namespace {

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <class T>
__global__ __launch_bounds__(256) void encode_kernel(CodeArgs a)
{
    // A group's rows are shared by `parts` blocks, up to 64 at a time, as they come: one group may have those of all.
    const GroupRows of = group_rows(a.groups, blockIdx.x / a.parts);
    const int each = min((of.end - of.begin + a.parts - 1) / a.parts, 64);
    for (int64_t first = of.begin + (int64_t)(blockIdx.x % a.parts) * each; first < of.end; first += (int64_t)a.parts * each) {
        const int items = (int)min((int64_t)each, of.end - first) * a.pieces;
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
                const bool there = at + i * 256 < items;
                checkpoint_store<T>(a.codes + p[i].row * a.row, a.scales + p[i].row * a.scale_row, p[i].col, there ? p[i].n : 0, v);
            }
        }
    }
}

template <class T>
__global__ __launch_bounds__(256) void decode_kernel(CodeArgs a)
{
    decode_rows<T>(a, blockIdx.x, gridDim.x);
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
uint32_t code_blocks(CodeArgs& a)
{
    a.each = (int32_t)std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(64, 2048 / a.pieces), a.rows / (8 * COMPUTE_UNITS)));
    return (uint32_t)std::min<int64_t>(up(a.rows, a.each), 1 << 22);
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
    const int64_t blocks = code_blocks(a);
    // Of several groups four blocks to a compute unit at least, of which most may be of groups without rows.
    a.parts = (int32_t)(groups.n > 1 ? std::min(rows, up(std::max<int64_t>(blocks, 4 * COMPUTE_UNITS), groups.n)) : blocks);
    with_type(dtype, [&](auto t) { hipLaunchKernelGGL(encode_kernel<decltype(t)>, dim3((uint32_t)(groups.n * a.parts)), dim3(256), 0, s, a); });
}

CodeArgs decode_args(int64_t rows, int64_t cols, const ps_checkpoint& from, int activation, const ps_matrix& x, int64_t cols_to, uint32_t* blocks)
{
    CodeArgs a = code_args(Groups{}, rows, cols, x, from);
    a.cols_to = (int32_t)cols_to;
    a.pieces = (int32_t)up(cols_to, 8);
    a.act = activation;
    *blocks = code_blocks(a);
    return a;
}

void launch_checkpoint_decode(int dtype, const CodeArgs& a, uint32_t blocks, hipStream_t s)
{
    with_type(dtype, [&](auto t) { hipLaunchKernelGGL(decode_kernel<decltype(t)>, dim3(blocks), dim3(256), 0, s, a); });
}

}  // namespace ps

extern "C" ps_status ps_checkpoint_encode(int32_t dtype, int64_t rows, int64_t cols, const ps_matrix* x, const ps_checkpoint* to, void* hip_stream)
{
    using namespace ps;
    static const char call[] = "ps_checkpoint_encode";
    const ps_status st = check_matrix_of_codes(call, dtype, rows, cols, x, to);
    if (st != PS_OK || !rows) return st;
    launch_checkpoint_encode(dtype, Groups{nullptr, nullptr, 1, 1, (int32_t)rows}, rows, cols, *x, *to, static_cast<hipStream_t>(hip_stream));
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
    uint32_t blocks;
    const CodeArgs a = decode_args(rows, cols, *from, activation, *x, cols, &blocks);
    launch_checkpoint_decode(dtype, a, blocks, static_cast<hipStream_t>(hip_stream));
    return launched(call);
}
