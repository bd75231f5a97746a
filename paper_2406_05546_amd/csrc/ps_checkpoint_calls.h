// Encoding and decoding of whole matrices (ps_checkpoint.hip), for the calls of ps_linear.hip.
#pragma once
#include "ps_linear.h"

namespace ps {

ps_status check_checkpoint(const char* call, const char* name, const ps_checkpoint* c, int64_t rows, int64_t cols);
// Rows in no group are left as they are.
void launch_checkpoint_encode(int dtype, const Groups& groups, int64_t rows, int64_t cols, const ps_matrix& x, const ps_checkpoint& to, hipStream_t s);

struct CodeArgs {
    void* x;
    uint8_t *codes, *scales;
    int64_t x_row, row, scale_row, rows;
    int32_t cols, cols_to, pieces, each, act;  // pieces of eight columns of a row; rows of a block
    int32_t parts;                             // encoding: blocks of a group
    Groups groups;
};

// A block takes `each` rows (up to 64), a thread pieces of eight columns of them.  Bound by memory: CODE_AHEAD pieces are asked for together,
// without a branch between them, at which the compiler would wait; a row's last piece, where it is partial, is read again.  8192 x
// 8192 in bf16: encoded in 35 us, 5.8 TB/s, decoded in 31, 6.5 TB/s.
constexpr int CODE_AHEAD = 4;

// Rows of cols_to >= cols elements, zeros behind; `blocks`: how many of them there are to be.
CodeArgs decode_args(int64_t rows, int64_t cols, const ps_checkpoint& from, int activation, const ps_matrix& x, int64_t cols_to, uint32_t* blocks);
void launch_checkpoint_decode(int dtype, const CodeArgs& a, uint32_t blocks, hipStream_t s);

#if defined(__HIPCC__)
struct Piece {
    int64_t row;
    int col, n;  // n: columns that exist
};
__device__ __forceinline__ Piece piece_of(const CodeArgs& a, int64_t first, int item)
{
    const int line = (int)((uint32_t)item / (uint32_t)a.pieces), col = (int)((uint32_t)item % (uint32_t)a.pieces) * 8;
    return {first + line, col, min(8, a.cols - col)};
}

// What block `block` of `blocks` decodes: x = act(values), zeros behind the columns up to cols_to.
template <class T>
__device__ __forceinline__ void decode_rows(const CodeArgs& a, int64_t block, int64_t blocks)
{
    for (int64_t first = block * a.each; first < a.rows; first += blocks * a.each) {
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

#endif

}  // namespace ps
