// AdamW over many tensors in one launch (include/ps_dense.h): every weight, its two states and its gradient rows are
// read once and written once, whatever the number, sizes and types of the tensors.
#include "ps_dense.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

namespace ps {

namespace {

constexpr int LANE_VALUES = 8;                            // consecutive elements of a lane: 16 bytes of a 16-bit type
constexpr int ADAMW_THREADS = 256;
constexpr int PIECE = ADAMW_THREADS * LANE_VALUES;        // elements of a block
constexpr int SCALE_LANES = PS_ADAMW_BLOCK / LANE_VALUES; // lanes that share a scale
constexpr int32_t LAUNCH_PIECES = 1 << 23;                // of one launch, which has less than 2^32 threads
static_assert(SCALE_LANES == 32 && PIECE % PS_ADAMW_BLOCK == 0, "half a wavefront holds one block of an 8-bit state");

struct Tensor {
    void* param;
    const void* grad;
    void* copy;
    void *m, *v;
    float *m_scale, *v_scale;
    int64_t numel, grad_row;
    int32_t param_type, grad_type, copy_type, bits;
    float decay;
    int32_t pad;
};
struct Piece {
    int32_t tensor, index;  // elements index * PIECE .. of it
};
struct Step {
    float beta1, beta1_rest, beta2, beta2_rest, eps, lr, lr_corrected, root_correction, grad_scale;
    int32_t n_rows;
};

template <class T>
__device__ __forceinline__ void load_part(const void* base, int64_t at, int n, float (&x)[LANE_VALUES])
{
    const T* p = static_cast<const T*>(base) + at;
    if (n == LANE_VALUES)
        load_n(p, x);
    else
        load_some(p, n, x);
}
template <class T>
__device__ __forceinline__ void store_part(void* base, int64_t at, int n, const float (&x)[LANE_VALUES])
{
    T* p = static_cast<T*>(base) + at;
    if (n == LANE_VALUES)
        store_n(p, x);
    else
        store_some(p, n, x);
}
__device__ __forceinline__ void load_typed(int type, const void* base, int64_t at, int n, float (&x)[LANE_VALUES])
{
    if (type == PS_F32)
        load_part<float>(base, at, n, x);
    else if (type == PS_BF16)
        load_part<bf16_t>(base, at, n, x);
    else
        load_part<f16_t>(base, at, n, x);
}
// Adds the rows from the second on to x, in order, with AHEAD of them on their way at once (64 rows of 813,258 fp32 gradients:
// 59 -> 50 us, 4.6 TB/s).
constexpr int AHEAD = 8;
template <class T>
__device__ __forceinline__ void add_rows(const void* base, int64_t at, int64_t row, int n_rows, int n, float (&x)[LANE_VALUES])
{
    int k = 1;
    for (; k + AHEAD <= n_rows; k += AHEAD) {
        float more[AHEAD][LANE_VALUES];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) load_part<T>(base, at + (k + u) * row, n, more[u]);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
#pragma unroll
            for (int i = 0; i < LANE_VALUES; ++i) x[i] += more[u][i];
    }
    for (; k < n_rows; ++k) {
        float more[LANE_VALUES];
        load_part<T>(base, at + k * row, n, more);
#pragma unroll
        for (int i = 0; i < LANE_VALUES; ++i) x[i] += more[i];
    }
}
__device__ __forceinline__ void store_typed(int type, void* base, int64_t at, int n, const float (&x)[LANE_VALUES])
{
    if (type == PS_F32)
        store_part<float>(base, at, n, x);
    else if (type == PS_BF16)
        store_part<bf16_t>(base, at, n, x);
    else
        store_part<f16_t>(base, at, n, x);
}

// Eight e4m3 codes -> values, and back (to the nearest, ties to even; magnitudes are at most 448 here, or NaN).
__device__ __forceinline__ void decode8(const void* base, int64_t at, int n, float scale, float (&x)[LANE_VALUES])
{
    const uint8_t* p = static_cast<const uint8_t*>(base) + at;
    uint32_t code[2] = {0, 0};
    if (n == LANE_VALUES) {
        __builtin_memcpy(code, p, 8);
    } else {
#pragma unroll
        for (int i = 0; i < LANE_VALUES; ++i)
            if (i < n) code[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        x[4 * i + 0] = __builtin_amdgcn_cvt_f32_fp8((int)code[i], 0) * scale;
        x[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8((int)code[i], 1) * scale;
        x[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8((int)code[i], 2) * scale;
        x[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8((int)code[i], 3) * scale;
    }
}

// Largest magnitude over the 32 lanes that share a scale; NaN if any of them is (as an integer NaN is the largest).
__device__ __forceinline__ float largest_of_block(const float (&x)[LANE_VALUES])
{
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < LANE_VALUES; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
    for (int off = 1; off < SCALE_LANES; off <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off, 64));
    return __uint_as_float(top);
}

// Rounds the block's values to codes and writes them and the scale.  ROOT: what is not 0 is not held as 0.
template <bool ROOT>
__device__ __forceinline__ void encode8(void* base, float* scales, int64_t at, int n, const float (&x)[LANE_VALUES])
{
    const float top = largest_of_block(x);
    // A scale made from less than 2^-100 would have an infinite inverse; states that small are held as 0 (roots as the
    // least code).  NaN stays.
    const float from = top < 0x1p-100f ? 0x1p-100f : top;
    const float inverse = 448.f / from;
    uint32_t code[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int c = 0;
        c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 0] * inverse, x[4 * i + 1] * inverse, c, false);
        c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inverse, x[4 * i + 3] * inverse, c, true);
        code[i] = (uint32_t)c;
        if (ROOT) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (x[4 * i + j] > 0.f && inverse > 0.f && (code[i] >> (8 * j) & 0xffu) == 0) code[i] |= 1u << (8 * j);
        }
    }
    uint8_t* p = static_cast<uint8_t*>(base) + at;
    if (n == LANE_VALUES) {
        __builtin_memcpy(p, code, 8);
    } else {
#pragma unroll
        for (int i = 0; i < LANE_VALUES; ++i)
            if (i < n) p[i] = (uint8_t)(code[i / 4] >> (8 * (i % 4)));
    }
    if (n > 0 && (threadIdx.x & (SCALE_LANES - 1)) == 0) scales[at / PS_ADAMW_BLOCK] = from * (1.f / 448.f);
}

// A block takes 2048 elements of one tensor, named by the piece list (so that the launch is one whatever the tensors),
// a lane eight consecutive ones.  Bound by memory: 201.6 M bf16 weights with 8-bit states 400-420 us, 4.8-5.1 TB/s (a
// copy of 2 GiB: 4.9).  A small table is bound by trips to memory that wait for each other, for the piece, the tensor, and then each
// operand, which is converted in its type's branch before the next is asked for: 813,258 fp32 weights 6.5 us, 3.5 TB/s; 1.2 M
// bf16 weights in 61 tensors, 8-bit states and two gradient rows 9.5.  MANY: several gradient rows, which take registers that others go without.
template <bool MANY>
__global__ __launch_bounds__(ADAMW_THREADS) void adamw_kernel(const Tensor* __restrict__ tensors, const Piece* __restrict__ pieces, Step s)
{
// An 8-bit state has one rounding for every operation written here, so that its codes can be checked one by one.
#pragma clang fp contract(off)
    const Piece piece = pieces[blockIdx.x];
    const Tensor t = tensors[piece.tensor];
    const int64_t at = (int64_t)piece.index * PIECE + threadIdx.x * LANE_VALUES;
    const int n = (int)max((int64_t)0, min((int64_t)LANE_VALUES, t.numel - at));
    if (t.bits != 8 && n == 0) return;  // the lanes of an 8-bit block meet below

    float p[LANE_VALUES], g[LANE_VALUES], m[LANE_VALUES], v[LANE_VALUES];
    const int64_t from = n ? at : 0;  // lanes past the end read nothing
    load_typed(t.param_type, t.param, from, n, p);
    if (t.bits == 8) {
        // Lanes past the end hold zeros, and read no scale: those of a block's other lanes meet them for the largest magnitude, and any
        // other block's scale may be NaN, or on its way to be written.
        const int64_t block = at / PS_ADAMW_BLOCK;
        decode8(t.m, from, n, n ? t.m_scale[block] : 0.f, m);
        decode8(t.v, from, n, n ? t.v_scale[block] : 0.f, v);
    } else {
        load_part<float>(t.m, from, n, m);
        load_part<float>(t.v, from, n, v);
    }
    load_typed(t.grad_type, t.grad, from, n, g);
    if constexpr (MANY) {
        if (t.grad_type == PS_F32)
            add_rows<float>(t.grad, from, t.grad_row, s.n_rows, n, g);
        else if (t.grad_type == PS_BF16)
            add_rows<bf16_t>(t.grad, from, t.grad_row, s.n_rows, n, g);
        else
            add_rows<f16_t>(t.grad, from, t.grad_row, s.n_rows, n, g);
    }
    const float kept = s.lr * t.decay;
#pragma unroll
    for (int i = 0; i < LANE_VALUES; ++i) {
        const float gi = g[i] * s.grad_scale;
        m[i] = m[i] * s.beta1 + gi * s.beta1_rest;
        const float old = t.bits == 8 ? v[i] * v[i] : v[i];
        const float vi = old * s.beta2 + gi * gi * s.beta2_rest;
        const float root = sqrtf(vi);
        v[i] = t.bits == 8 ? root : vi;
        p[i] = p[i] - p[i] * kept - s.lr_corrected * m[i] / (root * s.root_correction + s.eps);
    }
    if (n) {
        store_typed(t.param_type, t.param, at, n, p);
        if (t.copy) store_typed(t.copy_type, t.copy, at, n, p);
    }
    if (t.bits == 8) {
        encode8<false>(t.m, t.m_scale, at, n, m);
        encode8<true>(t.v, t.v_scale, at, n, v);
    } else {
        store_part<float>(t.m, at, n, m);
        store_part<float>(t.v, at, n, v);
    }
}

bool known_type(int t) { return t == PS_F32 || t == PS_BF16 || t == PS_F16; }

bool misaligned(const void* p, int size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; }

// The table's checks; counts its pieces.
ps_status check_tensors(const char* call, const ps_adamw_tensor* ts, int32_t n, int64_t* pieces)
{
    if (n < 0 || (n && !ts)) return dense_fail(PS_EINVAL, "%s: no tensors, or a negative number of them", call);
    int64_t total = 0;
    for (int32_t i = 0; i < n; ++i) {
        const ps_adamw_tensor& t = ts[i];
        if (t.numel < 0) return dense_fail(PS_EINVAL, "%s: tensor %d has a negative size", call, i);
        if (!known_type(t.param_dtype) || !known_type(t.grad_dtype) || (t.copy_dev && !known_type(t.copy_dtype)))
            return dense_fail(PS_EINVAL, "%s: tensor %d has an unknown type", call, i);
        if (t.state_bits != 8 && t.state_bits != 32) return dense_fail(PS_EINVAL, "%s: tensor %d: states have 8 or 32 bits", call, i);
        if (t.grad_rows < 1 || (t.grad_rows > 1 && t.grad_row < t.numel)) return dense_fail(PS_EINVAL, "%s: tensor %d: gradient rows overlap, or there are none", call, i);
        if (!(t.weight_decay >= 0.f)) return dense_fail(PS_EINVAL, "%s: tensor %d: weight decay below 0 or NaN", call, i);
        if (!t.numel) continue;
        if (!t.param_dev || !t.grad_dev || !t.m_dev || !t.v_dev || (t.state_bits == 8 && (!t.m_scale_dev || !t.v_scale_dev)))
            return dense_fail(PS_EINVAL, "%s: tensor %d has a null pointer", call, i);
        const int state = t.state_bits == 8 ? 1 : 4;
        if (misaligned(t.param_dev, dtype_size(t.param_dtype)) || misaligned(t.grad_dev, dtype_size(t.grad_dtype)) ||
            (t.copy_dev && misaligned(t.copy_dev, dtype_size(t.copy_dtype))) || misaligned(t.m_dev, state) || misaligned(t.v_dev, state) ||
            (state == 1 && (misaligned(t.m_scale_dev, 4) || misaligned(t.v_scale_dev, 4))))
            return dense_fail(PS_EINVAL, "%s: tensor %d is not aligned to its elements", call, i);
        total += (t.numel + PIECE - 1) / PIECE;
        if (total > INT32_MAX) return dense_fail(PS_EINVAL, "%s: more than 2^31 pieces of %d elements", call, PIECE);
    }
    *pieces = total;
    return PS_OK;
}

}  // namespace
}  // namespace ps

struct ps_adamw {
    const ps::Tensor* tensors;
    const ps::Piece* pieces;
    int32_t n_pieces, grad_rows;  // grad_rows: the least of any tensor
};

extern "C" ps_status ps_adamw_workspace_bytes(const ps_adamw_tensor* ts, int32_t n, uint64_t* bytes_out)
{
    using namespace ps;
    if (!bytes_out) return dense_fail(PS_EINVAL, "ps_adamw_workspace_bytes: no place for the result");
    int64_t pieces = 0;
    const ps_status st = check_tensors("ps_adamw_workspace_bytes", ts, n, &pieces);
    if (st == PS_OK) *bytes_out = (sizeof(Tensor) * (uint64_t)n + sizeof(Piece) * (uint64_t)pieces + 255) / 256 * 256;
    return st;
}

extern "C" ps_status ps_adamw_create(ps_adamw** out, const ps_adamw_tensor* ts, int32_t n, void* workspace, uint64_t bytes, void* hip_stream)
{
    using namespace ps;
    if (!out) return dense_fail(PS_EINVAL, "ps_adamw_create: no place for the handle");
    *out = nullptr;
    int64_t total = 0;
    const ps_status st = check_tensors("ps_adamw_create", ts, n, &total);
    if (st != PS_OK) return st;
    const uint64_t table = sizeof(Tensor) * (uint64_t)n, list = sizeof(Piece) * (uint64_t)total;
    if (table + list) {
        if (!workspace || misaligned(workspace, 16)) return dense_fail(PS_EINVAL, "ps_adamw_create: null or misaligned workspace");
        if (bytes < table + list) return dense_fail(PS_ENOMEM, "ps_adamw_create: workspace too small");
    }
    try {
        std::vector<char> host(table + list);
        Tensor* tensor = reinterpret_cast<Tensor*>(host.data());
        Piece* piece = reinterpret_cast<Piece*>(host.data() + table);
        int32_t rows = INT32_MAX;
        for (int32_t i = 0; i < n; ++i) {
            const ps_adamw_tensor& t = ts[i];
            tensor[i] = Tensor{t.param_dev, t.grad_dev, t.copy_dev, t.m_dev, t.v_dev, t.m_scale_dev, t.v_scale_dev, t.numel, t.grad_row,
                               t.param_dtype, t.grad_dtype, t.copy_dtype, t.state_bits, t.weight_decay, 0};
            for (int64_t at = 0, k = 0; at < t.numel; at += PIECE, ++k) *piece++ = Piece{i, (int32_t)k};
            rows = std::min(rows, t.grad_rows);
        }
        ps_adamw* h = new ps_adamw{static_cast<const Tensor*>(workspace), reinterpret_cast<const Piece*>(static_cast<const char*>(workspace) + table), (int32_t)total, rows};
        if (table + list) {
            hipStream_t s = static_cast<hipStream_t>(hip_stream);
            hipError_t e = hipMemcpyAsync(workspace, host.data(), table + list, hipMemcpyHostToDevice, s);
            if (e == hipSuccess) e = hipStreamSynchronize(s);
            if (e != hipSuccess) {
                delete h;
                return dense_fail(PS_EDEVICE, "ps_adamw_create: %s", hipGetErrorString(e));
            }
        }
        *out = h;
        return PS_OK;
    } catch (const std::bad_alloc&) {
        return dense_fail(PS_ENOMEM, "ps_adamw_create: no host memory for the table");
    }
}

extern "C" ps_status ps_adamw_destroy(ps_adamw* h)
{
    if (!h) return ps::dense_fail(PS_EINVAL, "ps_adamw_destroy: no handle");
    delete h;
    return PS_OK;
}

extern "C" ps_status ps_adamw_step(ps_adamw* h, const ps_adamw_options* o, void* hip_stream)
{
    using namespace ps;
    if (!h || !o) return dense_fail(PS_EINVAL, "ps_adamw_step: no handle or no options");
    if (!(o->lr >= 0) || !(o->beta1 >= 0 && o->beta1 < 1) || !(o->beta2 >= 0 && o->beta2 < 1) || !((float)o->eps > 0) || !std::isfinite(o->grad_scale) ||
        !std::isfinite(o->lr) || !std::isfinite(o->eps))
        return dense_fail(PS_EINVAL, "ps_adamw_step: learning rate, betas, eps or gradient scale out of range");
    if (o->step < 1) return dense_fail(PS_EINVAL, "ps_adamw_step: steps are counted from 1");
    if (o->n_rows < 1 || o->n_rows > h->grad_rows) return dense_fail(PS_EINVAL, "ps_adamw_step: %d gradient rows of %d", o->n_rows, h->grad_rows);
    if (!h->n_pieces) return PS_OK;
    const double c1 = 1 - std::pow(o->beta1, (double)o->step), c2 = 1 - std::pow(o->beta2, (double)o->step);
    const Step s{(float)o->beta1, (float)(1 - o->beta1), (float)o->beta2, (float)(1 - o->beta2), (float)o->eps, (float)o->lr,
                 (float)(o->lr / c1), (float)(1 / std::sqrt(c2)), (float)o->grad_scale, o->n_rows};
    for (int64_t first = 0; first < h->n_pieces; first += LAUNCH_PIECES)
        hipLaunchKernelGGL(o->n_rows > 1 ? adamw_kernel<true> : adamw_kernel<false>, dim3((uint32_t)std::min<int64_t>(h->n_pieces - first, LAUNCH_PIECES)), dim3(ADAMW_THREADS), 0,
                           static_cast<hipStream_t>(hip_stream), h->tensors, h->pieces + first, s);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? PS_OK : dense_fail(PS_EDEVICE, "ps_adamw_step: %s", hipGetErrorString(e));
}
