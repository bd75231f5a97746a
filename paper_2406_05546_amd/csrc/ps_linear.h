// Dense layers on the gfx950 matrix cores (include/ps_dense.h): forward, input gradient and weight gradient, in one group
// of rows or in many.
//
//   out[r][c] = sum_k R(r, k) C(c, k)
//
// R gives the rows of the result, C its (contiguous) columns.  Either operand lies k-contiguous ("KC": x and w of the
// forward pass, dz of the input gradient) or row-contiguous ("RC": w of the input gradient, dz and x of the weight
// gradient).  A block owns a BR x BC tile of the result, and its operands come in stages of 128 bytes of k (64 values of a
// 16-bit type, 32 of fp32) through LDS; wavefronts are arranged WR x WC and multiply 16 x 16 tiles
// (v_mfma_f32_16x16x32_bf16 / _f16, v_mfma_f32_16x16x4_f32) with C as the instruction's first operand, so that a lane
// gets consecutive columns of one row of the result.
//
// Bound by the matrix cores (and the chip's power) where rows are many: bf16 8192^3 1340-1410 TFLOP/s in all three kinds, the
// library's product of rows with rows 1330-1570 (the first and the third ten one after the other), of its two transposed forms
// 1170-1360 and 1040-1180; by memory where they are few.
#pragma once
#include "ps_checkpoint.h"
#include "ps_dense.h"
#include "ps_split.h"

#include <algorithm>
#include <type_traits>

namespace ps {

typedef uint32_t uintx2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr int LINEAR_XCDS = 8, COMPUTE_UNITS = 256;

#if defined(__HIPCC__)
// Value e of 16 bytes.  Values that wait in registers stay packed this way; arrays of 16-bit ones take a register each.
template <class T>
__device__ __forceinline__ float element(const uintx4& x, int e)
{
    if constexpr (sizeof(T) == 4)
        return __uint_as_float(x[e]);
    else if constexpr (__is_same(T, bf16_t))
        return __uint_as_float(e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16);
    else
        return to_float(f16_t{(uint16_t)(x[e / 2] >> (e & 1) * 16)});
}
#endif

// ---------------------------------------------------------------------------------------------------------------
// Groups

// Where the rows of the groups are, and which matrix each uses.  Offsets come from device memory and are whatever they
// are: every one is taken into 0 .. rows, a group that ends before it begins is empty.
struct Groups {
    const int32_t* offsets;  // [n + 1], or null: one group of all rows
    const int32_t* index;    // [n], or null: group g uses matrix g
    int32_t n, n_weights, rows;
};

struct GroupRows {
    int g, begin, end;
};

#if defined(__HIPCC__)

__device__ __forceinline__ int scalar(int v) { return __builtin_amdgcn_readfirstlane(v); }

// What lanes of a wavefront wrote to LDS before this is what its lanes read behind it: LDS serves a wavefront in order, so nothing is
// waited for, but the compiler moves and keeps nothing across it.
__device__ __forceinline__ void wave_meets()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ GroupRows group_rows(const Groups& gs, int g)
{
    if (!gs.offsets) return {g, 0, gs.rows};
    const int begin = min(max(gs.offsets[g], 0), gs.rows), end = min(max(gs.offsets[g + 1], begin), gs.rows);
    return {g, begin, end};
}

__device__ __forceinline__ int group_matrix(const Groups& gs, int g)
{
    const int i = gs.index ? gs.index[g] : g;
    return min(max(i, 0), gs.n_weights - 1);
}

// Tiles of `size` rows that 64 groups from g0 on are cut into, one group to a lane, summed up to each lane.  Rows are at most 2^28
// and tiles at least 16 rows, so that 64 groups (which may overlap, if the offsets are no offsets) stay below 2^30.
__device__ __forceinline__ int tiles_upto(const Groups& gs, int g0, int size, GroupRows& r, int& own)
{
    const int lane = threadIdx.x & 63;
    r = {g0 + lane, 0, 0};
    if (r.g < gs.n) r = group_rows(gs, r.g);
    own = (r.end - r.begin + size - 1) / size;
    int upto = own;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int other = __shfl_up(upto, d, 64);
        if (lane >= d) upto += other;
    }
    return upto;
}

// How many tiles there are, or (with many groups, which would take long to count) `bound`.
constexpr int COUNTED_GROUPS = 1024;
__device__ __forceinline__ int count_tiles(const Groups& gs, int size, int bound)
{
    if (!gs.offsets || gs.n > COUNTED_GROUPS) return bound;
    int total = 0;
    for (int g0 = 0; g0 < gs.n && total < bound; g0 += 64) {
        GroupRows r;
        int own;
        total += __builtin_amdgcn_readlane(tiles_upto(gs, g0, size, r, own), 63);
    }
    return min(total, bound);
}

// The group that has row `first` + lane, for a whole wavefront: the last one that begins there or before, if it ends behind it; -1 for
// rows of none.  One look at the offsets for every power of 64 groups, and one for 64 that begin among the rows: next to kernels that
// fill the memory's queues, each one takes microseconds.  Where more than 64 offsets do not ascend, the search need not find the last one, and
// what it finds goes by `first`: a multiple of 64, so that every call has the same.
__device__ __forceinline__ int groups_of_rows(const Groups& gs, int64_t first)
{
    const int lane = threadIdx.x & 63;
    const int64_t r = first + lane;
    if (!gs.offsets) return r < gs.rows ? 0 : -1;
    auto begins = [&](int g) __attribute__((always_inline)) { return min(max(gs.offsets[g], 0), gs.rows); };
    const int end_of_all = begins(gs.n);
    int lo = 0, hi = gs.n;  // groups before lo begin at `first` or before, those from hi on behind it
    bool disorder = false;
    while (lo < hi) {
        const int step = (hi - lo + 63) >> 6, g = lo + lane * step;
        const unsigned long long set = __ballot(g < hi && begins(min(g, gs.n)) <= first);
        const int before = __popcll(set);
        disorder |= (set & (set + 1)) != 0;  // not the first lanes'
        if (before == 0) break;
        hi = min(hi, lo + before * step);
        lo = lo + (before - 1) * step + 1;
    }
    int group = lo - 1;
    for (int g0 = lo; g0 < gs.n; g0 += 64) {
        const int begin = g0 + lane < gs.n ? begins(g0 + lane) : 0x7fffffff;
        unsigned long long among = __ballot(begin <= first + 63);
        // ascending, so those that begin among the rows are the first lanes' (if the offsets are none, any of them may be)
        for (; among; among &= among - 1) {
            const int i = __builtin_ctzll(among);
            if (__builtin_amdgcn_readlane(begin, i) <= r) group = g0 + i;
        }
        if (__builtin_amdgcn_readlane(begin, 63) > first + 63) break;
    }
    bool in = group >= 0 && r < gs.rows && (group + 1 < gs.n || r < end_of_all);
    if (disorder && in) in = begins(group) <= r && r < begins(group + 1);  // (else both were seen)
    return in ? group : -1;
}

// The group and the first row of the `tile`-th piece of `size` rows when the groups are cut up one after the other; false
// if there are not so many.  Every wavefront looks for itself, 64 groups at a time.
__device__ __forceinline__ bool find_rows(const Groups& gs, int tile, int size, GroupRows& found, int& first)
{
    if (!gs.offsets) {
        first = tile * size;
        found = {0, 0, gs.rows};
        return first < gs.rows;
    }
    int before = 0;  // tiles of the groups passed; stays at most `tile`
    for (int g0 = 0; g0 < gs.n; g0 += 64) {
        GroupRows r;
        int own;
        const int upto = tiles_upto(gs, g0, size, r, own);
        const unsigned long long beyond = __ballot(upto > tile - before);
        if (beyond) {
            const int l = __builtin_ctzll(beyond);
            found.g = scalar(g0 + l);
            found.begin = __builtin_amdgcn_readlane(r.begin, l);
            found.end = __builtin_amdgcn_readlane(r.end, l);
            first = found.begin + (tile - before - __builtin_amdgcn_readlane(upto - own, l)) * size;
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return false;
}

// ---------------------------------------------------------------------------------------------------------------
// Activations

// The normal distribution at z: the smaller of Phi(z) and 1 - Phi(z), and exp(-z^2 / 2).  With
// t = 1 / (1 + c |z|), exp(z^2 / 2) (1 - Phi(|z|)) is t times a polynomial in t, which with the coefficients as they stand is off by
// at most 2.0e-7 of the value for |z| up to 13.1 (beyond, both are below the smallest number).  The tail is measured to 5.4e-7 of it for |z| up
// to 2 and, as the exponent's rounding makes z^2 2^-24 of it, to 1.6e-6 at 5, 5.3e-6 at 10 and 7.7e-6 at 13.  The library's erfc takes five times as long, and with it the
// 256 x 256 tiles of a GELU layer spent a fifth of their time here.
struct NormalTail {
    float tail, bell;
};
__device__ __forceinline__ NormalTail normal_tail(float z)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.300520382f, fabsf(z), 1.f)), bell = __expf(-0.5f * z * z);
    float s = 0.0361404633f;
    s = fmaf(s, t, -0.158216909f);
    s = fmaf(s, t, 0.206578147f);
    s = fmaf(s, t, -0.0541327452f);
    s = fmaf(s, t, 0.128854472f);
    s = fmaf(s, t, 0.0999575415f);
    s = fmaf(s, t, 0.120983854f);
    s = fmaf(s, t, 0.11983513f);
    return {s * t * bell, bell};
}
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

template <int ACT>
__device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == PS_ACT_RELU) return z <= 0.f ? 0.f : z;
    if constexpr (ACT == PS_ACT_GELU) {
        const NormalTail n = normal_tail(z);
        return z * (z < 0.f ? n.tail : 1.f - n.tail);
    }
    if constexpr (ACT == PS_ACT_SILU) return z * logistic(z);
    return z;
}
__device__ __forceinline__ float activation_slope(float z, int act)
{
    if (act == PS_ACT_RELU) return z <= 0.f ? 0.f : 1.f;
    if (act == PS_ACT_GELU) {
        const NormalTail n = normal_tail(z);
        return fmaf(z * 0.39894228f, n.bell, z < 0.f ? n.tail : 1.f - n.tail);
    }
    if (act == PS_ACT_SILU) {
        const float s = logistic(z);
        return s * fmaf(z, 1.f - s, 1.f);
    }
    return 1.f;
}

// ---------------------------------------------------------------------------------------------------------------
// Matrix instructions: what 16 bytes of k of a row times 16 bytes of k of a column give.

template <class T>
struct Mma;
template <>
struct Mma<bf16_t> {
    static constexpr int E = 8;      // values in 16 bytes
    static constexpr int STEPS = 1;  // instructions
    static __device__ __forceinline__ void add(const uintx4& c, const uintx4& r, floatx4& acc)
    {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, c), __builtin_bit_cast(bf16x8, r), acc, 0, 0, 0);
    }
};
template <>
struct Mma<f16_t> {
    static constexpr int E = 8, STEPS = 1;
    static __device__ __forceinline__ void add(const uintx4& c, const uintx4& r, floatx4& acc)
    {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, c), __builtin_bit_cast(f16x8, r), acc, 0, 0, 0);
    }
};
template <>
struct Mma<float> {
    static constexpr int E = 4, STEPS = 4;
    static __device__ __forceinline__ void add(const uintx4& c, const uintx4& r, floatx4& acc)
    {
        // one k of each 16 bytes at a time
#pragma unroll
        for (int i = 0; i < 4; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(c[i]), __uint_as_float(r[i]), acc, 0, 0, 0);
    }
};

// ---------------------------------------------------------------------------------------------------------------
// 16 bytes for every lane from memory straight to LDS, one behind the other from `to` on (the same for all lanes).  Written as
// it is and not by its builtin, because the compiler has every transposing LDS read wait for all such loads that it knows of;
// it has no result that could be overwritten, and whoever reads what it brings waits for vmcnt himself.  (m0 cannot be named
// as changed: it is reserved, and the compiler sets it before each use of its own, of which there are none here.)
__device__ __forceinline__ void load_to_lds(uintx4 descriptor, uint32_t offset, int to)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" : : "v"(offset), "s"(descriptor), "s"(to) : "memory");
}
__device__ __forceinline__ int lds_address(const char* p) { return scalar((int)(uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p); }

// ---------------------------------------------------------------------------------------------------------------
// One operand's tile in LDS: ROWS rows (or columns) of the result, shared by W wavefronts along them, and 128 bytes of k;
// in HALVES pieces that are brought and read one after the other, each with its part of every wavefront's rows:
// row w * ROWS / W + h * EACH + i of the tile is row w * EACH + i of half h.
//
// KC: row r of a half at r * 128, its 16-byte pieces exchanged by a function of the row, so that 16 lanes that read the same
// piece of 16 rows, and 8 lanes that read it of 8, use all banks once.  RC: k at k * HROWS * sizeof(T), 32-byte groups
// (16 columns of a 16-bit type; 64 bytes of fp32) exchanged by a function of k for the same reason; the transposing LDS read
// (ds_read_b64_tr_b16: 16 lanes read 16 columns of four k, and each gets the four k of its column) turns 16-bit types.
// COLS: the operand that is the result's columns.  If it is KC, row 4q + e of the MFMA tiles 2t and 2t + 1 is column
// 32 t + 8 q + e and + 4, so that a lane ends up with eight consecutive columns.
//
// NT threads bring it, 16 bytes at a time.  DIRECT: memory to LDS without registers; rows start at multiples of 16 bytes
// and have multiples of 16 bytes, buffer bounds give zeros past the last row.  Else through registers, at any alignment.
template <class T, bool KC, bool COLS, int ROWS, int W, int HALVES, int NT, bool DIRECT>
struct Operand {
    static constexpr int SIZE = sizeof(T), E = 16 / SIZE, BK = 128 / SIZE;
    static constexpr int HROWS = ROWS / HALVES, EACH = HROWS / W;  // rows of a half, and of one wavefront in it
    static constexpr int HBYTES = HROWS * 128, BYTES = ROWS * 128, LOADS = HBYTES / (NT * 16);  // LOADS: instructions of a half
    static_assert(LOADS * NT * 16 == HBYTES, "every thread brings the same number of pieces");
    static constexpr int PIECES = HROWS / E;  // RC: pieces of one k
    static constexpr bool PERMUTED = KC && COLS;
    static_assert(EACH % (PERMUTED ? 32 : 16) == 0, "whole MFMA tiles, or pairs of them");
    static_assert(!DIRECT || (KC ? NT / 8 % 32 == 0 && (NT / 8 % EACH == 0 || EACH % (NT / 8) == 0) : NT / PIECES % 16 == 0), "the loads' places differ by the same for every thread");
    static constexpr int SUBS = 2;                            // reads of 16 bytes of k for each of the four lane groups
    static constexpr int READS = KC ? 1 : SIZE == 2 ? 2 : 4;  // LDS instructions of one
    // RC rows go on beside the tile's last column.  What is there enters only columns that nobody stores; but fp32 sums are all
    // looked at (those that the split cannot hold are formed again), so there those columns are left out.
    static constexpr bool CUT = DIRECT && !KC && SIZE == 4;

    const char* base;  // of the tile's first row (KC) or column (RC) and the first k of the next stage to be brought
    int64_t step;      // bytes from stage to stage
    int32_t pitch;     // bytes from row to row (KC) or from k to k (RC)
    int32_t left;      // k still to be brought
    int32_t rows;      // KC: valid rows of the tile; RC: valid columns
    uint32_t own_offset;  // byte from `base` of this thread's piece in the first load of the first half; past a row's end NOWHERE
    int32_t own_column;   // CUT: its first column, in every load of that half
    uintx4 reg[DIRECT ? 1 : LOADS];

    static __device__ __forceinline__ int kc_swap(int row)
    {
        return PERMUTED ? (row >> 1 & 1) | (row >> 3 & 1) << 1 | ((row ^ row >> 4) & 1) << 2 : (row >> 1 & 3) | ((row ^ row >> 3) & 1) << 2;
    }
    static __device__ __forceinline__ int rc_swap(int k)  // in 16-byte pieces
    {
        if (SIZE == 4) return (k >> 2 & 3) << 2;
        return HROWS >= 128 ? ((k & 3) | (k >> 3 & 1) << 2) << 1 : ((k >> 1 & 1) | (k >> 3 & 1) << 1) << 1;
    }
    // Piece i of thread t of a half: row (KC) or k (RC) of the tile, and element of k (KC) or column (RC) of the tile
    static __device__ __forceinline__ void place(int half, int i, int t, int& line, int& element)
    {
        const int f = i * NT + t;
        if (KC) {
            const int r = f >> 3;
            line = r / EACH * (EACH * HALVES) + half * EACH + r % EACH;
            element = ((f & 7) ^ kc_swap(r)) * E;
        } else {
            line = f / PIECES;
            const int c = ((f & (PIECES - 1)) ^ rc_swap(line)) * E;
            element = c / EACH * (EACH * HALVES) + half * EACH + c % EACH;
        }
    }

    // first: element of the tile's first row or column and the first k
    __device__ __forceinline__ void init(const T* first, int64_t stride, int valid, int depth, int t)
    {
        base = reinterpret_cast<const char*>(first);
        pitch = (int32_t)(stride * SIZE);
        step = KC ? 128 : (int64_t)pitch * BK;
        left = depth;
        rows = min(valid, ROWS);
        int line, element;
        place(0, 0, t, line, element);
        own_offset = line * pitch + element * SIZE;
        if (CUT) own_column = element;
        end_of_row(t);
    }
    static constexpr uint32_t NOWHERE = 0xfffffff0u;  // beyond what any descriptor allows, and so read as zero
    // KC: leaves out what is past the end of the rows, in the last stage and those behind it.
    __device__ __forceinline__ void end_of_row(int t)
    {
        if (KC && left < BK) {
            asm volatile("" : "+v"(t));  // worked out here, not kept in a register all along
            int line, element;
            place(0, 0, t, line, element);
            if (element >= left) own_offset = NOWHERE;
        }
    }

    // DIRECT: load i of a half of the next stage, or nothing past the last one, to the LDS address `tile` (of that half, and the wavefront's first piece).
    __device__ __forceinline__ void bring(int half, int i, int tile) const
    {
        // A load is at the same place for every thread but for what is the same for all of them, by which the descriptor's
        // base is moved.  What may be read ends, KC, with the last row; RC, with the last k.
        const int lines = KC ? rows : min(left, BK), last = (KC ? min(left, BK) : rows) * SIZE;
        const int bytes = (lines - 1) * pitch + last;  // without lines not above 0: they are no closer than they are long
        int line, element;
        place(half, i, 0, line, element);
        const int moved = line * pitch + element * SIZE;  // of thread 0, which is at 0 in the first load of the first half
        const uint64_t from = reinterpret_cast<uint64_t>(base) + (uint32_t)moved;
        uint32_t offset = own_offset;
        if (CUT && own_column + half * EACH >= rows) offset = NOWHERE;  // (columns are multiples of a piece)
        load_to_lds(uintx4{(uint32_t)scalar((int)from), (uint32_t)scalar((int)(from >> 32)) & 0xffffu, (uint32_t)scalar(max(bytes - moved, 0)), 0x00020000u}, offset,
                    tile + i * NT * 16);
    }
    // All of it
    __device__ __forceinline__ void bring(int half, int tile) const
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) bring(half, i, tile);
    }
    // Through registers: the whole next stage.
    __device__ __forceinline__ void load(int t)
    {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            int line, element;
            place(0, i, t, line, element);
            const int n = KC ? (line < rows ? left - element : 0) : (line < left ? rows - element : 0);
            const char* p = base + (int64_t)line * pitch + element * SIZE;
            uintx4 v = {0, 0, 0, 0};
            if (n >= E) {
                __builtin_memcpy(&v, p, 16);
            } else if (n > 0) {
                const T* q = reinterpret_cast<const T*>(p);
#pragma unroll
                for (int e = 0; e < E - 1; ++e) {
                    if (e >= n) continue;
                    if constexpr (SIZE == 4)
                        v[e] = __float_as_uint(q[e]);
                    else
                        v[e / 2] |= (uint32_t)q[e].bits << (16 * (e & 1));
                }
            }
            reg[i] = v;
        }
    }
    __device__ __forceinline__ void next_stage(int t)
    {
        base += step;
        left = max(left - BK, 0);
        if (DIRECT) end_of_row(t);
    }
    __device__ __forceinline__ void put(char* tile, int t) const
    {
        static_assert(DIRECT || HALVES == 1, "operands through registers come whole");
        if constexpr (!DIRECT) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) *reinterpret_cast<uintx4*>(tile + (i * NT + t) * 16) = reg[i];
        }
    }

    // 16 bytes of k of the lane's row in MFMA tile `tile16` of wavefront w's rows of a half, `tile`: k = (sub * 4 + lane / 16) * E ..
    static __device__ __forceinline__ uintx4 fetch(const char* tile, int w, int tile16, int sub, int lane)
    {
        const int l = lane & 15, q = lane >> 4, first = w * EACH;
        if constexpr (KC) {
            const int row = PERMUTED ? first + 32 * (tile16 >> 1) + 8 * (l >> 2) + 4 * (tile16 & 1) + (l & 3) : first + 16 * tile16 + l;
            return *reinterpret_cast<const uintx4*>(tile + row * 128 + (((sub * 4 + q) ^ kc_swap(row)) << 4));
        } else if constexpr (SIZE == 2) {
            typedef short shortx4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) shortx4* LdsPtr;
            const int k = 32 * sub + 8 * q + (l >> 2);
            const int piece = (2 * (first / 16 + tile16)) ^ rc_swap(k);
            const char* p = tile + k * (HROWS * 2) + piece * 16 + (l & 3) * 8;
            const uintx2 a = __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(shortx4*)p));
            const uintx2 b = __builtin_bit_cast(uintx2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(shortx4*)(p + 4 * HROWS * 2)));
            return uintx4{a[0], a[1], b[0], b[1]};
        } else {
            uintx4 v;
            const int col = first + 16 * tile16 + l;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int k = 16 * sub + 4 * q + e;
                v[e] = *reinterpret_cast<const uint32_t*>(tile + k * (HROWS * 4) + (((col >> 2) ^ rc_swap(k)) << 4) + (col & 3) * 4);
            }
            return v;
        }
    }
};

#endif  // __HIPCC__

// ---------------------------------------------------------------------------------------------------------------
// What becomes of the sums

struct Epilogue {
    // forward: y = act(sum + bias) + residual, pre = sum + bias; gradients: out = sum
    void* out;
    const void* bias;
    const void* residual;
    void* pre;
    int64_t out_row, residual_row, pre_row, bias_matrix, out_matrix;  // elements
    int32_t act;
    float* partial;  // if not null the sums go there instead, one result for each part of the contraction: [part][rows][cols]
    uint8_t *codes, *scales;  // KEPT: pre in 8 bits
    int64_t codes_row, scales_row;
};

#if defined(__HIPCC__)

// N consecutive columns of one row, of which `valid` exist: what is added to them (nothing is read where there is none),
// and what becomes of them.
template <class T, int N>
__device__ __forceinline__ void load_columns(const void* base, int64_t at, int valid, float (&x)[N])
{
    const T* p = static_cast<const T*>(base) + at;
    if (valid >= N)
        load_n(p, x);
    else
        load_some(p, valid, x);
}
template <class T, int N>
__device__ __forceinline__ void load_bias(const Epilogue& e, int matrix, int col, int valid, float (&x)[N])
{
    if (e.bias && valid > 0) load_columns<T>(e.bias, matrix * e.bias_matrix + col, valid, x);
}
template <class T, int N>
__device__ __forceinline__ void load_residual(const Epilogue& e, int64_t row, int col, int valid, float (&x)[N])
{
    if (e.residual && valid > 0) load_columns<T>(e.residual, row * e.residual_row + col, valid, x);
}
template <class T, int N>
__device__ __forceinline__ void store_columns(T* p, int valid, const float (&v)[N])
{
    if (valid >= N)
        store_n(p, v);
    else
        store_some(p, valid, v);
}
// sum + bias, rounded to T, in 8 bits; of a quad of lanes every one calls this, whatever `valid` is.
template <class T>
__device__ __forceinline__ void keep(const Epilogue& e, const float (&bias)[8], int64_t row, int col, int valid, const float (&v)[8])
{
    float z[8];
    if (e.bias) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = to_float(from_float<T>(v[i] + bias[i]));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = to_float(from_float<T>(v[i]));
    }
    if (valid < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = i < valid ? z[i] : 0.f;
    }
    checkpoint_store<T>(e.codes + row * e.codes_row, e.scales + row * e.scales_row, col, valid, z);
}
template <class T, bool RESIDUAL, int N>
__device__ __forceinline__ void finish(const Epilogue& e, const float (&bias)[N], const float (&residual)[N], int64_t row, int col, int valid, float (&v)[N])
{
    if (valid <= 0) return;
    if (e.bias) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += bias[i];
    }
    if (e.pre) store_columns(static_cast<T*>(e.pre) + row * e.pre_row + col, valid, v);
    if (e.act == PS_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activate<PS_ACT_RELU>(v[i]);
    } else if (e.act == PS_ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activate<PS_ACT_GELU>(v[i]);
    } else if (e.act == PS_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activate<PS_ACT_SILU>(v[i]);
    }
    if (RESIDUAL) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += residual[i];
    }
    store_columns(static_cast<T*>(e.out) + row * e.out_row + col, valid, v);
}

#endif

// ---------------------------------------------------------------------------------------------------------------
// The kernel

struct Product {
    const void *r, *c;                       // operands
    int64_t r_row, c_row, c_matrix;          // strides in elements; c_matrix between the matrices of C
    int32_t rows, cols, depth;               // of the result (RAGGED_K: per group) and of the contraction (RAGGED_K: of all groups), as the operands have them
    int32_t out_rows, out_cols;              // of the result as it is written: operands may be padded
    int32_t tiles_r, tiles_c;                // tiles along the rows (RAGGED_K: of all groups together) and columns
    int32_t parts, part_stages;              // the contraction in parts of so many stages each
    Groups groups;
    Epilogue epi;
};

// Which operand is ragged: rows of the result in groups (forward, input gradient), or the contraction (weight gradient).
enum { RAGGED_R = 0, RAGGED_K = 1 };

#if defined(__HIPCC__)

// Blocks are handed to the eight XCDs in turn; each XCD walks a contiguous range of tiles, in patches of `PATCH` tiles of
// rows, so that the tiles that run at the same time share their operands in the XCD's L2.
constexpr int PATCH = 4;
__device__ __forceinline__ bool tile_of_block(const Product& p, int tiles_r, int block, int& tr, int& tc, int& part)
{
    const int per_part = tiles_r * p.tiles_c, total = per_part * p.parts;
    const int per_xcd = (total + LINEAR_XCDS - 1) / LINEAR_XCDS, within = block / LINEAR_XCDS;
    int v = block % LINEAR_XCDS * per_xcd + within;
    if (within >= per_xcd || v >= total) return false;
    part = v / per_part;
    v -= part * per_part;
    const int band = v / (PATCH * p.tiles_c), first = band * PATCH, high = min(PATCH, tiles_r - first);
    v -= band * PATCH * p.tiles_c;
    tr = first + v % high;
    tc = v / high;
    return true;
}

// A dimension of a grid has less than 2^32 threads, which are 2^24 blocks of 256: tiles beyond ROW_OF_BLOCKS go along the second one.
constexpr int ROW_OF_BLOCKS = 1 << 23;
static_assert(ROW_OF_BLOCKS % LINEAR_XCDS == 0, "every row of blocks begins at the first XCD");

// One tile: its rows, columns and piece of the contraction.
struct Tile {
    int r0, r_valid, c0, c_valid, k_first, depth, matrix, group, part;
};
template <int BR, int BC, int BK, int RAGGED>
__device__ __forceinline__ bool find_tile(const Product& p, int tiles_r, int block, Tile& t)
{
    int tr, tc;
    if (!tile_of_block(p, tiles_r, block, tr, tc, t.part)) return false;
    GroupRows rows;
    t.depth = p.depth;
    t.k_first = 0;
    if (RAGGED == RAGGED_R) {
        if (!find_rows(p.groups, tr, BR, rows, t.r0)) return false;
        t.r_valid = rows.end - t.r0;
    } else {
        const int per_group = (p.rows + BR - 1) / BR;
        rows = group_rows(p.groups, tr / per_group);
        t.r0 = tr % per_group * BR;
        t.r_valid = p.rows - t.r0;
        t.k_first = rows.begin;
        t.depth = rows.end - rows.begin;
    }
    t.group = rows.g;
    t.matrix = RAGGED == RAGGED_R ? group_matrix(p.groups, rows.g) : 0;
    t.c0 = tc * BC;
    t.c_valid = p.cols - t.c0;
    if (p.parts > 1) {
        const int from = min(t.part * p.part_stages * BK, t.depth);
        t.k_first += from;
        t.depth = min(t.depth - from, p.part_stages * BK);
    }
    // the same for all lanes, which the compiler does not see behind a loop
    for (int* v : {&t.r0, &t.r_valid, &t.c0, &t.c_valid, &t.k_first, &t.depth, &t.matrix, &t.group, &t.part}) *v = scalar(*v);
    return true;
}

// Whether a kernel's blocks take one tile after the other, and the first operands of the next are on their way while the sums of
// this one are finished: those of 256 x 256, alone on their compute unit, for whose sums LDS has just room beside the operands
// (160 KB).  Against a block for each tile: bf16 8192 x 16384 x 4096 with GELU and pre-activations 959 -> 919 us, 32 groups of
// 512 rows 2048 -> 8192 890 -> 830.  Two blocks of 128 x 128 hide each other's beginnings and ends: 64 groups of 128
// rows, weight gradient 1568 -> 512, took 54 us with a block for each tile (49 now) and 60 this way.
constexpr bool linear_persistent(int tile_rows) { return tile_rows == 256; }

// The kernel's argument, read where it is used: the compiler would keep all of it in scalar registers, and have too few.
__device__ __forceinline__ const Product& argument()
{
    typedef const __attribute__((address_space(4))) Product* Constant;
    Constant p = (Constant)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return *(const Product*)p;
}

// s_waitcnt's argument: all but `n` of the wavefront's loads are done; everything of it is done.
constexpr int wait_vm(int n) { return (n & 15) | (n >> 4) << 14 | 0xf70; }
constexpr int WAIT_ALL = 0x0070;

// Barriers that wait for nothing in flight, and for the wavefront's own LDS reads; no memory access is moved across it.
__device__ __forceinline__ void block_barrier()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

__device__ __forceinline__ void block_barrier_after_reads()
{
    __builtin_amdgcn_s_waitcnt(0xc07f);
    block_barrier();
}

// KEPT: the forward pass keeps its pre-activations in 8 bits.
template <class T, bool R_KC, bool C_KC, int BR, int BC, int WR, int WC, bool DIRECT, int RAGGED, bool KEPT>
__global__ __launch_bounds__(64 * WR * WC, 2) void linear_kernel(Product p)
{
    constexpr int NT = 64 * WR * WC, TR = BR / WR / 16, TC = BC / WC / 16;
    constexpr bool SPLIT = sizeof(T) == 4, FORWARD_PASS = R_KC && C_KC;
    constexpr int HALVES = DIRECT && TR >= 4 && TC >= 4 ? 2 : 1, HR = TR / HALVES, HC = TC / HALVES;
    using OpR = Operand<T, R_KC, false, BR, WR, HALVES, NT, DIRECT>;
    using OpC = Operand<T, C_KC, true, BC, WC, HALVES, NT, DIRECT>;
    constexpr int BK = OpR::BK, SUBS = OpR::SUBS, STEPS = Mma<T>::STEPS;
    constexpr bool PERSISTENT = linear_persistent(BR);
    static_assert(!PERSISTENT || (HALVES == 2 && !SPLIT), "only this pipeline is begun ahead");
    constexpr int FINISH_PIECES = TC * 4;  // 16-byte pieces of a wavefront's row of sums
    constexpr int FINISH_BYTES = WR * WC * (PERSISTENT ? 1 : TR) * 16 * FINISH_PIECES * 16;
    // One array: where there are several, the compiler keeps account of what comes into which, and waits for more than it must.
    __shared__ __attribute__((aligned(256))) char lds[2 * (OpR::BYTES + OpC::BYTES) + (PERSISTENT ? FINISH_BYTES : 0)];
    static_assert(PERSISTENT || FINISH_BYTES <= 2 * (OpR::BYTES + OpC::BYTES), "the sums take the operands' place");
    constexpr int BUFFER = OpR::BYTES + OpC::BYTES;
    char *const r00 = lds, *const r01 = r00 + OpR::HBYTES, *const c00 = lds + OpR::BYTES, *const c01 = c00 + OpC::HBYTES;
    char *const r10 = r00 + BUFFER, *const c10 = c00 + BUFFER;

    const int tiles_r = RAGGED == RAGGED_R ? count_tiles(p.groups, BR, p.tiles_r) : p.tiles_r;
    const int tid = threadIdx.x, wave = scalar(tid >> 6);
    int lane = tid & 63;
    const int wr = wave / WC, wc = wave % WC;  // of eight wavefronts, two that share a SIMD have different rows
    Tile tile;
    int block = blockIdx.y * ROW_OF_BLOCKS + blockIdx.x;
    if (!find_tile<BR, BC, BK, RAGGED>(p, tiles_r, block, tile)) return;
    OpR opr;
    OpC opc;
    // What is worked out from the thread's number around the products is worked out there, not kept in registers all along.
    auto anew = [](int v) __attribute__((always_inline)) {
        asm volatile("" : "+v"(v));
        return v;
    };
    auto begin = [&]() __attribute__((always_inline)) {
        const Product& p = argument();
        const int tid = anew(threadIdx.x);
        opr.init(static_cast<const T*>(p.r) + (R_KC ? (int64_t)tile.r0 * p.r_row + tile.k_first : (int64_t)tile.k_first * p.r_row + tile.r0), p.r_row, tile.r_valid,
                     tile.depth, tid);
        opc.init(static_cast<const T*>(p.c) + tile.matrix * p.c_matrix + (C_KC ? (int64_t)tile.c0 * p.c_row + tile.k_first : (int64_t)tile.k_first * p.c_row + tile.c0),
                     p.c_row, tile.c_valid, tile.depth, tid);
    };
    begin();

    floatx4 acc[TR][TC];
    auto clear = [](auto& sums) __attribute__((always_inline)) {
        for (auto& row : sums)
            for (auto& sum : row) sum = floatx4{0.f, 0.f, 0.f, 0.f};
    };
    // fp32: the small terms of the split products, and whether the sums are to be formed without the split
    floatx4 small[SPLIT ? TR : 1][SPLIT ? TC : 1];
    uintx4 fr[HALVES][HR][SUBS], fc[HALVES][HC][SUBS];
    // where the wavefront's first piece of the first half comes in LDS, and the halves from there on
    const int to_first = lds_address(lds) + wave * 1024;
    constexpr int to_r[2] = {0, OpR::HBYTES}, to_c[2] = {OpR::BYTES, OpR::BYTES + OpC::HBYTES};
    auto bring_r = [&](int h, int buffer) __attribute__((always_inline)) { opr.bring(h, to_first + to_r[h] + buffer * BUFFER); };
    auto bring_c = [&](int h, int buffer) __attribute__((always_inline)) { opc.bring(h, to_first + to_c[h] + buffer * BUFFER); };
    auto fetch_r = [&](int h, const char* from, int sub) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < HR; ++i) fr[h][i][sub] = OpR::fetch(from, wr, i, sub, lane);
    };
    auto fetch_c = [&](const char* from, int sub, int set) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < HC; ++j) fc[set][j][sub] = OpC::fetch(from, wc, j, sub, lane);
    };
    auto multiply = [&](int hr, int hc, int sub, int set) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < HR; ++i)
#pragma unroll
            for (int j = 0; j < HC; ++j) Mma<T>::add(fc[set][j][sub], fr[hr][i][sub], acc[hr * HR + i][hc * HC + j]);
    };
    auto bring_two = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            bring_r(0, b);
            bring_c(0, b);
            bring_c(HALVES - 1, b);
            bring_r(HALVES - 1, b);
            opr.next_stage(tid);
            opc.next_stage(tid);
        }
    };
    if constexpr (PERSISTENT) bring_two();
    for (;;) {
        if constexpr (PERSISTENT && !R_KC) lane = anew(threadIdx.x) & 63;  // (for the other kinds this makes registers run out)
        clear(acc);
        const int stages = (tile.depth + BK - 1) / BK;
        if constexpr (SPLIT) {
            // fp32 products on the bf16 matrix instructions, operands split in three (ps_split.h), which are read as they are and split
            // by every wavefront that uses them: a column once a stage, a row's parts where they are used.  Splitting takes
            // 44 instructions, 176 cycles, for eight k of 16 rows, next to 96 cycles of matrix
            // instructions for each of the products that they enter.  4096^3: 677-735 us, six bf16 products at 1.1-1.2 PFLOP/s, of the
            // 1.3-1.4 that a bf16 product of such sizes gets from this chip's power; fp32 matrix instructions: 1050.  A block whose sums the split may not hold forms them all again with
            // fp32 matrix instructions: sums that are not finite, and those that are small next to what operands may have lost.  Parts are multiples
            // of 2^-133 (ps_split.h), so each product is off by at most 2^-133 of the largest operand that the wavefront meets (`top`), and a
            // sum of `depth` products that is 2^-109 depth top or more by 2^-24 of it; a sum of 0, where all of it may be lost, stands
            // if that is below 2^-80.  The largest takes four instructions beside the 44 (4096^3 651-673 -> 677-704 us).
            float top = 0.f;
            auto pass = [&](auto form) __attribute__((always_inline)) {
                constexpr bool exact = decltype(form)::value;
                auto products = [&](const char* r, const char* c) __attribute__((always_inline)) {
                    if constexpr (exact) {
#pragma unroll
                        for (int sub = 0; sub < SUBS; ++sub) {
#pragma unroll
                            for (int h = 0; h < HALVES; ++h) {
                                fetch_c(c + h * OpC::HBYTES, sub, h);
                                fetch_r(h, r + h * OpR::HBYTES, sub);
                            }
#pragma unroll
                            for (int h = 0; h < HALVES * HALVES; ++h) multiply(h / HALVES, h % HALVES, sub, h % HALVES);
                        }
                    } else {
                        auto parts = [&](const uintx4& x, const uintx4& y) __attribute__((always_inline)) {
                            float v[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e < 4 ? x[e] : y[e - 4]);
#pragma unroll
                            for (int e = 0; e < 8; e += 2) top = __builtin_elementwise_maximum(__builtin_elementwise_maximum(top, fabsf(v[e])), fabsf(v[e + 1]));
                            asm volatile("" : "+v"(top));  // now: left to the stage's end it would keep all operands in registers
                            return split8(v);
                        };
                        auto of_c = [&](int j, int sub) __attribute__((always_inline)) { return OpC::fetch(c + j / HC * OpC::HBYTES, wc, j % HC, sub, lane); };
                        auto of_r = [&](int i, int sub) __attribute__((always_inline)) { return OpR::fetch(r + i / HR * OpR::HBYTES, wr, i % HR, sub, lane); };
                        // The parts of one column or row are made while the matrix instructions of those before are under way, two vector
                        // instructions to each where there are 24 of them: columns during the first row's products (4096^3 3-5 % less time
                        // than without).
                        Split8 sc[TC], sr, next;
                        uintx4 x[2];
                        auto read = [&](int n) __attribute__((always_inline)) {  // column 0, row 0, columns 1 .., rows 1 ..
                            const bool column = n == 0 || (n > 1 && n <= TC);
                            const int k = n == 0 ? 0 : n == 1 ? 0 : column ? n - 1 : n - TC;
                            if (n >= TR + TC) return;
#pragma unroll
                            for (int sub = 0; sub < 2; ++sub) x[sub] = column ? of_c(k, sub) : of_r(k, sub);
                        };
                        // the read of that number, and then products with vector instructions between them
                        auto among = [](auto products, auto vector, int reads) __attribute__((always_inline)) {
                            if (reads < TR + TC) __builtin_amdgcn_sched_group_barrier(0x100, 2 * std::max(OpR::READS, OpC::READS), 0);
#pragma unroll
                            for (int k = 0; k < decltype(products)::value; ++k) {
                                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                                __builtin_amdgcn_sched_group_barrier(0x002, decltype(vector)::value, 0);
                            }
                            __builtin_amdgcn_sched_barrier(0);  // or all rows are fetched and split ahead, and registers run out
                        };
                        auto product = [&](int i, int j, int t) __attribute__((always_inline)) {
                            floatx4& to = t < SPLIT_SMALL ? small[i][j] : acc[i][j];
                            to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sc[j].part(TERM_A[t]), sr.part(TERM_B[t]), to, 0, 0, 0);
                        };
                        read(0);
                        const uintx4 first[2] = {x[0], x[1]};
                        read(1);
                        sc[0] = parts(first[0], first[1]);
                        sr = parts(x[0], x[1]);
                        read(2);
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int j = 0; j < TC; ++j) {
                            const uintx4 raw[2] = {x[0], x[1]};
                            read(j + 3);
                            if (j + 1 < TC)
                                sc[j + 1] = parts(raw[0], raw[1]);
                            else if (TR > 1)
                                next = parts(raw[0], raw[1]);
#pragma unroll
                            for (int t = 0; t <= SPLIT_SMALL; ++t) product(0, j, t);
                            among(std::integral_constant<int, SPLIT_SMALL + 1>{}, std::integral_constant<int, 8>{}, j + 3);
                        }
#pragma unroll
                        for (int i = 1; i < TR; ++i) {
                            sr = next;
                            const uintx4 raw[2] = {x[0], x[1]};
                            read(TC + i + 2);
                            if (i + 1 < TR) next = parts(raw[0], raw[1]);
#pragma unroll
                            for (int t = 0; t <= SPLIT_SMALL; ++t)
#pragma unroll
                                for (int j = 0; j < TC; ++j) product(i, j, t);
                            among(std::integral_constant<int, (SPLIT_SMALL + 1) * TC>{}, std::integral_constant<int, 2>{}, TC + i + 2);
                        }
                    }
                };
                if constexpr (DIRECT) {
                    constexpr int LOADS = HALVES * (OpR::LOADS + OpC::LOADS);
                    auto bring = [&](int buffer) __attribute__((always_inline)) {
#pragma unroll
                        for (int h = 0; h < HALVES; ++h) {
                            bring_r(h, buffer);
                            bring_c(h, buffer);
                        }
                        opr.next_stage(tid);
                        opc.next_stage(tid);
                    };
                    bring(0);
                    bring(1);
#pragma unroll 1
                    for (int s = 0; s < stages; ++s) {
                        int from = (s & 1) * BUFFER;  // unknown to the compiler, which would keep addresses for either buffer in registers
                        asm volatile("" : "+s"(from));
                        __builtin_amdgcn_s_waitcnt(wait_vm(LOADS));
                        block_barrier();
                        products(r00 + from, c00 + from);
                        block_barrier_after_reads();
                        bring(s & 1);
                    }
                    __builtin_amdgcn_s_waitcnt(wait_vm(0));  // LDS is given back with nothing on its way there
                } else {
                    for (int s = 0; s < stages; ++s) {
                        char *const r = s & 1 ? r10 : r00, *const c = s & 1 ? c10 : c00;
                        opr.load(tid);
                        opc.load(tid);
                        opr.put(r, tid);
                        opc.put(c, tid);
                        opr.next_stage(tid);
                        opc.next_stage(tid);
                        __syncthreads();
                        products(r, c);
                    }
                }
            };
            clear(small);
            pass(std::false_type{});
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) top = __builtin_elementwise_maximum(top, __shfl_xor(top, off, 64));
            const float reach = top * (float)tile.depth, least = fmaxf(SPLIT_TINY, reach * 0x1p-109f);  // (NaN only where sums are)
            const bool zero_too = reach >= 0x1p53f;
            bool lost = false;
#pragma unroll
            for (int i = 0; i < TR; ++i)
#pragma unroll
                for (int j = 0; j < TC; ++j) {
                    acc[i][j] += small[i][j];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float m = fabsf(acc[i][j][e]);
                        lost |= !(m < INFINITY) || (m < least && (m > 0.f || zero_too));
                    }
                }
            if (__syncthreads_or(lost)) {
                begin();
                clear(acc);
                pass(std::true_type{});
            }
        } else if constexpr (HALVES == 2) {
            // A stage in four phases, a quarter of the products each, in an order in which each phase needs one more half of an
            // operand: it is read from LDS in the phase before.
            //     products   R0 C0   R0 C1   R1 C1   R1 C0
            //     reads      C1      R1      R0'     C0'      (') of the next stage
            //     brings     R0"     C0"     C1"     R1"      (") of the stage after that, into this one's buffer
            // Two barriers a stage, behind the second and the fourth phase: past them everybody's part of what is read next is in
            // LDS, and nobody reads any more what is replaced next.  So a load has a stage and a half to arrive (with whole
            // operands and one barrier it had one).
            constexpr int FLIGHT = 2 * (OpR::LOADS + OpC::LOADS);
            static_assert(OpR::LOADS == 2 && OpC::LOADS == 2, "a phase places two loads");
            // A phase: the products of two halves, the reads of a third (`fetch`), and two loads, each behind a half of the products
            auto phase = [&](int hr, int hc, int set, auto fetch, auto load) __attribute__((always_inline)) {
                fetch();
                multiply(hr, hc, 0, set);
#pragma unroll
                for (int i = 0; i < HR * HC; ++i) {  // the reads among the products
                    __builtin_amdgcn_sched_group_barrier(0x008, STEPS, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, std::max(HR * OpR::READS, HC * OpC::READS) * SUBS / (HR * HC), 0);
                }
                __builtin_amdgcn_sched_barrier(0);
                load(0);
                multiply(hr, hc, 1, set);
                __builtin_amdgcn_sched_barrier(0);
                load(1);
            };
            auto arrived = [&]() __attribute__((always_inline)) {  // what is read next: everything but the last eight loads
                __builtin_amdgcn_s_waitcnt(wait_vm(FLIGHT) & ~0xf00);
                block_barrier();
            };
            // c0: the registers that hold C0 (those of C1 are free for the next stage's C0 when that is read)
            auto stage = [&](int buffer, int c0) __attribute__((always_inline)) {
                // unknown to the compiler, which would keep addresses for either buffer in registers, and have too few
                int from = buffer * BUFFER, from_next = BUFFER - from, to = to_first + from;
                asm volatile("" : "+s"(from), "+s"(from_next), "+s"(to));
                phase(0, 0, c0, [&]() __attribute__((always_inline)) {
                    fetch_c(c01 + from, 0, c0 ^ 1);
                    fetch_c(c01 + from, 1, c0 ^ 1);
                }, [&](int i) __attribute__((always_inline)) { opr.bring(0, i, to_r[0] + to); });
                phase(0, 1, c0 ^ 1, [&]() __attribute__((always_inline)) {
                    fetch_r(1, r01 + from, 0);
                    fetch_r(1, r01 + from, 1);
                }, [&](int i) __attribute__((always_inline)) { opc.bring(0, i, to_c[0] + to); });
                arrived();
                phase(1, 1, c0 ^ 1, [&]() __attribute__((always_inline)) {
                    fetch_r(0, r00 + from_next, 0);  // behind the last stage what lay there before, which nobody uses
                    fetch_r(0, r00 + from_next, 1);
                }, [&](int i) __attribute__((always_inline)) { opc.bring(1, i, to_c[1] + to); });
                phase(1, 0, c0, [&]() __attribute__((always_inline)) {
                    fetch_c(c00 + from_next, 0, c0 ^ 1);
                    fetch_c(c00 + from_next, 1, c0 ^ 1);
                }, [&](int i) __attribute__((always_inline)) { opr.bring(1, i, to_r[1] + to); });
                opr.next_stage(tid);
                opc.next_stage(tid);
                arrived();
            };
            if constexpr (!PERSISTENT) bring_two();
            arrived();
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub) {
                fetch_c(c00, sub, 0);
                fetch_r(0, r00, sub);
            }
            block_barrier_after_reads();
            // In a tile that is not whole, a wavefront without rows or columns of the result brings its share and no more.
            if (wr * (BR / WR) < tile.r_valid && wc * (BC / WC) < tile.c_valid) {
                for (int s = 0; s < stages; s += 2) {
                    stage(0, 0);
                    if (s + 1 < stages) stage(1, 1);
                }
            } else {
#pragma unroll 1
                for (int s = 0; s < stages; ++s) {
                    bring_r(0, s & 1);
                    bring_c(0, s & 1);
                    arrived();
                    bring_c(1, s & 1);
                    bring_r(1, s & 1);
                    opr.next_stage(tid);
                    opc.next_stage(tid);
                    arrived();
                }
            }
            __builtin_amdgcn_s_waitcnt(wait_vm(0));  // LDS is given back with nothing on its way there
        } else if constexpr (DIRECT) {
            // While the products of one half of a stage's k are formed, the operands of the next half are on their way from LDS to
            // registers, and those of the next stage from memory to LDS.  One barrier a stage, in its middle: past it everybody's
            // part of the next stage is in LDS, and nobody reads this one's buffer any more, which then takes the stage after next.
            auto bring = [&](int buffer) __attribute__((always_inline)) {
                bring_r(0, buffer);
                bring_c(0, buffer);
                opr.next_stage(tid);
                opc.next_stage(tid);
            };
            auto fetch = [&](const char* r, const char* c, int sub) __attribute__((always_inline)) {
                fetch_c(c, sub, 0);
                fetch_r(0, r, sub);
            };
            constexpr int LOADS = OpR::LOADS + OpC::LOADS;
            bring(0);
            bring(1);
            __builtin_amdgcn_s_waitcnt(wait_vm(LOADS));
            block_barrier();
            fetch(r00, c00, 0);
            auto stage = [&](int buffer) __attribute__((always_inline)) {
                fetch(buffer ? r10 : r00, buffer ? c10 : c00, 1);
                multiply(0, 0, 0, 0);
                __builtin_amdgcn_s_waitcnt(WAIT_ALL);
                block_barrier();
                fetch(buffer ? r00 : r10, buffer ? c00 : c10, 0);  // behind the last stage what lay there before, which nobody uses
                multiply(0, 0, 1, 0);
                bring(buffer);
            };
            for (int s = 0; s < stages; s += 2) {
                stage(0);
                if (s + 1 < stages) stage(1);
            }
            __builtin_amdgcn_s_waitcnt(wait_vm(0));  // LDS is given back with nothing on its way there
        } else {
            if (stages > 0) {
                opr.load(tid);
                opc.load(tid);
                opr.put(r00, tid);
                opc.put(c00, tid);
            }
            __syncthreads();
            for (int s = 0; s < stages; ++s) {
                const char *r = s & 1 ? r10 : r00, *c = s & 1 ? c10 : c00;
                char *r_next = s & 1 ? r00 : r10, *c_next = s & 1 ? c00 : c10;
                if (s + 1 < stages) {
                    opr.next_stage(tid);
                    opc.next_stage(tid);
                    opr.load(tid);
                    opc.load(tid);
                }
#pragma unroll
                for (int sub = 0; sub < SUBS; ++sub) {
                    fetch_c(c, sub, 0);
                    fetch_r(0, r, sub);
                    multiply(0, 0, sub, 0);
                }
                if (s + 1 < stages) {
                    opr.put(r_next, tid);
                    opc.put(c_next, tid);
                }
                __syncthreads();
            }
        }

        // Lane (q, l) has row 16 i + l, columns 16 j + 4 q + e, or, permuted, 32 j / 2 + 8 q + 4 (j & 1) + e.  The sums go through
        // LDS, 16 rows of a wavefront at a time, so that it stores whole cache lines, and the code that finishes them, of which only
        // one way is taken, is there once (a copy for every MFMA tile made 150 KB, and its way through the instruction cache
        // took 5 us a tile).
        // What comes to LDS for the next tile is older than the stores here, and the loads of what is added
        // wait for it too; so the bias is there before, once for the tile.
        Epilogue epi = argument().epi;  // copies: behind a store the argument would be read again
        if constexpr (KEPT) epi.pre = nullptr;
        const int rows = argument().out_rows, cols = argument().out_cols;
        constexpr int PIECES = FINISH_PIECES, LANES = TC * 2, AT_ONCE = 64 / LANES;  // lanes of a row, rows at once
        const Tile done = tile;
        const int lane = anew(threadIdx.x) & 63, l = lane & 15, q = lane >> 4;
        const int at = lane % LANES, c = wc * TC * 16 + 8 * at, c_valid = cols - done.c0 - c;  // the lane's eight columns
        const int r_valid = RAGGED == RAGGED_K ? rows - done.r0 : done.r_valid;
        float bias[8];
        if constexpr (FORWARD_PASS) load_bias<T>(epi, done.matrix, done.c0 + c, c_valid, bias);
        block_barrier();  // nobody reads what comes, or these sums, take the place of
        bool more = false;
        if constexpr (PERSISTENT) {
            block += gridDim.x;  // (as many as compute units, in one row)
            more = find_tile<BR, BC, BK, RAGGED>(argument(), tiles_r, block, tile);
            if (FORWARD_PASS && epi.bias) {
#pragma unroll
                for (int e = 0; e < 8; ++e) asm volatile("" : "+v"(bias[e]));
            }
            if (more) {
                begin();
                bring_two();
            }
        }
        constexpr int TURN = PERSISTENT ? 1 : TR;  // MFMA tiles of rows that go through LDS at once: all, where they take the operands' place
        char* const mine = lds + (PERSISTENT ? 2 * BUFFER : 0) + wave * (TURN * 16 * PIECES * 16);
#pragma unroll 1
        for (int i = 0; i < TR; i += TURN) {
#pragma unroll
            for (int k = 0; k < TR; ++k) {
                if (TURN == 1 && k != i) continue;  // the registers of a row of tiles have to be named
#pragma unroll
                for (int j = 0; j < TC; ++j) {
                    const int piece = OpC::PERMUTED ? 8 * (j / 2) + 2 * q + (j & 1) : 4 * j + q;
                    *reinterpret_cast<floatx4*>(mine + (k % TURN * 16 + l) * (PIECES * 16) + ((piece ^ (l & (PIECES - 1))) << 4)) = acc[k][j];
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            auto take = [&](int row, floatx4 (&x)[2]) __attribute__((always_inline)) {
#pragma unroll
                for (int e = 0; e < 2; ++e) x[e] = *reinterpret_cast<const floatx4*>(mine + row * (PIECES * 16) + (((2 * at + e) ^ (row & (PIECES - 1))) << 4));
            };
            // A loop of its own where there is a residual: behind its loads, taken or not, the compiler waits for all stores before.
            auto finish_rows = [&](auto residual_too) __attribute__((always_inline)) {
                constexpr bool RESIDUAL = decltype(residual_too)::value;
                floatx4 x[2];
                take(lane / LANES, x);
#pragma unroll 1
                for (int h = 0; h < TURN * 16; h += AT_ONCE) {
                    const int row = h + lane / LANES, r = (wr * TR + i) * 16 + row, valid = r < r_valid ? c_valid : 0;
                    float v[8], residual[8];
                    if constexpr (RESIDUAL) load_residual<T>(epi, done.r0 + r, done.c0 + c, valid, residual);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = x[e / 4][e % 4];
                    take(h + AT_ONCE < TURN * 16 ? row + AT_ONCE : row, x);
                    if constexpr (KEPT) {
                        if (r < r_valid && !epi.partial) keep<T>(epi, bias, done.r0 + r, done.c0 + c, c_valid, v);
                    }
                    if (valid <= 0) continue;
                    if (epi.partial) {
                        float* to = epi.partial + ((int64_t)done.part * rows + (done.r0 + r)) * cols + done.c0 + c;
                        store_columns(to, valid, v);
                    } else if constexpr (FORWARD_PASS) {
                        finish<T, RESIDUAL>(epi, bias, residual, done.r0 + r, done.c0 + c, valid, v);
                    } else {
                        store_columns(static_cast<T*>(epi.out) + (RAGGED == RAGGED_K ? done.group : 0) * epi.out_matrix + (done.r0 + r) * epi.out_row + done.c0 + c, valid, v);
                    }
                }
            };
            if constexpr (FORWARD_PASS) {
                if (epi.residual && !epi.partial)
                    finish_rows(std::true_type{});
                else
                    finish_rows(std::false_type{});
            } else {
                finish_rows(std::false_type{});
            }
            if constexpr (TURN < TR) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // read before the next rows are written
        }
        if (!more) return;
    }
}

#endif

// Launchers, one file each (kinds of operands): forward, input gradient, weight gradient.
void launch_linear_forward(const Product& p, int dtype, bool direct, int tile, hipStream_t s);
void launch_linear_forward_kept(const Product& p, int dtype, bool direct, int tile, hipStream_t s);
void launch_linear_dx(const Product& p, int dtype, bool direct, int tile, hipStream_t s);
void launch_linear_dw(const Product& p, int dtype, bool direct, int tile, hipStream_t s);

// Forward pass for few rows, 16 * row_tiles of a group (1 to 4) to a block; tiles_r counts these, tiles_c 16 columns each.
void launch_linear_few(const Product& p, int dtype, int row_tiles, hipStream_t s);
// Input gradient for few rows (row_tiles 1 or 2); tiles_c counts 16 * (16 bytes) of columns each, of which there are at least 16 bytes; the
// contraction in parts of part_stages steps of FEW_DX_STEP / (bytes of a value).
void launch_linear_few_dx(const Product& p, int dtype, int row_tiles, hipStream_t s);
constexpr int FEW_DX_STEP = 64;

// Sizes of square tiles, by number.
constexpr int LINEAR_TILE[3] = {64, 128, 256};

#if defined(__HIPCC__)
template <class T, bool R_KC, bool C_KC, bool DIRECT, int RAGGED, bool KEPT>
void start_linear(const Product& p, int tile, hipStream_t s)
{
    const int total = (p.tiles_r * p.tiles_c * p.parts + LINEAR_XCDS - 1) / LINEAR_XCDS * LINEAR_XCDS;
    const dim3 grid(std::min(total, ROW_OF_BLOCKS), (total + ROW_OF_BLOCKS - 1) / ROW_OF_BLOCKS);  // blocks past the last tile end at once
    if (tile == 0)
        hipLaunchKernelGGL((linear_kernel<T, R_KC, C_KC, 64, 64, 2, 2, DIRECT, RAGGED, KEPT>), grid, dim3(256), 0, s, p);
    else if (tile == 1 || !DIRECT || sizeof(T) == 4)
        hipLaunchKernelGGL((linear_kernel<T, R_KC, C_KC, 128, 128, 2, 2, DIRECT, RAGGED, KEPT>), grid, dim3(256), 0, s, p);
    else if constexpr (DIRECT && sizeof(T) == 2) {
        static_assert(linear_persistent(256), "a block for each tile would have to be counted as above");
        hipLaunchKernelGGL((linear_kernel<T, R_KC, C_KC, 256, 256, 2, 4, DIRECT, RAGGED, KEPT>), dim3(std::min(total, COMPUTE_UNITS)), dim3(512), 0, s, p);
    }
}
template <bool R_KC, bool C_KC, int RAGGED, bool KEPT = false>
void start_linear_typed(const Product& p, int dtype, bool direct, int tile, hipStream_t s)
{
    if (dtype == PS_F32)
        direct ? start_linear<float, R_KC, C_KC, true, RAGGED, KEPT>(p, tile, s) : start_linear<float, R_KC, C_KC, false, RAGGED, KEPT>(p, tile, s);
    else if (dtype == PS_BF16)
        direct ? start_linear<bf16_t, R_KC, C_KC, true, RAGGED, KEPT>(p, tile, s) : start_linear<bf16_t, R_KC, C_KC, false, RAGGED, KEPT>(p, tile, s);
    else
        direct ? start_linear<f16_t, R_KC, C_KC, true, RAGGED, KEPT>(p, tile, s) : start_linear<f16_t, R_KC, C_KC, false, RAGGED, KEPT>(p, tile, s);
}
#endif

}  // namespace ps
