// Log probabilities of given tokens, entropies, the most probable alternatives, and the gradient of the first two
// (include/ps_tokens.h).
//
// With t = (z - m) scale log2(e), a row needs s = sum 2^t and u = sum t 2^t for its largest z, m: L = log s and the entropy is
// log s - ln 2 u / s.  Each lane keeps m, s and u of the values that it has seen, in one pass: when m grows by d (in units of t),
// s becomes 2^-d s and u becomes 2^-d (u - d s).
#include "../../include/ps_tokens.h"
#include "ps_linear.h"
#include "ps_tokens.h"

#include <cmath>

namespace ps {
namespace {

constexpr int VECTORS = 4;  // of 16 bytes that a lane asks for together
constexpr float LOG2E = 1.44269504f, LN2 = 0.693147181f;
constexpr float NEVER = -300.f;  // 2^NEVER is 0, and times NEVER too: what -infinity is taken to where t is multiplied

__device__ __forceinline__ float negative_infinity() { return __uint_as_float(0xff800000u); }

// ---- keys of values ------------------------------------------------------------------------------------------------------

// Values in the order of their keys: the larger value first, among equals the lower index.  0 is no key of a value.
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t b = __float_as_uint(v + 0.f);  // -0 is 0
    return b ^ (uint32_t)((int32_t)b >> 31) ^ (b >> 31 ? 0u : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint64_t key)
{
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o >> 31 ? o ^ 0x80000000u : ~o);
}
__device__ __forceinline__ uint64_t key_of(float v, int index) { return (uint64_t)ordered(v) << 32 | (uint32_t)~index; }
__device__ __forceinline__ int index_of(uint64_t key) { return (int)~(uint32_t)key; }

// ---- forward -----------------------------------------------------------------------------------------------------------

struct ForwardArgs {
    const void *logits, *tokens;
    float *logp, *norm, *top_logp;
    int32_t* top_tokens;
    float* part_sums;      // [row][part][3], where a row is cut into parts
    uint64_t* part_lists;  // [row][part][top]
    int64_t row, token_stride, rows;
    int32_t vocab, token_bytes, top, parts, part_rounds;
    float scale;
};

__device__ __forceinline__ int64_t token_of_row(const void* tokens, int bytes, int64_t at)
{
    return bytes == 4 ? (int64_t) static_cast<const int32_t*>(tokens)[at] : static_cast<const int64_t*>(tokens)[at];
}

struct Sums {
    float m, s, u;
};
// c: scale log2(e)
__device__ __forceinline__ Sums join(Sums a, Sums b, float c)
{
    const float m = fmaxf(a.m, b.m);
    auto part = [&](const Sums& x, float& s, float& u) __attribute__((always_inline)) {
        const float d = x.m == m ? 0.f : fmaxf((x.m - m) * c, NEVER), f = __builtin_amdgcn_exp2f(d);
        s = x.s * f;
        u = (x.u + d * x.s) * f;
    };
    float s0, u0, s1, u1;
    part(a, s0, u0);
    part(b, s1, u1);
    return {m, s0 + s1, u0 + u1};
}
__device__ __forceinline__ Sums join_lanes(Sums x, float c)
{
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) x = join(x, Sums{__shfl_xor(x.m, off, 64), __shfl_xor(x.s, off, 64), __shfl_xor(x.u, off, 64)}, c);
    return x;
}

// What a row's sums and its token give; one thread.
template <class T>
__device__ __forceinline__ void finish_row(const ForwardArgs& a, int64_t row, const Sums& x, int64_t token, float at_token)
{
    const bool none = x.m == negative_infinity() && x.s == 0.f;
    const float log_s = logf(x.s);  // -infinity where there is none
    a.norm[row * 3] = x.m;
    a.norm[row * 3 + 1] = log_s;
    a.norm[row * 3 + 2] = none ? 0.f : log_s - LN2 * (x.u / x.s);
    if (a.logp) a.logp[row] = token < 0 || token >= a.vocab ? 0.f : none ? negative_infinity() : (at_token - x.m) * a.scale - log_s;
}
// The row's token and its logit, asked for before they are needed
template <class T>
__device__ __forceinline__ int64_t take_token(const ForwardArgs& a, int64_t row, float& at_token)
{
    int64_t t = -1;
    if (a.logp) t = token_of_row(a.tokens, a.token_bytes, row * a.token_stride);
    const T* z = static_cast<const T*>(a.logits) + row * a.row;
    at_token = to_float(z[min(max(t, (int64_t)0), (int64_t)a.vocab - 1)]);
    return t;
}

__device__ __forceinline__ void write_best(const ForwardArgs& a, int64_t row, int place, uint64_t key, const Sums& x)
{
    a.top_logp[row * a.top + place] = key ? (value_of(key) - x.m) * a.scale - logf(x.s) : negative_infinity();
    a.top_tokens[row * a.top + place] = key ? index_of(key) : -1;
}

// A row (or part of one) as WAVES wavefronts see it: vectors of 16 bytes at multiples of 16 bytes in memory, of which the row begins `ahead`
// values behind the first one's beginning.  Vector v has columns v * E - ahead on; those from `first` to `end` are the part's.
template <class T, int WAVES>
struct Range {
    static constexpr int E = 16 / sizeof(T), THREADS = WAVES * 64;
    const T* z;
    int first, end, ahead, vocab;

    __device__ __forceinline__ int column(int v) const { return v * E - ahead; }
    // A vector that goes past an end of the row is read where the row's first or last one is, so that nothing is read in a branch, where the compiler
    // would wait for it, or beside the row; `leave_out` makes -infinity of what is no column of the vector, or of a vector of none of the
    // range's.  `from`: the column of the first value that was read.
    __device__ __forceinline__ int from(int v) const { return vocab >= E ? min(max(column(v), 0), vocab - E) : column(v); }
    __device__ __forceinline__ void take(int v, uintx4& raw) const
    {
        if (vocab >= E) {
            __builtin_memcpy(&raw, z + from(v), 16);
        } else {
            T x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = z[min(max(column(v) + e, 0), vocab - 1)];
            __builtin_memcpy(&raw, x, 16);
        }
    }
    __device__ __forceinline__ void leave_out(int v, uintx4& raw) const
    {
        // from + e is in the vector and the row
        const int at = column(v), lo = max(at, 0) - from(v), hi = v < end ? min(at + E, vocab) - from(v) : 0;
        constexpr int IN_DWORD = E / 4;
        constexpr uint32_t LEFT_OUT = sizeof(T) == 4 ? 0xff800000u : __is_same(T, bf16_t) ? 0xff80ff80u : 0xfc00fc00u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t in = 0;
#pragma unroll
            for (int k = 0; k < IN_DWORD; ++k) {
                const int e = i * IN_DWORD + k;
                in |= e >= lo && e < hi ? (IN_DWORD == 1 ? ~0u : 0xffffu << 16 * k) : 0u;
            }
            raw[i] = (raw[i] & in) | (LEFT_OUT & ~in);
        }
    }
};

// The best `top` values of a range.  Each lane knows the largest of its own values; the top-th largest of these is a value that at least
// `top` values reach, and only lanes whose largest reaches it can have one of the best: these lanes' vectors, few, are read again, and
// what reaches it (but for its lower bits) is listed.  Where more than LIST do (equal values), what is above it is listed, and then the first that
// equal it; where that is too much as well (large values that fewer lanes have than there are alternatives), the top-th value itself is
// found bit by bit, in 32 passes over the row.  4096 rows of 50257 in bf16 with 5 alternatives: 95 us, masks of the lowest value 93, all equal
// 341, large values in three lanes only 3017.  A value's place is the number of listed keys above its own, so the order in which they were
// listed does not matter.
constexpr int LIST = 256;
template <int WAVES>
struct Scratch {
    uint64_t list[LIST + PS_LOGPROB_MAX_TOP], best[PS_LOGPROB_MAX_TOP];
    float high[WAVES * 64];
    uint16_t lanes[WAVES * 64];
    int n_lanes, count, wave_count[WAVES];
    uint32_t from;
};

template <int WAVES>
__device__ __forceinline__ void meet_all()
{
    if constexpr (WAVES > 1)
        __syncthreads();
    else
        wave_meets();
}

// The k-th largest of the lanes' values (with more than four wavefronts, of the largest of four lanes each), from bit `high_bit` to `low_bit` of
// its number; what is above is in `least`, what is below left out, so that as many reach it.  For a whole wavefront.
template <int WAVES>
__device__ __forceinline__ uint32_t kth_of_lanes(const float* high, int k, uint32_t least = 0, int high_bit = 31, int low_bit = 16)
{
    constexpr int EACH = WAVES < 4 ? WAVES : 4;
    uint32_t o[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        float v = high[i * 64 + (threadIdx.x & 63)];
#pragma unroll
        for (int w = i + EACH; w < WAVES; w += EACH) v = fmaxf(v, high[w * 64 + (threadIdx.x & 63)]);
        o[i] = ordered(v);
    }
    for (int b = high_bit; b >= low_bit; --b) {
        const uint32_t more = least | 1u << b;
        int n = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) n += __popcll(__ballot(o[i] >= more));
        if (n >= k) least = more;
    }
    return least;
}

template <class T, int WAVES>
__device__ __forceinline__ void best_of_range(const Range<T, WAVES>& r, Scratch<WAVES>& s, int top, int each, float high)
{
    constexpr int E = Range<T, WAVES>::E, THREADS = Range<T, WAVES>::THREADS;
    const int t = threadIdx.x % THREADS, wave = t / 64, lane = t & 63;
    s.high[t] = high;
    if (t == 0) s.n_lanes = s.count = 0;
    if (t < top) s.best[t] = 0;
    meet_all<WAVES>();
    if (wave == 0) {
        const uint32_t from = kth_of_lanes<WAVES>(s.high, top);
        if (lane == 0) s.from = from;
    }
    meet_all<WAVES>();
    uint32_t from = s.from;
    if (high > negative_infinity() && ordered(high) >= from) s.lanes[atomicAdd(&s.n_lanes, 1)] = (uint16_t)t;
    meet_all<WAVES>();
    auto list = [&](bool has, float v, int index) __attribute__((always_inline)) {
        if (!has) return;
        const int place = atomicAdd(&s.count, 1);
        if (place < LIST) s.list[place] = key_of(v, index);
    };
    // whether v is a value, and reaches or passes a number of `ordered`
    auto reaches = [](float v, uint32_t o) __attribute__((always_inline)) { return v > negative_infinity() && ordered(v) >= o; };
    auto passes = [](float v, uint32_t o) __attribute__((always_inline)) { return v > negative_infinity() && ordered(v) > o; };
    const int items = s.n_lanes * each;  // `each` vectors of a lane
    for (int i = t; i < items; i += THREADS) {
        const int q = s.lanes[i / each], n = i % each;
        const int v = r.first + (n * WAVES + q / 64) * 64 + (q & 63);
        uintx4 raw;
        const int at = r.from(v);
        r.take(v, raw);
        r.leave_out(v, raw);
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float x = element<T>(raw, e);
            list(reaches(x, from), x, at + e);
        }
    }
    meet_all<WAVES>();
    int n = s.count;
    if (n > LIST) {
        auto every = [&](auto f) __attribute__((always_inline)) {  // all values of the range
            for (int v = r.first + t; v < r.end; v += THREADS) {
                uintx4 raw;
                const int at = r.from(v);
                r.take(v, raw);
                r.leave_out(v, raw);
#pragma unroll
                for (int e = 0; e < E; ++e) f(element<T>(raw, e), at + e);
            }
        };
        auto list_above = [&]() __attribute__((always_inline)) {
            meet_all<WAVES>();
            if (t == 0) s.count = 0;
            meet_all<WAVES>();
            every([&](float x, int index) { list(passes(x, from), x, index); });
            meet_all<WAVES>();
            return s.count;
        };
        // the top-th largest lane's value to its last bit, so that what equals it is told from what is above
        if (wave == 0) {
            from = kth_of_lanes<WAVES>(s.high, top, from, 15, 0);
            if (lane == 0) s.from = from;
        }
        meet_all<WAVES>();
        from = s.from;
        n = list_above();
        if (n > LIST) {
            from = 0;
            for (int b = 31; b >= 0; --b) {
                meet_all<WAVES>();
                if (t == 0) s.count = 0;
                meet_all<WAVES>();
                int mine = 0;
                every([&](float x, int) { mine += reaches(x, from | 1u << b); });
                atomicAdd(&s.count, mine);
                meet_all<WAVES>();
                if (s.count >= top) from |= 1u << b;
            }
            n = list_above();  // fewer than `top`
        }
        // the first ones that equal it
        for (int v0 = r.first; n < top && v0 < r.end; v0 += THREADS) {
            uintx4 raw;
            const int at = r.from(v0 + t);
            r.take(v0 + t, raw);
            r.leave_out(v0 + t, raw);
            int mine = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float x = element<T>(raw, e);
                mine += reaches(x, from) && !passes(x, from);
            }
            int upto = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int other = __shfl_up(upto, d, 64);
                if (lane >= d) upto += other;
            }
            if (lane == 63) s.wave_count[wave] = upto;
            meet_all<WAVES>();
            int place = n + upto - mine, all = 0;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) {
                if (k < wave) place += s.wave_count[k];
                all += s.wave_count[k];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float x = element<T>(raw, e);
                if (!reaches(x, from) || passes(x, from)) continue;
                if (place < top) s.list[place] = key_of(x, at + e);
                ++place;
            }
            n = min(n + all, top);
            meet_all<WAVES>();
        }
    }
    for (int i = t; i < n; i += THREADS) {
        const uint64_t key = s.list[i];
        int place = 0;
#pragma unroll 4
        for (int k = 0; k < n; ++k) place += s.list[k] > key;
        if (place < top) s.best[place] = key;
    }
    meet_all<WAVES>();
}

// WAVES wavefronts take a row, or a part of one, in rounds of VECTORS vectors to a lane; the next round is asked for before the present
// one is worked on.  Where rows are few, parts of them are blocks of their own, and join_row_kernel finishes.  Bound by memory; behind it by
// the vector ALU: about ten operations and an exponential for a value.  bf16, 4096 rows of 50257: 83 us, 4.9 TB/s, with 5 alternatives 90; fp32 144 and
// 152 us, 5.7 TB/s.
template <class T, int WAVES, bool TOP>
__global__ __launch_bounds__(WAVES > 4 ? WAVES * 64 : 256) void logprob_kernel(ForwardArgs a)
{
    constexpr int E = 16 / sizeof(T), ROWS = WAVES < 4 ? 4 / WAVES : 1;  // rows of a block
    constexpr int EACH = 64 * VECTORS;                   // vectors of a wavefront in a round, 64 of each 64 * WAVES
    __shared__ Scratch<WAVES> scratch[TOP ? ROWS : 1];
    __shared__ Sums meet[ROWS * WAVES];
    const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6), w = wave % WAVES, of = wave / WAVES;
    const float c = a.scale * LOG2E;
    const int64_t total = a.rows * a.parts;
    for (int64_t block = (int64_t)blockIdx.x * ROWS; block < total; block += (int64_t)gridDim.x * ROWS) {
        const bool there = block + of < total;
        const int64_t item = there ? block + of : total - 1, row = item / a.parts;
        const int part = (int)(item - row * a.parts);
        Range<T, WAVES> r;
        r.z = static_cast<const T*>(a.logits) + row * a.row;
        r.vocab = a.vocab;
        r.ahead = (int)(reinterpret_cast<uintptr_t>(r.z) / sizeof(T) % E);
        const int vectors = (a.vocab + r.ahead + E - 1) / E, of_part = a.part_rounds * (WAVES * EACH);
        r.first = part * of_part;
        r.end = part + 1 < a.parts ? min(r.first + of_part, vectors) : vectors;
        float at_token = 0.f;
        const int64_t token = a.parts == 1 ? take_token<T>(a, row, at_token) : -1;
        Sums sums{negative_infinity(), 0.f, 0.f};
        // Vector j of a round is v + j * WAVES * 64; `all` of n from v on are whole ones of the range.
        auto all = [&](int v, int n) __attribute__((always_inline)) { return r.column(v) >= 0 && r.column(v + n) <= a.vocab && v + n <= r.end; };
        auto take = [&](int v, uintx4 (&raw)[VECTORS]) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < VECTORS; ++j) r.take(v + j * WAVES * 64 + lane, raw[j]);
        };
        auto add = [&](const auto& raw) __attribute__((always_inline)) {
            float high = negative_infinity();
            for (const uintx4& x : raw) {
#pragma unroll
                for (int e = 0; e < E; ++e) high = fmaxf(high, element<T>(x, e));
            }
            if (high > sums.m) {
                const float d = fmaxf((sums.m - high) * c, NEVER), f = __builtin_amdgcn_exp2f(d);  // (nothing yet: 0)
                sums.u = (sums.u + d * sums.s) * f;
                sums.s *= f;
                sums.m = high;
            }
            const float m = sums.m == negative_infinity() ? 0.f : sums.m;
            for (const uintx4& x : raw) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float t = (element<T>(x, e) - m) * c, p = __builtin_amdgcn_exp2f(t);
                    sums.s += p;
                    sums.u = fmaf(p, fmaxf(t, NEVER), sums.u);
                }
            }
        };
        uintx4 now[VECTORS], then[VECTORS];
        int v = r.first + w * 64;
        if (v < r.end) take(v, now);
        for (; v < r.end; v += WAVES * EACH) {
            if (v + WAVES * EACH < r.end) take(v + WAVES * EACH, then);
            if (all(v, (VECTORS - 1) * WAVES * 64 + 64)) {
                add(now);
            } else {
#pragma unroll
                for (int j = 0; j < VECTORS; ++j) {
                    const int vj = v + j * WAVES * 64;
                    if (vj >= r.end) continue;
                    uintx4 one[1] = {now[j]};
                    if (!all(vj, 64)) r.leave_out(vj + lane, one[0]);
                    add(one);
                }
            }
#pragma unroll
            for (int j = 0; j < VECTORS; ++j) now[j] = then[j];
        }
        const float high = sums.m;
        sums = join_lanes(sums, c);
        if constexpr (TOP) best_of_range<T, WAVES>(r, scratch[of], a.top, (r.end - r.first + WAVES * 64 - 1) / (WAVES * 64), high);
        if constexpr (WAVES > 1) {
            if (lane == 0) meet[wave] = sums;
            __syncthreads();
            sums = meet[0];
            if (w == 0) {
#pragma unroll
                for (int k = 1; k < WAVES; ++k) sums = join(sums, meet[k], c);
            }
        }
        if (there && w == 0) {
            if (a.parts > 1) {
                if (lane == 0) {
                    a.part_sums[item * 3] = sums.m;
                    a.part_sums[item * 3 + 1] = sums.s;
                    a.part_sums[item * 3 + 2] = sums.u;
                }
                if (TOP && lane < a.top) a.part_lists[item * a.top + lane] = scratch[of].best[lane];
            } else {
                if (lane == 0) finish_row<T>(a, row, sums, token, at_token);
                if (TOP && lane < a.top) write_best(a, row, lane, scratch[of].best[lane], sums);
            }
        }
        meet_all<WAVES>();  // what is in LDS is written again
    }
}

// Finishes rows that were cut into parts: a block to a row.  Bound by its dependent trips to memory: 4.6 us for one row in 16 parts.
constexpr int MOST_PARTS = 64;

template <class T, bool TOP>
__global__ __launch_bounds__(256) void join_row_kernel(ForwardArgs a)
{
    __shared__ uint64_t list[TOP ? MOST_PARTS * PS_LOGPROB_MAX_TOP : 1], best[TOP ? PS_LOGPROB_MAX_TOP : 1];
    __shared__ float high[64];
    __shared__ int count;
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63;
    const float c = a.scale * LOG2E;
    float at_token;
    const int64_t token = take_token<T>(a, row, at_token);
    Sums x{negative_infinity(), 0.f, 0.f};
    if (lane < a.parts) {
        const float* p = a.part_sums + (row * a.parts + lane) * 3;
        x = Sums{p[0], p[1], p[2]};
    }
    if constexpr (TOP) {
        // Of parts that have i keys or more each, the i-th keys of n parts are reached by n * i: none of the best is below the n-th largest
        // i-th key, where n * i is `top` or more.
        const uint64_t* const lists = a.part_lists + row * a.parts * a.top;
        const int i = (a.top + a.parts - 1) / a.parts, n = (a.top + i - 1) / i;
        if (threadIdx.x < 64) {
            const uint64_t key = lists[min(lane, a.parts - 1) * a.top + i - 1];
            high[lane] = lane < a.parts && key ? value_of(key) : negative_infinity();
        }
        if (threadIdx.x < (uint32_t)a.top) best[threadIdx.x] = 0;
        if (threadIdx.x == 0) count = 0;
        __syncthreads();
        const uint32_t from = kth_of_lanes<1>(high, n);
        for (int k = threadIdx.x; k < a.parts * a.top; k += 256) {
            const uint64_t key = lists[k];
            if (key && (uint32_t)(key >> 32) >= from) list[atomicAdd(&count, 1)] = key;
        }
        __syncthreads();
        // the order in which they were listed does not matter
        for (int k = threadIdx.x; k < count; k += 256) {
            const uint64_t key = list[k];
            int place = 0;
#pragma unroll 8
            for (int o = 0; o < count; ++o) place += list[o] > key;
            if (place < a.top) best[place] = key;
        }
        __syncthreads();
    }
    x = join_lanes(x, c);
    if (threadIdx.x == 0) finish_row<T>(a, row, x, token, at_token);
    if (TOP && threadIdx.x < (uint32_t)a.top) write_best(a, row, threadIdx.x, best[threadIdx.x], x);
}

// ---- backward ----------------------------------------------------------------------------------------------------------

struct BackwardArgs {
    const void *logits, *tokens;
    const float *norm, *dlogp, *dentropy;
    void* dlogits;
    int64_t row, out_row, token_stride, dlogp_stride, dentropy_stride, rows;
    int32_t vocab, token_bytes, per_row;  // blocks of a row
    float scale;
};

// dz = scale (gl ([j is the token] - p) - gh p (log p + H)), so scale p (A + B t) and for the token scale gl more, with t = log2 p, A = -(gl + gh H),
// B = -gh ln 2.  The scale comes last: with it A may be infinite, and 0 where p is 0 would be NaN, or among the smallest numbers, and lose bits.
// Bound by memory: bf16 8192 rows of 32768 184 us, 5.8 TB/s; of 32767, whose rows begin anywhere, 224, 4.8 TB/s (fp32 372 and 389); 4096 of
// 50257 146 us, 5.6 TB/s.
template <class T>
__global__ __launch_bounds__(256) void logprob_backward_kernel(BackwardArgs a)
{
    constexpr int E = 16 / sizeof(T), EACH = 256 * VECTORS * E;
    const int64_t total = a.rows * a.per_row;
    for (int64_t b = blockIdx.x; b < total; b += gridDim.x) {
        const int64_t row = b / a.per_row;
        const int first = (int)(b - row * a.per_row) * EACH, base = first + threadIdx.x * E;
        const T* const z = static_cast<const T*>(a.logits) + row * a.row;
        T* const out = static_cast<T*>(a.dlogits) + row * a.out_row;
        const float m = a.norm[row * 3], c = a.scale * LOG2E, log2_s = a.norm[row * 3 + 1] * LOG2E, entropy = a.norm[row * 3 + 2];
        int64_t token = -1;
        float gl = 0.f;
        if (a.dlogp) {
            token = token_of_row(a.tokens, a.token_bytes, row * a.token_stride);
            gl = a.dlogp[row * a.dlogp_stride];
            if (token < 0 || token >= a.vocab) gl = 0.f;
        }
        const float gh = a.dentropy ? a.dentropy[row * a.dentropy_stride] : 0.f;
        const float A = -(gl + gh * entropy), B = -gh * LN2;
        const bool none = m == negative_infinity() && log2_s == negative_infinity();
        auto give = [&](int64_t at, int n, const uintx4& raw) __attribute__((always_inline)) {
            float d[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float t = (element<T>(raw, e) - m) * c - log2_s;
                d[e] = __builtin_amdgcn_exp2f(t) * fmaf(B, fmaxf(t, NEVER), A);
            }
            if (token >= at && token < at + E) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (token == at + e) d[e] += gl;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) d[e] *= a.scale;
            if (none) {
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] = 0.f;
            }
            store_columns(out + at, n, d);
        };
        if (first + EACH <= a.vocab) {
            // without a branch between them, at which the compiler would wait
            uintx4 raw[VECTORS];
#pragma unroll
            for (int j = 0; j < VECTORS; ++j) __builtin_memcpy(&raw[j], z + base + j * 256 * E, 16);
#pragma unroll
            for (int j = 0; j < VECTORS; ++j) give(base + j * 256 * E, E, raw[j]);
        } else {
            for (int at = base; at < a.vocab; at += 256 * E) {
                const int n = min(E, a.vocab - at);
                T x[E] = {};
                uintx4 raw;
                if (n == E) {
                    __builtin_memcpy(&raw, z + at, 16);
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (e < n) x[e] = z[at + e];
                    __builtin_memcpy(&raw, x, 16);
                }
                give(at, n, raw);
            }
        }
    }
}

ps_status check_logprob(const char* call, const ps_logprob* l)
{
    if (!l) return dense_fail(PS_EINVAL, "%s: no description", call);
    if (l->dtype != PS_F32 && l->dtype != PS_BF16 && l->dtype != PS_F16) return dense_fail(PS_EINVAL, "%s: unknown type", call);
    if (l->rows < 0 || l->rows > PS_DENSE_MAX_ROWS) return dense_fail(PS_EINVAL, "%s: rows outside 0 .. %d", call, PS_DENSE_MAX_ROWS);
    if (l->vocab < 1 || l->vocab > PS_DENSE_MAX_STRIDE) return dense_fail(PS_EINVAL, "%s: vocab outside 1 .. %d", call, PS_DENSE_MAX_STRIDE);
    if (l->top < 0 || l->top > PS_LOGPROB_MAX_TOP) return dense_fail(PS_EINVAL, "%s: alternatives outside 0 .. %d", call, PS_LOGPROB_MAX_TOP);
    const float scale = (float)l->scale;
    if (!(scale > 0.f) || !std::isfinite(scale * LOG2E)) return dense_fail(PS_EINVAL, "%s: the scale is not above 0, or too large", call);
    return PS_OK;
}

ps_status check_numbers(const char* call, const char* name, const void* p, int64_t stride)
{
    if (reinterpret_cast<uintptr_t>(p) & 3) return dense_fail(PS_EINVAL, "%s: misaligned %s", call, name);
    if (stride < 0 || stride > PS_DENSE_MAX_STRIDE) return dense_fail(PS_EINVAL, "%s: %s is too far apart", call, name);
    return PS_OK;
}

// Whether sixteen wavefronts take a row: where there is a compute unit for each row, which takes 64 k values in about the time of a second
// launch (256 rows of 50257 in bf16 with 5 alternatives 20.8 us in parts, 15.4 this way; one of 131072 with 20 17.3 and 17.3, alone 33 and 37).
bool sixteen(const ps_logprob& l) { return l.rows <= COMPUTE_UNITS && l.vocab <= 65536; }

// Parts of a row, so many rounds of four wavefronts each: as many as make two blocks for a compute unit of all rows, one from 257 rows on.  us:
//   two blocks, and eight, 5 alternatives   bf16 512 rows of 20000 13.0, 17.6   of 131072 31.3, 36.7   128 of 131072 16.7, 20.4   one 16.7, 15.8
//                                           fp32 512 of 50000 21.5, 30.2
//   one part, and two, no alternatives      bf16 260 rows of 20000 7.0, 9.5     of 50257 11.8, 14.2    of 131072 25.6, 23.1      fp32 of 50000 14.5, 16.0
//                                           384 of 20000 7.2, 9.7               of 50257 13.5, 15.2    of 131072 26.9, 24.7      16.0, 19.3
//                                           511 of 20000 7.5, 11.2              of 50257 14.9, 18.5    of 131072 27.9, 29.9      19.0, 23.4
struct Cut {
    int parts, rounds;
};
Cut cut_rows(const ps_logprob& l)
{
    if (sixteen(l)) return {1, 0};
    const int64_t round = 4 * 64 * VECTORS * 16 / dtype_size(l.dtype), rounds = (l.vocab + round - 1) / round;  // (a part more for what is ahead of a row)
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(rounds, MOST_PARTS), l.rows ? 2 * COMPUTE_UNITS / l.rows : 1));
    const int64_t each = (rounds + parts - 1) / parts;
    return {(int)((rounds + each - 1) / each), (int)each};
}
uint64_t sums_bytes(const ps_logprob& l, const Cut& c) { return ((uint64_t)l.rows * c.parts * 12 + 255) / 256 * 256; }

template <class T, bool TOP>
void start_forward(const ForwardArgs& a, hipStream_t s)
{
    // One wavefront to a row that it takes in one round, and in up to eight where there are rows for two wavefronts to a SIMD: no row waits for
    // four.  us of one, and of four, without and with 5 alternatives:
    //   bf16   2048 rows of 8000 10.3, 13.3 and 11.0, 17.8    8192 of 4000 17.9, 22.7 and 26.1, 53.5    8192 of 16000 47.7, 61.6 and 52.0, 73.2
    //          2048 of 20000 as long                          4096 of 50257 with alternatives 98, 91
    //   fp32   16384 of 4000 42.3, 56.5 and 44.5, 99.9        8192 of 8000 43.5, 59.8 and 41.2, 61.8
    // (A row of a few values leaves most lanes without one: 8192 rows of 10 classes in fp32 7.5 us, for the call's 10.)
    constexpr int ROUND = 64 * VECTORS * 16 / (int)sizeof(T);  // of a wavefront
    const int64_t most = 1 << 20;
    if (a.vocab <= ROUND || (a.vocab <= 8 * ROUND && a.rows >= 8 * COMPUTE_UNITS)) {
        hipLaunchKernelGGL((logprob_kernel<T, 1, TOP>), dim3((uint32_t)std::min((a.rows + 3) / 4, most)), dim3(256), 0, s, a);
        return;
    }
    if (a.part_rounds == 0) {
        hipLaunchKernelGGL((logprob_kernel<T, 16, TOP>), dim3((uint32_t)a.rows), dim3(1024), 0, s, a);
        return;
    }
    hipLaunchKernelGGL((logprob_kernel<T, 4, TOP>), dim3((uint32_t)std::min(a.rows * a.parts, most)), dim3(256), 0, s, a);
    if (a.parts > 1) hipLaunchKernelGGL((join_row_kernel<T, TOP>), dim3((uint32_t)a.rows), dim3(256), 0, s, a);
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

}  // namespace
}  // namespace ps

extern "C" ps_status ps_logprob_workspace_bytes(const ps_logprob* l, uint64_t* bytes_out)
{
    using namespace ps;
    const ps_status st = check_logprob("ps_logprob_workspace_bytes", l);
    if (st != PS_OK) return st;
    if (!bytes_out) return dense_fail(PS_EINVAL, "ps_logprob_workspace_bytes: no place for the result");
    const Cut cut = cut_rows(*l);
    *bytes_out = cut.parts > 1 ? sums_bytes(*l, cut) + (uint64_t)l->rows * cut.parts * l->top * 8 : 0;
    return PS_OK;
}

extern "C" ps_status ps_logprob_forward(const ps_logprob* l, const ps_tokens* tokens, const ps_matrix* logits, float* logp, float* norm, float* top_logp,
                                        int32_t* top_tokens, void* workspace, uint64_t workspace_bytes, void* hip_stream)
{
    using namespace ps;
    static const char call[] = "ps_logprob_forward";
    ps_status st = check_logprob(call, l);
    if (st != PS_OK) return st;
    if ((st = check_tokens(call, tokens, l->rows, logp != nullptr)) != PS_OK) return st;
    if ((st = check_rows(call, "logits", l->dtype, logits, l->rows, l->vocab, 1)) != PS_OK) return st;
    if (l->rows && !norm) return dense_fail(PS_EINVAL, "%s: norm is missing", call);
    if (l->rows && l->top && (!top_logp || !top_tokens)) return dense_fail(PS_EINVAL, "%s: no place for the alternatives", call);
    for (const void* p : {(const void*)logp, (const void*)norm, (const void*)top_logp, (const void*)top_tokens})
        if ((st = check_numbers(call, "result", p, 0)) != PS_OK) return st;
    if (!l->rows) return PS_OK;
    const Cut cut = cut_rows(*l);
    uint64_t need = 0;
    if ((st = ps_logprob_workspace_bytes(l, &need)) != PS_OK) return st;
    if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))) return dense_fail(PS_EINVAL, "%s: null or misaligned workspace", call);
    if (workspace_bytes < need) return dense_fail(PS_ENOMEM, "%s: workspace too small", call);
    ForwardArgs a{};
    a.parts = cut.parts;
    a.part_rounds = cut.rounds;
    a.part_sums = static_cast<float*>(workspace);
    a.part_lists = reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + sums_bytes(*l, cut));
    a.logits = logits->data_dev;
    a.row = logits->row;
    if (logp) {
        a.tokens = tokens->data_dev;
        a.token_stride = tokens->stride;
        a.token_bytes = tokens->bytes;
    }
    a.logp = logp;
    a.norm = norm;
    a.top_logp = top_logp;
    a.top_tokens = top_tokens;
    a.rows = l->rows;
    a.vocab = (int32_t)l->vocab;
    a.top = l->top;
    a.scale = (float)l->scale;
    with_type(l->dtype, [&](auto t) {
        using T = decltype(t);
        if (a.top)
            start_forward<T, true>(a, static_cast<hipStream_t>(hip_stream));
        else
            start_forward<T, false>(a, static_cast<hipStream_t>(hip_stream));
    });
    return tokens_launched(call);
}

extern "C" ps_status ps_logprob_backward(const ps_logprob* l, const ps_tokens* tokens, const ps_matrix* logits, const float* norm, const ps_vector* dlogp,
                                         const ps_vector* dentropy, const ps_matrix* dlogits, void* hip_stream)
{
    using namespace ps;
    static const char call[] = "ps_logprob_backward";
    ps_status st = check_logprob(call, l);
    if (st != PS_OK) return st;
    const bool of_logp = dlogp && dlogp->data_dev, of_entropy = dentropy && dentropy->data_dev;
    if ((st = check_tokens(call, tokens, l->rows, of_logp)) != PS_OK) return st;
    if ((st = check_rows(call, "logits", l->dtype, logits, l->rows, l->vocab, 1)) != PS_OK) return st;
    if ((st = check_rows(call, "dlogits", l->dtype, dlogits, l->rows, l->vocab, 1)) != PS_OK) return st;
    if (l->rows && !norm) return dense_fail(PS_EINVAL, "%s: norm is missing", call);
    if ((st = check_numbers(call, "norm", norm, 0)) != PS_OK) return st;
    if (of_logp && (st = check_numbers(call, "dlogp", dlogp->data_dev, dlogp->stride)) != PS_OK) return st;
    if (of_entropy && (st = check_numbers(call, "dentropy", dentropy->data_dev, dentropy->stride)) != PS_OK) return st;
    if (!l->rows) return PS_OK;
    BackwardArgs a{};
    a.logits = logits->data_dev;
    a.row = logits->row;
    a.dlogits = dlogits->data_dev;
    a.out_row = dlogits->row;
    a.norm = norm;
    if (of_logp) {
        a.tokens = tokens->data_dev;
        a.token_stride = tokens->stride;
        a.token_bytes = tokens->bytes;
        a.dlogp = dlogp->data_dev;
        a.dlogp_stride = dlogp->stride;
    }
    if (of_entropy) a.dentropy = dentropy->data_dev, a.dentropy_stride = dentropy->stride;
    a.rows = l->rows;
    a.vocab = (int32_t)l->vocab;
    a.scale = (float)l->scale;
    with_type(l->dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int EACH = 256 * VECTORS * 16 / (int)sizeof(T);
        a.per_row = (a.vocab + EACH - 1) / EACH;
        hipLaunchKernelGGL(logprob_backward_kernel<T>, dim3((uint32_t)std::min<int64_t>(a.rows * a.per_row, 1 << 22)), dim3(256), 0, static_cast<hipStream_t>(hip_stream), a);
    });
    return tokens_launched(call);
}
