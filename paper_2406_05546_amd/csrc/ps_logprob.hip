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

constexpr float LOG2E = 1.44269504f, LN2 = 0.693147181f;
constexpr float NEVER = -300.f;  // 2^NEVER is 0, and times NEVER too: what -infinity is taken to where t is multiplied

__device__ __forceinline__ float negative_infinity() { return __uint_as_float(0xff800000u); }

// ---- the best of a row ---------------------------------------------------------------------------------------------------

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

// A wavefront's candidates: a list in LDS, in no order until `cut` keeps the best `top` of it in theirs.
constexpr int LIST = 256;

struct Best {
    uint64_t* list;
    int count, top;
    uint64_t least;  // what a candidate has to be above: 0, or the last of `top` that were kept

    __device__ __forceinline__ void cut()
    {
        const int lane = threadIdx.x & 63;
        __builtin_amdgcn_wave_barrier();
        uint64_t mine[LIST / 64];
        int rank[LIST / 64];
#pragma unroll
        for (int i = 0; i < LIST / 64; ++i) {
            rank[i] = 0;
            mine[i] = i * 64 + lane < count ? list[i * 64 + lane] : 0;
        }
#pragma unroll 4
        for (int k = 0; k < count; ++k) {
            const uint64_t other = list[k];
#pragma unroll
            for (int i = 0; i < LIST / 64; ++i) rank[i] += other > mine[i];
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < LIST / 64; ++i)
            if (i * 64 + lane < count && rank[i] < top) list[rank[i]] = mine[i];
        __builtin_amdgcn_wave_barrier();
        if (count >= top) {
            count = top;
            least = list[top - 1];
        }
    }
    // One value from each lane that has one
    __device__ __forceinline__ void add(bool has, float v, int index)
    {
        uint64_t key = key_of(v, index);
        has = has && key > least;
        unsigned long long who = __ballot(has);
        if (!who) return;
        if (count + __popcll(who) > LIST) {
            cut();
            has = has && key > least;
            who = __ballot(has);
        }
        if (has) list[count + __popcll(who & ((1ull << (threadIdx.x & 63)) - 1))] = key;
        count += __popcll(who);
    }
};

// The k-th largest of one value from each lane (of their `ordered` numbers).
__device__ __forceinline__ uint32_t kth_of_lanes(uint32_t o, int k)
{
    uint32_t least = 0;
    for (int b = 31; b >= 0; --b) {
        const uint32_t more = least | 1u << b;
        if (__popcll(__ballot(o >= more)) >= k) least = more;
    }
    return least;
}

// ---- forward -----------------------------------------------------------------------------------------------------------

struct ForwardArgs {
    const void *logits, *tokens;
    float *logp, *norm, *top_logp;
    int32_t* top_tokens;
    int64_t row, token_stride, rows;
    int32_t vocab, token_bytes, top;
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
        const float d = x.m == m ? 0.f : fmaxf((x.m - m) * c, NEVER), f = exp2f(d);
        s = x.s * f;
        u = (x.u + d * x.s) * f;
    };
    float s0, u0, s1, u1;
    part(a, s0, u0);
    part(b, s1, u1);
    return {m, s0 + s1, u0 + u1};
}

// WAVES wavefronts take a row, each 64 * VECTORS * 16 bytes at a time.  Bound by memory; behind it by the vector ALU: about ten
// operations and an exponential for a value.
constexpr int VECTORS = 4;

template <class T, int WAVES, bool TOP>
__global__ __launch_bounds__(WAVES * 64 < 256 ? 256 : WAVES * 64) void logprob_kernel(ForwardArgs a)
{
    constexpr int E = 16 / sizeof(T), ROWS = WAVES < 4 ? 4 / WAVES : 1;  // rows of a block
    constexpr int EACH = 64 * VECTORS * E;
    __shared__ uint64_t lists[TOP ? ROWS * WAVES * LIST : 1];
    __shared__ Sums meet[ROWS * WAVES];
    __shared__ int counts[ROWS * WAVES];
    const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6), w = wave % WAVES;
    const float c = a.scale * LOG2E;
    const int64_t step = (int64_t)gridDim.x * ROWS;
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < a.rows; row0 += step) {
        const int64_t row = row0 + wave / WAVES;
        const bool there = row < a.rows;
        const T* const z = static_cast<const T*>(a.logits) + (there ? row : 0) * a.row;
        Sums sums{negative_infinity(), 0.f, 0.f};
        Best best{lists + (TOP ? wave * LIST : 0), 0, a.top, 0};
        for (int64_t base = (int64_t)w * EACH; there && base < a.vocab; base += WAVES * EACH) {
            T raw[VECTORS][E];
#pragma unroll
            for (int j = 0; j < VECTORS; ++j) {
                const int64_t at = base + j * 64 * E + lane * E;
                if (at + E <= a.vocab) {
                    __builtin_memcpy(raw[j], z + at, 16);
                } else {
                    const T* p = z + at;
                    asm volatile("" : "+v"(p));
#pragma unroll
                    for (int e = 0; e < E; ++e) raw[j][e] = at + e < a.vocab ? p[e] : from_float<T>(negative_infinity());
                }
            }
            float high = negative_infinity(), highs[VECTORS];
#pragma unroll
            for (int j = 0; j < VECTORS; ++j) {
                highs[j] = negative_infinity();
#pragma unroll
                for (int e = 0; e < E; ++e) highs[j] = fmaxf(highs[j], to_float(raw[j][e]));
                high = fmaxf(high, highs[j]);
            }
            if (high > sums.m) {
                const float d = sums.m == negative_infinity() ? 0.f : fmaxf((sums.m - high) * c, NEVER), f = exp2f(d);
                sums.u = (sums.u + d * sums.s) * f;
                sums.s *= f;
                sums.m = high;
            }
            const float m = sums.m == negative_infinity() ? 0.f : sums.m;
#pragma unroll
            for (int j = 0; j < VECTORS; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float t = (to_float(raw[j][e]) - m) * c, p = __builtin_amdgcn_exp2f(t);
                    sums.s += p;
                    sums.u = fmaf(p, fmaxf(t, NEVER), sums.u);
                }
            if constexpr (TOP) {
                // Values of later rounds have higher indexes, so those that only equal the last kept one come too late.
                const float over = best.least ? value_of(best.least) : negative_infinity();
                const unsigned long long some = __ballot(high > over);
                if (some) {
                    // the largest values of `top` lanes are `top` values: what is below all of these is no candidate
                    float from = over;
                    if (__popcll(some) >= a.top) from = fmaxf(from, value_of((uint64_t)kth_of_lanes(ordered(high), a.top) << 32));
#pragma unroll
                    for (int j = 0; j < VECTORS; ++j) {
                        if (!__ballot(highs[j] >= from && highs[j] > negative_infinity())) continue;
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            const float v = to_float(raw[j][e]);
                            best.add(v >= from && v > negative_infinity(), v, (int)(base + j * 64 * E + lane * E + e));
                        }
                    }
                    if (best.count >= a.top) best.cut();
                }
            }
        }
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) sums = join(sums, Sums{__shfl_xor(sums.m, off, 64), __shfl_xor(sums.s, off, 64), __shfl_xor(sums.u, off, 64)}, c);
        if constexpr (TOP) {
            best.cut();  // in order, also where there are fewer
            if (lane == 0) counts[wave] = best.count;
        }
        if (WAVES > 1) {
            if (lane == 0) meet[wave] = sums;
            __syncthreads();
            sums = meet[0];
            for (int k = 1; k < WAVES; ++k) sums = join(sums, meet[k], c);
        } else {
            __builtin_amdgcn_wave_barrier();
        }
        if (there) {
            const bool none = sums.m == negative_infinity() && sums.s == 0.f;
            const float log_s = logf(sums.s);  // -infinity where there is none
            if (w == 0 && lane == 0) {
                a.norm[row * 3] = sums.m;
                a.norm[row * 3 + 1] = log_s;
                a.norm[row * 3 + 2] = none ? 0.f : log_s - LN2 * (sums.u / sums.s);
                if (a.logp) {
                    const int64_t t = token_of_row(a.tokens, a.token_bytes, row * a.token_stride);
                    float v = 0.f;
                    if (t >= 0 && t < a.vocab) v = none ? negative_infinity() : (to_float(z[t]) - sums.m) * a.scale - log_s;
                    a.logp[row] = v;
                }
            }
            if constexpr (TOP) {
                // the lists of the row's wavefronts, each in order: an entry's place is how many are before it
                const int first = wave / WAVES * WAVES;
                int total = 0;
                for (int k = 0; k < WAVES; ++k) total += counts[first + k];
                for (int i = w * 64 + lane; i < WAVES * a.top; i += WAVES * 64) {
                    const int of = i / a.top, at = i % a.top;
                    if (at >= counts[first + of]) continue;
                    const uint64_t key = lists[(first + of) * LIST + at];
                    int place = at;
                    for (int k = 0; k < WAVES; ++k) {
                        if (k == of) continue;
                        const int n = counts[first + k];
                        for (int x = 0; x < n; ++x) place += lists[(first + k) * LIST + x] > key;
                    }
                    if (place < a.top) {
                        a.top_logp[row * a.top + place] = (value_of(key) - sums.m) * a.scale - log_s;
                        a.top_tokens[row * a.top + place] = index_of(key);
                    }
                }
                for (int i = total + w * 64 + lane; i < a.top; i += WAVES * 64) {
                    a.top_logp[row * a.top + i] = negative_infinity();
                    a.top_tokens[row * a.top + i] = -1;
                }
            }
        }
        if (WAVES > 1) __syncthreads();  // what met in LDS is written again
    }
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

// dz = scale (gl ([j is the token] - p) - gh p (log p + H)), so -p (A + B t) with t = log2 p, A = scale (gl + gh H), B = scale gh ln 2.
template <class T>
__global__ __launch_bounds__(256) void logprob_backward_kernel(BackwardArgs a)
{
    constexpr int E = 16 / sizeof(T), EACH = 256 * VECTORS * E;
    const int64_t total = a.rows * a.per_row;
    for (int64_t b = blockIdx.x; b < total; b += gridDim.x) {
        const int64_t row = b / a.per_row;
        const int base = (int)(b - row * a.per_row) * EACH + threadIdx.x * E;
        const T* const z = static_cast<const T*>(a.logits) + row * a.row;
        T* const out = static_cast<T*>(a.dlogits) + row * a.out_row;
        T raw[VECTORS][E];
#pragma unroll
        for (int j = 0; j < VECTORS; ++j) {
            const int64_t at = base + (int64_t)j * 256 * E;
            if (at + E <= a.vocab) {
                __builtin_memcpy(raw[j], z + at, 16);
            } else {
                const T* p = z + at;
                asm volatile("" : "+v"(p));
#pragma unroll
                for (int e = 0; e < E; ++e) raw[j][e] = at + e < a.vocab ? p[e] : T{};
            }
        }
        const float m = a.norm[row * 3], c = a.scale * LOG2E, log2_s = a.norm[row * 3 + 1] * LOG2E;
        int64_t token = -1;
        float gl = 0.f;
        if (a.dlogp) {
            token = token_of_row(a.tokens, a.token_bytes, row * a.token_stride);
            if (token >= 0 && token < a.vocab) gl = a.dlogp[row * a.dlogp_stride];
        }
        const float gh = a.dentropy ? a.dentropy[row * a.dentropy_stride] : 0.f;
        const float A = -a.scale * (gl + gh * a.norm[row * 3 + 2]), B = -a.scale * gh * LN2;
        const bool none = m == negative_infinity() && log2_s == negative_infinity();
#pragma unroll
        for (int j = 0; j < VECTORS; ++j) {
            const int64_t at = base + (int64_t)j * 256 * E;
            if (at >= a.vocab) continue;
            float d[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float t = (to_float(raw[j][e]) - m) * c - log2_s;
                d[e] = __builtin_amdgcn_exp2f(t) * fmaf(B, fmaxf(t, NEVER), A);
            }
            if (token >= at && token < at + E) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (token == at + e) d[e] = fmaf(a.scale, gl, d[e]);
            }
            if (none) {
#pragma unroll
                for (int e = 0; e < E; ++e) d[e] = 0.f;
            }
            store_columns(out + at, (int)min((int64_t)E, a.vocab - at), d);
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

template <class T, bool TOP>
void start_forward(const ForwardArgs& a, hipStream_t s)
{
    // a wavefront to a row of a few rounds, sixteen where rows are too few to fill the chip with four
    constexpr int ROUND = 64 * VECTORS * 16 / (int)sizeof(T);
    const int64_t most = 1 << 20;
    if (a.vocab <= ROUND)
        hipLaunchKernelGGL((logprob_kernel<T, 1, TOP>), dim3((uint32_t)std::min((a.rows + 3) / 4, most)), dim3(256), 0, s, a);
    else if (a.rows > 2 * COMPUTE_UNITS || a.vocab <= 4 * ROUND)
        hipLaunchKernelGGL((logprob_kernel<T, 4, TOP>), dim3((uint32_t)std::min(a.rows, most)), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((logprob_kernel<T, 16, TOP>), dim3((uint32_t)std::min(a.rows, most)), dim3(1024), 0, s, a);
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

extern "C" ps_status ps_logprob_forward(const ps_logprob* l, const ps_tokens* tokens, const ps_matrix* logits, float* logp, float* norm, float* top_logp,
                                        int32_t* top_tokens, void* hip_stream)
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
    ForwardArgs a{};
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
