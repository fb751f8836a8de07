// Beam search over whole rows of logits: for every sentence the B best continuations of its B hypotheses,
//   total(b, t) = score[b] + logit(b, t) - log sum over allowed t' of exp(logit(b, t')),
// in the order total descending, then b, then t; and the reordering of what follows the hypotheses.
//
// Selection is one pass over the logits.  A workgroup keeps a piece of one row in registers, finds its maximum and
// sum of exponentials, and its B best; a second kernel joins the pieces of a sentence.  The sums of hypotheses are
// compared in 64 bits, because two hypotheses of a sentence can be closer than 32 bits tell apart: exponentials are
// added in 64 bits too, but for eight at a time in three levels of 32 (a running sum in 32 bits rounds every one of
// a few different values the same way again and again: 2.4e-7 of the sum was met).
//
// The B best of a piece: each lane of a workgroup's four wavefronts knows the largest of its own values, and the
// smallest of the wavefronts' ceil(B / 4)-th largest of these is a bound that at least B values reach.  The values at or
// above it, a few times B as a rule, are gathered and each is ranked by counting those before it.  Where more than
// GATHER values reach the bound (long ties, ascending rows), at most B rounds over the piece take one value after the
// other, with all that share it.
//
// What bounds it: the vector units.  A 16-bit value takes 11 of their issue slots (mask 2, range and maximum 1, the
// exponential and its correction 8), and about 170 instructions of a wavefront stand around its 48 values a lane.  Counted
// for 256 x 250,000 with masks and a tenth ended (kernel, us; cycles of a vector unit, the same at 2.4 GHz in us; bytes at
// 5.1 TB/s): fp16 35, 57,000, 24; 24.  bf16 42, 73,000, 30; 24 (each value is bounded twice, in `settle` and `minus`).  fp32 53,
// 79,000, 33; 46.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "vp.h"
#include "vp_kernels.h"
#include "typed.h"
#include "wave_ops.h"

namespace {

constexpr int THREADS = 256;
constexpr int WAVES = THREADS / 64;
constexpr int GATHER = 1024;       // values that are ranked by counting
constexpr int VECTORS = 512;       // vectors of eight that hold them
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

__device__ inline float minus_inf() { return -__builtin_inff(); }

__device__ inline double wave_sum_double(double v)
{
#define VP_DPP_ADD64(ctrl, rows)                                                                            \
    {                                                                                                       \
        const long long b = __builtin_bit_cast(long long, v);                                               \
        const unsigned int lo = (unsigned int)__builtin_amdgcn_update_dpp(0, (int)b, ctrl, rows, 0xf, false); \
        const unsigned int hi = (unsigned int)__builtin_amdgcn_update_dpp(0, (int)(b >> 32), ctrl, rows, 0xf, false); \
        v += __builtin_bit_cast(double, ((unsigned long long)hi << 32) | lo);                               \
    }
    VP_DPP_ADD64(0x111, 0xf)
    VP_DPP_ADD64(0x112, 0xf)
    VP_DPP_ADD64(0x114, 0xf)
    VP_DPP_ADD64(0x118, 0xf)
    VP_DPP_ADD64(0x142, 0xa)
    VP_DPP_ADD64(0x143, 0xc)
#undef VP_DPP_ADD64
    const long long b = __builtin_bit_cast(long long, v);
    const unsigned int lo = (unsigned int)__builtin_amdgcn_readlane((int)b, 63);
    const unsigned int hi = (unsigned int)__builtin_amdgcn_readlane((int)(b >> 32), 63);
    return __builtin_bit_cast(double, ((unsigned long long)hi << 32) | lo);
}

// Larger key: larger value, then smaller index (-0 ties with +0).
__device__ inline unsigned long long key_of(float v, int i)
{
    unsigned int hi = __float_as_uint(v + 0.f);
    hi ^= (hi & 0x80000000u) ? 0xffffffffu : 0x80000000u;
    return ((unsigned long long)hi << 32) | ~(unsigned int)i;
}
__device__ inline float value_of(unsigned long long key)
{
    unsigned int hi = (unsigned int)(key >> 32);
    hi ^= (hi & 0x80000000u) ? 0x80000000u : 0xffffffffu;
    return __uint_as_float(hi);
}
__device__ inline int index_of(unsigned long long key) { return (int)~(unsigned int)key; }

// The B-th largest of the lanes' values, each lane counted once, and the largest; `low`, which every value
// reaches, if fewer are above it.
__device__ inline float nth_of_lanes(float v, float low, int B, float &most)
{
    const int lane = threadIdx.x & 63;
    float best = low;
    most = low;
    for (int r = 0; r < B; ++r) {
        best = wave_max_float(v);
        most = r == 0 ? best : most;
        if (best == low) break;
        const unsigned long long at = __ballot(v == best);
        if (lane == __ffsll((long long)at) - 1) v = low;
    }
    return best;
}

// Eight neighbouring values of a row in registers.  What is not there (masked, past the row's end, NaN, -inf) is held
// as the type's lowest finite value `low`: differences to it are numbers, and its exponential is nothing.  Where
// too few are above it they are looked up again (`allowed_value`), since a logit may be that low.
__device__ inline unsigned int pk_max_f16(unsigned int a, unsigned int b)
{
    unsigned int o;
    asm("v_pk_max_f16 %0, %1, %2" : "=v"(o) : "v"(a), "v"(b));
    return o;
}
// bytes of ones for bits 2 p and 2 p + 1 of a mask, one in each half
__device__ inline unsigned int pair_mask(unsigned int bits, int p)
{
    const unsigned int lo = (unsigned int)__builtin_amdgcn_sbfe((int)bits, 2 * p, 1), hi = (unsigned int)__builtin_amdgcn_sbfe((int)bits, 2 * p + 1, 1);
    return (lo & 0xffffu) | (hi & 0xffff0000u);
}

template <typename T> struct Eight;
template <> struct Eight<Half> {
    static constexpr float low = -65504.f;
    u32x4 w;
    __device__ void load(const Half *p) { w = *(const u32x4_any2 *)p; }
    __device__ void clear() { w = u32x4{0xfbfffbffu, 0xfbfffbffu, 0xfbfffbffu, 0xfbfffbffu}; }
    __device__ void set(int j, Half x)   // (j a constant)
    {
        w[j / 2] = j % 2 ? (w[j / 2] & 0xffffu) | ((unsigned int)x.b << 16) : (w[j / 2] & 0xffff0000u) | x.b;
    }
    __device__ void mask(unsigned int bits)
    {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const unsigned int m = pair_mask(bits, p);
            w[p] = (w[p] & m) | (0xfbfffbffu & ~m);
        }
    }
    // into range (NaN becomes `low`, a signalling one a quiet one); the largest of the numbers
    __device__ float settle()
    {
#pragma unroll
        for (int p = 0; p < 4; ++p) w[p] = pk_max_f16(w[p], 0xfbfffbffu);
        const unsigned int m = pk_max_f16(pk_max_f16(w[0], w[1]), pk_max_f16(w[2], w[3]));
        return value(Half{(uint16_t)pk_max_f16(m, m >> 16)});
    }
    __device__ float at(int j) const { return value(Half{(uint16_t)(w[j / 2] >> (j % 2 * 16))}); }
    __device__ float raw(int j) const { return at(j); }      // of a vector that is not settled
    __device__ float minus(int j, float most) const   // at(j) - most in one instruction
    {
        float o;
        if (j % 2) asm("v_fma_mix_f32 %0, %1, 1.0, -%2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(o) : "v"(w[j / 2]), "v"(most));
        else asm("v_fma_mix_f32 %0, %1, 1.0, -%2 op_sel_hi:[1,0,0]" : "=v"(o) : "v"(w[j / 2]), "v"(most));
        return o;
    }
};
template <> struct Eight<Bf16> {
    static constexpr float low = -3.3895314e38f;
    u32x4 w;
    __device__ void load(const Bf16 *p) { w = *(const u32x4_any2 *)p; }
    __device__ void clear() { w = u32x4{0xff7fff7fu, 0xff7fff7fu, 0xff7fff7fu, 0xff7fff7fu}; }
    __device__ void set(int j, Bf16 x)
    {
        w[j / 2] = j % 2 ? (w[j / 2] & 0xffffu) | ((unsigned int)x.b << 16) : (w[j / 2] & 0xffff0000u) | x.b;
    }
    __device__ void mask(unsigned int bits)
    {
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            const unsigned int m = pair_mask(bits, p);
            w[p] = (w[p] & m) | (0xff7fff7fu & ~m);
        }
    }
    __device__ float raw(int j) const { return __uint_as_float(j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16); }
    __device__ float at(int j) const { return fmaxf(raw(j), low); }
    __device__ float settle()
    {
        float m = at(0);
#pragma unroll
        for (int j = 1; j < 8; ++j) m = fmaxf(m, at(j));
        return m;
    }
    __device__ float minus(int j, float most) const { return at(j) - most; }
};
template <> struct Eight<float> {
    static constexpr float low = -3.4028235e38f;
    float v[8];
    __device__ void load(const float *p) { load8(p, v); }
    __device__ void clear()
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = low;
    }
    __device__ void set(int j, float x) { v[j] = x; }
    __device__ void mask(unsigned int bits)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (bits >> j) & 1 ? v[j] : low;
    }
    __device__ float settle()
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaxf(v[j], low);
        return fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
    }
    __device__ float at(int j) const { return v[j]; }
    __device__ float raw(int j) const { return v[j]; }
    __device__ float minus(int j, float most) const { return v[j] - most; }
};

// the next float above `low` (all three types' lowest values are floats)
__device__ inline float above_low(float low) { return __uint_as_float(__float_as_uint(low) - 1); }

// exp(d) for d <= 0, to the exponential instruction's own error: what rounding d * log2(e) lost comes back as a factor
// 1 + c, for the same reason as the sums above.  d may be as low as two lowest values apart in the type (the product is finite, or the exponential's zero
// meets a finite c): for fp32 it is bounded first.
template <typename T> __device__ inline float exp_of(float d)
{
    if (!std::is_same<T, Half>::value) d = fmaxf(d, -200.f);
    const float a = d * LOG2E, e = __builtin_amdgcn_exp2f(a);
    return fmaf(e, fmaf(-a, LN2, d), e);
}

struct Piece {
    double sum;    // of exp(x - most)
    float most;
    float pad;
};

struct SelectArgs {
    const void *logits;
    long stride, allowed_stride;      // elements, 32-bit words
    const float *scores;
    const uint32_t *allowed;          // or NULL
    const uint8_t *done;              // or NULL
    int n, V, B, pieces, eos;
    Piece *part;                      // [n, pieces]
    unsigned long long *best;         // [n, pieces, B]: keys, 0: none
    float *out_scores;
    int32_t *out_parent, *out_token;
    uint8_t *out_done;                // or NULL
};

__device__ inline bool live(const SelectArgs &A, int row)
{
    return !(A.done && A.done[row]) && A.scores[row] > minus_inf();
}

template <typename T> __device__ inline bool allowed_value(const SelectArgs &A, int row, int t)
{
    if (A.allowed && !((A.allowed[(size_t)row * A.allowed_stride + (t >> 5)] >> (t & 31)) & 1)) return false;
    return value(((const T *)A.logits)[(size_t)row * A.stride + t]) > minus_inf();
}

// The eight values from column c of a row on as they lie in memory, and a bit for each that is there and allowed.
template <typename T> __device__ inline unsigned int load_again(const SelectArgs &A, int row, long c, Eight<T> &e)
{
    const T *const x = (const T *)A.logits + (size_t)row * A.stride + c;
    unsigned int there = 0;
    if (c + 8 <= A.V) {
        e.load(x);
        there = 255;
    } else {
        e.clear();
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < A.V) e.set(j, x[j]), there |= 1u << j;
    }
    if (A.allowed && there) there &= A.allowed[(size_t)row * A.allowed_stride + (c >> 5)] >> (c & 31);
    return there;
}

// The threads whose `is` holds put (value, token) behind m keys, in the order of the threads, as long as there are fewer
// than B: how many did.  (Every thread calls it.)
__device__ inline int put_in_order(bool is, int token, float value, int m, int B, unsigned long long *keys, int *wave_i)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned long long all = __ballot(is);
    __syncthreads();
    if (lane == 0) wave_i[wave] = (int)__popcll(all);
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        before += w < wave ? wave_i[w] : 0;
        total += wave_i[w];
    }
    const int at = m + before + (int)__popcll(all & ((1ull << lane) - 1ull));
    if (is && at < B) keys[at] = key_of(value, token);
    return min(total, B - m);
}

// U: vectors of eight values to a thread; a piece is 2048 U values.
template <typename T, int U>
__global__ __launch_bounds__(THREADS) void select_piece_kernel(const SelectArgs A)
{
    __shared__ float wave_f[WAVES], wave_t[WAVES];
    __shared__ double wave_d[WAVES];
    __shared__ int reaching, gathered, wave_i[WAVES];
    __shared__ Eight<T> vectors[VECTORS];
    __shared__ int vector_at[VECTORS];
    __shared__ unsigned long long keys[GATHER];
    constexpr float low = Eight<T>::low;
    const int row = blockIdx.x / A.pieces, piece = blockIdx.x % A.pieces;
    if (!live(A, row)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int first = piece * (2048 * U) + threadIdx.x * 8;
    const T *const x = (const T *)A.logits + (size_t)row * A.stride;
    Eight<T> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const long c = (long)first + u * 2048;
        if (c + 8 <= A.V) {
            v[u].load(x + c);
        } else {
            v[u].clear();
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (c + j < A.V) v[u].set(j, x[c + j]);
        }
    }
    if (A.allowed) {
        const uint32_t *const bits = A.allowed + (size_t)row * A.allowed_stride;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long c = (long)first + u * 2048;
            v[u].mask(c < A.V ? bits[c >> 5] >> (c & 31) : 0);
        }
    }
    float top[U], mine = low;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        top[u] = v[u].settle();
        mine = fmaxf(mine, top[u]);
    }
    float wave_most;
    const float bound = nth_of_lanes(mine, low, (A.B + WAVES - 1) / WAVES, wave_most);
    if (threadIdx.x == 0) reaching = gathered = 0;
    if (lane == 0) {
        wave_f[wave] = wave_most;
        wave_t[wave] = bound;
    }
    __syncthreads();
    float most = wave_f[0], floor = wave_t[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) most = fmaxf(most, wave_f[w]), floor = fminf(floor, wave_t[w]);
    if (floor == low) {   // a wavefront has little (the row's end, few tokens allowed): the best wavefront's B-th largest
        const float alone = nth_of_lanes(mine, low, A.B, wave_most);
        __syncthreads();
        if (lane == 0) wave_t[wave] = alone;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) floor = fmaxf(floor, wave_t[w]);
    }
    unsigned long long *const best = A.best + ((size_t)row * A.pieces + piece) * A.B;
    Piece *const part = A.part + (size_t)row * A.pieces + piece;
    if (most == __builtin_inff()) {
        if (threadIdx.x == 0) *part = {0.0, most, 0.f};
        for (int r = threadIdx.x; r < A.B; r += THREADS) best[r] = 0;
        return;
    }
    // vectors that reach the bound are put down whole, and their values looked at by all threads alike behind the
    // exponentials (eight comparisons and branches a vector, in every wavefront that has one, cost a quarter of the pass)
    const bool few = floor == low;
    floor = fmaxf(floor, above_low(low));
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (top[u] >= floor) {
            const int k = atomicAdd(&reaching, 1);
            if (k < VECTORS) {
                vectors[k] = v[u];
                vector_at[k] = first + u * 2048;
            }
        }
    double s = 0.0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = exp_of<T>(v[u].minus(j, most));
        s += (double)(((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7])));
    }
    if (most <= low + 200.f || s != s) {
        // What is held as `low` would count among values so near to it; and a signalling NaN among fp16 logits, which one
        // maximum makes a quiet one instead of `low`, is in the sum: the sum once more, of what is there.
        s = 0.0;
#pragma unroll 1
        for (int u = 0; u < U; ++u) {
            Eight<T> e;
            const unsigned int there = load_again(A, row, (long)first + u * 2048, e);
#pragma unroll
            for (int j = 0; j < 8; ++j) s += (there >> j & 1) && e.raw(j) > minus_inf() ? (double)exp_of<float>(e.raw(j) - most) : 0.0;
        }
    }
    const double d = wave_sum_double(s);
    if (lane == 0) wave_d[wave] = d;
    __syncthreads();
    const int put = min(reaching, VECTORS);
    for (int e = threadIdx.x; e < put * 8; e += THREADS) {
        const float at = value(((const T *)&vectors[e >> 3])[e & 7]);
        if (at >= floor) {
            const int k = atomicAdd(&gathered, 1);
            if (k < GATHER) keys[k] = key_of(at, vector_at[e >> 3] + (e & 7));
        }
    }
    __syncthreads();
    int m = reaching <= VECTORS ? gathered : GATHER + 1;
    bool at_low = false;
    if (few && m < A.B) {   // tokens at the lowest value itself, if there are any, come next
        bool mine_low = false;
#pragma unroll 1
        for (int u = 0; u < U; ++u) {
            Eight<T> e;
            const unsigned int there = load_again(A, row, (long)first + u * 2048, e);
#pragma unroll
            for (int j = 0; j < 8; ++j) mine_low |= (there >> j & 1) && e.raw(j) == low;
        }
        if (lane == 0) wave_f[wave] = 0.f;
        if (__any(mine_low) && lane == 0) wave_f[wave] = 1.f;
        __syncthreads();
        at_low = wave_f[0] + wave_f[1] + wave_f[2] + wave_f[3] > 0.f;
    }
    if (threadIdx.x == 0) *part = {wave_d[0] + wave_d[1] + wave_d[2] + wave_d[3], m > 0 || at_low ? most : minus_inf(), 0.f};
    if (at_low) {
        // in order of their tokens until B are there
        for (int t0 = piece * (2048 * U); t0 < min((long)A.V, (long)(piece + 1) * (2048 * U)) && m < A.B; t0 += THREADS) {
            const int t = t0 + threadIdx.x;
            const bool is = t < A.V && allowed_value<T>(A, row, t) && value(x[t]) == low;
            m += put_in_order(is, t, low, m, A.B, keys, wave_i);
        }
    } else if (m > GATHER) {
        // Value after value: the largest below the last, and all that are equal to it; at the last one only the first tokens
        // that there is room for.  (From memory: with the registers' values every call had registers for three wavefronts a
        // SIMD instead of seven.)
        const int base = piece * (2048 * U);
        float prev = __builtin_inff();
        m = 0;
        while (m < A.B) {
            float next = low;
#pragma unroll 1
            for (int u = 0; u < U; ++u) {
                Eight<T> e;
                const unsigned int there = load_again(A, row, (long)first + u * 2048, e);
#pragma unroll
                for (int j = 0; j < 8; ++j) next = (there >> j & 1) && e.raw(j) < prev ? fmaxf(next, e.raw(j)) : next;
            }
            next = wave_max_float(next);
            __syncthreads();
            if (lane == 0) wave_f[wave] = next;
            if (threadIdx.x == 0) gathered = m;
            __syncthreads();
            next = fmaxf(fmaxf(wave_f[0], wave_f[1]), fmaxf(wave_f[2], wave_f[3]));
#pragma unroll 1
            for (int u = 0; u < U; ++u) {
                Eight<T> e;
                const unsigned int there = load_again(A, row, (long)first + u * 2048, e);
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if ((there >> j & 1) && e.raw(j) == next) {
                        const int k = atomicAdd(&gathered, 1);
                        if (k < A.B) keys[k] = key_of(next, first + u * 2048 + j);
                    }
            }
            __syncthreads();
            if (gathered <= A.B) {
                m = gathered;
            } else {
                for (int t0 = base; t0 < base + 2048 * U && m < A.B; t0 += THREADS) {
                    const int t = t0 + threadIdx.x;
                    const bool is = t < A.V && allowed_value<T>(A, row, t) && value(x[t]) == next;
                    m += put_in_order(is, t, next, m, A.B, keys, wave_i);
                }
            }
            prev = next;
        }
    }
    __syncthreads();
    // Many are cut to the B best of every 64 first.
    const unsigned long long *from = keys;
    if (m > 96) {
        unsigned long long *const fewer = (unsigned long long *)vectors;
        if (threadIdx.x == 0) gathered = 0;
        __syncthreads();
        for (int e0 = wave * 64; e0 < m; e0 += THREADS) {
            const unsigned long long k = e0 + lane < m ? keys[e0 + lane] : 0;
            int r = 0;
            for (int o = 0; o < 64; ++o) {
                const unsigned int lo = (unsigned int)__builtin_amdgcn_readlane((int)k, o), hi = (unsigned int)__builtin_amdgcn_readlane((int)(k >> 32), o);
                r += (((unsigned long long)hi << 32) | lo) > k;
            }
            if (k && r < A.B) fewer[atomicAdd(&gathered, 1)] = k;
        }
        __syncthreads();
        m = gathered;
        from = fewer;
    }
    for (int e = threadIdx.x; e < m; e += THREADS) {
        const unsigned long long k = from[e];
        int r = 0;
#pragma unroll 4
        for (int o = 0; o < m; ++o) r += from[o] > k;
        if (r < A.B) best[r] = k;
    }
    for (int r = m + threadIdx.x; r < A.B; r += THREADS) best[r] = 0;
}
static_assert(sizeof(Eight<Half>) * VECTORS >= GATHER * 8, "room for the keys of a second look");

// Total descending, then hypothesis and token ascending (both in `at`, b * 2^32 + t).
struct Choice {
    double total;
    unsigned long long at;
};
__device__ inline bool before(double t, unsigned long long a, double t2, unsigned long long a2)
{
    return (t > t2) | ((t == t2) & (a < a2));
}

// One workgroup per sentence.  The first of every piece's list gives the bound that B choices reach; the lists descend,
// so each is read only as far as it reaches the bound (in all about B steps).
constexpr int JOIN_THREADS = 512, JOIN_WAVES = JOIN_THREADS / 64;
constexpr int AHEAD = 3;     // entries of a thread's first list that are loaded at once

__global__ __launch_bounds__(JOIN_THREADS) void select_join_kernel(const SelectArgs A)
{
    // of every hypothesis: its score, whether it has ended, and its log-sum-exp; NaN: it has no continuation
    __shared__ double score_of[VP_MAX_BEAMS], lse[VP_MAX_BEAMS];
    __shared__ bool ended[VP_MAX_BEAMS];
    __shared__ float wave_t[JOIN_WAVES];
    __shared__ int gathered;
    __shared__ Choice kept[GATHER];
    __shared__ Choice wave_best[JOIN_WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int B = A.B, row0 = blockIdx.x * B, lists = B * A.pieces;
    // (on its way while the sums are joined; a row that is not live has none, and its entries are not looked at)
    unsigned long long ahead[AHEAD] = {};
    if ((int)threadIdx.x < lists && live(A, row0 + (int)threadIdx.x / A.pieces)) {
#pragma unroll
        for (int r = 0; r < AHEAD; ++r)
            if (r < B) ahead[r] = A.best[((size_t)row0 * A.pieces + threadIdx.x) * B + r];
    }
    for (int b = wave; b < B; b += JOIN_WAVES) {
        const int row = row0 + b;
        double s = 0.0;
        float most = minus_inf();
        const float score = A.scores[row];
        const bool over = A.done && A.done[row];
        if (lane == 0) {
            score_of[b] = (double)score;
            ended[b] = over;
        }
        if (!over && score > minus_inf()) {
            const Piece *const part = A.part + (size_t)row * A.pieces;
            Piece held = {0.0, minus_inf(), 0.f};
            if (lane < A.pieces) held = part[lane];
            most = held.most;
            for (int p = lane + 64; p < A.pieces; p += 64) most = fmaxf(most, part[p].most);
            most = wave_max_float(most);
            if (most > minus_inf() && most < __builtin_inff()) {
                if (held.most > minus_inf()) s = held.sum * exp((double)held.most - (double)most);
                for (int p = lane + 64; p < A.pieces; p += 64) {
                    const Piece q = part[p];
                    if (q.most > minus_inf()) s += q.sum * exp((double)q.most - (double)most);
                }
            }
        }
        s = wave_sum_double(s);
        if (lane == 0) lse[b] = s > 0.0 ? (double)most + log(s) : __builtin_nan("");
    }
    if (threadIdx.x == 0) gathered = 0;
    __syncthreads();
    // entry r of list b * pieces + p; total -inf: none
    auto choice_of = [&](int b, int p, int r, bool known, unsigned long long k) -> Choice {
        const double score = score_of[b];
        if (ended[b]) {
            const bool there = p == 0 && r == 0 && A.eos >= 0 && A.eos < A.V && score > -__builtin_inf();
            return {there ? score : -__builtin_inf(), ((unsigned long long)b << 32) | (unsigned int)A.eos};
        }
        if (!(lse[b] == lse[b])) return {-__builtin_inf(), 0};
        if (!known) k = A.best[((size_t)(row0 + b) * A.pieces + p) * B + r];
        if (k == 0) return {-__builtin_inf(), 0};
        const double t = score + ((double)value_of(k) - lse[b]);
        return {t == t ? t : -__builtin_inf(), ((unsigned long long)b << 32) | (unsigned int)index_of(k)};
    };
    auto choice = [&](int b, int p, int r) { return choice_of(b, p, r, false, 0); };
    float mine = minus_inf();
    Choice held = {-__builtin_inf(), 0};      // (of this thread's first list)
    for (int e = threadIdx.x; e < lists; e += JOIN_THREADS) {
        const int b = e / A.pieces;
        const Choice c = choice_of(b, e - b * A.pieces, 0, e == (int)threadIdx.x, ahead[0]);
        if (e == (int)threadIdx.x) held = c;
        mine = fmaxf(mine, (float)c.total);
    }
    float unused;
    const float bound = nth_of_lanes(mine, minus_inf(), B, unused);
    if (lane == 0) wave_t[wave] = bound;
    __syncthreads();
    float least = wave_t[0];
#pragma unroll
    for (int w = 1; w < JOIN_WAVES; ++w) least = fmaxf(least, wave_t[w]);
    if (mine >= least)
        for (int e = threadIdx.x; e < lists; e += JOIN_THREADS) {
            const int b = e / A.pieces, p = e - b * A.pieces;
            Choice c = e == (int)threadIdx.x ? held : choice(b, p, 0);
            for (int r = 1; c.total > -__builtin_inf() && (float)c.total >= least; ++r) {
                const int k = atomicAdd(&gathered, 1);
                if (k < GATHER) kept[k] = c;
                if (r == B) break;
                c = e == (int)threadIdx.x && r < AHEAD ? choice_of(b, p, r, true, r == 1 ? ahead[1] : ahead[2]) : choice(b, p, r);
            }
        }
    __syncthreads();
    const int m = gathered;
    auto write = [&](int r, double t, unsigned long long at) {
        const int o = row0 + r;
        const int b = (int)(at >> 32), token = (int)(unsigned int)at;
        A.out_scores[o] = (float)t;
        A.out_parent[o] = b;
        A.out_token[o] = token;
        if (A.out_done) A.out_done[o] = ended[b] || token == A.eos;
    };
    auto write_none = [&](int r) {
        const int o = row0 + r;
        A.out_scores[o] = minus_inf();
        A.out_parent[o] = -1;
        A.out_token[o] = -1;
        if (A.out_done) A.out_done[o] = 0;
    };
    if (m <= GATHER) {
        for (int e = threadIdx.x; e < m; e += JOIN_THREADS) {
            const Choice c = kept[e];
            int r = 0;
#pragma unroll 4
            for (int o = 0; o < m; ++o) r += before(kept[o].total, kept[o].at, c.total, c.at);
            if (r < B) write(r, c.total, c.at);
        }
        for (int r = m + threadIdx.x; r < B; r += JOIN_THREADS) write_none(r);
        return;
    }
    double prev_t = __builtin_inf();
    unsigned long long prev_a = 0;
    for (int r = 0; r < B; ++r) {
        Choice top = {-__builtin_inf(), ~0ull};
        for (int e = threadIdx.x; e < lists * B; e += JOIN_THREADS) {
            const int l = e / B, b = l / A.pieces;
            const Choice c = choice(b, l - b * A.pieces, e - l * B);
            const bool open = r == 0 || before(prev_t, prev_a, c.total, c.at);
            if (c.total > -__builtin_inf() && open && before(c.total, c.at, top.total, top.at)) top = c;
        }
        for (int o = 32; o; o >>= 1) {
            const Choice other = {__shfl_xor(top.total, o), __shfl_xor(top.at, o)};
            if (before(other.total, other.at, top.total, top.at)) top = other;
        }
        __syncthreads();
        if (lane == 0) wave_best[wave] = top;
        __syncthreads();
        for (int w = 0; w < JOIN_WAVES; ++w)
            if (before(wave_best[w].total, wave_best[w].at, top.total, top.at)) top = wave_best[w];
        if (threadIdx.x == 0) {
            if (top.at == ~0ull) write_none(r);
            else write(r, top.total, top.at);
        }
        prev_t = top.total;
        prev_a = top.at;
    }
}

// ---------------------------------------------------------------- reordering
// Every state's row s B + b becomes what row s B + parent[s B + b] was, in place: a thread takes 16 bytes of a place
// (or one element, at the end of a run) of all B rows of a sentence, reads what moves and then writes it, so no
// byte is read after it was written over and nothing is copied twice.  The bytes wait in registers (in LDS, one
// wavefront of 32 rows took 676 us where the registers take 236: 12 layers x 32 rows x 16 x 500 x 64, fp16).
constexpr int DIMS = 4;
struct StateArgs {
    char *base;
    long row_stride, sizes[DIMS], strides[DIMS];   // bytes; the places outside the contiguous run
    long run;                                      // bytes
    int elem, dims;
    unsigned int chunks;                           // of a run: 16-byte ones, then elements
    unsigned int groups;                           // workgroups for each sentence
};
constexpr int STATES = 8;
struct ReorderArgs {
    StateArgs state[STATES];
    int states, S, B;
    const int32_t *parent;
    long first;            // the launch's first workgroup, of those that all states need
};

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef i32x4 i32x4_any1 __attribute__((aligned(1)));

__device__ inline i32x4 load_chunk(const char *p, bool whole, int elem)
{
    if (whole) return *(const i32x4_any1 *)p;
    i32x4 v = {0, 0, 0, 0};
    if (elem == 1) v[0] = *(const uint8_t *)p;
    else if (elem == 2) v[0] = *(const uint16_t *)p;
    else if (elem == 4) v[0] = *(const int *)p;
    else v[0] = ((const int *)p)[0], v[1] = ((const int *)p)[1];
    return v;
}
__device__ inline void store_chunk(char *p, bool whole, int elem, i32x4 v)
{
    if (whole) *(i32x4_any1 *)p = v;
    else if (elem == 1) *(uint8_t *)p = (uint8_t)v[0];
    else if (elem == 2) *(uint16_t *)p = (uint16_t)v[0];
    else if (elem == 4) *(int *)p = v[0];
    else ((int *)p)[0] = v[0], ((int *)p)[1] = v[1];
}

// MOST: rows that wait in registers, at least B.
template <int MOST>
__global__ __launch_bounds__(THREADS) void reorder_kernel(const ReorderArgs A)
{
    long group = A.first + blockIdx.x;
    int k = 0;
    while (k + 1 < A.states && group >= (long)A.state[k].groups * A.S) group -= (long)A.state[k].groups * A.S, ++k;
    const StateArgs &st = A.state[k];
    const int sentence = (int)(group / st.groups);
    const unsigned int id = (unsigned int)(group % st.groups) * THREADS + threadIdx.x;
    unsigned int place = id / st.chunks;
    const unsigned int chunk = id - place * st.chunks;
    const unsigned int whole_chunks = (unsigned int)(st.run / 16);
    const bool whole = chunk < whole_chunks;
    char *at = st.base + (size_t)sentence * A.B * st.row_stride +
               (whole ? (size_t)chunk * 16 : (size_t)whole_chunks * 16 + (size_t)(chunk - whole_chunks) * st.elem);
    for (int i = 0; i < st.dims; ++i) {
        const unsigned int size = (unsigned int)st.sizes[i], q = place / size;
        at += (long)(place - q * size) * st.strides[i];
        place = q;
    }
    if (place) return;      // past the last place
    const int32_t *const parent = A.parent + (size_t)sentence * A.B;
    auto moves = [&](int b, int &from) {
        from = parent[b];
        return from >= 0 && from < A.B && from != b;
    };
    i32x4 v[MOST];
#pragma unroll
    for (int b = 0; b < MOST; ++b) {
        int from;
        if (b < A.B && moves(b, from)) v[b] = load_chunk(at + (size_t)from * st.row_stride, whole, st.elem);
    }
#pragma unroll
    for (int b = 0; b < MOST; ++b) {
        int from;
        if (b < A.B && moves(b, from)) store_chunk(at + (size_t)b * st.row_stride, whole, st.elem, v[b]);
    }
}

struct SelectLayout {
    int U, pieces;
    size_t part, best, total;
};

// Vectors to a thread: as many as leave room for eight wavefronts a SIMD (six 16-bit ones, 36 us for 256 x 250,000 fp16;
// four 38, eight 41; four of fp32), fewer where few rows would leave compute units without a piece (5 rows fp32: one
// vector, 123 pieces a row, 5.7 us).
void select_layout(int n, int V, int B, int type, SelectLayout *L)
{
    int U = type == VP_F32 ? 4 : 6;
    while (U > 1 && (long)n * layer_ceil_div(V, 2048 * U) < 1024) U = U == 6 ? 4 : U / 2;
    L->U = U;
    L->pieces = (int)layer_ceil_div(V, 2048 * U);
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o += layer_align_up(bytes); return at; };
    L->part = take((size_t)n * L->pieces * sizeof(Piece));
    L->best = take((size_t)n * L->pieces * B * 8);
    L->total = o;
}

vp_status select_sizes(const char *fn, int32_t S, int32_t B, int32_t V)
{
    if (S < 0 || B < 1 || B > VP_MAX_BEAMS || V < 1 || V > (1 << 30) || (long)S * B > VP_MAX_ROWS)
        return (vp_status)vpi_fail(VP_ERR_UNSUPPORTED, "%s: S = %d, B = %d, V = %d (need 1 <= B <= %d, S * B <= %d, 1 <= V <= 2^30)", fn, S, B, V, VP_MAX_BEAMS, VP_MAX_ROWS);
    return VP_OK;
}

// What a reorder needs to know of its states, or why there is none: nothing is launched.
vp_status reorder_states(const vp_state *states, int32_t count, int32_t S, int32_t B, ReorderArgs *A, long *groups_in_all)
{
    if (S < 0 || B < 1 || B > VP_MAX_BEAMS || (long)S * B > VP_MAX_ROWS)
        return (vp_status)vpi_fail(VP_ERR_UNSUPPORTED, "vp_beam_reorder: S = %d, B = %d (need 1 <= B <= %d, S * B <= %d)", S, B, VP_MAX_BEAMS, VP_MAX_ROWS);
    if (count < 0 || count > STATES) return (vp_status)vpi_fail(VP_ERR_UNSUPPORTED, "vp_beam_reorder: %d states: at most %d a call", count, STATES);
    if (count > 0 && !states) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_reorder: null pointer argument");
    long total = 0;
    for (int i = 0; i < count; ++i) {
        const vp_state &in = states[i];
        if (in.elem_bytes != 1 && in.elem_bytes != 2 && in.elem_bytes != 4 && in.elem_bytes != 8)
            return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_reorder: state %d: elements of %d bytes", i, in.elem_bytes);
        if (in.dims < 1 || in.dims > VP_STATE_DIMS || in.row_dim < 0 || in.row_dim >= in.dims)
            return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_reorder: state %d: %d dimensions, rows along %d", i, in.dims, in.row_dim);
        if (in.sizes[in.row_dim] != (int64_t)S * B)
            return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_reorder: state %d has %lld rows, %lld hypotheses", i, (long long)in.sizes[in.row_dim], (long long)S * B);
        // the dimensions by stride; they must not overlap (what lies inside a step is smaller than the step)
        int order[VP_STATE_DIMS], kept = 0;
        bool empty = S == 0;
        for (int j = 0; j < in.dims; ++j) {
            if (in.sizes[j] < 0 || in.strides[j] < 0) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_reorder: state %d: a negative size or stride", i);
            empty = empty || in.sizes[j] == 0;
            if (in.sizes[j] > 1) order[kept++] = j;
        }
        if (empty) continue;
        if (!in.data || !layer_aligned(in.data, in.elem_bytes)) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_reorder: state %d: null or misaligned address", i);
        std::sort(order, order + kept, [&](int a, int b) { return in.strides[a] < in.strides[b]; });
        int64_t reach = 1;
        for (int j = 0; j < kept; ++j) {
            if (in.strides[order[j]] < reach) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_reorder: state %d overlaps itself", i);
            // (so that no product below overflows)
            int64_t span;
            if (__builtin_mul_overflow(in.sizes[order[j]] - 1, in.strides[order[j]], &span) || __builtin_add_overflow(span, reach, &reach) || reach > (1ll << 48))
                return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_reorder: state %d reaches past any memory", i);
        }
        StateArgs &st = A->state[A->states];
        st.base = (char *)in.data;
        st.elem = in.elem_bytes;
        st.row_stride = (long)in.strides[in.row_dim] * in.elem_bytes;
        st.run = in.elem_bytes;
        // dimensions that continue each other become one; those that continue the run lengthen it
        for (int j = 0; j < kept; ++j) {
            const int o = order[j];
            if (o == in.row_dim) continue;
            const long size = (long)in.sizes[o], stride = (long)in.strides[o] * in.elem_bytes;
            if (st.dims == 0 && stride == st.run) st.run *= size;
            else if (st.dims > 0 && stride == st.sizes[st.dims - 1] * st.strides[st.dims - 1]) st.sizes[st.dims - 1] *= size;
            else if (st.dims == DIMS) return (vp_status)vpi_fail(VP_ERR_UNSUPPORTED, "vp_beam_reorder: state %d: more than %d separate dimensions around its runs", i, DIMS);
            else st.sizes[st.dims] = size, st.strides[st.dims++] = stride;
        }
        const long chunks = st.run / 16 + st.run % 16 / st.elem;
        long places = 1;
        for (int j = 0; j < st.dims; ++j) places *= st.sizes[j];
        const long groups = layer_ceil_div(chunks * places, THREADS);
        if (chunks * places >= (1l << 31))   // (numbered in 32 bits within a sentence)
            return (vp_status)vpi_fail(VP_ERR_UNSUPPORTED, "vp_beam_reorder: state %d is too large", i);
        st.chunks = (unsigned int)chunks;
        st.groups = (unsigned int)groups;
        total += groups * S;
        ++A->states;
    }
    *groups_in_all = total;
    return VP_OK;
}

}  // namespace

extern "C" {

size_t vp_beam_select_workspace_bytes(int32_t S, int32_t B, int32_t V)
{
    if (select_sizes("vp_beam_select", S, B, V) != VP_OK) return 0;
    SelectLayout L;
    // (of the type that takes more: its pieces are the shorter ones)
    select_layout(std::max(S * B, 1), V, B, VP_F32, &L);
    return L.total;
}

vp_status vp_beam_select(const void *logits, int32_t type, int64_t stride, const float *scores, int32_t S, int32_t B,
                         int32_t V, const uint32_t *allowed, int64_t allowed_stride, const uint8_t *done, int32_t eos,
                         float *out_scores, int32_t *out_parent, int32_t *out_token, uint8_t *out_done,
                         void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const vp_status s = select_sizes("vp_beam_select", S, B, V);
    if (s != VP_OK) return s;
    if (!type_known(type)) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_select: unknown type %d", type);
    if (stride < V || (allowed && allowed_stride < layer_ceil_div(V, 32)))
        return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_select: rows of %d at a stride of %lld, bits at %lld words", V, (long long)stride, (long long)allowed_stride);
    if (S == 0) return VP_OK;
    if (!logits || !scores || !out_scores || !out_parent || !out_token || !workspace)
        return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_select: null pointer argument");
    if (!layer_aligned(logits, type_size(type)) || !layer_aligned(scores, 4) || !layer_aligned(allowed, 4))
        return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_select: an address that is no multiple of its element's size");
    if (!layer_aligned(workspace, LAYER_ALIGN)) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    const int n = S * B;
    SelectLayout L;
    select_layout(n, V, B, type, &L);
    if (workspace_bytes < L.total) return (vp_status)vpi_fail(VP_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, L.total);
    if ((long)n * L.pieces >= (1l << 32) / THREADS) return (vp_status)vpi_fail(VP_ERR_UNSUPPORTED, "vp_beam_select: %d rows of %d are too many", n, V);
    const hipStream_t st = (hipStream_t)hip_stream;
    const SelectArgs A = {logits, (long)stride, (long)allowed_stride, scores, allowed, done, n, V, B, L.pieces, eos,
                          (Piece *)((char *)workspace + L.part), (unsigned long long *)((char *)workspace + L.best),
                          out_scores, out_parent, out_token, out_done};
    const dim3 grid((unsigned int)n * (unsigned int)L.pieces);
    with_type(type, [&](auto t) {
        typedef decltype(t) T;
        if constexpr (sizeof(T) == 2) {
            if (L.U == 6) {
                hipLaunchKernelGGL((select_piece_kernel<T, 6>), grid, dim3(THREADS), 0, st, A);
                return;
            }
        }
        if (L.U == 4) hipLaunchKernelGGL((select_piece_kernel<T, 4>), grid, dim3(THREADS), 0, st, A);
        else if (L.U == 2) hipLaunchKernelGGL((select_piece_kernel<T, 2>), grid, dim3(THREADS), 0, st, A);
        else hipLaunchKernelGGL((select_piece_kernel<T, 1>), grid, dim3(THREADS), 0, st, A);
    });
    hipLaunchKernelGGL(select_join_kernel, dim3(S), dim3(JOIN_THREADS), 0, st, A);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (vp_status)vpi_fail(VP_ERR_HIP, "vp_beam_select: %s", hipGetErrorString(e));
    return VP_OK;
}

vp_status vp_beam_reorder_check(const vp_state *states, int32_t count, int32_t S, int32_t B)
{
    ReorderArgs A = {};
    long total = 0;
    return reorder_states(states, count, S, B, &A, &total);
}

vp_status vp_beam_reorder(const vp_state *states, int32_t count, const int32_t *parent, int32_t S, int32_t B,
                          void *hip_stream)
{
    ReorderArgs A = {};
    long total = 0;
    const vp_status s = reorder_states(states, count, S, B, &A, &total);
    if (s != VP_OK) return s;
    if (S > 0 && count > 0 && !parent) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_beam_reorder: null pointer argument");
    A.S = S;
    A.B = B;
    A.parent = parent;
    if (total == 0 || B == 1) return VP_OK;
    const hipStream_t st = (hipStream_t)hip_stream;
    constexpr long most = LAUNCH_THREADS / THREADS;     // workgroups of a launch
    for (; A.first < total; A.first += most) {
        const dim3 grid((unsigned int)std::min<long>(most, total - A.first));
        if (B <= 4) hipLaunchKernelGGL((reorder_kernel<4>), grid, dim3(THREADS), 0, st, A);
        else if (B <= 8) hipLaunchKernelGGL((reorder_kernel<8>), grid, dim3(THREADS), 0, st, A);
        else if (B <= 16) hipLaunchKernelGGL((reorder_kernel<16>), grid, dim3(THREADS), 0, st, A);
        else hipLaunchKernelGGL((reorder_kernel<32>), grid, dim3(THREADS), 0, st, A);
    }
    static_assert(VP_MAX_BEAMS <= 32, "rows in registers");
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (vp_status)vpi_fail(VP_ERR_HIP, "vp_beam_reorder: %s", hipGetErrorString(e));
    return VP_OK;
}

}  // extern "C"
