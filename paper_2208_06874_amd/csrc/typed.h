// Elements of the three types the layer kernels take (vp_type), moved eight at a time.  Rows of an odd number of
// 16-bit elements start at any even address: the vectors are declared with the alignment of one element, for which
// gfx950 has the same 16-byte memory instructions (unaligned access is on), so no kernel needs a second form.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vp.h"

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef u32x4 u32x4_any2 __attribute__((aligned(2)));
typedef u32x2 u32x2_any2 __attribute__((aligned(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef f32x4 f32x4_any4 __attribute__((aligned(4)));

struct Half { uint16_t b; };
struct Bf16 { uint16_t b; };

__device__ inline float value(Half x) { return (float)__builtin_bit_cast(_Float16, x.b); }
__device__ inline float value(Bf16 x) { return __uint_as_float((unsigned int)x.b << 16); }
__device__ inline float value(float x) { return x; }

// one rounding, nearest with ties to even
__device__ inline void round_to(float v, Half &o) { o.b = __builtin_bit_cast(uint16_t, (_Float16)v); }
__device__ inline void round_to(float v, Bf16 &o) { o.b = __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ inline void round_to(float v, float &o) { o = v; }

template <typename T> __device__ inline float rounded(float v)
{
    T t;
    round_to(v, t);
    return value(t);
}

__device__ inline void load8(const float *p, float (&v)[8])
{
    const f32x4 a = *(const f32x4_any4 *)p, b = *(const f32x4_any4 *)(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
}
template <typename T> __device__ inline void load8(const T *p, float (&v)[8])
{
    const u32x4 a = *(const u32x4_any2 *)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = value(T{(uint16_t)(a[i] & 0xffffu)});
        v[2 * i + 1] = value(T{(uint16_t)(a[i] >> 16)});
    }
}
__device__ inline void store8(float *p, const float (&v)[8])
{
    f32x4 a, b;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = v[i], b[i] = v[4 + i];
    *(f32x4_any4 *)p = a;
    *(f32x4_any4 *)(p + 4) = b;
}
template <typename T> __device__ inline u32x4 packed8(const float (&v)[8])
{
    u32x4 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        T lo, hi;
        round_to(v[2 * i], lo);
        round_to(v[2 * i + 1], hi);
        a[i] = (unsigned int)lo.b | ((unsigned int)hi.b << 16);
    }
    return a;
}
template <typename T> __device__ inline void store8(T *p, const float (&v)[8]) { *(u32x4_any2 *)p = packed8<T>(v); }

// A store past the L2's lines.  (Between two empty asm statements: where the other branch of a condition stores the same
// value to the same place, the compiler makes one ordinary store of the two.)
#define VP_STREAM_STORE(p, v)                       \
    do {                                            \
        asm volatile("");                           \
        __builtin_nontemporal_store((v), (p));      \
        asm volatile("");                           \
    } while (0)

// Eight elements at column c of a row of d: what lies at or past d reads as 0 and is not written.
template <typename T> __device__ inline void load8_within(const T *row, int c, int d, float (&v)[8])
{
    if (c + 8 <= d) {
        load8(row + c, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i < d ? value(row[c + i]) : 0.f;
}
template <typename T> __device__ inline void store8_within(T *row, int c, int d, const float (&v)[8])
{
    if (c + 8 <= d) {
        store8(row + c, v);
        return;
    }
    const int left = d - c;
    if (left <= 0) return;
    // four, two and one, as many as are left
    if constexpr (sizeof(T) == 4) {
        // (as vectors: of the array the compiler would make a choice of addresses, and keep it in memory)
        const f32x4 lo = {v[0], v[1], v[2], v[3]}, hi = {v[4], v[5], v[6], v[7]};
        if (left & 4) *(f32x4_any4 *)(row + c) = lo;
        const int at = left & 4;
        const f32x4 rest = at ? hi : lo;
        const float x = rest[0], y = rest[1], z = rest[2];
        if (left & 2) row[c + at] = x, row[c + at + 1] = y;
        if (left & 1) row[c + left - 1] = left & 2 ? z : x;
    } else {
        const u32x4 a = packed8<T>(v);
        typedef uint32_t u32_any2 __attribute__((aligned(2)));
        if (left & 4) *(u32x2_any2 *)(row + c) = u32x2{a[0], a[1]};
        const int at = left & 4;
        const uint32_t x = at ? a[2] : a[0], y = at ? a[3] : a[1];
        if (left & 2) *(u32_any2 *)(row + c + at) = x;
        if (left & 1) row[c + left - 1].b = (uint16_t)(left & 2 ? y : x);
    }
}

// Four at a time: for fp32 results, so that a wavefront's store is one run of bytes.
__device__ inline void load4(const float *p, float (&v)[4])
{
    const f32x4 a = *(const f32x4_any4 *)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i];
}
template <typename T> __device__ inline void load4(const T *p, float (&v)[4])
{
    const u32x2 a = *(const u32x2_any2 *)p;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        v[2 * i] = value(T{(uint16_t)(a[i] & 0xffffu)});
        v[2 * i + 1] = value(T{(uint16_t)(a[i] >> 16)});
    }
}
template <typename T> __device__ inline void load_within(const T *row, int c, int d, float (&v)[8]) { load8_within(row, c, d, v); }
template <typename T> __device__ inline void load_within(const T *row, int c, int d, float (&v)[4])
{
    if (c + 4 <= d) {
        load4(row + c, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = c + i < d ? value(row[c + i]) : 0.f;
}
template <typename T> __device__ inline void store_within(T *row, int c, int d, const float (&v)[8]) { store8_within(row, c, d, v); }
__device__ inline void store_within(float *row, int c, int d, const float (&v)[4])
{
    if (c + 4 <= d) {
        f32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = v[i];
        *(f32x4_any4 *)(row + c) = a;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (c + i < d) row[c + i] = v[i];
}
// The same past the L2's lines where `stream` is set (the same for every lane): for results larger than the L2, whose
// other data then stay there (the embedding gradient of 250,000 x 1,024: 301 -> 226 us).
__device__ inline void put_within(float *row, int c, int d, const float (&v)[4], bool stream)
{
    if (stream && c + 4 <= d) {
        const f32x4 a = {v[0], v[1], v[2], v[3]};
        VP_STREAM_STORE((f32x4_any4 *)(row + c), a);
        return;
    }
    store_within(row, c, d, v);
}
__device__ inline void put_within(float *row, int c, int d, const float (&v)[8], bool) { store8_within(row, c, d, v); }   // (half lines at a time: the L2 joins them)
template <typename T> __device__ inline void put_within(T *row, int c, int d, const float (&v)[8], bool stream)
{
    if (stream && c + 8 <= d) {
        VP_STREAM_STORE((u32x4_any2 *)(row + c), packed8<T>(v));
        return;
    }
    store_within(row, c, d, v);
}
// Results of a call that are read next are better left in the L2s when they fit: 256 and 4,096 rows through embedding, norm
// and product are 3 and 0 % slower with all results streamed, 16,384 rows 1 % (the norm alone 40 -> 31 us).
constexpr long STREAM_BYTES = 16l << 20;     // half of the eight L2s

// E elements at column c of a row of d, in two steps: the load, which never branches, so that any number of them can be on
// their way together, and the values, which read as 0 at and past d.  Where the row ends inside the piece (or in front of
// it) the row's last E elements are loaded and moved down.  (As one step with a branch around the row's end, the
// conversions sat in the branch, every load was waited for before the next, and rows of 4,095 took twice those of 4,096.)
template <typename T, int E> struct RowPiece {
    static constexpr int DWORDS = E * sizeof(T) / 4;
    uint32_t w[DWORDS];

    __device__ void load(const T *row, int c, int d)
    {
        if (d >= E) {      // (the same for every lane)
            const T *const p = row + min(c, d - E);
            if constexpr (DWORDS == 2) {
                const u32x2 a = *(const u32x2_any2 *)p;
                w[0] = a[0], w[1] = a[1];
            } else {
#pragma unroll
                for (int q = 0; q < DWORDS / 4; ++q) {
                    const u32x4 a = *((const u32x4_any2 *)p + q);
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[4 * q + i] = a[i];
                }
            }
            return;
        }
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < E; ++i) w[i] = c + i < d ? __builtin_bit_cast(uint32_t, row[c + i]) : 0u;
        } else {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                const uint32_t lo = c + 2 * i < d ? row[c + 2 * i].b : 0, hi = c + 2 * i + 1 < d ? row[c + 2 * i + 1].b : 0;
                w[i] = lo | hi << 16;
            }
        }
    }
    __device__ void values(int c, int d, float (&v)[E])
    {
        const int s = d >= E ? c - (d - E) : 0;     // elements that lie in front of c
        if (s > 0) {
            const int by = sizeof(T) == 2 ? s >> 1 : s;
#pragma unroll
            for (int k = DWORDS / 2; k; k /= 2)
#pragma unroll
                for (int i = 0; i < DWORDS; ++i) w[i] = by & k ? i + k < DWORDS ? w[i + k] : 0u : w[i];
#pragma unroll
            for (int i = 0; i < DWORDS; ++i) w[i] = by >= DWORDS ? 0u : w[i];
            if (sizeof(T) == 2 && (s & 1)) {
#pragma unroll
                for (int i = 0; i < DWORDS; ++i) w[i] = w[i] >> 16 | (i + 1 < DWORDS ? w[i + 1] << 16 : 0u);
            }
        }
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) {
                v[2 * i] = value(T{(uint16_t)(w[i] & 0xffffu)});
                v[2 * i + 1] = value(T{(uint16_t)(w[i] >> 16)});
            }
        }
    }
};

// elements a lane takes of a row that ends up as T
template <typename T> constexpr int LANE_ELEMENTS = 16 / sizeof(T);

inline size_t type_size(int t) { return t == VP_F32 ? 4 : 2; }
inline bool type_known(int t) { return t == VP_F16 || t == VP_BF16 || t == VP_F32; }

// f(T{}) for the type t (checked by the caller)
template <typename F> inline void with_type(int t, F f)
{
    if (t == VP_F16) f(Half{});
    else if (t == VP_BF16) f(Bf16{});
    else f(float{});
}

// A launch counts the threads of a dimension in 32 bits: calls of more rows than fit take several launches of at most these
// many threads.
constexpr long LAUNCH_THREADS = 1l << 31;

constexpr size_t LAYER_ALIGN = 256;
inline size_t layer_align_up(size_t x) { return (x + LAYER_ALIGN - 1) / LAYER_ALIGN * LAYER_ALIGN; }
inline bool layer_aligned(const void *p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline long layer_ceil_div(long a, long b) { return (a + b - 1) / b; }

}  // namespace
