// Root-mean-square norm of the sum of a row and its residual, and its gradient.
//   s = x + residual, rounded once to their type (the stream that goes on); the norm is that of the rounded sum
//   rstd = (mean of s^2 + eps)^(-1/2), y = s * rstd * weight
//   norm = y rounded once; and in 8 bits per block of 128 columns: scale = max(max |y|, 1e-30) / 448, q = y / scale
//   rounded to e4m3 (1e-30 keeps a block of zeros from dividing by zero; 448 is the largest e4m3 value)
// One to eight wavefronts keep a row in registers, eight columns to a lane, 512 to a wavefront, so every byte is read once and a block of 128 columns is 16 neighbouring lanes, whose maximum four
// data-parallel moves find.  (One wavefront a row whatever its width kept four to eight times the registers: one or two
// wavefronts a SIMD, and 6,000 x 4,096 bf16 took 46 and 125 us forward and backward.)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "vp.h"
#include "vp_kernels.h"
#include "typed.h"
#include "wave_ops.h"

namespace {

constexpr int waves_of(int W) { return W < 3 ? 4 : W; }     // of a workgroup, for W to a row
constexpr int STEP = 512;          // columns of a wavefront's step
constexpr int BLOCK = 128;         // columns that share a scale
constexpr float TINY = 1e-30f;
constexpr float E4M3_MAX = 448.f;

// Largest unsigned over the 16 lanes of a row, to each of them.  (The bits of magnitudes: NaN above infinity above
// every number, so that neither is lost.)
__device__ inline unsigned int row_max(unsigned int v)
{
#define VP_ROW_MAX(ctrl) v = max(v, (unsigned int)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, 0xf, 0xf, false));
    VP_ROW_MAX(0x121)   // row_ror:1
    VP_ROW_MAX(0x122)   // row_ror:2
    VP_ROW_MAX(0x124)   // row_ror:4
    VP_ROW_MAX(0x128)   // row_ror:8
#undef VP_ROW_MAX
    return v;
}

template <typename T> __device__ inline void load8_of(const T *p, int c, int d, float (&v)[8])
{
    RowPiece<T, 8> piece;
    piece.load(p, c, d);
    piece.values(c, d, v);
}
__device__ inline void load8_any(const void *p, int type, int c, int d, float (&v)[8])
{
    if (type == VP_F16) load8_of((const Half *)p, c, d, v);
    else if (type == VP_BF16) load8_of((const Bf16 *)p, c, d, v);
    else load8_of((const float *)p, c, d, v);
}

struct NormArgs {
    const void *x, *residual, *weight;
    long x_stride, residual_stride, n;
    int d, weight_type;
    float eps;
    void *sum, *norm;     // NULL: not wanted
    int norm_type;
    uint8_t *q;           // NULL: not wanted; rows of a multiple of 128 bytes
    float *scales;
    float *rstd;
    bool stream;

    // on to the rows behind these (elements of `size` bytes)
    void skip(long rows, size_t size)
    {
        const long blocks = (d + BLOCK - 1) / BLOCK;
        x = (const char *)x + rows * x_stride * size;
        if (residual) residual = (const char *)residual + rows * residual_stride * size;
        if (sum) sum = (char *)sum + rows * d * size;
        if (norm) norm = (char *)norm + rows * d * type_size(norm_type);
        if (q) q += rows * blocks * BLOCK, scales += rows * blocks;
        if (rstd) rstd += rows;
    }
};

// Sum over the W wavefronts of a row; `slot`: one of two places, in turn where calls follow each other.
template <int W> __device__ inline float row_sum_of(float v, int slot)
{
    constexpr int WAVES = waves_of(W);
    v = wave_sum_float(v);
    if (W == 1) return v;
    __shared__ float part[2][WAVES];
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) part[slot][wave] = v;
    __syncthreads();
    const int first = wave / W * W;
    v = part[slot][first];
#pragma unroll
    for (int w = 1; w < W; ++w) v += part[slot][first + w];
    return v;
}

// W wavefronts to a row, 512 columns to each.
template <typename T, int W>
__global__ __launch_bounds__(64 * waves_of(W)) void add_norm_kernel(const NormArgs A)
{
    constexpr int WAVES = waves_of(W);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long row = (long)blockIdx.x * (WAVES / W) + wave / W;
    const int c = (wave % W) * STEP + lane * 8;
    const int d = A.d;
    const long at = min(row, A.n - 1);      // (a row past the last one is worked on, and not written)
    RowPiece<T, 8> x, r;
    x.load((const T *)A.x + (size_t)at * A.x_stride, c, d);
    if (A.residual) r.load((const T *)A.residual + (size_t)at * A.residual_stride, c, d);
    float f[8], w[8];
    load8_any(A.weight, A.weight_type, c, d, w);
    x.values(c, d, f);
    if (A.residual) {
        float g[8];
        r.values(c, d, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = rounded<T>(f[j] + g[j]);
    }
    float squares = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) squares += f[j] * f[j];
    const float rstd = 1.f / sqrtf(row_sum_of<W>(squares, 0) / (float)d + A.eps);
    if (row >= A.n) return;
    if (A.rstd && lane == 0 && wave % W == 0) A.rstd[row] = rstd;
    const int blocks = (d + BLOCK - 1) / BLOCK;
    if (A.sum) put_within((T *)A.sum + (size_t)row * d, c, d, f, A.stream);
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = f[j] * rstd * w[j];
    // past d no part in the scale and bytes of zero, though rstd or the scale may be no number or infinite (the bytes without a
    // branch: with one around what was packed, 16,384 x 1,536 bf16 took 33.3 us instead of 33.0)
    const int left = d - c;
    if (left < 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = j < left ? y[j] : 0.f;
    }
    if (A.norm) {
        const size_t at = (size_t)row * d;
        if (A.norm_type == VP_F16) put_within((Half *)A.norm + at, c, d, y, A.stream);
        else if (A.norm_type == VP_BF16) put_within((Bf16 *)A.norm + at, c, d, y, A.stream);
        else put_within((float *)A.norm + at, c, d, y, A.stream);
    }
    if (A.q) {
        unsigned int most = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) most = max(most, __float_as_uint(y[j]) & 0x7fffffffu);
        most = max(row_max(most), __float_as_uint(TINY));
        const float scale = __uint_as_float(most) / E4M3_MAX;
        u32x2 packed;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float p[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) p[j] = h * 4 + j < left ? y[h * 4 + j] / scale : 0.f;
            int word = __builtin_amdgcn_cvt_pk_fp8_f32(p[0], p[1], 0, false);
            packed[h] = (unsigned int)__builtin_amdgcn_cvt_pk_fp8_f32(p[2], p[3], word, true);
        }
        if (c < blocks * BLOCK) {
            u32x2 *const to = (u32x2 *)(A.q + (size_t)row * blocks * BLOCK + c);
            if (A.stream) VP_STREAM_STORE(to, packed);
            else *to = packed;
            if ((lane & 15) == 0) A.scales[(size_t)row * blocks + c / BLOCK] = scale;
        }
    }
}

// ---------------------------------------------------------------- gradient
//   h = s * rstd,   dx = rstd * (w * dnorm - h * mean(w * dnorm * h)) + dsum,   dweight = sum over rows of dnorm * h
// (h is of the order of one whatever the row's size; rstd^3 and w * dnorm * s leave 32 bits' range long before rstd does)
// A workgroup takes every so many rows (W wavefronts to each) and keeps its share of dweight in registers; what its
// wavefronts have of the same columns is joined in LDS, and a second kernel adds up the workgroups' in a fixed order.
constexpr int GRAD_GROUPS = 1024;

struct NormGradArgs {
    const void *dnorm, *s, *dsum, *weight;
    long dnorm_stride, s_stride, dsum_stride, n;
    int d, weight_type;
    const float *rstd;
    void *dx;
    float *partial;   // [groups, d]
    bool stream;
};

template <typename T, int W>
__global__ __launch_bounds__(64 * waves_of(W)) void add_norm_grad_kernel(const NormGradArgs A)
{
    constexpr int WAVES = waves_of(W), ROWS = WAVES / W;     // rows at a time
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = (wave % W) * STEP + lane * 8;
    const int d = A.d;
    float w[8], dw[8] = {};
    load8_any(A.weight, A.weight_type, c, d, w);
    const float per = 1.f / (float)d;
    struct Row { RowPiece<T, 8> f, g, e; float r; } next;
    auto load = [&](long row, Row &to) {
        const long at = min(row, A.n - 1);     // (a row past the last one counts nothing)
        to.f.load((const T *)A.s + (size_t)at * A.s_stride, c, d);
        to.g.load((const T *)A.dnorm + (size_t)at * A.dnorm_stride, c, d);
        if (A.dsum) to.e.load((const T *)A.dsum + (size_t)at * A.dsum_stride, c, d);
        to.r = A.rstd[at];
    };
    const long mine = (long)blockIdx.x * ROWS, step = (long)gridDim.x * ROWS;
    if (mine < A.n) load(mine + wave / W, next);
    int slot = 0;
    for (long row0 = mine; row0 < A.n; row0 += step, slot ^= 1) {
        const long row = row0 + wave / W;
        Row now = next;
        if (row0 + step < A.n) load(row + step, next);     // (on its way during this one: 38 -> 30 us for 16,384 x 1,024 bf16)
        const float r = now.r;
        float f[8], g[8];
        now.f.values(c, d, f);
        now.g.values(c, d, g);
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            f[j] *= r;
            dw[j] = row < A.n ? fmaf(g[j], f[j], dw[j]) : dw[j];     // (not by r = 0: the row that is read may hold infinities)
            g[j] *= w[j];
            dot += g[j] * f[j];
        }
        const float k = per * row_sum_of<W>(dot, slot);
        float o[8], e[8] = {};
        if (A.dsum) now.e.values(c, d, e);
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = r * (g[j] - f[j] * k) + e[j];
        if (row < A.n) put_within((T *)A.dx + (size_t)row * d, c, d, o, A.stream);
    }
    if (ROWS > 1) {
        __shared__ float part[WAVES][STEP];
        if (wave >= W) {
#pragma unroll
            for (int j = 0; j < 8; ++j) part[wave][j * 64 + lane] = dw[j];
        }
        __syncthreads();
        if (wave >= W) return;
#pragma unroll
        for (int v = 1; v < ROWS; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) dw[j] += part[wave + v * W][j * 64 + lane];
    }
    store8_within(A.partial + (size_t)blockIdx.x * d, c, d, dw);
}

// dweight[c] = sum over the groups: 16 columns x 32 strands of groups to a workgroup, the strands joined by halves.
constexpr int STRANDS = 32;
__global__ __launch_bounds__(16 * STRANDS) void dweight_kernel(const float *__restrict__ partial, int groups, int d,
                                                               float *__restrict__ dweight)
{
    __shared__ float part[STRANDS][16];
    const int col = threadIdx.x & 15, strand = threadIdx.x >> 4;
    const int c = blockIdx.x * 16 + col;
    float acc = 0.f;
    if (c < d)
#pragma unroll 8
        for (int g = strand; g < groups; g += STRANDS) acc += partial[(size_t)g * d + c];
    part[strand][col] = acc;
    for (int half = STRANDS / 2; half; half /= 2) {
        __syncthreads();
        if (strand < half) part[strand][col] += part[strand + half][col];
    }
    if (strand == 0 && c < d) dweight[c] = part[0][col];
}

// f(wavefronts to a row)
template <typename F> void with_waves(int d, F f)
{
    const int steps = (d + STEP - 1) / STEP;
    if (steps <= 1) f(std::integral_constant<int, 1>{});
    else if (steps == 2) f(std::integral_constant<int, 2>{});
    else if (steps == 3) f(std::integral_constant<int, 3>{});
    else if (steps == 4) f(std::integral_constant<int, 4>{});
    else if (steps <= 6) f(std::integral_constant<int, 6>{});
    else f(std::integral_constant<int, 8>{});
}
static_assert(VP_MAX_DIM <= 8 * STEP, "up to eight wavefronts");
inline int rows_at_once(int d) { return d <= STEP ? 4 : d <= 2 * STEP ? 2 : 1; }
inline int grad_groups(int64_t n, int d) { return (int)std::max<int64_t>(1, std::min<int64_t>(GRAD_GROUPS, layer_ceil_div(n, rows_at_once(d)))); }

vp_status norm_sizes(const char *fn, int64_t n, int32_t d)
{
    if (d < 1 || d > VP_MAX_DIM) return (vp_status)vpi_fail(VP_ERR_UNSUPPORTED, "%s: d = %d: need 1 <= d <= %d", fn, d, VP_MAX_DIM);
    if (n < 0 || n >= (1ll << 31)) return (vp_status)vpi_fail(VP_ERR_UNSUPPORTED, "%s: n = %lld out of range", fn, (long long)n);
    return VP_OK;
}

}  // namespace

extern "C" {

vp_status vp_add_norm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, int32_t type,
                      const void *weight, int32_t weight_type, int64_t n, int32_t d, float eps, void *sum, void *norm,
                      int32_t norm_type, uint8_t *q, float *scales, float *rstd, void *hip_stream)
{
    const vp_status s = norm_sizes("vp_add_norm", n, d);
    if (s != VP_OK) return s;
    if (!type_known(type) || !type_known(weight_type) || (norm && !type_known(norm_type)))
        return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_add_norm: unknown type %d, %d or %d", type, weight_type, norm_type);
    if (x_stride < d || (residual && residual_stride < d))
        return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_add_norm: rows of %d at a stride of %lld or %lld", d, (long long)x_stride, (long long)residual_stride);
    if (!(eps >= 0.f)) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_add_norm: eps = %g", (double)eps);
    if ((q == nullptr) != (scales == nullptr)) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_add_norm: q and scales go together");
    if (n == 0) return VP_OK;
    if (!x || !weight) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_add_norm: null pointer argument");
    // (a row's sum would lie on another row's elements)
    if (n > 1 && sum && ((sum == x && x_stride != d) || (sum == residual && residual_stride != d)))
        return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_add_norm: sum over rows that are not contiguous");
    const size_t a = type_size(type);
    if (!layer_aligned(x, a) || !layer_aligned(residual, a) || !layer_aligned(sum, a) || !layer_aligned(weight, type_size(weight_type)) ||
        (norm && !layer_aligned(norm, type_size(norm_type))) || !layer_aligned(q, 8) || !layer_aligned(scales, 4) || !layer_aligned(rstd, 4))
        return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_add_norm: an address that is no multiple of its element's size (q: of 8)");
    NormArgs A = {x, residual, weight, (long)x_stride, (long)residual_stride, 0, d, weight_type, eps, sum, norm, norm_type, q, scales, rstd,
                  n * d * (long)((sum ? a : 0) + (norm ? type_size(norm_type) : 0) + (q ? 1 : 0)) > STREAM_BYTES};
    with_type(type, [&](auto t) {
        with_waves(d, [&](auto waves) {
            constexpr int W = decltype(waves)::value, ROWS = waves_of(W) / W;
            constexpr long most = LAUNCH_THREADS / (64 * W);
            for (long at = 0; at < n; at += most) {
                A.n = std::min<long>(most, n - at);
                hipLaunchKernelGGL((add_norm_kernel<decltype(t), W>), dim3((unsigned int)layer_ceil_div(A.n, ROWS)), dim3(64 * waves_of(W)), 0, (hipStream_t)hip_stream, A);
                A.skip(most, a);
            }
        });
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (vp_status)vpi_fail(VP_ERR_HIP, "vp_add_norm: %s", hipGetErrorString(e));
    return VP_OK;
}

size_t vp_add_norm_grad_workspace_bytes(int64_t n, int32_t d)
{
    if (norm_sizes("vp_add_norm_grad", n, d) != VP_OK) return 0;
    return layer_align_up((size_t)grad_groups(n, d) * d * 4);
}

vp_status vp_add_norm_grad(const void *dnorm, int64_t dnorm_stride, const void *s, int64_t s_stride, const void *dsum,
                           int64_t dsum_stride, int32_t type, const void *weight, int32_t weight_type,
                           const float *rstd, int64_t n, int32_t d, void *dx, float *dweight, void *workspace,
                           size_t workspace_bytes, void *hip_stream)
{
    const vp_status st = norm_sizes("vp_add_norm_grad", n, d);
    if (st != VP_OK) return st;
    if (!type_known(type) || !type_known(weight_type)) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_add_norm_grad: unknown type %d or %d", type, weight_type);
    if (dnorm_stride < d || s_stride < d || (dsum && dsum_stride < d))
        return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_add_norm_grad: rows of %d at a stride of %lld, %lld or %lld", d, (long long)dnorm_stride, (long long)s_stride, (long long)dsum_stride);
    if ((n > 0 && (!dnorm || !s || !rstd || !dx)) || !weight || !dweight || !workspace)
        return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_add_norm_grad: null pointer argument");
    const size_t a = type_size(type);
    if (!layer_aligned(dnorm, a) || !layer_aligned(s, a) || !layer_aligned(dsum, a) || !layer_aligned(dx, a) ||
        !layer_aligned(weight, type_size(weight_type)) || !layer_aligned(rstd, 4) || !layer_aligned(dweight, 4))
        return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_add_norm_grad: an address that is no multiple of its element's size");
    if (!layer_aligned(workspace, LAYER_ALIGN)) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    const size_t need = vp_add_norm_grad_workspace_bytes(n, d);
    if (workspace_bytes < need) return (vp_status)vpi_fail(VP_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, need);
    const int groups = grad_groups(n, d);
    const NormGradArgs A = {dnorm, s, dsum, weight, (long)dnorm_stride, (long)s_stride, (long)dsum_stride, (long)n, d, weight_type, rstd, dx, (float *)workspace, n * d * (long)a > STREAM_BYTES};
    with_type(type, [&](auto t) {
        with_waves(d, [&](auto waves) {
            hipLaunchKernelGGL((add_norm_grad_kernel<decltype(t), decltype(waves)::value>), dim3(groups), dim3(64 * waves_of(decltype(waves)::value)), 0, (hipStream_t)hip_stream, A);
        });
    });
    hipLaunchKernelGGL(dweight_kernel, dim3((unsigned int)layer_ceil_div(d, 16)), dim3(16 * STRANDS), 0, (hipStream_t)hip_stream, (const float *)workspace, groups, d, dweight);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (vp_status)vpi_fail(VP_ERR_HIP, "vp_add_norm_grad: %s", hipGetErrorString(e));
    return VP_OK;
}

}  // extern "C"
