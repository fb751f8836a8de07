// The embedding of tokens, out[i, :] = scale * table[ids[i], :], and its gradient,
// grad[t, :] = scale * sum of dout[i, :] over the i with ids[i] = t.  Both move rows and compute next to nothing.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "vp.h"
#include "vp_kernels.h"
#include "typed.h"
#include "wave_ops.h"

namespace {

constexpr int THREADS = 256, WAVES = THREADS / 64;

// ---------------------------------------------------------------- the lookup
// A row is taken by the smallest power of two of threads that covers it with 16 bytes of output each (at most the
// workgroup), so that a step of few rows has all of its bytes in flight at once and narrow rows share wavefronts.
// The last columns overlap the ones before where d is no multiple of a thread's.
template <typename T, typename O>
__global__ __launch_bounds__(THREADS) void embed_kernel(const T *__restrict__ table, long stride, int V, int d,
                                                        const int32_t *__restrict__ ids, long n, float scale,
                                                        int row_threads, bool stream, O *__restrict__ out)
{
    const long i = (long)blockIdx.x * (THREADS / row_threads) + threadIdx.x / row_threads;
    if (i >= n) return;
    const int id = ids[i];
    const bool there = id >= 0 && id < V;
    const T *const row = table + (size_t)(there ? id : 0) * stride;
    O *const to = out + (size_t)i * d;
    constexpr int E = LANE_ELEMENTS<O>;
    for (int c = (threadIdx.x & (row_threads - 1)) * E; c < d; c += row_threads * E) {
        const int at = d >= E ? min(c, d - E) : 0;
        float v[E];
        RowPiece<T, E> piece;
        piece.load(row, at, d);      // (of row 0, for an id outside)
        piece.values(at, d, v);
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = there ? v[j] * scale : 0.f;
        put_within(to, at, d, v, stream);
    }
}

// ---------------------------------------------------------------- the gradient
// The tokens' positions are put into one list per token (count, room, place); the order inside a list is whatever
// the atomics gave, and is put right by whoever sums the list, so the sums run in ascending position and are the
// same every time.  Lists of up to SHORT positions are one wavefront's.  Longer ones are cut by position into
// windows of about WINDOW entries, which workgroups sum apart and a last kernel joins.
constexpr int SHORT = 16;
constexpr int WINDOW = 128;
constexpr int ALLOC_THREADS = 1024;
constexpr int TOKENS = 16;          // tokens of a workgroup: four for each of its wavefronts
constexpr int ITEM_COLS = 512;      // columns of a long list's item: eight for each lane
constexpr int SMALL_SORT = 256;     // entries that are ordered by comparing each with each
constexpr int SPAN = 8192;          // positions that are ordered as bits at a time
constexpr int MAX_ITEM_GROUPS = 1024;

struct GradState {
    int32_t cursor;   // list entries handed out
    int32_t items;    // windows of long lists
    int32_t joins;    // long lists of more than one window
};
struct GradItem {
    int32_t token, window, windows, pad;
};
struct GradJoin {
    int32_t token, first, windows, pad;
};

__host__ __device__ inline int windows_of(int count) { return (count + WINDOW - 1) / WINDOW; }

__device__ inline bool counts(int id, int V, int padding_id) { return id >= 0 && id < V && id != padding_id; }

__global__ __launch_bounds__(THREADS) void grad_clear_kernel(int32_t *__restrict__ count, int V, GradState *state)
{
    for (long t = (long)blockIdx.x * THREADS + threadIdx.x; t < V; t += (long)gridDim.x * THREADS) count[t] = 0;
    if (blockIdx.x == 0 && threadIdx.x < 3) ((int32_t *)state)[threadIdx.x] = 0;
}

// How many positions every token has, and a number for every position among its token's.  A workgroup counts its own
// positions in a table in LDS first and asks once for each of its tokens: requests to one counter are served one by one,
// and a frequent token has hundreds (9.4 us for 65,536 tokens of which one in a hundred is the same, against 6).
constexpr int COUNT_THREADS = 1024, SLOTS = 2048;

__global__ __launch_bounds__(COUNT_THREADS) void grad_count_kernel(const int32_t *__restrict__ ids, long n, int V,
                                                                   int padding_id, int32_t *__restrict__ count,
                                                                   int32_t *__restrict__ rank)
{
    __shared__ int token[SLOTS], many[SLOTS];
    const long i = (long)blockIdx.x * COUNT_THREADS + threadIdx.x;
    const int id = i < n ? ids[i] : -1;
    const bool in = counts(id, V, padding_id);
    for (int k = threadIdx.x; k < SLOTS; k += COUNT_THREADS) token[k] = -1, many[k] = 0;
    __syncthreads();
    int slot = 0, place = 0;
    if (in) {
        slot = (int)((unsigned int)id * 2654435761u >> 21);
        for (;;) {   // (at most COUNT_THREADS of the SLOTS are ever taken)
            const int was = atomicCAS(&token[slot], -1, id);
            if (was == -1 || was == id) break;
            slot = (slot + 1) & (SLOTS - 1);
        }
        place = atomicAdd(&many[slot], 1);
    }
    __syncthreads();
    for (int k = threadIdx.x; k < SLOTS; k += COUNT_THREADS)
        if (many[k]) many[k] = atomicAdd(&count[token[k]], many[k]);
    __syncthreads();
    if (i < n) rank[i] = many[slot] + place;
}
static_assert(SLOTS == 1 << (32 - 21), "the hash's bits");

// Room for every token's list, one atomic a workgroup; the windows of long lists.
__global__ __launch_bounds__(ALLOC_THREADS) void grad_room_kernel(const int32_t *__restrict__ count, int V,
                                                                  int32_t *__restrict__ start, GradState *state,
                                                                  GradItem *__restrict__ items,
                                                                  GradJoin *__restrict__ joins)
{
    __shared__ int sums[ALLOC_THREADS / 64];
    __shared__ int base;
    const long t = (long)blockIdx.x * ALLOC_THREADS + threadIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int c = t < V ? count[t] : 0;
    const int upto = wave_inclusive_sum(c);
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < ALLOC_THREADS / 64; ++w) {
        before += w < wave ? sums[w] : 0;
        total += sums[w];
    }
    if (threadIdx.x == 0) base = total ? atomicAdd(&state->cursor, total) : 0;
    __syncthreads();
    if (t < V) start[t] = base + before + upto - c;
    // (one request a wavefront for its long lists)
    const int nw = c > SHORT ? windows_of(c) : 0;
    if (!__ballot(nw > 0)) return;
    const int upto_items = wave_inclusive_sum(nw);
    const unsigned long long joined = __ballot(nw > 1);
    int first_item = 0, first_join = 0;
    if (lane == 63) {
        first_item = atomicAdd(&state->items, upto_items);
        if (joined) first_join = atomicAdd(&state->joins, (int)__popcll(joined));
    }
    first_item = __builtin_amdgcn_readlane(first_item, 63) + upto_items - nw;
    first_join = __builtin_amdgcn_readlane(first_join, 63) + (int)__popcll(joined & ((1ull << lane) - 1ull));
    for (int w = 0; w < nw; ++w) items[first_item + w] = {(int32_t)t, w, nw, 0};
    if (nw > 1) joins[first_join] = {(int32_t)t, first_item, nw, 0};
}

__global__ __launch_bounds__(THREADS) void grad_place_kernel(const int32_t *__restrict__ ids, long n, int V,
                                                             int padding_id, const int32_t *__restrict__ start,
                                                             const int32_t *__restrict__ rank,
                                                             int32_t *__restrict__ list)
{
    const long i = (long)blockIdx.x * THREADS + threadIdx.x;
    if (i >= n) return;
    const int id = ids[i];
    if (counts(id, V, padding_id)) list[start[id] + rank[i]] = (int32_t)i;
}

// acc += row for rows list[from .. to): E columns from c on and, for C > 1, the same of the next C - 1 wavefronts' widths;
// four loads in flight (eight leave room for five wavefronts instead of eight, and were slower)
template <typename T, typename At, int C, int E>
__device__ inline void add_rows(const T *__restrict__ dout, long stride, int d, int c, int from, int to, At at,
                                float (&acc)[C][E])
{
    constexpr int ROWS = C >= 4 ? 1 : 4 / C;
    int e = from;
    for (; e + ROWS <= to; e += ROWS) {
        RowPiece<T, E> v[ROWS][C];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const T *const row = dout + (size_t)at(e + u) * stride;
#pragma unroll
            for (int k = 0; k < C; ++k) v[u][k].load(row, c + k * 64 * E, d);
        }
#pragma unroll
        for (int u = 0; u < ROWS; ++u)
#pragma unroll
            for (int k = 0; k < C; ++k) {
                float x[E];
                v[u][k].values(c + k * 64 * E, d, x);
#pragma unroll
                for (int j = 0; j < E; ++j) acc[k][j] += x[j];
            }
    }
    for (; e < to; ++e) {
        const T *const row = dout + (size_t)at(e) * stride;
        RowPiece<T, E> v[C];
#pragma unroll
        for (int k = 0; k < C; ++k) v[k].load(row, c + k * 64 * E, d);
#pragma unroll
        for (int k = 0; k < C; ++k) {
            float x[E];
            v[k].values(c + k * 64 * E, d, x);
#pragma unroll
            for (int j = 0; j < E; ++j) acc[k][j] += x[j];
        }
    }
}

// Rows of zeros, one behind the other from `first` on: those of `rows` that which(row) picks, 16 bytes a thread whatever row
// they belong to, so that narrow rows take no more stores than wide ones (a wavefront a row: 36 us for 250,000 rows of 100
// fp16, so 12).
template <int E, typename G, typename Which>
__device__ inline void zero_rows(G *first, int rows, int d, Which which, int thread, int threads)
{
    const int all = rows * d;
    for (int f = thread * E; f < all; f += threads * E) {
        const int u0 = f / d, u1 = (min(f + E, all) - 1) / d;
        if (u1 - u0 <= 1 && f + E <= all && which(u0) && which(u1)) {
            const float zero[E] = {};
            put_within(first, f, all, zero, true);
        } else {
            for (int j = 0; j < E && f + j < all; ++j)
                if (which((f + j) / d)) round_to(0.f, first[f + j]);
        }
    }
}

struct ItemRoom {
    union {
        int32_t few[SMALL_SORT];
        uint16_t many[SPAN];
        float part[3][ITEM_COLS];
    };
    int32_t sorted[SMALL_SORT];
    uint32_t bits[SPAN / 32];
    int32_t wave_sum[4];
    int32_t n;
};
static_assert(SPAN / 32 == THREADS, "a word of bits for every thread");
static_assert(SHORT == 16 && TOKENS == 16, "16 lanes for each of a wavefront's four tokens");

// One window of a long list: columns cols .. cols + 512 of the sum over the token's positions in [lo, hi).  These are found in
// the list, or among the ids of [lo, hi) where that is shorter: a list of c is cut into c / WINDOW windows, and looking
// through all of it in each of them goes with the square of c (4,194,304 positions of one token, d = 4: 160 ms, so 3).
template <typename T, typename G>
__device__ void grad_item(const T *__restrict__ dout, long stride, const int32_t *__restrict__ ids, long n, int d, float scale, const GradItem it,
                          int item, int cols, const int32_t *__restrict__ list, int count, ItemRoom &R,
                          float *__restrict__ partial, G *__restrict__ grad)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long width = (n + it.windows - 1) / it.windows;
    const long lo = it.window * width, hi = min(n, lo + width);
    const int c = cols + lane * 8;
    float acc[1][8] = {};
    if (threadIdx.x == 0) R.n = 0;
    __syncthreads();
    const bool shorter = hi - lo < count;
    const int entries = shorter ? (int)max(hi - lo, 0l) : count;
    for (int e = threadIdx.x; e < entries; e += THREADS) {
        const int p = shorter ? (int)lo + e : list[e];
        if (shorter ? ids[p] == it.token : p >= lo && p < hi) {
            const int k = atomicAdd(&R.n, 1);
            if (k < SMALL_SORT) R.few[k] = p;
        }
    }
    __syncthreads();
    const int m = R.n;
    if (m <= SMALL_SORT) {
        if ((int)threadIdx.x < m) {
            const int p = R.few[threadIdx.x];
            int r = 0;
            for (int e = 0; e < m; ++e) r += R.few[e] < p;
            R.sorted[r] = p;
        }
        __syncthreads();
        if (c < d) add_rows(dout, stride, d, c, m * wave / 4, m * (wave + 1) / 4, [&](int e) { return R.sorted[e]; }, acc);
    } else {
        for (long at = lo; at < hi; at += SPAN) {
            const long end = min(hi, at + SPAN);
            __syncthreads();
            R.bits[threadIdx.x] = 0;
            __syncthreads();
            if (end - at < count) {
                for (int e = threadIdx.x; e < (int)(end - at); e += THREADS)
                    if (ids[at + e] == it.token) atomicOr(&R.bits[e >> 5], 1u << (e & 31));
            } else {
                for (int e = threadIdx.x; e < count; e += THREADS) {
                    const int p = list[e];
                    if (p >= at && p < end) atomicOr(&R.bits[(p - at) >> 5], 1u << ((p - at) & 31));
                }
            }
            __syncthreads();
            // every thread lists the positions of its word, behind those of the words before
            const uint32_t word = R.bits[threadIdx.x];
            const int mine = __popc(word);
            const int upto = wave_inclusive_sum(mine);
            if (lane == 63) R.wave_sum[wave] = upto;
            __syncthreads();
            int k = upto - mine, total = 0;
            for (int w = 0; w < 4; ++w) {
                k += w < wave ? R.wave_sum[w] : 0;
                total += R.wave_sum[w];
            }
            for (uint32_t b = word; b; b &= b - 1) R.many[k++] = (uint16_t)(threadIdx.x * 32 + __ffs((int)b) - 1);
            __syncthreads();
            if (c < d)
                add_rows(dout, stride, d, c, total * wave / 4, total * (wave + 1) / 4,
                         [&](int e) { return at + R.many[e]; }, acc);
        }
    }
    __syncthreads();
    if (wave > 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) R.part[wave - 1][j * 64 + lane] = acc[0][j];
    }
    __syncthreads();
    if (wave == 0 && c < d) {
#pragma unroll
        for (int w = 0; w < 3; ++w)
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[0][j] += R.part[w][j * 64 + lane];
        if (it.windows == 1) {
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[0][j] *= scale;
            store8_within(grad + (size_t)it.token * d, c, d, acc[0]);
        } else {
            store8_within(partial + (size_t)item * d, c, d, acc[0]);
        }
    }
    __syncthreads();
}

// Workgroups 0 .. item_groups - 1 take the windows of long lists, so that these begin first; the others write the
// rows of TOKENS tokens each from `first` on, a wavefront a row: zeros, or the sum over its list, ordered by counting.
template <typename T, typename G>
__global__ __launch_bounds__(THREADS) void grad_rows_kernel(const T *__restrict__ dout, long stride,
                                                            const int32_t *__restrict__ ids, long n, int V, int d,
                                                            float scale, const int32_t *__restrict__ count,
                                                            const int32_t *__restrict__ start,
                                                            const int32_t *__restrict__ list,
                                                            const GradState *__restrict__ state,
                                                            const GradItem *__restrict__ items, int item_groups, long first,
                                                            float *__restrict__ partial, G *__restrict__ grad)
{
    __shared__ ItemRoom R;
    if ((int)blockIdx.x < item_groups) {
        const int cols = (d + ITEM_COLS - 1) / ITEM_COLS;
        const long total = (long)state->items * cols;
        for (long k = blockIdx.x; k < total; k += item_groups) {
            const int item = (int)(k / cols);
            const GradItem it = items[item];
            grad_item(dout, stride, ids, n, d, scale, it, item, (int)(k % cols) * ITEM_COLS, list + start[it.token],
                      count[it.token], R, partial, grad);
        }
        return;
    }
    constexpr int E = LANE_ELEMENTS<G>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // a wavefront's four tokens; their lists, 16 lanes each, in one load, and ordered by counting: a lane's place is the
    // number of smaller positions among its 16
    const long t0 = first + (long)(blockIdx.x - item_groups) * TOKENS + wave * (TOKENS / 4);
    const long mine = t0 + (lane >> 4);
    const int many = mine < V ? count[mine] : -1;
    const int at = lane & 15;
    // rows of zeros wait for nothing
    const unsigned long long none = __ballot(many == 0);
    if (none) zero_rows<E>(grad + (size_t)t0 * d, TOKENS / 4, d, [&](int u) { return (none >> (16 * u) & 1) != 0; }, lane, 64);
    const int p = at < many && many <= SHORT ? list[start[mine] + at] : 0x7fffffff;
    int place = 0;
#define VP_COUNT_SMALLER(k) place += __builtin_amdgcn_update_dpp(0, p, 0x120 + k, 0xf, 0xf, false) < p;   // row_ror:k
    VP_COUNT_SMALLER(1) VP_COUNT_SMALLER(2) VP_COUNT_SMALLER(3) VP_COUNT_SMALLER(4) VP_COUNT_SMALLER(5)
    VP_COUNT_SMALLER(6) VP_COUNT_SMALLER(7) VP_COUNT_SMALLER(8) VP_COUNT_SMALLER(9) VP_COUNT_SMALLER(10)
    VP_COUNT_SMALLER(11) VP_COUNT_SMALLER(12) VP_COUNT_SMALLER(13) VP_COUNT_SMALLER(14) VP_COUNT_SMALLER(15)
#undef VP_COUNT_SMALLER
    // (lanes without a position all count `many`, a place that none of the others has)
    const int ordered = __builtin_amdgcn_ds_permute(((lane & 48) + place) * 4, p);
    // narrow rows: the four at once, 16 lanes each (65,536 positions, 250,000 x 100 fp16: 71 us one after the other, 57 so)
    if (d <= 16 * E) {
        const int m = many > SHORT ? 0 : max(many, 0), c = at * E;
        const int most = max(max(__builtin_amdgcn_readlane(m, 0), __builtin_amdgcn_readlane(m, 16)),
                             max(__builtin_amdgcn_readlane(m, 32), __builtin_amdgcn_readlane(m, 48)));
        float acc[E] = {};
        for (int e = 0; e < most; ++e) {
            const int row = __builtin_amdgcn_ds_bpermute(((lane & 48) + e) * 4, ordered);
            if (e < m) {
                RowPiece<T, E> v;
                v.load(dout + (size_t)row * stride, c, d);
                float x[E];
                v.values(c, d, x);
#pragma unroll
                for (int j = 0; j < E; ++j) acc[j] += x[j];
            }
        }
        if (m > 0) {
#pragma unroll
            for (int j = 0; j < E; ++j) acc[j] *= scale;
            put_within(grad + (size_t)mine * d, c, d, acc, true);
        }
        return;
    }
    for (int u = 0; u < TOKENS / 4; ++u) {
        const int m = __builtin_amdgcn_readlane(many, u * 16);
        if (m <= 0 || m > SHORT) continue;
        G *const to = grad + (size_t)(t0 + u) * d;
        constexpr int C = 16 / E;   // 1,024 columns at a time
        for (int c0 = 0; c0 < d; c0 += C * 64 * E) {   // (every lane stays in the loop: the list is read across lanes)
            const int c = c0 + lane * E;
            float acc[C][E] = {};
            add_rows(dout, stride, d, c, 0, m, [&](int e) { return __builtin_amdgcn_readlane(ordered, u * 16 + e); }, acc);
#pragma unroll
            for (int k = 0; k < C; ++k) {
                if (c0 + k * 64 * E >= d) break;
#pragma unroll
                for (int j = 0; j < E; ++j) acc[k][j] *= scale;
                put_within(to, c + k * 64 * E, d, acc[k], true);
            }
        }
    }
}

// The rows of long lists of several windows: their sums in order.
template <typename G>
__global__ __launch_bounds__(THREADS) void grad_join_kernel(int d, float scale, const GradState *__restrict__ state,
                                                            const GradJoin *__restrict__ joins,
                                                            const float *__restrict__ partial, G *__restrict__ grad)
{
    const int total = state->joins;
    for (int k = blockIdx.x; k < total; k += gridDim.x) {
        const GradJoin jn = joins[k];
        for (int c = blockIdx.y * THREADS + threadIdx.x; c < d; c += gridDim.y * THREADS) {
            float acc = 0.f;
#pragma unroll 4
            for (int w = 0; w < jn.windows; ++w) acc += partial[(size_t)(jn.first + w) * d + c];
            round_to(acc * scale, grad[(size_t)jn.token * d + c]);
        }
    }
}

// ---------------------------------------------------------------- few positions
// Up to FEW positions: no lists in memory.  A workgroup takes TAKEN tokens and one wavefront's width of columns, looks
// through all ids for its tokens' positions, in order, and writes its rows: one launch instead of six (a call of 500
// rows, 5,000 x 256: 9 us against 24).  Lists longer than TOGETHER are summed by all four wavefronts, a quarter each.
constexpr int FEW = 1024, TOGETHER = 32;

template <int TAKEN, typename T, typename G>
__global__ __launch_bounds__(THREADS) void grad_few_kernel(const T *__restrict__ dout, long stride,
                                                           const int32_t *__restrict__ ids, int n, int V, int d,
                                                           float scale, int padding_id, int first, G *__restrict__ grad)
{
    constexpr int E = LANE_ELEMENTS<G>, PER = FEW / THREADS;
    __shared__ uint32_t list[FEW];               // (token - t0) * 2^16 + position, ascending positions
    __shared__ uint16_t mine[WAVES][FEW];        // a wavefront's own: one token's positions
    __shared__ int many[TAKEN], sums[WAVES];
    __shared__ float part[WAVES - 1][64 * E];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t0 = first + (int)blockIdx.x * TAKEN, c = blockIdx.y * 64 * E + lane * E;
    if (threadIdx.x < TAKEN) many[threadIdx.x] = 0;
    int id[PER], found = 0;
#pragma unroll
    for (int u = 0; u < PER; ++u) {
        const int i = threadIdx.x * PER + u;
        id[u] = i < n ? ids[i] : -1;
        if (!counts(id[u], V, padding_id) || id[u] < t0 || id[u] - t0 >= TAKEN) id[u] = -1;
        found += id[u] >= 0;
    }
    const int upto = wave_inclusive_sum(found);
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int at = upto - found, total = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        at += w < wave ? sums[w] : 0;
        total += sums[w];
    }
#pragma unroll
    for (int u = 0; u < PER; ++u)
        if (id[u] >= 0) {
            list[at++] = (uint32_t)(id[u] - t0) << 16 | (uint32_t)(threadIdx.x * PER + u);
            atomicAdd(&many[id[u] - t0], 1);
        }
    __syncthreads();
    // token u's positions in order into this wavefront's list
    auto collect = [&](int u) {
        int k = 0;
        for (int e0 = 0; e0 < total; e0 += 64) {
            const uint32_t entry = e0 + lane < total ? list[e0 + lane] : 0xffffffffu;
            const bool is = (int)(entry >> 16) == u;
            const unsigned long long all = __ballot(is);
            if (is) mine[wave][k + (int)__popcll(all & ((1ull << lane) - 1ull))] = (uint16_t)entry;
            k += (int)__popcll(all);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    const auto position = [&](int e) { return mine[wave][e]; };
    const bool narrow = d <= 32 * E;     // (one width of columns then: the workgroup has its rows whole)
    if (narrow) {
        zero_rows<E>(grad + (size_t)t0 * d, min(TAKEN, V - t0), d, [&](int u) { return many[u] == 0; }, threadIdx.x, THREADS);
    }
    // tokens by 64: every fourth is this wavefront's, those of long lists all wavefronts'
    constexpr unsigned long long FOURTH = 0x1111111111111111ull;
    for (int h = 0; h < TAKEN; h += 64) {
        const int of = h + lane < min(TAKEN, V - t0) ? many[(h + lane) & (TAKEN - 1)] : -1;
        unsigned long long some = __ballot(of > 0 && of <= TOGETHER) & FOURTH << wave, none = narrow ? 0 : __ballot(of == 0) & FOURTH << wave;
        for (; none; none &= none - 1) {
            const float zero[E] = {};
            if (c < d) put_within(grad + (size_t)(t0 + h + __ffsll((long long)none) - 1) * d, c, d, zero, true);
        }
        for (; some; some &= some - 1) {
            const int u = h + __ffsll((long long)some) - 1;
            collect(u);
            float acc[1][E] = {};
            if (c >= d) continue;
            add_rows(dout, stride, d, c, 0, many[u], position, acc);
#pragma unroll
            for (int j = 0; j < E; ++j) acc[0][j] *= scale;
            put_within(grad + (size_t)(t0 + u) * d, c, d, acc[0], true);
        }
    }
    for (int h = 0; h < TAKEN; h += 64) {
        const int of = h + lane < TAKEN ? many[(h + lane) & (TAKEN - 1)] : 0;
        for (unsigned long long all = __ballot(of > TOGETHER); all; all &= all - 1) {
            const int u = h + __ffsll((long long)all) - 1, m = many[u];
            collect(u);
            float acc[1][E] = {};
            if (c < d) add_rows(dout, stride, d, c, m * wave / WAVES, m * (wave + 1) / WAVES, position, acc);
            if (wave > 0) {
#pragma unroll
                for (int j = 0; j < E; ++j) part[wave - 1][j * 64 + lane] = acc[0][j];
            }
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int w = 0; w < WAVES - 1; ++w)
#pragma unroll
                    for (int j = 0; j < E; ++j) acc[0][j] += part[w][j * 64 + lane];
#pragma unroll
                for (int j = 0; j < E; ++j) acc[0][j] *= scale;
                if (c < d) put_within(grad + (size_t)(t0 + u) * d, c, d, acc[0], true);
            }
            __syncthreads();
        }
    }
}

struct GradLayout {
    size_t state, count, start, rank, list, items, joins, partial, total;
    long max_items, max_joins;
};

void grad_layout(int64_t n, int V, int d, GradLayout *L)
{
    if (n <= FEW) n = 0;      // (no lists in memory)
    // windows: sum of ceil(c / WINDOW) over lists with c > SHORT
    L->max_joins = n / (WINDOW + 1);
    L->max_items = n / WINDOW + n / (SHORT + 1);
    size_t o = 0;
    auto take = [&](size_t bytes) { size_t at = o; o += layer_align_up(bytes); return at; };
    L->state = take(sizeof(GradState));
    L->count = take((size_t)V * 4);
    L->start = take((size_t)V * 4);
    L->rank = take((size_t)n * 4);
    L->list = take((size_t)n * 4);
    L->items = take((size_t)L->max_items * sizeof(GradItem));
    L->joins = take((size_t)L->max_joins * sizeof(GradJoin));
    L->partial = take((size_t)L->max_items * d * 4);
    L->total = o;
}

vp_status embed_sizes(const char *fn, int64_t n, int32_t V, int32_t d)
{
    if (d < 1 || d > VP_MAX_DIM) return (vp_status)vpi_fail(VP_ERR_UNSUPPORTED, "%s: d = %d: need 1 <= d <= %d", fn, d, VP_MAX_DIM);
    if (V < 1 || V >= (1ll << 31) - 16) return (vp_status)vpi_fail(VP_ERR_UNSUPPORTED, "%s: V = %d out of range", fn, V);
    if (n < 0 || n >= (1ll << 31) - 65536) return (vp_status)vpi_fail(VP_ERR_UNSUPPORTED, "%s: n = %lld out of range", fn, (long long)n);
    return VP_OK;
}

}  // namespace

extern "C" {

vp_status vp_embed(const void *table, int32_t table_type, int64_t table_stride, int32_t V, int32_t d,
                   const int32_t *ids, int64_t n, float scale, void *out, int32_t out_type, void *hip_stream)
{
    const vp_status s = embed_sizes("vp_embed", n, V, d);
    if (s != VP_OK) return s;
    if (!type_known(table_type) || !type_known(out_type)) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_embed: unknown type %d or %d", table_type, out_type);
    if (table_stride < d) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_embed: rows of %d at a stride of %lld", d, (long long)table_stride);
    if (n == 0) return VP_OK;
    if (!table || !ids || !out) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_embed: null pointer argument");
    if (!layer_aligned(table, type_size(table_type)) || !layer_aligned(ids, 4) || !layer_aligned(out, type_size(out_type)))
        return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_embed: an address that is no multiple of its element's size");
    int row_threads = 4;
    while (row_threads < THREADS && row_threads * (int)(16 / type_size(out_type)) < d) row_threads *= 2;
    const long most = LAUNCH_THREADS / row_threads;
    const bool stream = n * d * (long)type_size(out_type) > STREAM_BYTES;
    with_type(table_type, [&](auto t) {
        with_type(out_type, [&](auto o) {
            for (long at = 0; at < n; at += most) {
                const long rows = std::min<long>(most, n - at);
                hipLaunchKernelGGL((embed_kernel<decltype(t), decltype(o)>), dim3((unsigned int)layer_ceil_div(rows, THREADS / row_threads)), dim3(THREADS), 0,
                                   (hipStream_t)hip_stream, (const decltype(t) *)table, (long)table_stride, V, d, ids + at, rows, scale, row_threads, stream,
                                   (decltype(o) *)out + at * d);
            }
        });
    });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (vp_status)vpi_fail(VP_ERR_HIP, "vp_embed: %s", hipGetErrorString(e));
    return VP_OK;
}

size_t vp_embed_grad_workspace_bytes(int64_t n, int32_t V, int32_t d)
{
    if (embed_sizes("vp_embed_grad", n, V, d) != VP_OK) return 0;
    GradLayout L;
    grad_layout(n, V, d, &L);
    return L.total;
}

vp_status vp_embed_grad(const void *dout, int32_t dout_type, int64_t dout_stride, const int32_t *ids, int64_t n,
                        int32_t V, int32_t d, float scale, int32_t padding_id, void *grad, int32_t grad_type,
                        void *workspace, size_t workspace_bytes, void *hip_stream)
{
    const vp_status s = embed_sizes("vp_embed_grad", n, V, d);
    if (s != VP_OK) return s;
    if (!type_known(dout_type) || !type_known(grad_type)) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_embed_grad: unknown type %d or %d", dout_type, grad_type);
    if (dout_stride < d) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_embed_grad: rows of %d at a stride of %lld", d, (long long)dout_stride);
    if ((n > 0 && (!dout || !ids)) || !grad || !workspace) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_embed_grad: null pointer argument");
    if (!layer_aligned(dout, type_size(dout_type)) || !layer_aligned(ids, 4) || !layer_aligned(grad, type_size(grad_type)))
        return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "vp_embed_grad: an address that is no multiple of its element's size");
    if (!layer_aligned(workspace, LAYER_ALIGN)) return (vp_status)vpi_fail(VP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
    GradLayout L;
    grad_layout(n, V, d, &L);
    if (workspace_bytes < L.total) return (vp_status)vpi_fail(VP_ERR_WORKSPACE, "workspace of %zu bytes, %zu needed", workspace_bytes, L.total);
    const hipStream_t st = (hipStream_t)hip_stream;
    if (n <= FEW) {
        auto launch = [&](auto taken) {
            constexpr int TAKEN = decltype(taken)::value;
            constexpr long most = LAUNCH_THREADS / THREADS;      // workgroups of a launch
            for (long at = 0; at < layer_ceil_div(V, TAKEN); at += most) {
                const dim3 grid((unsigned int)std::min<long>(most, layer_ceil_div(V, TAKEN) - at), (unsigned int)layer_ceil_div(d, 64 * (16 / type_size(grad_type))));
                with_type(dout_type, [&](auto t) {
                    with_type(grad_type, [&](auto g) {
                        hipLaunchKernelGGL((grad_few_kernel<TAKEN, decltype(t), decltype(g)>), grid, dim3(THREADS), 0, st, (const decltype(t) *)dout,
                                           (long)dout_stride, ids, (int)n, V, d, scale, padding_id, (int)(at * TAKEN), (decltype(g) *)grad);
                    });
                });
            }
        };
        // (every workgroup looks through all ids: 500 positions in 250,000 tokens of 24 take 24 us with 32 tokens to a workgroup)
        if (V <= 32768) launch(std::integral_constant<int, 32>{});
        else launch(std::integral_constant<int, 128>{});
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (vp_status)vpi_fail(VP_ERR_HIP, "vp_embed_grad: %s", hipGetErrorString(e));
        return VP_OK;
    }
    char *const ws = (char *)workspace;
    GradState *const state = (GradState *)(ws + L.state);
    int32_t *const count = (int32_t *)(ws + L.count), *const start = (int32_t *)(ws + L.start);
    int32_t *const rank = (int32_t *)(ws + L.rank), *const list = (int32_t *)(ws + L.list);
    GradItem *const items = (GradItem *)(ws + L.items);
    GradJoin *const joins = (GradJoin *)(ws + L.joins);
    float *const partial = (float *)(ws + L.partial);
    hipLaunchKernelGGL(grad_clear_kernel, dim3((unsigned int)std::min<long>(1024, layer_ceil_div(V, THREADS))), dim3(THREADS), 0, st, count, V, state);
    {
        const dim3 grid((unsigned int)layer_ceil_div(n, THREADS));
        hipLaunchKernelGGL(grad_count_kernel, dim3((unsigned int)layer_ceil_div(n, COUNT_THREADS)), dim3(COUNT_THREADS), 0, st, ids, (long)n, V, padding_id, count, rank);
        hipLaunchKernelGGL(grad_room_kernel, dim3((unsigned int)layer_ceil_div(V, ALLOC_THREADS)), dim3(ALLOC_THREADS), 0, st, count, V, start, state, items, joins);
        hipLaunchKernelGGL(grad_place_kernel, grid, dim3(THREADS), 0, st, ids, (long)n, V, padding_id, start, rank, list);
    }
    const int cols = (d + ITEM_COLS - 1) / ITEM_COLS;
    const int item_groups = (int)std::min<long>(MAX_ITEM_GROUPS, L.max_items * cols);
    constexpr long most = LAUNCH_THREADS / THREADS;
    for (long at = 0; at < layer_ceil_div(V, TOKENS); at += most) {
        const int windows = at == 0 ? item_groups : 0;
        const dim3 grid((unsigned int)(windows + std::min<long>(most, layer_ceil_div(V, TOKENS) - at)));
        with_type(dout_type, [&](auto t) {
            with_type(grad_type, [&](auto g) {
                hipLaunchKernelGGL((grad_rows_kernel<decltype(t), decltype(g)>), grid, dim3(THREADS), 0, st,
                                   (const decltype(t) *)dout, (long)dout_stride, ids, (long)n, V, d, scale, count, start, list,
                                   state, items, windows, at * TOKENS, partial, (decltype(g) *)grad);
            });
        });
    }
    if (L.max_joins > 0)
        with_type(grad_type, [&](auto g) {
            hipLaunchKernelGGL((grad_join_kernel<decltype(g)>), dim3((unsigned int)std::min<long>(256, L.max_joins), (unsigned int)layer_ceil_div(d, THREADS)),
                               dim3(THREADS), 0, st, d, scale, state, joins, partial, (decltype(g) *)grad);
        });
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return (vp_status)vpi_fail(VP_ERR_HIP, "vp_embed_grad: %s", hipGetErrorString(e));
    return VP_OK;
}

}  // extern "C"
