// Rows of features along the grouping of slots by transit: into the order of the groups, back to the samples with
// weights, summed per group, and the gradient of the weights.  Slot q belongs to row q / m, as the slots of a k-hop
// step belong to their parents.
//
//     by transit    out[p] = w[q] x[q / m],                 q = sorted_slots[p]
//     to samples    out[r] = sum_j w[r m + j] z[index[r m + j]]
//     weight grad   dw[r m + j] = dy[r] . z[index[r m + j]]
//     group sum     out[u] = sum over group u's pairs of w[q] x[q / m]
//
// Every one is bound by the rows it moves.  A lane holds 16 bytes of a row and the lanes of a workgroup are dealt out
// over (row, piece) without gaps, so that rows of any length use all lanes; a row's last piece reaches back over the one
// before it where the length is no multiple of a piece (both write the same numbers), and rows shorter than a piece go
// number by number.  Sums are 32-bit, in an order that sizes alone decide; no atomics.
//
// 16,385 rows of 1,024 bf16 with four slots each, 134 MB of slots' rows: there 37 us, back 36, weight grad 34, 4.5 to 4.9 TB/s
// with the rows they belong to, where a copy reaches 5.5.  Rows out of a table are bound by its lines: 233,000 rows of 25 slots
// x 128 bf16, 1.49 GB in pieces of 256 bytes out of 60 MB, 193 us where few rows are met often (7.7 TB/s, part of it from L2),
// and 327 for the sums per group, whose rows are met equally often (4.6 TB/s from the last-level cache).
#include <type_traits>

#include "nd_philox.h"
#include "nd_rows.h"
#include "nd_wave.h"

namespace nd {
namespace {

constexpr int kThreads = 256;

// A workgroup's lanes over rows and pieces: lane -> (row within the workgroup, piece of it).
struct Deal {
    FastDiv pieces;       // pieces of a row that one workgroup holds (at most kThreads)
    uint32_t all_pieces;  // pieces of a row
    uint32_t rows;        // rows of a workgroup
    uint32_t lanes;       // rows * pieces
};
inline Deal make_deal(int32_t d, int vec, uint32_t threads = kThreads) {
    Deal t;
    t.all_pieces = (uint32_t)((d + vec - 1) / vec);
    const uint32_t most = threads < kThreads ? threads : kThreads;
    const uint32_t here = t.all_pieces < most ? t.all_pieces : most;
    t.pieces = make_fastdiv(here);
    t.rows = threads / here;
    t.lanes = t.rows * here;
    return t;
}
// A launch holds fewer than 2^32 lanes, so workgroups go on to further rows from here on.
constexpr int64_t kMaxGroups = 1 << 20;
inline unsigned workgroups(int64_t n) { return (unsigned)(n < kMaxGroups ? n : kMaxGroups); }
inline unsigned deal_threads(const Deal& t) { return (t.lanes + 63u) / 64u * 64u; }
inline unsigned deal_columns(const Deal& t) { return (t.all_pieces + t.pieces.d - 1) / t.pieces.d; }

// Where this lane's piece starts; false where the lane has none.
template <int VEC>
__device__ __forceinline__ bool deal_lane(const Deal& t, int32_t d, uint32_t* row, int32_t* at) {
    *row = fastdiv(threadIdx.x, t.pieces);
    const uint32_t piece = blockIdx.y * t.pieces.d + (threadIdx.x - *row * t.pieces.d);
    const int32_t start = (int32_t)piece * VEC;
    *at = start + VEC <= d ? start : d - VEC;
    return threadIdx.x < t.lanes && piece < t.all_pieces;
}

// Live pairs: all of them, or as many as the grouping found.
__device__ __forceinline__ int64_t live(int64_t all, const int64_t* counts, int which) {
    if (!counts) return all;
    const int64_t c = counts[which];
    return c < all ? (c > 0 ? c : 0) : all;
}

__global__ __launch_bounds__(kThreads) void positions_clear_kernel(int32_t* __restrict__ position, int64_t n_slots) {
    const int64_t q = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (q < n_slots) position[q] = -1;
}
__global__ __launch_bounds__(kThreads) void positions_kernel(const int32_t* __restrict__ slots, int64_t n_pairs,
                                                             const int64_t* __restrict__ counts, int64_t n_slots,
                                                             int32_t* __restrict__ position) {
    const int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (p >= live(n_pairs, counts, 0)) return;
    const uint32_t q = (uint32_t)slots[p];
    if (q < n_slots) position[q] = (int32_t)p;
}

template <typename T, int VEC, int ROUNDS>
__global__ __launch_bounds__(kThreads) void by_transit_kernel(const T* __restrict__ x, int64_t x_stride, int32_t d, Deal t,
                                                              const int32_t* __restrict__ slots, int64_t n_pairs,
                                                              const int64_t* __restrict__ counts, FastDiv m,
                                                              uint32_t n_slots, const float* __restrict__ weights,
                                                              T* __restrict__ out, int64_t out_stride) {
    uint32_t row;
    int32_t at;
    if (!deal_lane<VEC>(t, d, &row, &at)) return;
    const int64_t pairs = live(n_pairs, counts, 0);
    for (int64_t p0 = (int64_t)blockIdx.x * (ROUNDS * t.rows) + row; p0 < pairs; p0 += (int64_t)gridDim.x * (ROUNDS * t.rows)) {
        uint32_t q[ROUNDS];
        Piece<T, VEC> v[ROUNDS];
        float w[ROUNDS];
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            const int64_t p = p0 + (int64_t)i * t.rows;
            q[i] = p < pairs ? (uint32_t)slots[p] : ~0u;
        }
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            v[i] = Piece<T, VEC>{};
            w[i] = 1.f;
            if (q[i] < n_slots) {
                v[i] = load_piece<T, VEC>(x + (int64_t)fastdiv(q[i], m) * x_stride + at);
                if (weights) w[i] = weights[q[i]];
            }
        }
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i) {
            const int64_t p = p0 + (int64_t)i * t.rows;
            if (p >= pairs) break;
            if (weights && q[i] < n_slots) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[i].v[e] = (T)((float)v[i].v[e] * w[i]);
            }
            store_piece<T, VEC>(out + p * out_stride + at, v[i]);
        }
    }
}

// A lane adds up its piece of every `step`-th slot's row from `first` on, four loads under way at a time (eight or sixteen take
// registers from wavefronts: 199 and 253 us where four take 194, 233,000 rows of 25 slots x 128 bf16).
constexpr int kAhead = 4;
template <typename T, int VEC>
__device__ __forceinline__ void add_slots(const T* __restrict__ z, int64_t z_stride, uint32_t n_z, const int32_t* idx,
                                          const float* w, int32_t first, int32_t m, int32_t step, int32_t at,
                                          float (&sum)[VEC]) {
    for (int32_t j0 = first; j0 < m; j0 += kAhead * step) {
        uint32_t place[kAhead];
        Piece<T, VEC> v[kAhead];
        float f[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) place[i] = j0 + i * step < m ? (uint32_t)idx[j0 + i * step] : ~0u;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            v[i] = Piece<T, VEC>{};
            f[i] = 0.f;
            if (place[i] < n_z) {
                v[i] = load_piece<T, VEC>(z + (int64_t)place[i] * z_stride + at);
                f[i] = w ? w[j0 + i * step] : 1.f;
            }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[e] = fmaf(f[i], (float)v[i].v[e], sum[e]);
    }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_sum(T* __restrict__ to, const float (&sum)[VEC]) {
    Piece<T, VEC> o;
#pragma unroll
    for (int e = 0; e < VEC; ++e) o.v[e] = (T)sum[e];
    store_piece<T, VEC>(to, o);
}

template <typename T, int VEC>
__global__ __launch_bounds__(kThreads) void to_samples_kernel(const T* __restrict__ z, int64_t z_stride, uint32_t n_z, int32_t d,
                                                              Deal t, const int32_t* __restrict__ index, int64_t n, int32_t m,
                                                              const float* __restrict__ weights, T* __restrict__ out,
                                                              int64_t out_stride) {
    uint32_t row;
    int32_t at;
    if (!deal_lane<VEC>(t, d, &row, &at)) return;
    for (int64_t r = (int64_t)blockIdx.x * t.rows + row; r < n; r += (int64_t)gridDim.x * t.rows) {
        float sum[VEC] = {};
        add_slots<T, VEC>(z, z_stride, n_z, index + r * m, weights ? weights + r * m : nullptr, 0, m, 1, at, sum);
        store_sum<T, VEC>(out + r * out_stride + at, sum);
    }
}

// Few rows: the slots of one are shared out over the rows of a workgroup's lanes and joined in their order.
constexpr uint32_t kShareThreads = 1024;
template <typename T, int VEC>
__global__ __launch_bounds__(kShareThreads) void to_samples_share_kernel(const T* __restrict__ z, int64_t z_stride, uint32_t n_z,
                                                                         int32_t d, Deal t, const int32_t* __restrict__ index,
                                                                         int32_t m, const float* __restrict__ weights,
                                                                         T* __restrict__ out, int64_t out_stride) {
    extern __shared__ float shared_sums[];
    uint32_t row;
    int32_t at;
    const bool mine = deal_lane<VEC>(t, d, &row, &at);
    const int64_t r = blockIdx.x;
    float sum[VEC] = {};
    if (mine)
        add_slots<T, VEC>(z, z_stride, n_z, index + r * m, weights ? weights + r * m : nullptr, (int32_t)row, m, (int32_t)t.rows,
                          at, sum);
#pragma unroll
    for (int e = 0; e < VEC; ++e) shared_sums[threadIdx.x * VEC + e] = sum[e];
    __syncthreads();
    if (!mine || row != 0) return;
    for (uint32_t k = 1; k < t.rows; ++k)
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[e] += shared_sums[(threadIdx.x + k * t.pieces.d) * VEC + e];
    store_sum<T, VEC>(out + r * out_stride + at, sum);
}

// Of HELD sums over lanes the upper half of the lanes goes on with the upper half, the lower with the others; *first: the
// first of what a lane goes on with.
template <int HELD, int N>
__device__ __forceinline__ void fold(float (&dot)[N], int lane, int* s, int* first) {
    if constexpr (HELD > 1) {
        const bool upper = lane & *s;
#pragma unroll
        for (int i = 0; i < HELD / 2; ++i) {
            const float keep = upper ? dot[HELD / 2 + i] : dot[i], give = upper ? dot[i] : dot[HELD / 2 + i];
            dot[i] = keep + __shfl_xor(give, *s);
        }
        if (upper) *first += HELD / 2;
        *s >>= 1;
        fold<HELD / 2>(dot, lane, s, first);
    }
}

// 2^log_lanes lanes of a wavefront share the dot products of one row with SLOTS of its slots' rows, whose pieces are under
// way together (four: 231 us for 233,000 rows of 25 slots x 128 bf16; eight 288).  In the first steps of the sum over the
// lanes, half of them go on with half of the products each.
template <typename T, int VEC, int SLOTS>
__global__ __launch_bounds__(kThreads) void weight_grad_kernel(const T* __restrict__ dy, int64_t dy_stride,
                                                               const T* __restrict__ z, int64_t z_stride, uint32_t n_z,
                                                               int32_t d, const int32_t* __restrict__ index, int64_t n,
                                                               int32_t m, FastDiv shares, int log_lanes,
                                                               float* __restrict__ dweights) {
    const int lanes = 1 << log_lanes, lane = threadIdx.x & (lanes - 1);
    const int64_t per = kThreads >> log_lanes, items = n * shares.d;
    for (int64_t i0 = (int64_t)blockIdx.x * per; i0 < items; i0 += (int64_t)gridDim.x * per) {
        const int64_t item = i0 + (threadIdx.x >> log_lanes);
        const bool mine = item < items;
        const int64_t r = mine ? fastdiv((uint32_t)item, shares) : 0;
        const int32_t j0 = (int32_t)(item - r * shares.d) * SLOTS;
        uint32_t place[SLOTS];
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) place[i] = mine && j0 + i < m ? (uint32_t)index[r * m + j0 + i] : ~0u;
        float dot[SLOTS] = {};
        for (int32_t c = lane * VEC; mine && c < d; c += lanes * VEC) {
            const int32_t at = c + VEC <= d ? c : d - VEC;
            const Piece<T, VEC> a = load_piece<T, VEC>(dy + r * dy_stride + at);
            Piece<T, VEC> b[SLOTS];
#pragma unroll
            for (int i = 0; i < SLOTS; ++i) {
                b[i] = Piece<T, VEC>{};
                if (place[i] < n_z) b[i] = load_piece<T, VEC>(z + (int64_t)place[i] * z_stride + at);
            }
            if (c == at) {
#pragma unroll
                for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) dot[i] = fmaf((float)a.v[e], (float)b[i].v[e], dot[i]);
            } else {  // the last piece reaches back; what was counted is skipped
#pragma unroll
                for (int i = 0; i < SLOTS; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (e >= c - at) dot[i] = fmaf((float)a.v[e], (float)b[i].v[e], dot[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < SLOTS; ++i)
            if (place[i] >= n_z) dot[i] = 0.f;  // also where dy is infinite or no number
        int s = lanes >> 1, first = 0;
        fold<SLOTS>(dot, lane, &s, &first);
        const int rest = (s << 1) - 1;  // lanes that hold parts of the same product
        for (; s > 0; s >>= 1) dot[0] += __shfl_xor(dot[0], s);
        if (mine && (rest <= 0 || (lane & rest) == 0) && j0 + first < m) dweights[r * m + j0 + first] = dot[0];
    }
}

// ------------------------------------------------------------------------------------------------- sums per group
// Pairs are cut into tiles of equal length, whatever the groups: a hub's pairs are spread over as many workgroups as
// they fill tiles.  A group inside one tile is summed there; of one that crosses tiles every tile leaves what it holds
// (32-bit floats: `first` if the group began before the tile, `last` otherwise), and a second launch adds those up.
__device__ __forceinline__ int64_t live_groups(const GroupSum& g) {
    return g.ctl ? (int64_t)g.ctl->U : live(g.n_groups, g.counts, 1);
}
__device__ __forceinline__ int64_t start_of(const GroupSum& g, int64_t u, int64_t pairs) {
    const int64_t s = g.start[u];
    return s < 0 ? 0 : (s < pairs ? s : pairs);
}
// Live pairs that are in a group.
__device__ __forceinline__ int64_t grouped_pairs(const GroupSum& g, int64_t groups) {
    const int64_t pairs = g.ctl ? (int64_t)g.ctl->P : live(g.n_pairs, g.counts, 0);
    return groups > 0 ? start_of(g, groups, pairs) : 0;
}
// Row of the output that group u's sum goes to, or -1.
__device__ __forceinline__ int64_t row_of_group(const GroupSum& g, int64_t u) {
    if (!g.group_row) return u;
    const int64_t r = g.group_row[u];
    return r >= 0 && r < g.out_rows ? r : -1;
}

// Which group the first pair in a tile that is in one belongs to: the tile's first pair, or, where the offsets begin behind it,
// the first group's.  Tiles in front of that are not marked, and not read.
__device__ __forceinline__ void mark_tiles(const GroupSum& g, int64_t groups, int64_t pairs, int64_t u) {
    int64_t first = 0, last = -1;  // the group's tiles
    if (u < groups) {
        const int64_t a = start_of(g, u, pairs), b = start_of(g, u + 1, pairs);
        if (b > a) {
            first = a > start_of(g, 0, pairs) ? (a + g.tile - 1) / g.tile : a / g.tile;
            last = (b - 1) / g.tile;
        }
    }
    if (g.mark && u < groups) g.mark[g.mark_key[u]] = (int32_t)u;
    // few: every lane its own; many (a hub): the wavefront together
    uint64_t many = __ballot(last - first >= 8);
    if (last - first < 8)
        for (int64_t t = first; t <= last; ++t) g.tile_group[t] = (int32_t)u;
    while (many) {
        const int from = __ffsll((unsigned long long)many) - 1;
        many &= many - 1;
        const int64_t a = __shfl(first, from), b = __shfl(last, from), v = __shfl(u, from);
        for (int64_t t = a + lane_id(); t <= b; t += kWave) g.tile_group[t] = (int32_t)v;
    }
}

// Rows that no group names are zero: a workgroup marks the named ones of 256 rows and clears the others.
template <typename T, int VEC>
__device__ __forceinline__ void clear_rows(const GroupSum& g, int64_t groups, int64_t pairs, int32_t d, const Deal& t,
                                           int64_t r0, T* __restrict__ out) {
    __shared__ uint32_t named[kThreads];
    const int64_t r1 = r0 + kThreads < g.out_rows ? r0 + kThreads : g.out_rows;
    int64_t lo = 0, hi = groups;  // first group with a row of r0 or more; every lane looks at one place at a time
    while (lo < hi) {
        const int64_t step = (hi - lo + kThreads - 1) / kThreads, at = lo + threadIdx.x * step;
        const int64_t less = __syncthreads_count(at < hi && (int64_t)g.group_row[at] < r0);
        hi = lo + less * step < hi ? lo + less * step : hi;
        if (less > 0) lo += (less - 1) * step + 1;
    }
    named[threadIdx.x] = 0;
    __syncthreads();
    // rows ascend, so that at most as many groups as rows follow
    const int64_t u = lo + threadIdx.x;
    if (u < groups) {
        const int64_t r = g.group_row[u];
        const bool holds = start_of(g, u + 1, pairs) > start_of(g, u, pairs);
        if (r >= r0 && r < r1 && holds) named[r - r0] = 1;
    }
    __syncthreads();
    const uint32_t row = fastdiv(threadIdx.x, t.pieces);
    if (threadIdx.x >= t.lanes) return;
    for (uint32_t c = threadIdx.x - row * t.pieces.d; c < t.all_pieces; c += t.pieces.d) {
        const int32_t at = (int32_t)(c + 1) * VEC <= d ? (int32_t)c * VEC : d - VEC;
        for (int64_t r = r0 + row; r < r1; r += t.rows)
            if (!named[r - r0]) store_piece<T, VEC>(out + r * g.out_stride + at, Piece<T, VEC>{});
    }
}

// The first `tile_blocks` workgroups do the one, the others the other.
template <typename T, int VEC>
__global__ __launch_bounds__(kThreads) void group_tiles_kernel(int32_t d, Deal t, GroupSum g, int64_t tile_blocks,
                                                               T* __restrict__ out) {
    const int64_t groups = live_groups(g), pairs = grouped_pairs(g, groups);
    if (blockIdx.x < tile_blocks)
        mark_tiles(g, groups, pairs, (int64_t)blockIdx.x * kThreads + threadIdx.x);
    else
        clear_rows<T, VEC>(g, groups, pairs, d, t, (blockIdx.x - tile_blocks) * kThreads, out);
}

template <typename T, typename O, int VEC>
__global__ __launch_bounds__(kThreads) void group_sum_kernel(const T* __restrict__ x, int64_t x_stride, int32_t d, Deal t,
                                                             FastDiv m, uint32_t n_slots,
                                                             const float* __restrict__ weights, GroupSum g,
                                                             O* __restrict__ out) {
    uint32_t row;
    int32_t at;
    if (!deal_lane<VEC>(t, d, &row, &at)) return;
    const uint32_t groups = (uint32_t)live_groups(g), pairs = (uint32_t)grouped_pairs(g, groups);
    const uint32_t first_pair = groups > 0 ? (uint32_t)start_of(g, 0, pairs) : 0;  // those before it are in no group
    for (int64_t tile = (int64_t)blockIdx.x * t.rows + row; tile * g.tile < pairs; tile += (int64_t)gridDim.x * t.rows) {
        const uint32_t tile_first = (uint32_t)(tile * g.tile);
        const uint32_t p1 = pairs - tile_first < (uint32_t)g.tile ? pairs : tile_first + g.tile;
        if (p1 <= first_pair) continue;
        const uint32_t p0 = tile_first < first_pair ? first_pair : tile_first;
        uint32_t u = (uint32_t)g.tile_group[tile];
        if (u >= groups) u = groups - 1;
        bool before = start_of(g, u, pairs) < p0;
        // of this group and the next, so that no group waits for where it ends
        uint32_t end = (uint32_t)start_of(g, u + 1, pairs), next = u + 1 < groups ? u + 1 : u,
                 next_end = (uint32_t)start_of(g, next + 1, pairs);
        int64_t to = row_of_group(g, u), next_to = row_of_group(g, next);
        float sum[VEC] = {};
        uint32_t q[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) q[i] = (uint32_t)i < p1 - p0 ? (uint32_t)g.slots[p0 + i] : ~0u;
        for (uint32_t p = p0; p < p1; p += kAhead) {
            Piece<T, VEC> v[kAhead];
            float f[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                v[i] = Piece<T, VEC>{};
                f[i] = 0.f;
                if (q[i] < n_slots) {
                    v[i] = load_piece<T, VEC>(x + (int64_t)fastdiv(q[i], m) * x_stride + at);
                    f[i] = weights ? weights[q[i]] : 1.f;
                }
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) q[i] = (uint32_t)(kAhead + i) < p1 - p ? (uint32_t)g.slots[p + kAhead + i] : ~0u;
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if ((uint32_t)i >= p1 - p) break;
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] = fmaf(f[i], (float)v[i].v[e], sum[e]);
                const uint32_t after = p + i + 1;
                if (after < end && after < p1) continue;
                // the group ends here, or the tile does
                if (!before && end <= p1) {
                    if (to >= 0) store_sum<O, VEC>(out + to * g.out_stride + at, sum);
                } else {
                    store_sum<float, VEC>(g.parts + (tile * 2 + (before ? 0 : 1)) * d + at, sum);
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] = 0.f;
                before = false;
                while (end <= after && u + 1 < groups) {  // groups without pairs are passed over
                    u = next;
                    end = next_end;
                    to = next_to;
                    next = u + 1 < groups ? u + 1 : u;
                    next_end = (uint32_t)start_of(g, next + 1, pairs);
                    next_to = row_of_group(g, next);
                }
            }
        }
    }
}

template <typename T, int VEC>
__device__ __forceinline__ void store_group(const GroupSum& g, int64_t u, int32_t at, const float (&sum)[VEC],
                                            T* __restrict__ out) {
    const int64_t r = row_of_group(g, u);
    if (r >= 0) store_sum<T, VEC>(out + r * g.out_stride + at, sum);
}

// Adds up what tiles left of a group.
template <typename T, int VEC>
__global__ __launch_bounds__(kThreads) void group_join_kernel(int32_t d, Deal t, GroupSum g, T* __restrict__ out) {
    __shared__ float shared[kThreads * VEC];
    uint32_t row;
    int32_t at;
    const bool mine = deal_lane<VEC>(t, d, &row, &at);
    const int64_t groups = live_groups(g), pairs = grouped_pairs(g, groups);
    // A workgroup looks through 64 groups at a time, from all over the order, since large groups are often neighbours (hubs
    // have low ids in many graphs): those of few tiles are joined a row of lanes each, the others by the whole workgroup.
    // Groups without pairs are zero rows.
    constexpr int64_t kFew = 8;
    const int64_t rounds = (groups + kWave - 1) / kWave;
    for (int64_t round = blockIdx.x; round < rounds; round += gridDim.x) {
        const auto group = [&](int64_t i) { return i * rounds + round; };
        int64_t a = 0, b = 1;
        if (group(lane_id()) < groups) {
            a = start_of(g, group(lane_id()), pairs);
            b = start_of(g, group(lane_id()) + 1, pairs);
        }
        const int64_t t0 = a / g.tile, t1 = b > a ? (b - 1) / g.tile : t0 - 1;
        // the same in every wavefront
        const uint64_t few = __ballot(b <= a ? !g.group_row : t1 != t0 && t1 - t0 < kFew);
        uint64_t many = __ballot(b > a && t1 - t0 >= kFew);
        for (uint32_t i = row; mine && i < kWave; i += t.rows) {
            if (!((few >> i) & 1u)) continue;
            const int64_t ua = start_of(g, group(i), pairs), ub = start_of(g, group(i) + 1, pairs);
            const int64_t k0 = ua / g.tile, k1 = ub > ua ? (ub - 1) / g.tile : k0 - 1;
            float sum[VEC] = {};
            for (int64_t k = k0; k <= k1; ++k) {
                const Piece<float, VEC> v = load_piece<float, VEC>(g.parts + (k * 2 + (k == k0 ? 1 : 0)) * d + at);
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[e] += v.v[e];
            }
            store_group(g, group(i), at, sum, out);
        }
        while (many) {
            const int from = __ffsll((unsigned long long)many) - 1;
            many &= many - 1;
            const int64_t k0 = __shfl(t0, from), k1 = __shfl(t1, from);
            float sum[VEC] = {};
            if (mine)
                for (int64_t k = k0 + row; k <= k1; k += t.rows) {
                    const Piece<float, VEC> v = load_piece<float, VEC>(g.parts + (k * 2 + (k == k0 ? 1 : 0)) * d + at);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum[e] += v.v[e];
                }
            __syncthreads();
#pragma unroll
            for (int e = 0; e < VEC; ++e) shared[threadIdx.x * VEC + e] = sum[e];
            __syncthreads();
            if (mine && row == 0) {
                for (uint32_t k = 1; k < t.rows; ++k)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) sum[e] += shared[(threadIdx.x + k * t.pieces.d) * VEC + e];
                store_group(g, group(from), at, sum, out);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------------ launches
// Pairs of a tile: few enough that 2,048 wavefronts, eight per compute unit, have one, since a tile's rows are fetched
// four at a time one after the other; more where there are enough, since a tile leaves up to two rows of floats (5.8
// million pairs x 128 bf16: tiles of 64 pairs 333 us and 40 to join them, of 128 333 and 21, of 256 394 and 15).
constexpr int32_t kLeastTile = 8, kMostTile = 128;
int32_t tile_pairs(int64_t n_pairs, int32_t d, int bytes) {
    const int vec = d * bytes >= 16 ? 16 / bytes : 1;
    const int64_t pieces = (d + vec - 1) / vec;
    int32_t tile = kMostTile;
    while (tile > kLeastTile && n_pairs / tile * pieces < 2048 * kWave) tile /= 2;
    return tile;
}

struct GroupSumPlan {
    int64_t tiles;
    size_t o_parts, total;
};
GroupSumPlan plan_group_sum(int64_t n_pairs, int32_t d) {
    GroupSumPlan p;
    // the type is not known here: as many tiles as the one with the smaller ones has
    int32_t tile = tile_pairs(n_pairs, d, 2);
    if (tile_pairs(n_pairs, d, 4) < tile) tile = tile_pairs(n_pairs, d, 4);
    p.tiles = (n_pairs + tile - 1) / tile;
    p.o_parts = ((size_t)p.tiles * 4 + 255) / 256 * 256;
    p.total = p.o_parts + (size_t)p.tiles * 2 * (size_t)d * 4 + 256;
    return p;
}


template <typename T, typename O, int VEC>
int launch_group_sum(const T* x, int64_t x_stride, int64_t n, int32_t d, int32_t m, const float* weights, GroupSum g, O* out,
                     hipStream_t stream) {
    const Deal t = make_deal(d, VEC);
    g.tile = tile_pairs(g.n_pairs, d, (int)sizeof(T));
    const int64_t tiles = (g.n_pairs + g.tile - 1) / g.tile;
    const bool sums = g.n_groups > 0 && tiles > 0;
    const int64_t tile_blocks = sums ? (g.n_groups + kThreads - 1) / kThreads : 0;
    const int64_t clear_blocks = g.group_row ? (g.out_rows + kThreads - 1) / kThreads : 0;
    if (tile_blocks + clear_blocks > 0)
        hipLaunchKernelGGL((group_tiles_kernel<O, VEC>), dim3((unsigned)(tile_blocks + clear_blocks)), dim3(kThreads), 0, stream,
                           d, t, g, tile_blocks, out);
    if (sums)
        hipLaunchKernelGGL((group_sum_kernel<T, O, VEC>), dim3(workgroups((tiles + t.rows - 1) / t.rows), deal_columns(t)),
                           dim3(deal_threads(t)), 0, stream, x, x_stride, d, t, make_fastdiv((uint32_t)m), (uint32_t)(n * m),
                           weights, g, out);
    if (g.n_groups > 0)
        hipLaunchKernelGGL((group_join_kernel<O, VEC>), dim3(workgroups((g.n_groups + kWave - 1) / kWave), deal_columns(t)),
                           dim3(deal_threads(t)), 0, stream, d, t, g, out);
    ND_HIP_CHECK(hipGetLastError());
    return ND_OK;
}

template <typename F>
int by_type(int dtype, F&& f) {
    switch (dtype) {
        case ND_F32: return f((float*)nullptr);
        case ND_BF16: return f((bf16_t*)nullptr);
        default: return f((f16_t*)nullptr);
    }
}
// 16 bytes at a time, or single numbers where a row has fewer.
template <typename T, typename F>
int by_width(int32_t d, F&& f) {
    constexpr int kWide = 16 / (int)sizeof(T);
    if (d >= kWide) return f(std::integral_constant<int, kWide>());
    return f(std::integral_constant<int, 1>());
}

int check_slots(int64_t n, int32_t m, int64_t n_pairs) {
    if (n < 0 || n_pairs < 0 || m < 1) {
        set_error("n and n_pairs must not be negative and m at least 1");
        return ND_ERR_BAD_ARGUMENT;
    }
    if (m > ND_MAX_ROW_SLOTS || n >= (1ll << 31) || n * (int64_t)m >= (1ll << 31) || n_pairs >= (1ll << 31)) {
        set_error("at most %d slots per row, and fewer than 2^31 slots and pairs per call", ND_MAX_ROW_SLOTS);
        return ND_ERR_TOO_LARGE;
    }
    return ND_OK;
}

}  // namespace

int64_t group_sum_tiles(int64_t n_pairs, int32_t d, int dtype) {
    const int32_t tile = tile_pairs(n_pairs, d, (int)dtype_bytes(dtype));
    return (n_pairs + tile - 1) / tile;
}
// Rows of whole pieces only.
template <typename T>
int group_sum_floats(const T* x, int64_t x_stride, int64_t n, int32_t d, int32_t m, const float* weights, const GroupSum& g,
                     float* out, hipStream_t stream) {
    return launch_group_sum<T, float, 16 / (int)sizeof(T)>(x, x_stride, n, d, m, weights, g, out, stream);
}
template int group_sum_floats<bf16_t>(const bf16_t*, int64_t, int64_t, int32_t, int32_t, const float*, const GroupSum&, float*,
                                      hipStream_t);
template int group_sum_floats<f16_t>(const f16_t*, int64_t, int64_t, int32_t, int32_t, const float*, const GroupSum&, float*,
                                     hipStream_t);

}  // namespace nd

using namespace nd;

extern "C" {

int nd_group_positions(const int32_t* sorted_slots_dev, int64_t n_pairs, const int64_t* counts_dev, int64_t n_slots,
                       int32_t* position_dev, void* hip_stream) {
    if (n_pairs < 0 || n_slots < 0) {
        set_error("n_pairs and n_slots must not be negative");
        return ND_ERR_BAD_ARGUMENT;
    }
    if (n_pairs >= (1ll << 31) || n_slots >= (1ll << 31)) {
        set_error("fewer than 2^31 slots and pairs per call");
        return ND_ERR_TOO_LARGE;
    }
    if ((n_pairs > 0 && !sorted_slots_dev) || (n_slots > 0 && !position_dev)) {
        set_error("a required pointer is NULL");
        return ND_ERR_NULL_POINTER;
    }
    if (n_slots == 0) return ND_OK;
    hipStream_t stream = (hipStream_t)hip_stream;
    hipLaunchKernelGGL(positions_clear_kernel, dim3((unsigned)((n_slots + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                       stream, position_dev, n_slots);
    if (n_pairs > 0)
        hipLaunchKernelGGL(positions_kernel, dim3((unsigned)((n_pairs + kThreads - 1) / kThreads)), dim3(kThreads), 0,
                           stream, sorted_slots_dev, n_pairs, counts_dev, n_slots, position_dev);
    ND_HIP_CHECK(hipGetLastError());
    return ND_OK;
}

int nd_rows_by_transit(const void* x_dev, int64_t x_stride, int dtype, int64_t n, int32_t d,
                       const int32_t* sorted_slots_dev, int64_t n_pairs, const int64_t* counts_dev, int32_t m,
                       const float* weights_dev, void* out_dev, int64_t out_stride, void* hip_stream) {
    int rc = check_row_type(dtype, d);
    if (rc == ND_OK) rc = check_slots(n, m, n_pairs);
    if (rc == ND_OK) rc = check_rows("x_dev", x_dev, n, d, x_stride, dtype);
    if (rc == ND_OK) rc = check_rows("out_dev", out_dev, n_pairs, d, out_stride, dtype);
    if (rc != ND_OK) return rc;
    if (n_pairs > 0 && !sorted_slots_dev) {
        set_error("sorted_slots_dev is NULL");
        return ND_ERR_NULL_POINTER;
    }
    if (n_pairs == 0) return ND_OK;
    hipStream_t stream = (hipStream_t)hip_stream;
    return by_type(dtype, [&](auto* type) -> int {
        using T = std::remove_pointer_t<decltype(type)>;
        return by_width<T>(d, [&](auto width) -> int {
            constexpr int VEC = decltype(width)::value;
            constexpr int kRounds = 4;
            const Deal t = make_deal(d, VEC);
            const int64_t per = (int64_t)t.rows * kRounds;
            hipLaunchKernelGGL((by_transit_kernel<T, VEC, kRounds>), dim3(workgroups((n_pairs + per - 1) / per), deal_columns(t)),
                               dim3(deal_threads(t)), 0, stream, (const T*)x_dev, x_stride, d, t, sorted_slots_dev, n_pairs,
                               counts_dev, make_fastdiv((uint32_t)m), (uint32_t)(n * m), weights_dev, (T*)out_dev, out_stride);
            ND_HIP_CHECK(hipGetLastError());
            return ND_OK;
        });
    });
}

int nd_rows_to_samples(const void* z_dev, int64_t z_stride, int dtype, int64_t n_z, int32_t d, const int32_t* index_dev,
                       int64_t n, int32_t m, const float* weights_dev, void* out_dev, int64_t out_stride,
                       void* hip_stream) {
    int rc = check_row_type(dtype, d);
    if (rc == ND_OK) rc = check_slots(n, m, n_z);
    if (rc == ND_OK) rc = check_rows("z_dev", z_dev, n_z, d, z_stride, dtype);
    if (rc == ND_OK) rc = check_rows("out_dev", out_dev, n, d, out_stride, dtype);
    if (rc != ND_OK) return rc;
    if (n > 0 && !index_dev) {
        set_error("index_dev is NULL");
        return ND_ERR_NULL_POINTER;
    }
    if (n == 0) return ND_OK;
    hipStream_t stream = (hipStream_t)hip_stream;
    return by_type(dtype, [&](auto* type) -> int {
        using T = std::remove_pointer_t<decltype(type)>;
        return by_width<T>(d, [&](auto width) -> int {
            constexpr int VEC = decltype(width)::value;
            const Deal t = make_deal(d, VEC);
            // Up to 2,048 wavefronts of rows, eight per compute unit, a row's slots are shared out: 1 row of 30,000 slots x 128
            // bf16 199 us (5,510 with lanes that add up a row each), 200 rows of 30 3.9 (9.7), 6,000 rows of 30, just below,
            // 10.7 (15.3).  Above, lanes are busy without it.
            if (m > kAhead && n * t.all_pieces < 2048 * kWave) {
                uint32_t threads = kWave;
                while (threads < kShareThreads && (int64_t)threads * kAhead < (int64_t)m * t.all_pieces) threads *= 2;
                const Deal share = make_deal(d, VEC, threads);
                hipLaunchKernelGGL((to_samples_share_kernel<T, VEC>), dim3((unsigned)n, deal_columns(share)), dim3(threads),
                                   threads * VEC * sizeof(float), stream, (const T*)z_dev, z_stride, (uint32_t)n_z, d, share,
                                   index_dev, m, weights_dev, (T*)out_dev, out_stride);
                ND_HIP_CHECK(hipGetLastError());
                return ND_OK;
            }
            hipLaunchKernelGGL((to_samples_kernel<T, VEC>), dim3(workgroups((n + t.rows - 1) / t.rows), deal_columns(t)),
                               dim3(deal_threads(t)), 0, stream, (const T*)z_dev, z_stride, (uint32_t)n_z, d, t, index_dev,
                               n, m, weights_dev, (T*)out_dev, out_stride);
            ND_HIP_CHECK(hipGetLastError());
            return ND_OK;
        });
    });
}

int nd_rows_weight_grad(const void* dy_dev, int64_t dy_stride, const void* z_dev, int64_t z_stride, int dtype,
                        int64_t n_z, int32_t d, const int32_t* index_dev, int64_t n, int32_t m, float* dweights_dev,
                        void* hip_stream) {
    int rc = check_row_type(dtype, d);
    if (rc == ND_OK) rc = check_slots(n, m, n_z);
    if (rc == ND_OK) rc = check_rows("dy_dev", dy_dev, n, d, dy_stride, dtype);
    if (rc == ND_OK) rc = check_rows("z_dev", z_dev, n_z, d, z_stride, dtype);
    if (rc != ND_OK) return rc;
    if (n > 0 && (!index_dev || !dweights_dev)) {
        set_error("a required pointer is NULL");
        return ND_ERR_NULL_POINTER;
    }
    if (n == 0) return ND_OK;
    hipStream_t stream = (hipStream_t)hip_stream;
    return by_type(dtype, [&](auto* type) -> int {
        using T = std::remove_pointer_t<decltype(type)>;
        return by_width<T>(d, [&](auto width) -> int {
            constexpr int VEC = decltype(width)::value;
            constexpr int SLOTS = 4;
            int log_lanes = 0;  // at least as many lanes as slots, which the sum over them expects
            while ((1 << log_lanes) < SLOTS || (log_lanes < 6 && (VEC << log_lanes) < d)) ++log_lanes;
            const int32_t shares = (m + SLOTS - 1) / SLOTS;
            const int64_t per = kThreads >> log_lanes;
            hipLaunchKernelGGL((weight_grad_kernel<T, VEC, SLOTS>), dim3(workgroups((n * shares + per - 1) / per)),
                               dim3(kThreads), 0, stream, (const T*)dy_dev, dy_stride, (const T*)z_dev, z_stride, (uint32_t)n_z,
                               d, index_dev, n, m, make_fastdiv((uint32_t)shares), log_lanes, dweights_dev);
            ND_HIP_CHECK(hipGetLastError());
            return ND_OK;
        });
    });
}

size_t nd_rows_group_sum_workspace_bytes(int64_t n_pairs, int32_t d) {
    if (n_pairs < 0 || n_pairs >= (1ll << 31) || d < 1 || d > ND_MAX_ROW) return 0;
    return plan_group_sum(n_pairs, d).total;
}

int nd_rows_group_sum(const void* x_dev, int64_t x_stride, int dtype, int64_t n, int32_t d,
                      const int32_t* sorted_slots_dev, int64_t n_pairs, const int32_t* group_start_dev,
                      int64_t n_groups, const int64_t* counts_dev, int32_t m, const float* weights_dev,
                      const int32_t* group_row_dev, void* out_dev, int64_t out_stride, int64_t out_rows,
                      void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    int rc = check_row_type(dtype, d);
    if (rc == ND_OK) rc = check_slots(n, m, n_pairs);
    if (rc != ND_OK) return rc;
    if (n_groups < 0 || out_rows < 0) {
        set_error("n_groups and out_rows must not be negative");
        return ND_ERR_BAD_ARGUMENT;
    }
    if (!group_row_dev && out_rows < n_groups) {
        set_error("%lld rows for %lld groups", (long long)out_rows, (long long)n_groups);
        return ND_ERR_BAD_ARGUMENT;
    }
    if (out_rows >= (1ll << 31) || n_groups >= (1ll << 31) || out_rows + n_groups >= (1ll << 32) - 1024) {
        set_error("fewer than 2^31 rows and groups");
        return ND_ERR_TOO_LARGE;
    }
    rc = check_rows("x_dev", x_dev, n, d, x_stride, dtype);
    if (rc == ND_OK) rc = check_rows("out_dev", out_dev, out_rows, d, out_stride, dtype);
    if (rc != ND_OK) return rc;
    const GroupSumPlan plan = plan_group_sum(n_pairs, d);
    if ((n_pairs > 0 && !sorted_slots_dev) || (n_groups > 0 && !group_start_dev) || (n_groups > 0 && !workspace_dev)) {
        set_error("a required pointer is NULL");
        return ND_ERR_NULL_POINTER;
    }
    if (n_groups > 0 && (workspace_bytes < plan.total || ((uintptr_t)workspace_dev % 256) != 0)) {
        set_error("workspace needs %zu bytes aligned to 256", plan.total);
        return ND_ERR_WORKSPACE;
    }
    if (out_rows == 0) return ND_OK;
    hipStream_t stream = (hipStream_t)hip_stream;
    GroupSum g{};
    g.slots = sorted_slots_dev;
    g.start = group_start_dev;
    g.counts = counts_dev;
    g.group_row = group_row_dev;
    g.n_pairs = n_pairs;
    g.n_groups = n_groups;
    g.out_rows = out_rows;
    g.out_stride = out_stride;
    g.tile_group = (int32_t*)workspace_dev;
    g.parts = (float*)((char*)workspace_dev + plan.o_parts);
    return by_type(dtype, [&](auto* type) -> int {
        using T = std::remove_pointer_t<decltype(type)>;
        return by_width<T>(d, [&](auto width) -> int {
            constexpr int VEC = decltype(width)::value;
            return launch_group_sum<T, T, VEC>((const T*)x_dev, x_stride, n, d, m, weights_dev, g, (T*)out_dev, stream);
        });
    });
}

}  // extern "C"
