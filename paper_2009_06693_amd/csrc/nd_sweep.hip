#include "nd_sweep.h"

#include <cfloat>
#include <type_traits>

#include "nd_philox.h"
#include "nd_wave.h"

// With h a tile of held rows and p a block of 32 passing rows, a wavefront makes
//
//     S[p][h] = p . h,    P = exp(S - top) or g (c exp(S - lse) - count),    O[h] += sum_p P[p][h] p
//
// in 32 x 32 x 16 matrix instructions.  S is made with the passing rows as the instruction's rows, so that a lane holds 16
// passing rows of one held row: maxima and sums stay inside the lane, and the rounded P is at once the operand of
// the second product, whose other operand, the passing rows read down their columns, comes from the same tile in LDS
// through transposing reads.
namespace nd {
namespace {

constexpr int kThreads = 256;
constexpr int kRing = 4;           // units in LDS
constexpr float kLog2e = 1.44269504088896340736f;

typedef float Acc __attribute__((ext_vector_type(16)));
typedef float Float4 __attribute__((ext_vector_type(4)));
typedef short Short4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Eight {
    typedef T V __attribute__((ext_vector_type(8)));
};
__device__ __forceinline__ Acc multiply(Eight<bf16_t>::V a, Eight<bf16_t>::V b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ Acc multiply(Eight<f16_t>::V a, Eight<f16_t>::V b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

template <int MODE, int D>
struct Shape {
    // Held rows of a wavefront, in columns of 32.  What they take of the 512 registers: D / 8 for the rows, D / 2 for the
    // sums, per column.
    static constexpr int kColumns = MODE == kSweepLse || D <= 128 ? 2 : 1;
    static constexpr int kHeld = 4 * 32 * kColumns;
    static constexpr int kSteps = D / 16;              // instructions along a row
    static constexpr int kPieces = D / 8;              // 16-byte pieces of a row
    static constexpr int kUnitBytes = kSweepUnit * D * 2;
    static constexpr int kLoads = kUnitBytes / (kThreads * 16);  // pieces that a lane moves per unit
    // kSweepDw: counts of labels, a byte per (held row, passing row) of a unit, for two units
    static constexpr int kCountBytes = MODE == kSweepDw ? kHeld * kSweepUnit : 0;
    static constexpr int kLds = kRing * kUnitBytes + 2 * kCountBytes + (MODE == kSweepDw ? 64 : 0);
};

// Byte position of piece c of row r of a unit: pieces change places so that 16 rows' reads of one piece, and 4 rows' reads of
// 64 bytes, fall on different banks.
template <int D>
__device__ __forceinline__ int place(int r, int c) {
    if (D == 64) return (r * 8 + (c ^ ((((r >> 1) & 1) << 2) | ((r >> 2) & 3)))) * 16;
    return (r * (D / 8) + (c ^ (((r & 3) << 2) | ((r >> 2) & 3)))) * 16;
}

struct SweepArgs {
    const void *held, *passing;
    int64_t held_stride, passing_stride;
    SweepParts parts;
    void* out;
    int64_t out_stride;
};

template <typename T, int D, int MODE>
__global__ __attribute__((amdgpu_waves_per_eu(1, 1))) __launch_bounds__(kThreads) void sweep_kernel(LossArgs a, SweepArgs s) {
    using Sh = Shape<MODE, D>;
    using V8 = typename Eight<T>::V;
    constexpr int COLS = Sh::kColumns, HELD = Sh::kHeld, STEPS = Sh::kSteps;
    constexpr bool kSums = MODE != kSweepLse, kOnline = MODE != kSweepDw;
    // fp16 ends at 2^-24: exponentials are taken times 2^8 and may outgrow the maximum that they are relative to by 2^6
    constexpr float kRaise = std::is_same<T, f16_t>::value ? 8.f : 0.f;
    constexpr float kSlack = 4.f;  // e^4 < 2^6
    extern __shared__ __align__(16) char lds[];
    const int lane = lane_id(), wave = wave_id(), half = lane >> 5, col = lane & 31;
    const int64_t live = a.header->n_live;
    const int64_t held_rows = MODE == kSweepDw ? a.V : live, passing_rows = MODE == kSweepDw ? live : a.V;
    if (held_rows == 0 || passing_rows == 0) return;
    const SweepDeal deal(held_rows, HELD, passing_rows);
    if ((int64_t)blockIdx.x >= deal.groups) return;
    const T* held = (const T*)s.held;
    const T* passing = (const T*)s.passing;
    uint8_t* counts = (uint8_t*)(lds + kRing * Sh::kUnitBytes);
    uint32_t* touched = (uint32_t*)(lds + kRing * Sh::kUnitBytes + 2 * Sh::kCountBytes);  // a bit per (32 passing, 32 held)

    const int64_t end = deal.first((int64_t)blockIdx.x + 1);
    for (int64_t x = deal.first(blockIdx.x); x < end;) {
        const int64_t tile = x / deal.units;
        const int64_t u0 = x - tile * deal.units, u1 = end - x < deal.units - u0 ? u0 + (end - x) : deal.units;
        const int64_t row0 = tile * HELD + wave * (32 * COLS);
        x += u1 - u0;

        uint4 ahead[Sh::kLoads];
        auto load = [&](int64_t u) {
#pragma unroll
            for (int i = 0; i < Sh::kLoads; ++i) {
                const int e = i * kThreads + (int)threadIdx.x;
                int64_t r = u * kSweepUnit + e / Sh::kPieces;
                if (MODE != kSweepDw && r >= passing_rows) r = passing_rows - 1;  // gathered rows are padded
                ahead[i] = *reinterpret_cast<const uint4*>(passing + r * s.passing_stride + e % Sh::kPieces * 8);
            }
        };
        auto keep = [&](int slot) {
#pragma unroll
            for (int i = 0; i < Sh::kLoads; ++i) {
                const int e = i * kThreads + (int)threadIdx.x;
                *reinterpret_cast<uint4*>(lds + slot * Sh::kUnitBytes + place<D>(e / Sh::kPieces, e % Sh::kPieces)) = ahead[i];
            }
        };

        // held rows, as operands
        V8 rows[COLS][STEPS];
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
            int64_t r = row0 + c * 32 + col;
            r = r < held_rows ? r : held_rows - 1;
#pragma unroll
            for (int k = 0; k < STEPS; ++k)
                rows[c][k] = *reinterpret_cast<const V8*>(held + r * s.held_stride + k * 16 + half * 8);
        }
        Acc sums[COLS][D / 32];
        float top[COLS], top2[COLS], total[COLS];  // maximum, the same in the exponent of 2, sum
#pragma unroll
        for (int c = 0; c < COLS; ++c) {
            top[c] = -FLT_MAX;
            top2[c] = 0.f;
            total[c] = 0.f;
#pragma unroll
            for (int j = 0; j < D / 32; ++j) sums[c][j] = Acc{};
        }

        // labels of a unit's rows that are among the held ones
        constexpr int kLabelLoads = MODE == kSweepDw ? 3 : 1;
        const uint32_t unit_labels = (uint32_t)(kSweepUnit * a.k);
        int32_t met[kLabelLoads];
        auto load_labels = [&](int64_t u) {
#pragma unroll
            for (int i = 0; i < kLabelLoads; ++i) {
                const uint32_t e = (uint32_t)(i * kThreads) + threadIdx.x;
                met[i] = e < unit_labels ? a.labels_of[u * unit_labels + e] : -1;
            }
        };
        auto count_label = [&](int32_t v, uint32_t e, int buffer) {
            const int64_t h = (int64_t)v - tile * HELD;
            if (v < 0 || h < 0 || h >= HELD) return;
            const uint32_t r = fastdiv(e, a.div_k);
            // [held row][passing row]
            atomicAdd((uint32_t*)(counts + buffer * Sh::kCountBytes + (uint32_t)h * kSweepUnit + (r & ~3u)), 1u << (8u * (r & 3u)));
            atomicOr(&touched[buffer], 1u << ((uint32_t)h / 32u * 2u + r / 32u));
        };
        auto count_labels = [&](int64_t u, int buffer) {
#pragma unroll
            for (int i = 0; i < kLabelLoads; ++i) count_label(met[i], (uint32_t)(i * kThreads) + threadIdx.x, buffer);
            for (uint32_t e = (uint32_t)(kLabelLoads * kThreads) + threadIdx.x; e < unit_labels; e += kThreads)
                count_label(a.labels_of[u * unit_labels + e], e, buffer);
        };

        __syncthreads();  // the segment before has read its units
        if (MODE == kSweepDw) {
            for (int e = threadIdx.x * 16; e < 2 * Sh::kCountBytes; e += kThreads * 16)
                *reinterpret_cast<uint4*>(counts + e) = uint4{0, 0, 0, 0};
            if (threadIdx.x < 2) touched[threadIdx.x] = 0;
        }
        load(u0);
        keep(0);
        if (u0 + 1 < u1) {
            load(u0 + 1);
            keep(1);
        }
        if (u0 + 2 < u1) load(u0 + 2);
        if (MODE == kSweepDw) load_labels(u0);
        __syncthreads();
        if (MODE == kSweepDw) {
            count_labels(u0, 0);
            if (u0 + 1 < u1) load_labels(u0 + 1);
            __syncthreads();
        }

        // products of block b (0, 1) of the unit in `slot` with the held rows
        auto scores = [&](Acc (&out)[COLS], int slot, int b) {
            const char* from = lds + slot * Sh::kUnitBytes;
#pragma unroll
            for (int c = 0; c < COLS; ++c) out[c] = Acc{};
#pragma unroll
            for (int k = 0; k < STEPS; ++k) {
                const V8 p = *reinterpret_cast<const V8*>(from + place<D>(b * 32 + col, k * 2 + half));
#pragma unroll
                for (int c = 0; c < COLS; ++c) out[c] = multiply(p, rows[c][k], out[c]);
            }
        };
        // sums += rows of the block, weighted
        auto add_rows = [&](const V8 (&weight)[COLS][2], int slot, int b) {
            const char* from = lds + slot * Sh::kUnitBytes;
            const int sub = lane & 15, right = (lane >> 4) & 1;
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    union {
                        V8 v;
                        Short4 q[2];
                    } p;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int r = b * 32 + t * 16 + e * 8 + half * 4 + (sub >> 2), at = j * 32 + right * 16 + (sub & 3) * 4;
                        p.q[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            (__attribute__((address_space(3))) Short4*)(from + place<D>(r, at / 8) + (at & 4) * 2));
                    }
#pragma unroll
                    for (int c = 0; c < COLS; ++c) sums[c][j] = multiply(p.v, weight[c][t], sums[c][j]);
                }
        };

        V8 weight[2][COLS][2];  // of the two blocks under way
        Acc score[2][COLS];
#pragma unroll
        for (int c = 0; c < COLS; ++c)
#pragma unroll
            for (int t = 0; t < 2; ++t) weight[1][c][t] = V8{};

        // Block b of unit u: its weights from its scores, while the next block's scores and the sums over the block before
        // are made.
        auto block = [&](int64_t u, int b) {
            const int slot = (int)(u - u0) & (kRing - 1);
            const int next_slot = b == 0 ? slot : (slot + 1) & (kRing - 1);
            const int before_slot = b == 1 || u == u0 ? slot : (slot + kRing - 1) & (kRing - 1);
            const int before_b = b == 1 ? 0 : (u == u0 ? 0 : 1);
            Acc(&now)[COLS] = score[b];
            if (kOnline) {
                if (u == deal.units - 1) {  // behind the last passing row
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (u * kSweepUnit + b * 32 + 8 * (r / 4) + 4 * half + r % 4 >= passing_rows)
#pragma unroll
                            for (int c = 0; c < COLS; ++c) now[c][r] = -INFINITY;
                }
                float most[COLS];
                bool more = false;
#pragma unroll
                for (int c = 0; c < COLS; ++c) {
                    most[c] = now[c][0];
#pragma unroll
                    for (int r = 1; r < 16; ++r) most[c] = fmaxf(most[c], now[c][r]);
                    more = more || most[c] > top[c] + kSlack;
                }
                // The maximum moves only where an exponential would outgrow it: seldom after the first blocks.
                // Weights of the block before, not yet summed, are rounded once more then.
                if (__ballot(more)) {
#pragma unroll
                    for (int c = 0; c < COLS; ++c) {
                        const float t = fmaxf(top[c], fmaxf(most[c], __shfl_xor(most[c], 32)));
                        const float f = exp2_of((top[c] - t) * kLog2e);
                        total[c] *= f;
                        if (kSums) {
#pragma unroll
                            for (int j = 0; j < D / 32; ++j) sums[c][j] *= f;
#pragma unroll
                            for (int i = 0; i < 2; ++i)
#pragma unroll
                                for (int e = 0; e < 8; ++e) weight[b ^ 1][c][i][e] = (T)((float)weight[b ^ 1][c][i][e] * f);
                        }
                        top[c] = t;
                        top2[c] = t * kLog2e - kRaise;
                    }
                }
                scores(score[b ^ 1], next_slot, b ^ 1);
                if (kSums) add_rows(weight[b ^ 1], before_slot, before_b);
#pragma unroll
                for (int c = 0; c < COLS; ++c)
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float p = exp2_of(fmaf(now[c][t * 8 + e], kLog2e, -top2[c]));
                            total[c] += p;
                            if (kSums) weight[b][c][t][e] = (T)p;
                        }
            } else {
                const int buffer = (int)(u - u0) & 1;
                const uint32_t held_here = wave_uniform(touched[buffer]) >> (wave * COLS * 2 + b);
                scores(score[b ^ 1], next_slot, b ^ 1);
                add_rows(weight[b ^ 1], before_slot, before_b);
                const int64_t p0 = u * kSweepUnit + b * 32 + half * 4;
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) {
                    const Float4 lse = *reinterpret_cast<const Float4*>(a.place_lse + p0 + r4 * 8);
                    const Float4 count = *reinterpret_cast<const Float4*>(a.count + p0 + r4 * 8);
                    const Float4 g = *reinterpret_cast<const Float4*>(a.weight + p0 + r4 * 8);
                    const float scale = a.header->scale;
#pragma unroll
                    for (int c = 0; c < COLS; ++c) {
                        uint32_t held4 = 0;
                        if ((held_here >> (c * 2)) & 1u)
                            held4 = *reinterpret_cast<const uint32_t*>(counts + buffer * Sh::kCountBytes +
                                                                       (wave * COLS * 32 + c * 32 + col) * kSweepUnit + b * 32 + r4 * 8 + half * 4);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float f = g[e] * scale;
                            float p = f * count[e] * exp2_of((now[c][r4 * 4 + e] - lse[e]) * kLog2e);
                            if (count[e] == 0.f) p = 0.f;
                            p -= f * (float)((held4 >> (8 * e)) & 255u);
                            weight[b][c][r4 / 2][r4 % 2 * 4 + e] = (T)p;
                        }
                    }
                }
            }
        };

        scores(score[0], 0, 0);
        for (int64_t u = u0; u < u1; ++u) {
            const int slot = (int)(u - u0) & (kRing - 1);
            if (u + 2 < u1) {
                keep((slot + 2) & (kRing - 1));
                if (u + 3 < u1) load(u + 3);
            }
            block(u, 0);
            block(u, 1);
            if (MODE == kSweepDw) {
                const int buffer = (int)(u - u0) & 1;
                if (u + 1 < u1) {
                    count_labels(u + 1, buffer ^ 1);
                    if (u + 2 < u1) load_labels(u + 2);
                }
                __syncthreads();
                // this unit's counts are cleared for the unit after the next
                const uint32_t dirty = wave_uniform(touched[buffer]);
                if ((dirty >> (wave * COLS * 2)) & ((1u << (COLS * 2)) - 1u)) {
                    uint4* mine = reinterpret_cast<uint4*>(counts + buffer * Sh::kCountBytes + wave * COLS * 32 * kSweepUnit);
                    for (int e = lane; e < COLS * 32 * kSweepUnit / 16; e += kWave) mine[e] = uint4{0, 0, 0, 0};
                }
                __syncthreads();
                if (threadIdx.x == 0) touched[buffer] = 0;
            }
            __syncthreads();
        }
        if (kSums) add_rows(weight[1], (int)(u1 - 1 - u0) & (kRing - 1), 1);

        // out
        const bool whole = u0 == 0 && u1 == deal.units;
        if (kOnline) {
            const int64_t segment = (int64_t)blockIdx.x + tile;
            const float lower = exp2_of(-kRaise);
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                const float both = (total[c] + __shfl_xor(total[c], 32)) * lower;
                const int64_t at = segment * HELD + wave * (32 * COLS) + c * 32 + col;
                if (half == 0) {
                    s.parts.top[at] = top[c];
                    s.parts.sum[at] = both;
                }
                if (kSums)
#pragma unroll
                    for (int j = 0; j < D / 32; ++j)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const Float4 v = {sums[c][j][r * 4], sums[c][j][r * 4 + 1], sums[c][j][r * 4 + 2], sums[c][j][r * 4 + 3]};
                            *reinterpret_cast<Float4*>(s.parts.rows + at * D + j * 32 + r * 8 + half * 4) = v * lower;
                        }
            }
        } else {
            const float back = 1.f / a.header->scale;
            const int64_t segment = (int64_t)blockIdx.x * 2 + (u0 == 0 ? 1 : 0);  // one that ends a tile, one that begins one
#pragma unroll
            for (int c = 0; c < COLS; ++c) {
                const int64_t v = row0 + c * 32 + col;
#pragma unroll
                for (int j = 0; j < D / 32; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int e0 = j * 32 + r * 8 + half * 4;
                        const Float4 o = {sums[c][j][r * 4], sums[c][j][r * 4 + 1], sums[c][j][r * 4 + 2], sums[c][j][r * 4 + 3]};
                        if (!whole) {
                            *reinterpret_cast<Float4*>(s.parts.rows + (segment * HELD + wave * (32 * COLS) + c * 32 + col) * D + e0) = o;
                        } else if (v < held_rows) {
                            T* to = (T*)s.out + v * s.out_stride + e0;
                            if (e0 + 4 <= a.d) {
                                Piece<T, 4> q;
#pragma unroll
                                for (int e = 0; e < 4; ++e) q.v[e] = (T)(o[e] * back);
                                store_piece<T, 4>(to, q);
                            } else {
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (e0 + e < a.d) to[e] = (T)(o[e] * back);
                            }
                        }
                    }
            }
        }
    }
}

// Rows of dw whose tile several workgroups had a part of; all of them where there was nothing to sum.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void dw_join_kernel(LossArgs a, SweepParts parts, T* __restrict__ dw, int64_t dw_stride) {
    constexpr int HELD = Shape<kSweepDw, D>::kHeld;
    const int64_t live = a.header->n_live;
    const SweepDeal deal(a.V, HELD, live);
    const float back = 1.f / a.header->scale;
    for (int64_t v = (int64_t)blockIdx.x * 4 + wave_id(); v < a.V; v += (int64_t)gridDim.x * 4) {
        int64_t x0 = 0, g0 = 0, g1 = -1;
        if (live > 0) {
            x0 = v / HELD * deal.units;
            g0 = deal.group_of(x0);
            g1 = deal.group_of(x0 + deal.units - 1);
            if (g0 == g1) continue;
        }
        for (int e = lane_id(); e < a.d; e += kWave) {
            float sum = 0.f;
            for (int64_t g = g0; g <= g1; ++g) {
                const int64_t segment = g * 2 + (deal.first(g) <= x0 ? 1 : 0);
                sum += parts.rows[(segment * HELD + v % HELD) * D + e];
            }
            dw[v * dw_stride + e] = (T)(sum * back);
        }
    }
}

// lse, loss and dx of a gathered row, a wavefront each.
template <typename T, int D, int MODE>
__global__ __launch_bounds__(kThreads) void finish_kernel(LossArgs a, const T* __restrict__ rows, const T* __restrict__ w,
                                                          int64_t w_stride, SweepParts parts, T* __restrict__ dx, int64_t dx_stride) {
    constexpr int HELD = Shape<MODE, D>::kHeld;
    constexpr int PER = (D + 63) / 64;  // numbers of a lane: lane, lane + 64, ...
    const int64_t live = a.header->n_live;
    const SweepDeal deal(live, HELD, a.V);
    for (int64_t p = (int64_t)blockIdx.x * 4 + wave_id(); p < live; p += (int64_t)gridDim.x * 4) {
        const int64_t tile = p / HELD, x0 = tile * deal.units;
        const int64_t g0 = deal.group_of(x0), g1 = deal.group_of(x0 + deal.units - 1);
        const int64_t in_tile = p % HELD;
        float top = -FLT_MAX, sum = 0.f;
        for (int64_t g = g0 + lane_id(); g <= g1; g += kWave) {
            const float t2 = parts.top[(g + tile) * HELD + in_tile], s2 = parts.sum[(g + tile) * HELD + in_tile], t = fmaxf(top, t2);
            sum = sum * exp2_of((top - t) * kLog2e) + s2 * exp2_of((t2 - t) * kLog2e);
            top = t;
        }
        for (int s = 32; s > 0; s >>= 1) {
            const float t2 = __shfl_xor(top, s), s2 = __shfl_xor(sum, s), t = fmaxf(top, t2);
            sum = sum * exp2_of((top - t) * kLog2e) + s2 * exp2_of((t2 - t) * kLog2e);
            top = t;
        }
        const float lse = top + logf(sum);
        const int64_t row = a.row_of[p];
        const float c = a.count[p];
        float grad[PER] = {}, mine[PER];
        if (MODE == kSweepDx) {
            for (int64_t g = g0; g <= g1; ++g) {
                const int64_t at = (g + tile) * HELD + in_tile;
                const float f = exp2_of((parts.top[at] - top) * kLog2e);
#pragma unroll
                for (int i = 0; i < PER; ++i) grad[i] = fmaf(f, parts.rows[at * D + i * 64 + lane_id()], grad[i]);
            }
#pragma unroll
            for (int i = 0; i < PER; ++i) grad[i] *= c / sum;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) mine[i] = (float)rows[p * D + i * 64 + lane_id()];
        float met = 0.f;
        for (int32_t j = 0; j < a.k; ++j) {
            const int32_t v = wave_uniform(a.labels_of[p * a.k + j]);
            if (v < 0) continue;
            float dot = 0.f;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = i * 64 + lane_id();
                const float b = (float)w[(int64_t)v * w_stride + e];
                dot = fmaf(mine[i], b, dot);
                grad[i] -= b;
            }
            met += dot;
        }
        for (int s = 32; s > 0; s >>= 1) met += __shfl_xor(met, s);
        if (lane_id() == 0) {
            a.place_lse[p] = lse;
            a.lse[row] = lse;
            a.loss[row] = c * lse - met;
        }
        if (MODE == kSweepDx) {
            const float g = a.weight[p];
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int e = i * 64 + lane_id();
                if (e < a.d) dx[row * dx_stride + e] = (T)(g * grad[i]);
            }
        }
    }
}

// A launch holds fewer than 2^32 lanes: wavefronts go on to further rows from here on.
inline dim3 wave_per(int64_t rows) {
    const int64_t groups = (rows + 3) / 4;
    return dim3((unsigned)(groups < (1 << 20) ? groups : 1 << 20));
}

template <typename F>
int by_width(int32_t dp, F&& f) {
    switch (dp) {
        case 64: return f(std::integral_constant<int, 64>());
        case 128: return f(std::integral_constant<int, 128>());
        default: return f(std::integral_constant<int, 256>());
    }
}
template <typename T, int D, int MODE>
int launch_sweep(const LossArgs& a, const SweepArgs& s, hipStream_t stream) {
    constexpr int kLds = Shape<MODE, D>::kLds;
    static_assert(kLds <= 160 * 1024, "a compute unit's LDS");
    if (kLds > 64 * 1024)
        ND_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(&sweep_kernel<T, D, MODE>),
                                         hipFuncAttributeMaxDynamicSharedMemorySize, kLds));
    hipLaunchKernelGGL((sweep_kernel<T, D, MODE>), dim3(kSweepGroups), dim3(kThreads), kLds, stream, a, s);
    ND_HIP_CHECK(hipGetLastError());
    return ND_OK;
}

}  // namespace

int sweep_width(int32_t d) { return d <= 64 ? 64 : d <= 128 ? 128 : d <= 256 ? 256 : 0; }
int sweep_held(int mode, int32_t dp) { return mode == kSweepLse || dp <= 128 ? 256 : 128; }
int64_t sweep_segments(int mode, int64_t held, int32_t dp) {
    if (mode == kSweepDw) return 2 * kSweepGroups;
    const int h = sweep_held(mode, dp);
    return kSweepGroups + (held + h - 1) / h;
}

template <typename T>
int sweep(int mode, const LossArgs& a, const T* rows, const T* w, int64_t w_stride, const SweepParts& parts, T* dw,
          int64_t dw_stride, hipStream_t stream) {
    SweepArgs s{};
    s.parts = parts;
    s.out = dw;
    s.out_stride = dw_stride;
    s.held = mode == kSweepDw ? w : rows;
    s.held_stride = mode == kSweepDw ? w_stride : a.dp;
    s.passing = mode == kSweepDw ? rows : w;
    s.passing_stride = mode == kSweepDw ? a.dp : w_stride;
    return by_width(a.dp, [&](auto width) -> int {
        constexpr int D = decltype(width)::value;
        static_assert(Shape<kSweepDx, D>::kHeld == Shape<kSweepDw, D>::kHeld, "sweep_held");
        if (mode == kSweepLse) return launch_sweep<T, D, kSweepLse>(a, s, stream);
        if (mode == kSweepDx) return launch_sweep<T, D, kSweepDx>(a, s, stream);
        const int rc = launch_sweep<T, D, kSweepDw>(a, s, stream);
        if (rc != ND_OK) return rc;
        hipLaunchKernelGGL((dw_join_kernel<T, D>), wave_per(a.V), dim3(kThreads), 0, stream, a, parts, dw,
                           dw_stride);
        ND_HIP_CHECK(hipGetLastError());
        return ND_OK;
    });
}

template <typename T>
int sweep_finish(int mode, const LossArgs& a, const T* rows, const T* w, int64_t w_stride, const SweepParts& parts, T* dx,
                 int64_t dx_stride, hipStream_t stream) {
    return by_width(a.dp, [&](auto width) -> int {
        constexpr int D = decltype(width)::value;
        const dim3 grid = wave_per(a.n), block(kThreads);
        if (mode == kSweepLse)
            hipLaunchKernelGGL((finish_kernel<T, D, kSweepLse>), grid, block, 0, stream, a, rows, w, w_stride, parts, dx, dx_stride);
        else
            hipLaunchKernelGGL((finish_kernel<T, D, kSweepDx>), grid, block, 0, stream, a, rows, w, w_stride, parts, dx, dx_stride);
        ND_HIP_CHECK(hipGetLastError());
        return ND_OK;
    });
}

template int sweep<bf16_t>(int, const LossArgs&, const bf16_t*, const bf16_t*, int64_t, const SweepParts&, bf16_t*, int64_t,
                           hipStream_t);
template int sweep<f16_t>(int, const LossArgs&, const f16_t*, const f16_t*, int64_t, const SweepParts&, f16_t*, int64_t,
                          hipStream_t);
template int sweep_finish<bf16_t>(int, const LossArgs&, const bf16_t*, const bf16_t*, int64_t, const SweepParts&, bf16_t*, int64_t,
                                  hipStream_t);
template int sweep_finish<f16_t>(int, const LossArgs&, const f16_t*, const f16_t*, int64_t, const SweepParts&, f16_t*, int64_t,
                                 hipStream_t);

}  // namespace nd
