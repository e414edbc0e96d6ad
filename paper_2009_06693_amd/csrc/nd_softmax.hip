// Softmax loss over all vertices and its gradient, in pieces of the vertices.
//
//     s_nv = x_n . w_v        lse_n = log sum_v exp s_nv        loss_n = c_n lse_n - sum_j s_n,label[n][j]
//     dx_n = g_n (c_n sum_v p_nv w_v - sum_j w_label[n][j])     dw_v = sum_n g_n (c_n p_nv - #{j: label = v}) x_n
//
// Rows with labels are gathered once into a dense, zero-padded array, so that every product below works on full tiles of
// rows that count, whatever rows without labels hold.  The logits are a matrix product whose tiles leave a running maximum
// and sum per row and, where rows are long, themselves; for the gradient what is kept, or made again a piece of vertices at a
// time, is turned into a vertex's weight, rounded to the rows' type and multiplied by w (for dx) and by x (for dw).  Rows of
// 16 bits that are short go through sweeps instead, and a few rows without gradient through a kernel of their own.
#include <cfloat>
#include <type_traits>

#include "nd_philox.h"
#include "nd_rows.h"
#include "nd_sweep.h"

namespace nd {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 128;         // rows of a product's tile
constexpr int kChunk = 16;         // bytes that a lane moves at once
// Probabilities that lie in the workspace at a time: so many, or those of one tile of vertices where rows are more than a million
// (fp32: half as many).  fp32 scores that are kept have theirs in their place.
constexpr size_t kPieceBytes = (size_t)512 << 20;
constexpr int64_t kKeptBytes = (int64_t)4 << 30;    // scores that are kept at most

typedef float Acc __attribute__((ext_vector_type(16)));
typedef short Short4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int32_t labels_of_row(const LossArgs& a, int64_t row, bool* bad) {
    int32_t c = 0;
    for (int32_t j = 0; j < a.k; ++j) {
        const int32_t v = a.labels[row * a.k + j];
        if (v >= 0) {
            if ((int64_t)v < a.V)
                ++c;
            else
                *bad = true;
        }
    }
    return c;
}

// What the scale goes by: an infinite weight or one that is no number must not take the others' gradients with it.
__device__ __forceinline__ float weight_size(const LossArgs& a, int64_t row) {
    const float w = a.row_weight ? fabsf(a.row_weight[row]) : 1.f;
    return w <= FLT_MAX ? w : 0.f;
}

__global__ __launch_bounds__(kTile) void count_kernel(LossArgs a) {
    __shared__ uint32_t s_live[2], s_bad[2];
    __shared__ float s_weight[2];
    const int64_t row = (int64_t)blockIdx.x * kTile + threadIdx.x;
    bool bad = false;
    const bool live = row < a.n && labels_of_row(a, row, &bad) > 0;
    float w = live ? weight_size(a, row) : 0.f;
    for (int s = 32; s > 0; s >>= 1) w = fmaxf(w, __shfl_xor(w, s));
    const uint64_t lives = __ballot(live), bads = __ballot(bad);
    if (lane_id() == 0) {
        s_weight[wave_id()] = w;
        s_live[wave_id()] = (uint32_t)__popcll(lives);
        s_bad[wave_id()] = bads != 0;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        a.block_live[blockIdx.x] = s_live[0] + s_live[1];
        a.block_bad[blockIdx.x] = s_bad[0] | s_bad[1];
        a.block_weight[blockIdx.x] = fmaxf(s_weight[0], s_weight[1]);
    }
}

template <typename T>
__device__ __forceinline__ void write_header(const LossArgs& a, uint32_t live, uint32_t bad, float top) {
    a.header->status = bad;
    a.header->n_live = live;
    // fp16 holds 2^-24 to 65,504: the largest product of a weight and a count of labels becomes at most 2^15
    float scale = 1.f;
    if (std::is_same<T, f16_t>::value && top > 0.f)
        scale = exp2f(fminf(fmaxf(floorf(log2f(32768.f / (float)a.k) - log2f(top)), -60.f), 60.f));
    a.header->scale = scale;
}

// Many blocks: each block's count becomes that of the blocks before it, by one workgroup, which also writes the header.  Up to
// kScanBlocks every block adds up what is before it by itself, a launch less and as many reads as the square of the blocks.
// Placing without and with the scan, us: 4,096 blocks 13.9 and 12.3, 8,192 38.9 and 19.1, 32,768 441 and 57; 2,048 blocks take
// 9.0 without, and a scan is 5 by itself.
constexpr int32_t kScanBlocks = 2048;
constexpr int kScanThreads = 1024;
template <typename T>
__global__ __launch_bounds__(kScanThreads) void scan_blocks_kernel(LossArgs a, int32_t blocks) {
    constexpr int kEach = 4;
    __shared__ uint32_t s_scan[kScanThreads / kWave + 1];
    __shared__ float s_weight[kScanThreads / kWave];
    uint32_t before = 0, bad = 0;
    float top = 0.f;
    for (int64_t b0 = 0; b0 < blocks; b0 += kScanThreads * kEach) {
        const int64_t mine = b0 + (int64_t)threadIdx.x * kEach;
        uint32_t live[kEach], sum = 0, all;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            live[i] = 0;
            if (mine + i < blocks) {
                live[i] = a.block_live[mine + i];
                bad |= a.block_bad[mine + i];
                top = fmaxf(top, a.block_weight[mine + i]);
            }
            sum += live[i];
        }
        uint32_t at = before + block_exclusive_scan<uint32_t, kScanThreads>(sum, s_scan, &all);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (mine + i < blocks) a.block_live[mine + i] = at;
            at += live[i];
        }
        before += all;
        __syncthreads();  // s_scan is used again
    }
    for (int s = 32; s > 0; s >>= 1) top = fmaxf(top, __shfl_xor(top, s));
    if (lane_id() == 0) s_weight[wave_id()] = top;
    bad = __syncthreads_or(bad != 0);
    if (threadIdx.x != 0) return;
    for (int i = 1; i < kScanThreads / kWave; ++i) top = fmaxf(top, s_weight[i]);
    write_header<T>(a, before, bad, top);
}

// Deals out places: rows with labels from the front, the others behind them.
template <typename T>
__global__ __launch_bounds__(kTile) void place_kernel(LossArgs a, int32_t blocks) {
    __shared__ uint32_t s_before[2], s_all[2], s_bad[2], s_wave[2];
    __shared__ float s_weight[2];
    uint32_t before = 0, all = 0, bad_any = 0;
    float top = 0.f;
    const int64_t row = (int64_t)blockIdx.x * kTile + threadIdx.x;
    bool bad = false;
    const int32_t c = row < a.n ? labels_of_row(a, row, &bad) : 0;
    const bool scanned = blocks > kScanBlocks;
    if (scanned) {
        before = threadIdx.x == 0 ? a.block_live[blockIdx.x] : 0;
    } else if (blocks == 1) {  // nothing was counted
        all = c > 0;
        bad_any = bad;
        top = c > 0 ? weight_size(a, row) : 0.f;
    } else {
        for (int32_t b = threadIdx.x; b < blocks; b += kTile) {
            const uint32_t l = a.block_live[b];
            all += l;
            if (b < (int32_t)blockIdx.x) before += l;
            bad_any |= a.block_bad[b];
            top = fmaxf(top, a.block_weight[b]);
        }
    }
    for (int s = 32; s > 0; s >>= 1) {
        before += __shfl_xor(before, s);
        all += __shfl_xor(all, s);
        bad_any |= __shfl_xor(bad_any, s);
        top = fmaxf(top, __shfl_xor(top, s));
    }
    const uint64_t lives = __ballot(c > 0);
    if (lane_id() == 0) {
        s_before[wave_id()] = before;
        s_all[wave_id()] = all;
        s_bad[wave_id()] = bad_any;
        s_weight[wave_id()] = top;
        s_wave[wave_id()] = (uint32_t)__popcll(lives);
    }
    __syncthreads();
    before = s_before[0] + s_before[1];
    all = scanned ? a.header->n_live : s_all[0] + s_all[1];
    if (!scanned && blockIdx.x == 0 && threadIdx.x == 0)
        write_header<T>(a, all, s_bad[0] | s_bad[1], fmaxf(s_weight[0], s_weight[1]));
    if (row >= a.n) return;
    // rows with labels in front of this one
    const int64_t at = before + (wave_id() == 1 ? s_wave[0] : 0u) + (uint32_t)__popcll(lives & lanes_below(lane_id()));
    if (c > 0) {
        a.row_of[at] = (int32_t)row;
        a.count[at] = (float)c;
        a.weight[at] = a.row_weight ? a.row_weight[row] : 1.f;
    } else {
        a.row_of[all + (row - at)] = (int32_t)row;
    }
}

// Lanes over places and 16-byte pieces of a padded row.
struct Spread {
    FastDiv lanes;   // of a place (at most kThreads)
    uint32_t places; // of a workgroup
};
inline Spread make_spread(int32_t dp, int vec) {
    const uint32_t pieces = (uint32_t)(dp / vec), lanes = pieces < kThreads ? pieces : kThreads;
    return Spread{make_fastdiv(lanes), kThreads / lanes};
}
inline dim3 spread_grid(const Spread& s, int64_t places) {
    const int64_t groups = (places + s.places - 1) / s.places;
    return dim3((unsigned)(groups < (1 << 20) ? groups : 1 << 20));
}
// A row of d numbers as one of dp, zeros behind.
template <typename T>
__device__ __forceinline__ void pad_row(const T* __restrict__ from, T* __restrict__ to, int32_t d, int32_t dp, uint32_t lane,
                                        uint32_t lanes) {
    constexpr int VEC = kChunk / (int)sizeof(T);
    for (int32_t e = (int32_t)lane * VEC; e < dp; e += (int32_t)lanes * VEC) {
        Piece<T, VEC> v{};
        if (e + VEC <= d) {
            v = load_piece<T, VEC>(from + e);
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (e + i < d) v.v[i] = from[e + i];
        }
        store_piece<T, VEC>(to + e, v);
    }
}

// The rows with labels one after the other, then zeros up to a whole tile; what rows without labels get.
template <typename T>
__global__ __launch_bounds__(kThreads) void gather_kernel(LossArgs a, Spread s, const T* __restrict__ x, int64_t x_stride,
                                                          T* __restrict__ rows, T* __restrict__ dx, int64_t dx_stride) {
    if (a.label_row)  // none yet
        for (int64_t v = (int64_t)blockIdx.x * kThreads + threadIdx.x; v < a.V; v += (int64_t)gridDim.x * kThreads)
            a.label_row[v] = -1;
    const uint32_t in_group = fastdiv(threadIdx.x, s.lanes), lane = threadIdx.x - in_group * s.lanes.d;
    if (in_group >= s.places) return;
    const int64_t live = a.header->n_live, padded = (live + kTile - 1) / kTile * kTile;
    for (int64_t p = (int64_t)blockIdx.x * s.places + in_group; p < a.n_pad; p += (int64_t)gridDim.x * s.places) {
        if (p < live) {
            const int64_t row = a.row_of[p];
            pad_row(x + row * x_stride, rows + p * a.dp, a.d, a.dp, lane, s.lanes.d);
            for (int32_t j = (int32_t)lane; j < a.k; j += (int32_t)s.lanes.d) {
                const int32_t v = a.labels[row * a.k + j];
                const uint32_t mine = v >= 0 && (int64_t)v < a.V ? (uint32_t)v : ~0u;
                int32_t to = j;
                if (a.label_score) {  // ascending
                    to = 0;
#pragma unroll 4
                    for (int32_t i = 0; i < a.k; ++i) {
                        const int32_t u = a.labels[row * a.k + i];
                        const uint32_t other = u >= 0 && (int64_t)u < a.V ? (uint32_t)u : ~0u;
                        to += other < mine || (other == mine && i < j);
                    }
                }
                a.labels_of[p * a.k + to] = (int32_t)mine;
            }
            continue;
        }
        if (p < padded) {
            pad_row((const T*)nullptr, rows + p * a.dp, 0, a.dp, lane, s.lanes.d);
            if (lane == 0) {
                a.count[p] = a.weight[p] = a.place_lse[p] = 0.f;
                if (a.place_factor) a.place_factor[p] = INFINITY;
            }
        }
        for (int32_t j = (int32_t)lane; j < a.k; j += (int32_t)s.lanes.d) a.labels_of[p * a.k + j] = -1;
        if (p < a.n) {
            const int64_t row = a.row_of[p];
            if (lane == 0) a.loss[row] = a.lse[row] = 0.f;
            if (dx)
                for (int32_t e = (int32_t)lane; e < a.d; e += (int32_t)s.lanes.d) dx[row * dx_stride + e] = (T)0.f;
        }
    }
}

// Rows of d numbers at any stride to rows of dp, zeros behind.
template <typename T>
__global__ __launch_bounds__(kThreads) void pad_kernel(const T* __restrict__ w, int64_t stride, int64_t rows, int32_t d,
                                                       int32_t dp, Spread s, T* __restrict__ out) {
    const uint32_t in_group = fastdiv(threadIdx.x, s.lanes), lane = threadIdx.x - in_group * s.lanes.d;
    if (in_group >= s.places) return;
    for (int64_t r = (int64_t)blockIdx.x * s.places + in_group; r < rows; r += (int64_t)gridDim.x * s.places)
        pad_row(w + r * stride, out + r * dp, d, dp, lane, s.lanes.d);
}

// ------------------------------------------------------------------------------------------------ product of tiles
// C[m][n] = sum_k A(m, k) B(n, k) for a tile of 256 x 128, four wavefronts of 128 x 64 each in 32 x 32 matrix
// instructions: eight of them use six operands, so that LDS, which gives a wavefront's operand of 1 KB in 5 to 9 cycles
// (transposed reads) and has four SIMDs to feed, keeps ahead of them.  An operand lies in memory with the summed
// dimension along its rows (ACROSS = false) or down its columns (ACROSS = true), and in LDS as it does in memory, 16-byte
// pieces of a row exchanged so that the reads of a wavefront fall on different banks.  Bound by the matrix instructions and
// what it takes to feed them: 2,304 x 57,000 x 1,024 fp16 310 to 330 us, 815 to 870 TFLOP/s; 4,096 x 4,096 x 128 in fp32 48 us,
// 90 TFLOP/s, where a tile has eight steps and as much again to begin and end.
template <typename T>
struct Operand {
    const T* base;
    int64_t stride;
    int64_t rows;   // of the array: reads behind it are of its last row
    int32_t cols;   // ACROSS: numbers in a row (a multiple of a piece): pieces behind are the last one again
};

constexpr int kTileM = 256, kTileN = 128;
constexpr int kStepBytes = 64;                               // of the summed dimension at a time
constexpr int kLdsM = kTileM * kStepBytes, kLdsN = kTileN * kStepBytes, kLdsBytes = 2 * (kLdsM + kLdsN);

template <typename T>
struct Kind {
    static constexpr int kVec = kChunk / (int)sizeof(T);       // numbers in a piece
    static constexpr int kStep = kStepBytes / (int)sizeof(T);  // of the summed dimension in a tile
    static constexpr bool kWide = sizeof(T) == 4;
};

// Byte position in LDS of piece c of row r of a tile SIZE wide: SIZE rows of 4 pieces, or kStep rows of SIZE numbers.
template <typename T, bool ACROSS, int SIZE>
__device__ __forceinline__ int lds_place(int r, int c) {
    if (!ACROSS) return (r * 4 + (c ^ ((r >> 2) & 3))) * kChunk;
    constexpr int kPieces = SIZE / Kind<T>::kVec;
    if (Kind<T>::kWide) return (r * kPieces + (c ^ (((r >> 2) & 1) << 3))) * kChunk;
    return (r * kPieces + (c ^ (((r & 3) << 2) | ((r >> 2) & 3)))) * kChunk;
}

typedef uint32_t Word4 __attribute__((ext_vector_type(4)));

// A lane's pieces of an operand's tile, on their way to LDS.
template <typename T, bool ACROSS, int SIZE>
struct Mover {
    static constexpr int kCount = SIZE * kStepBytes / (kThreads * kChunk);
    static constexpr int kPieces = ACROSS ? SIZE / Kind<T>::kVec : 4;  // of a row of the tile
    Word4 v[2][kCount];    // two steps are under way
    const T* at[ACROSS ? 1 : kCount];       // the lane's rows,
    int32_t column[ACROSS ? kCount : 1];    // or its columns
    __device__ __forceinline__ Mover(const Operand<T>& o, int64_t m0) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int e = i * kThreads + (int)threadIdx.x, r = e / kPieces, p = e % kPieces;
            if (!ACROSS) {
                const int64_t row = m0 + r < o.rows ? m0 + r : o.rows - 1;
                at[i] = o.base + row * o.stride + p * Kind<T>::kVec;
            } else {
                const int64_t col = m0 + p * Kind<T>::kVec, last = o.cols - Kind<T>::kVec;
                column[i] = (int32_t)(col < last ? col : last);
            }
        }
    }
    template <int SET>
    __device__ __forceinline__ void fetch(const Operand<T>& o, int64_t k) {
        const int64_t k_row = k < o.rows ? k : o.rows - 1;
        const uint32_t left = o.rows - k_row < Kind<T>::kStep ? (uint32_t)(o.rows - k_row) : (uint32_t)Kind<T>::kStep;
        const T* across = o.base + k_row * o.stride;
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            if (!ACROSS) {
                v[SET][i] = *reinterpret_cast<const Word4*>(at[i] + k);
            } else {
                const uint32_t r = ((uint32_t)(i * kThreads) + threadIdx.x) / kPieces;
                v[SET][i] = *reinterpret_cast<const Word4*>(
                    across + ((uint64_t)(r < left ? r : left - 1u) * (uint32_t)o.stride + (uint32_t)column[i]));
            }
        }
    }
    template <int SET>
    __device__ __forceinline__ void keep(char* lds) const {
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            const int e = i * kThreads + (int)threadIdx.x;
            *reinterpret_cast<Word4*>(lds + lds_place<T, ACROSS, SIZE>(e / kPieces, e % kPieces)) = v[SET][i];
        }
    }
};

// A lane's share of a 32-row block for one group of the summed dimension: 16-bit types 16 of it, lane l holds row l % 32
// and the eight from 8 (l / 32) on; fp32 8 of it, the four from 4 (l / 32) on, one for each of four instructions.
template <typename T>
struct Fragment {
    T v[Kind<T>::kVec];
};
template <typename T, bool ACROSS, int SIZE>
__device__ __forceinline__ Fragment<T> fragment(const char* lds, int block_row, int group) {
    const int lane = lane_id(), half = lane >> 5;
    Fragment<T> f;
    if (!ACROSS) {
        const int r = block_row + (lane & 31);
        f = *reinterpret_cast<const Fragment<T>*>(lds + lds_place<T, false, SIZE>(r, group * 2 + half));
    } else if (Kind<T>::kWide) {
        const int col = block_row + (lane & 31);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            f.v[e] = *reinterpret_cast<const T*>(lds + lds_place<T, true, SIZE>(group * 8 + half * 4 + e, col / 4) + col % 4 * 4);
    } else {
        // 16 lanes hand in 4 rows x 16 columns and get a column of four rows each
        const int sub = lane & 15, col = block_row + ((lane >> 4) & 1) * 16 + (sub & 3) * 4;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int r = group * 16 + half * 8 + e * 4 + (sub >> 2);
            const char* at = lds + lds_place<T, true, SIZE>(r, col / 8) + (col & 4) * 2;
            const Short4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) Short4*)at);
            __builtin_memcpy(&f.v[e * 4], &t, 8);
        }
    }
    return f;
}
__device__ __forceinline__ Acc multiply(const Fragment<float>& a, const Fragment<float>& b, Acc c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
    return c;
}
__device__ __forceinline__ Acc multiply(const Fragment<bf16_t>& a, const Fragment<bf16_t>& b, Acc c) {
    typedef bf16_t V8 __attribute__((ext_vector_type(8)));
    V8 x, y;
    __builtin_memcpy(&x, &a, 16);
    __builtin_memcpy(&y, &b, 16);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
}
__device__ __forceinline__ Acc multiply(const Fragment<f16_t>& a, const Fragment<f16_t>& b, Acc c) {
    typedef f16_t V8 __attribute__((ext_vector_type(8)));
    V8 x, y;
    __builtin_memcpy(&x, &a, 16);
    __builtin_memcpy(&y, &b, 16);
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, c, 0, 0, 0);
}

// A barrier for what lies in LDS only: loads from memory stay under way across it.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The tile at (m0, n0) summed over [k0, k1), k1 - k0 a multiple of Kind::kStep; lds: kLdsBytes.  Ends with a barrier.
// Result: lane l of wavefront w holds column n = 64 (w % 2) + 32 j + l % 32 and rows m = 128 (w / 2) + 32 i + 8 (r / 4) +
// 4 (l / 32) + r % 4 in acc[i][j][r].
typedef Acc AccTile[4][2];
template <typename T, bool A_ACROSS, bool B_ACROSS>
__device__ __forceinline__ void product(const Operand<T>& a, const Operand<T>& b, int64_t m0, int64_t n0, int64_t k0,
                                        int64_t k1, char* lds, AccTile& acc) {
    const int wm = wave_id() / 2 * 128, wn = wave_id() % 2 * 64;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = Acc{};
    if (k0 >= k1) return;
    Mover<T, A_ACROSS, kTileM> ma(a, m0);
    Mover<T, B_ACROSS, kTileN> mb(b, n0);
    constexpr int kStep = Kind<T>::kStep;
    const int64_t last = k1 - kStep;  // behind it the last step is fetched again
    ma.template fetch<0>(a, k0);
    mb.template fetch<0>(b, k0);
    ma.template fetch<1>(a, k0 < last ? k0 + kStep : last);
    mb.template fetch<1>(b, k0 < last ? k0 + kStep : last);
    auto step = [&](int64_t k, auto set) {
        constexpr int SET = decltype(set)::value;
        char* la = lds + SET * (kLdsM + kLdsN);
        char* lb = la + kLdsM;
        ma.template keep<SET>(la);
        mb.template keep<SET>(lb);
        lds_barrier();
        const int64_t next = k + 2 * kStep < last ? k + 2 * kStep : last;
        ma.template fetch<SET>(a, next);
        mb.template fetch<SET>(b, next);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            Fragment<T> fa[4], fb[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) fb[j] = fragment<T, B_ACROSS, kTileN>(lb, wn + j * 32, g);
#pragma unroll
            for (int i = 0; i < 4; ++i) fa[i] = fragment<T, A_ACROSS, kTileM>(la, wm + i * 32, g);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = multiply(fa[i], fb[j], acc[i][j]);
        }
    };
    int64_t k = k0;
    for (; k + kStep < k1; k += 2 * kStep) {
        step(k, std::integral_constant<int, 0>());
        step(k + kStep, std::integral_constant<int, 1>());
    }
    if (k < k1) step(k, std::integral_constant<int, 0>());
    __syncthreads();
}
__device__ __forceinline__ int acc_row(int i, int r) {
    return wave_id() / 2 * 128 + i * 32 + 8 * (r / 4) + 4 * (lane_id() >> 5) + r % 4;
}
__device__ __forceinline__ int acc_col(int j) { return wave_id() % 2 * 64 + j * 32 + (lane_id() & 31); }

// A wavefront's part of a tile, from the place of its lane's first number on: the `left` rows there are, and the columns
// that are asked for; ADD: to what lies there.  One address that goes from row to row (with one for every number, dw of
// 4,096 x 4,096 x 128 fp32 took 54 us, so 48).
template <typename O, bool ADD>
__device__ __forceinline__ void store_tile(const AccTile& acc, float factor, O* __restrict__ to, int64_t stride, int left,
                                           bool first, bool second) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            if (i * 32 + 8 * (r / 4) + r % 4 < left) {
                if (first) to[0] = (O)((ADD ? to[0] : 0.f) + acc[i][0][r] * factor);
                if (second) to[32] = (O)((ADD ? to[32] : 0.f) + acc[i][1][r] * factor);
            }
            to += (r % 4 == 3 ? 5 : 1) * stride;
            asm volatile("" : "+v"(to));
        }
}

// Workgroups go round the eight XCDs, each with an L2 of its own: tiles next to each other, which share an operand, are
// given to workgroups of one XCD.
__device__ __forceinline__ int64_t tile_id() {
    const int64_t all = gridDim.x, b = blockIdx.x, xcd = b % 8, per = all / 8, more = all % 8;
    return xcd * per + (xcd < more ? xcd : more) + b / 8;
}

// ------------------------------------------------------------------------------------------------------- forward
// A workgroup takes 128 rows and every groups-th tile of 256 vertices; a lane keeps maximum and sum of its two columns.
// scores (may be null): the products themselves, as [vertex][row].
template <typename T>
__global__ __attribute__((amdgpu_waves_per_eu(2, 2))) __launch_bounds__(kThreads)
void stats_kernel(LossArgs a, Operand<T> w, Operand<T> x,
                                                         float* __restrict__ scores) {
    __shared__ __align__(16) char lds[kLdsBytes];
    const int64_t id = tile_id(), blocks = a.n_pad / kTile, group = id / blocks, n0 = id % blocks * kTile;
    if (n0 >= (int64_t)a.header->n_live) return;
    float top[2] = {-FLT_MAX, -FLT_MAX}, sum[2] = {};
    for (int64_t v0 = group * kTileM; v0 < a.V; v0 += (int64_t)a.groups * kTileM) {
        AccTile acc;
        product<T, false, false>(w, x, v0, n0, 0, a.dp, lds, acc);
        if (a.V - v0 < kTileM) {  // behind the last vertex
            const int left = (int)(a.V - v0) - acc_row(0, 0);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (i * 32 + 8 * (r / 4) + r % 4 >= left) acc[i][j][r] = -INFINITY;
        }
        if (scores) {
            // the row's address is the wavefront's, where in it the lane's: one register for all stores
            const int wave = __builtin_amdgcn_readfirstlane(wave_id());
            float* at = scores + (v0 + wave / 2 * 128) * a.n_pad + n0 + wave % 2 * 64;
            const uint32_t lane = (uint32_t)(lane_id() >> 5) * 4u * (uint32_t)a.n_pad + (lane_id() & 31);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    at[lane] = acc[i][0][r];
                    at[lane + 32] = acc[i][1][r];
                    at += (r % 4 == 3 ? 5 : 1) * a.n_pad;
                    asm volatile("" : "+s"(at));
                }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float t = top[j];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) t = fmaxf(t, acc[i][j][r]);
            float s = sum[j] * exp_of(top[j] - t);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) s += exp_of(acc[i][j][r] - t);
            top[j] = t;
            sum[j] = s;
        }
    }
    // the two halves of a wavefront, then the two wavefronts with the same columns
    float* shared = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float t2 = __shfl_xor(top[j], 32), s2 = __shfl_xor(sum[j], 32), t = fmaxf(top[j], t2);
        sum[j] = sum[j] * exp_of(top[j] - t) + s2 * exp_of(t2 - t);
        top[j] = t;
        if (wave_id() >= 2 && lane_id() < 32) {
            shared[acc_col(j) * 2] = top[j];
            shared[acc_col(j) * 2 + 1] = sum[j];
        }
    }
    __syncthreads();
    if (wave_id() < 2 && lane_id() < 32)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float t2 = shared[acc_col(j) * 2], s2 = shared[acc_col(j) * 2 + 1], t = fmaxf(top[j], t2);
            const int64_t at = group * a.n_pad + n0 + acc_col(j);
            a.part_max[at] = t;
            a.part_sum[at] = sum[j] * exp_of(top[j] - t) + s2 * exp_of(t2 - t);
        }
}

// Scores of the labels of 16-bit rows, 32 a wavefront: the diagonal of a tile of places against their labels.  It takes a
// thirty-second of what is computed, but has the numbers that the other products have, to the last bit: the same instructions
// over the same operands (x's rows as the instruction's rows, or w's), in the same order.  Bound by fetching both rows, four steps
// at a time: 74,000 labels of 128 bf16 6.4 us, 2,049 of 1,024 fp16, sixty-five wavefronts, 20.
template <typename T, bool W_ROWS>
__global__ __launch_bounds__(kThreads) void label_scores_kernel(LossArgs a, const T* __restrict__ rows, const T* __restrict__ w,
                                                                int64_t w_stride) {
    constexpr int kAtOnce = 4;
    const int lane = lane_id(), col = lane & 31, half = lane >> 5;
    const int64_t slots = (int64_t)a.header->n_live * a.k;
    for (int64_t s0 = ((int64_t)blockIdx.x * 4 + wave_id()) * 32; s0 < slots; s0 += (int64_t)gridDim.x * 128) {
        const int64_t slot = s0 + col < slots ? s0 + col : slots - 1;
        const int32_t label = a.labels_of[slot];
        const T* of_x = rows + (int64_t)fastdiv((uint32_t)slot, a.div_k) * a.dp + half * 8;
        const T* of_w = w + (int64_t)(label >= 0 ? label : 0) * w_stride + half * 8;
        Acc acc = Acc{};
        for (int32_t e = 0; e < a.dp; e += 16 * kAtOnce) {  // rows are padded to 64 numbers
            Fragment<T> x[kAtOnce], v[kAtOnce];
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) {
                x[i] = *reinterpret_cast<const Fragment<T>*>(of_x + e + i * 16);
                v[i] = *reinterpret_cast<const Fragment<T>*>(of_w + e + i * 16);
            }
#pragma unroll
            for (int i = 0; i < kAtOnce; ++i) acc = W_ROWS ? multiply(v[i], x[i], acc) : multiply(x[i], v[i], acc);
        }
        // row `col` of column `col`
        float score = acc[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) score = 8 * (r / 4) + r % 4 == (col & 27) ? acc[r] : score;
        if (half == ((col >> 2) & 1) && s0 + col < slots) a.label_score[slot] = score;
    }
}

// What a vertex weighs in a row's gradient: c p times the row's weight, scaled and rounded to the type.
template <typename T>
__device__ __forceinline__ T weight_of(float score, float lse, float count, float weight) {
    return (T)(weight * (count * exp_of(score - lse)));
}

// lse and loss of the gathered rows, a wavefront each: parts joined, then the products with the labels' rows, or (scores of
// labels are there) what labels weigh in the gradients.
template <typename T>
__global__ __launch_bounds__(kThreads) void loss_kernel(LossArgs a, const T* __restrict__ rows, const T* __restrict__ w,
                                                        int64_t w_stride) {
    const int64_t live = a.header->n_live;
    for (int64_t p = (int64_t)blockIdx.x * 4 + wave_id(); p < live; p += (int64_t)gridDim.x * 4) {
        float top = -FLT_MAX, sum = 0.f;
        for (int32_t g = lane_id(); g < a.groups; g += kWave) {
            const float t2 = a.part_max[(int64_t)g * a.n_pad + p], s2 = a.part_sum[(int64_t)g * a.n_pad + p];
            const float t = fmaxf(top, t2);
            sum = sum * exp_of(top - t) + s2 * exp_of(t2 - t);
            top = t;
        }
        for (int s = 32; s > 0; s >>= 1) {
            const float t2 = __shfl_xor(top, s), s2 = __shfl_xor(sum, s), t = fmaxf(top, t2);
            sum = sum * exp_of(top - t) + s2 * exp_of(t2 - t);
            top = t;
        }
        const int64_t row = a.row_of[p];
        if constexpr (!Kind<T>::kWide)
            if (a.label_score) {
                const int64_t slot = p * a.k + lane_id();
                const bool mine = lane_id() < a.k;
                const int32_t label = mine ? a.labels_of[slot] : -1;
                const float score = label >= 0 ? a.label_score[slot] : 0.f, c = a.count[p], g = a.weight[p], scale = a.header->scale;
                const LabelTerms terms = label_terms<false>(label, score, c, top, sum);
                // The products round a label's weight with all others; it is made here to the last bit, so that taking it off
                // again leaves what the label is in 32 bits.
                const float rounded = (float)weight_of<T>(score, terms.lse, c, g * scale) * (1.f / scale);
                if (mine) a.label_weight[slot] = terms.first ? g * terms.rate + rounded : 0.f;
                float met = score;
                for (int s = 32; s > 0; s >>= 1) met += __shfl_xor(met, s);
                if (lane_id() == 0) {
                    a.place_lse[p] = a.lse[row] = terms.lse;
                    a.loss[row] = c * terms.lse - met;
                }
                continue;
            }
        const float lse = top + logf(sum);
        float met = 0.f;
        constexpr int kAtOnce = 4;  // labels' rows under way
        for (int32_t j0 = 0; j0 < a.k; j0 += kAtOnce) {
            int32_t v[kAtOnce];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) v[j] = j0 + j < a.k ? a.labels_of[p * a.k + j0 + j] : -1;
            for (int32_t e = lane_id(); e < a.d; e += kWave) {
                const float mine = (float)rows[p * a.dp + e];
                float of[kAtOnce];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) of[j] = v[j] >= 0 ? (float)w[(int64_t)v[j] * w_stride + e] : 0.f;
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    if (v[j] >= 0) met = fmaf(mine, of[j], met);
            }
        }
        for (int s = 32; s > 0; s >>= 1) met += __shfl_xor(met, s);
        if (lane_id() == 0) {
            a.place_lse[p] = lse;
            a.lse[row] = lse;
            a.loss[row] = a.count[p] * lse - met;
        }
    }
}

// ------------------------------------------------------------------------------------------------------- few rows
// Up to eight rows against all vertices, forward only: w is read once, as it lies in memory, at the rate it comes, and
// nothing is prepared.  2^log_lanes lanes share a vertex's row, 16 bytes each at a time, four vertices under way; the
// rows of x wait in LDS as floats.  Every workgroup leaves a maximum and a sum per row, a second launch joins them.
constexpr int kFewRows = 8, kFewFloats = 8192, kFewAtOnce = 4, kFewGroups = 1024;

__device__ __forceinline__ float lane_sum(float v, int log_lanes) {
    if (log_lanes > 0) v += __uint_as_float(dpp_moved<0xB1, 0xf>(__float_as_uint(v)));   // lanes 1, 0, 3, 2 of four
    if (log_lanes > 1) v += __uint_as_float(dpp_moved<0x4E, 0xf>(__float_as_uint(v)));   // 2, 3, 0, 1
    if (log_lanes > 2) v += __uint_as_float(dpp_moved<0x141, 0xf>(__float_as_uint(v)));  // eight lanes mirrored
    if (log_lanes > 3) v += __uint_as_float(dpp_moved<0x140, 0xf>(__float_as_uint(v)));  // sixteen
    return v;
}
__device__ __forceinline__ void join_sums(float& top, float& sum, float top2, float sum2) {
    const float t = fmaxf(top, top2);
    sum = sum * exp_of(top - t) + sum2 * exp_of(top2 - t);
    top = t;
}

template <typename T, int VEC, int N>
__global__ __launch_bounds__(kThreads) void few_kernel(LossArgs a, const T* __restrict__ x, int64_t x_stride,
                                                       const T* __restrict__ w, int64_t w_stride, int log_lanes) {
    extern __shared__ __align__(16) float rows[];  // [N][pitch]: a last piece that reaches back has zeros for what it shares
    __shared__ float s_top[4][N], s_sum[4][N];
    const int32_t pitch = (a.d + VEC - 1) / VEC * VEC, back = pitch - a.d, shared_from = pitch - VEC;
    for (int32_t i = threadIdx.x; i < N * pitch; i += kThreads) {
        const int32_t n = i / pitch, e = i - n * pitch;
        const bool held = n < (int32_t)a.n && (e < shared_from || e - shared_from >= back);
        rows[i] = held ? (float)x[n * x_stride + (e < shared_from ? e : e - back)] : 0.f;
    }
    __syncthreads();
    const int lanes = 1 << log_lanes, lane = lane_id() & (lanes - 1), per_wave = kWave >> log_lanes;
    const int64_t per_group = 4 * per_wave * kFewAtOnce;
    const bool upper = lane & (lanes >> 1), odd = lane & (lanes >> 2);
    const int mine = (upper ? 2 : 0) + (odd ? 1 : 0);  // of the vertices under way
    float top[N], sum[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
        top[n] = -FLT_MAX;
        sum[n] = 0.f;
    }
    for (int64_t v0 = blockIdx.x * per_group; v0 < a.V; v0 += gridDim.x * per_group) {
        const int64_t v = v0 + wave_id() * (per_wave * kFewAtOnce) + (lane_id() >> log_lanes);
        float dot[kFewAtOnce][N] = {};
        for (int32_t c = lane * VEC; c < a.d; c += lanes * VEC) {
            const int32_t at = c + VEC <= a.d ? c : a.d - VEC, skip = c - at;  // the last piece reaches back
            Piece<T, VEC> p[kFewAtOnce];
#pragma unroll
            for (int u = 0; u < kFewAtOnce; ++u) {
                const int64_t row = v + u * per_wave < a.V ? v + u * per_wave : a.V - 1;
                p[u] = load_piece<T, VEC>(w + row * w_stride + at);
            }
            if (skip > 0)  // what another lane has is counted there
#pragma unroll
                for (int u = 0; u < kFewAtOnce; ++u)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) p[u].v[e] = e < skip ? (T)0.f : p[u].v[e];
#pragma unroll
            for (int n = 0; n < N; ++n) {
                Piece<float, VEC> f;
                __builtin_memcpy(&f, __builtin_assume_aligned(rows + n * pitch + c, VEC >= 4 ? 16 : 4), sizeof(f));
#pragma unroll
                for (int e = 0; e < VEC; ++e)
#pragma unroll
                    for (int u = 0; u < kFewAtOnce; ++u) dot[u][n] = fmaf((float)p[u].v[e], f.v[e], dot[u][n]);
            }
        }
        // each quarter of the lanes goes on with one of the four vertices, so that an exponential is taken four times less
        // often and fewer sums cross the lanes
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float half[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const float keep = upper ? dot[2 + u][n] : dot[u][n], give = upper ? dot[u][n] : dot[2 + u][n];
                half[u] = keep + __shfl_xor(give, lanes >> 1);
            }
            float score = (odd ? half[1] : half[0]) + __shfl_xor(odd ? half[0] : half[1], lanes >> 2);
            score = lane_sum(score, log_lanes - 2);
            if (v + mine * per_wave < a.V) join_sums(top[n], sum[n], score, 1.f);
        }
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
        for (int s = 32; s >= lanes >> 2; s >>= 1) join_sums(top[n], sum[n], __shfl_xor(top[n], s), __shfl_xor(sum[n], s));
        if (lane_id() == 0) {
            s_top[wave_id()][n] = top[n];
            s_sum[wave_id()][n] = sum[n];
        }
    }
    __syncthreads();
    if (threadIdx.x < N) {
        float t = s_top[0][threadIdx.x], s = s_sum[0][threadIdx.x];
        for (int i = 1; i < 4; ++i) join_sums(t, s, s_top[i][threadIdx.x], s_sum[i][threadIdx.x]);
        a.part_max[(int64_t)blockIdx.x * N + threadIdx.x] = t;
        a.part_sum[(int64_t)blockIdx.x * N + threadIdx.x] = s;
    }
}

// A workgroup per row.
template <typename T>
__global__ __launch_bounds__(kThreads) void few_finish_kernel(LossArgs a, const T* __restrict__ x, int64_t x_stride,
                                                              const T* __restrict__ w, int64_t w_stride, int32_t rows) {
    __shared__ float s_top[4], s_sum[4], s_met[4];
    const int64_t n = blockIdx.x;
    bool bad = false;
    const int32_t c = labels_of_row(a, n, &bad);
    if (n == 0) {
        for (int64_t e = threadIdx.x; e < a.n * a.k; e += kThreads) bad = bad || (int64_t)a.labels[e] >= a.V;
        bad = __syncthreads_or(bad);
        if (threadIdx.x == 0) a.header->status = bad;
    }
    float top = -FLT_MAX, sum = 0.f, met = 0.f;
    for (int32_t g = threadIdx.x; g < a.groups; g += kThreads)
        join_sums(top, sum, a.part_max[(int64_t)g * rows + n], a.part_sum[(int64_t)g * rows + n]);
    for (int s = 32; s > 0; s >>= 1) join_sums(top, sum, __shfl_xor(top, s), __shfl_xor(sum, s));
    for (int32_t j = wave_id(); j < a.k; j += 4) {
        const int32_t v = a.labels[n * a.k + j];
        if (v < 0 || (int64_t)v >= a.V) continue;
        for (int32_t e = lane_id(); e < a.d; e += kWave)
            met = fmaf((float)x[n * x_stride + e], (float)w[(int64_t)v * w_stride + e], met);
    }
    for (int s = 32; s > 0; s >>= 1) met += __shfl_xor(met, s);
    if (lane_id() == 0) {
        s_top[wave_id()] = top;
        s_sum[wave_id()] = sum;
        s_met[wave_id()] = met;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    for (int i = 1; i < 4; ++i) {
        join_sums(top, sum, s_top[i], s_sum[i]);
        met += s_met[i];
    }
    const float lse = top + logf(sum);
    a.lse[n] = c > 0 ? lse : 0.f;
    a.loss[n] = c > 0 ? (float)c * lse - met : 0.f;
}

// ------------------------------------------------------------------------------------------------------ gradient
// How often each of 256 vertices from v0 on is among the labels of 128 places from n0 on: counts[place][vertex], a lane a
// place.
constexpr int kCountPitch = kTileM + 4;
__device__ __forceinline__ void count_labels(const LossArgs& a, int64_t v0, int64_t n0, uint8_t* counts) {
    if (threadIdx.x < kTile) {
        uint8_t* mine = counts + threadIdx.x * kCountPitch;
        for (int e = 0; e < kTileM / 4; ++e) reinterpret_cast<uint32_t*>(mine)[e] = 0;
        for (int32_t j = 0; j < a.k; ++j) {
            const int64_t v = a.labels_of[(n0 + threadIdx.x) * a.k + j];
            if (v >= v0 && v < v0 + kTileM) mine[v - v0]++;
        }
    }
    __syncthreads();
}

// What a vertex weighs in a row's gradient, as [vertex][row]: 256 vertices of the piece from v_first on, 128 rows.  In fp32
// it is g (c p - count).  In 16 bits, to which it is rounded for the matrix instructions, it is g c p alone: one label can
// outweigh all vertices, and the rounding of its count would be that of the whole gradient (fp16, relative to 64 bits, 3.2e-4
// and without it 2.1e-4, which is the rounding of the result).  There the labels' rows are taken off afterwards, in 32 bits,
// with the rounded g c p of theirs: where a row is fitted its rounding, 2^-9 of it in bf16, would outweigh g (c p - count).
template <typename T>
__global__ __attribute__((amdgpu_waves_per_eu(2, 2))) __launch_bounds__(kThreads)
void probs_kernel(LossArgs a, Operand<T> w, Operand<T> x, int64_t v_first,
                                                         T* __restrict__ probs) {
    __shared__ __align__(16) char lds[kLdsBytes];
    const int64_t id = tile_id(), blocks = a.n_pad / kTile;
    const int64_t n0 = id % blocks * kTile, m0 = id / blocks * kTileM, v0 = v_first + m0;
    if (n0 >= (int64_t)a.header->n_live) return;
    AccTile acc;
    product<T, false, false>(w, x, v0, n0, 0, a.dp, lds, acc);
    uint8_t* counts = reinterpret_cast<uint8_t*>(lds);
    if constexpr (Kind<T>::kWide) count_labels(a, v0, n0, counts);
    const float scale = a.header->scale;
    const int left = (int)(a.V - v0 < kTileM ? a.V - v0 : kTileM) - acc_row(0, 0);
    float lse[2], c[2], g[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t place = n0 + acc_col(j);
        lse[j] = a.place_lse[place];
        c[j] = a.count[place];
        g[j] = a.weight[place] * scale;
    }
    T* to = probs + (m0 + acc_row(0, 0)) * a.n_pad + n0 + acc_col(0);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                T weight = (T)0.f;
                if (i * 32 + 8 * (r / 4) + r % 4 < left && c[j] > 0.f) {
                    if constexpr (Kind<T>::kWide)
                        weight = g[j] * (c[j] * exp_of(acc[i][j][r] - lse[j]) -
                                         (float)counts[acc_col(j) * kCountPitch + acc_row(i, r)]);
                    else
                        weight = weight_of<T>(acc[i][j][r], lse[j], c[j], g[j]);
                }
                to[j * 32] = weight;
            }
            to += (r % 4 == 3 ? 5 : 1) * a.n_pad;
            asm volatile("" : "+v"(to));
        }
}

// The same from scores that were kept, of the piece of vertices from v_first on; fp32: in their place.  A lane has four places.
template <typename T>
__global__ __launch_bounds__(kThreads) void kept_kernel(LossArgs a, const float* scores, int64_t v_first, T* probs) {
    __shared__ __align__(16) uint8_t counts[Kind<T>::kWide ? kTile * kCountPitch : 16];
    constexpr int kLanes = kTile / 4, kRows = kThreads / kLanes, kAtOnce = 8;
    const int64_t id = tile_id(), blocks = a.n_pad / kTile;
    const int64_t n0 = id % blocks * kTile, m0 = id / blocks * kTileM, v0 = v_first + m0;
    if (n0 >= (int64_t)a.header->n_live) return;
    if constexpr (Kind<T>::kWide) count_labels(a, v0, n0, counts);
    const float scale = a.header->scale;
    const int col = threadIdx.x % kLanes * 4, first = threadIdx.x / kLanes;
    float lse[4], c[4], g[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        lse[e] = a.place_lse[n0 + col + e];
        c[e] = a.count[n0 + col + e];
        g[e] = a.weight[n0 + col + e] * scale;
    }
    for (int r0 = first; r0 < kTileM; r0 += kRows * kAtOnce) {
        Piece<float, 4> s[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) s[i] = load_piece<float, 4>(scores + (v0 + r0 + i * kRows) * a.n_pad + n0 + col);
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            const int row = r0 + i * kRows;
            Piece<T, 4> p;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p.v[e] = (T)0.f;
                if (v0 + row < a.V && c[e] > 0.f) {
                    if constexpr (Kind<T>::kWide)
                        p.v[e] = g[e] * (c[e] * exp_of(s[i].v[e] - lse[e]) - (float)counts[(col + e) * kCountPitch + row]);
                    else
                        p.v[e] = weight_of<T>(s[i].v[e], lse[e], c[e], g[e]);
                }
            }
            store_piece<T, 4>(probs + (m0 + row) * a.n_pad + n0 + col, p);
        }
    }
}

// The rows under every vertex that is a label, summed: by vertex, the row of the sums or -1 (null: nothing to take off).
struct Labels {
    const int32_t* row;
    const float* sums;
};

// dw of 256 vertices of the piece and 128 numbers of their rows, over a share of the rows with labels: the result where
// there is one share, else its part.
template <typename T>
__global__ __attribute__((amdgpu_waves_per_eu(2, 2))) __launch_bounds__(kThreads)
void dw_kernel(LossArgs a, Operand<T> probs, Operand<T> x, int64_t v_first,
                                                      T* __restrict__ dw, int64_t dw_stride, float* __restrict__ parts,
                                                      int64_t part_rows, int32_t shares, Labels labels) {
    __shared__ __align__(16) char lds[kLdsBytes];
    // the tiles of one share, and of one tile of vertices, next to each other
    const int64_t id = tile_id(), d_tiles = (a.dp + kTileN - 1) / kTileN, v_tiles = gridDim.x / (d_tiles * shares);
    const int64_t d0 = id % d_tiles * kTileN, m0 = id / d_tiles % v_tiles * kTileM, share = id / (d_tiles * v_tiles);
    const int64_t steps = ((int64_t)a.header->n_live + Kind<T>::kStep - 1) / Kind<T>::kStep;
    const int64_t k0 = steps * share / shares * Kind<T>::kStep, k1 = steps * (share + 1) / shares * Kind<T>::kStep;
    AccTile acc;
    product<T, false, true>(probs, x, m0, d0, k0, k1, lds, acc);
    const float scale = a.header->scale, back = 1.f / scale;  // a power of two
    if constexpr (!Kind<T>::kWide)
        if (labels.row && shares == 1) {
            // Few vertices are labels: the wavefront's 128 as bits, and what is taken off only where one is.  All of it before
            // the first store, which a load's wait would wait for too.
            int32_t sum[2];
            uint64_t any[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t v = v_first + m0 + wave_id() / 2 * 128 + h * 64 + lane_id();
                sum[h] = v < a.V ? labels.row[v] : -1;
                any[h] = __ballot(sum[h] >= 0);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int at = i * 32 + 8 * (r / 4) + r % 4;  // and 4 behind, the other half of the wavefront
                    if (((any[at / 64] >> (at % 64)) & 0x11u) == 0) continue;
                    const int32_t mine = __shfl(sum[at / 64], at % 64 + 4 * (lane_id() >> 5));
                    if (mine >= 0)
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            if (d0 + acc_col(j) < a.dp)
                                acc[i][j][r] -= labels.sums[(int64_t)mine * a.dp + d0 + acc_col(j)] * scale;
                }
        }
    const int64_t m = m0 + acc_row(0, 0), e = d0 + acc_col(0);
    const int left = (int)(a.V - v_first - m < kTileM ? a.V - v_first - m : kTileM);  // rows from here on
    if (shares == 1)
        store_tile<T, false>(acc, back, dw + (v_first + m) * dw_stride + e, dw_stride, left, e < a.d, e + 32 < a.d);
    else
        store_tile<float, false>(acc, 1.f, parts + (share * part_rows + m) * a.dp + e, a.dp, left, e < a.d, e + 32 < a.d);
}

// Four numbers of a row, summed over the shares' parts: a wavefront has 256 numbers of one row, eight parts under way.
template <typename T>
__device__ __forceinline__ void join_parts(const float* __restrict__ parts, int32_t shares, int64_t share_size, float back,
                                           const float (&less)[4], int32_t e, int32_t d, T* __restrict__ to) {
    constexpr int kAtOnce = 8;
    float sum[4] = {};
    for (int32_t s0 = 0; s0 < shares; s0 += kAtOnce) {
        Piece<float, 4> v[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
            v[i] = Piece<float, 4>{};
            if (s0 + i < shares) v[i] = load_piece<float, 4>(parts + (s0 + i) * share_size + e);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[q] += v[i].v[q];
    }
    Piece<T, 4> o;
#pragma unroll
    for (int q = 0; q < 4; ++q) o.v[q] = (T)(sum[q] * back - less[q]);
    if (e + 4 <= d) {
        store_piece<T, 4>(to + e, o);
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (e + q < d) to[e + q] = o.v[q];
    }
}
constexpr int kLeastShare = 64;  // of the summed dimension: a multiple of every Kind's step
constexpr int kJoinWidth = kWave * 4;
template <typename T>
__global__ __launch_bounds__(kThreads) void dw_join_kernel(LossArgs a, const float* __restrict__ parts, int32_t shares,
                                                           int64_t part_rows, int64_t v_first, int64_t here, T* __restrict__ dw,
                                                           int64_t dw_stride, Labels labels) {
    const float back = 1.f / a.header->scale;
    const int32_t across = (a.d + kJoinWidth - 1) / kJoinWidth;
    for (int64_t i = (int64_t)blockIdx.x * 4 + wave_id(); i < here * across; i += (int64_t)gridDim.x * 4) {
        const int64_t m = i / across;
        const int32_t e = (int32_t)(i - m * across) * kJoinWidth + lane_id() * 4;
        if (e >= a.d) continue;
        float less[4] = {};
        const int32_t at = labels.row ? labels.row[v_first + m] : -1;
        if (at >= 0) {
            const Piece<float, 4> v = load_piece<float, 4>(labels.sums + (int64_t)at * a.dp + e);
#pragma unroll
            for (int q = 0; q < 4; ++q) less[q] = v.v[q];
        }
        join_parts<T>(parts + m * a.dp, shares, part_rows * a.dp, back, less, e, a.d, dw + (v_first + m) * dw_stride);
    }
}

// dx of 256 rows and 128 numbers, summed over a share of the piece's vertices.
template <typename T>
__global__ __attribute__((amdgpu_waves_per_eu(2, 2))) __launch_bounds__(kThreads)
void dx_kernel(LossArgs a, Operand<T> probs, Operand<T> w, int64_t v_first,
                                                      int64_t v_share, int64_t v_end, int first_piece,
                                                      float* __restrict__ parts) {
    __shared__ __align__(16) char lds[kLdsBytes];
    // the tiles of one share, and of one tile of rows, next to each other
    const int64_t id = tile_id(), d_tiles = (a.dp + kTileN - 1) / kTileN, n_tiles = a.n_pad / kTileM;
    const int64_t d0 = id % d_tiles * kTileN, n0 = id / d_tiles % n_tiles * kTileM, share = id / (d_tiles * n_tiles);
    if (n0 >= (int64_t)a.header->n_live) return;
    const int64_t k0 = share * v_share;
    const int64_t k1 = k0 + v_share < v_end ? k0 + v_share : v_end;
    Operand<T> piece = w;
    piece.base += v_first * w.stride;
    piece.rows -= v_first;
    AccTile acc;
    product<T, true, true>(probs, piece, n0, d0, k0, k1, lds, acc);
    const int64_t e = d0 + acc_col(0);
    float* to = parts + (share * a.n_pad + n0 + acc_row(0, 0)) * a.dp + e;
    if (first_piece)
        store_tile<float, false>(acc, 1.f, to, a.dp, kTileM, e < a.dp, e + 32 < a.dp);
    else
        store_tile<float, true>(acc, 1.f, to, a.dp, kTileM, e < a.dp, e + 32 < a.dp);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void dx_join_kernel(LossArgs a, const float* __restrict__ parts, int32_t shares,
                                                           Operand<T> w, T* __restrict__ dx, int64_t dx_stride) {
    const float back = 1.f / a.header->scale;
    const int32_t across = (a.d + kJoinWidth - 1) / kJoinWidth;
    const int64_t all = (int64_t)a.header->n_live * across;
    for (int64_t i = (int64_t)blockIdx.x * 4 + wave_id(); i < all; i += (int64_t)gridDim.x * 4) {
        const int64_t p = i / across;
        const int32_t e = (int32_t)(i - p * across) * kJoinWidth + lane_id() * 4;
        if (e >= a.d) continue;
        float less[4] = {};
        if constexpr (!Kind<T>::kWide) {  // the rows of the labels
            constexpr int kAtOnce = 4;
            for (int32_t j0 = 0; j0 < a.k; j0 += kAtOnce) {
                Piece<T, 4> v[kAtOnce];
                float f[kAtOnce];
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    const int32_t label = j0 + j < a.k ? a.labels_of[p * a.k + j0 + j] : -1;
                    v[j] = Piece<T, 4>{};
                    f[j] = 0.f;
                    if (label >= 0) {
                        v[j] = load_piece<T, 4>(w.base + label * w.stride + e);
                        f[j] = a.label_weight[p * a.k + j0 + j];
                    }
                }
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
                    for (int q = 0; q < 4; ++q) less[q] = fmaf(f[j], (float)v[j].v[q], less[q]);
            }
        }
        join_parts<T>(parts + p * a.dp, shares, a.n_pad * a.dp, back, less, e, a.d, dx + a.row_of[p] * dx_stride);
    }
}

// --------------------------------------------------------------------------------------------------------- layout
// A launch holds fewer than 2^32 lanes: wavefronts go on to further rows from here on.
inline dim3 wave_per(int64_t rows) {
    const int64_t groups = (rows + 3) / 4;
    return dim3((unsigned)(groups < (1 << 20) ? groups : 1 << 20));
}
inline size_t up256(size_t x) { return (x + 255) / 256 * 256; }

struct LossPlan {
    int64_t n_pad, blocks, piece;   // piece: vertices at a time (a multiple of a tile)
    int32_t dp, groups, shares, dw_shares;
    bool few;                       // few rows, forward
    bool sweep;                     // rows short enough for nd_sweep.hip
    bool kept;                      // the scores of all rows and vertices stay for the gradient
    // labels by vertex: the grouping's arrays, sums of their rows
    int64_t label_groups;
    SortPlan sort;
    size_t o_ctl, o_keys[2], o_vals[2], o_hist, o_scratch, o_gkey, o_gstart, o_label_row, o_label_sums, o_tile_group,
        o_label_parts;
    size_t o_label_score, o_label_weight, o_factor;
    size_t o_labels, o_live, o_weight, o_bad, o_row, o_count, o_gweight, o_lse, o_max, o_sum, o_rows, o_w, o_probs, o_scores,
        o_parts, o_dw_parts, total;
};
// 57,000 vertices, rows of 128 numbers in bf16: 8.4 us for one row, 17.8 for eight; nine rows the other way 24.5 (fp32: 19 for
// eight, 48 for nine; rows of 1,000 in bf16: 49 and 87).
bool few_rows(int64_t n, int32_t d, bool grad) {
    if (grad || n < 1 || n > kFewRows) return false;
    int rows = 1;
    while (rows < n) rows *= 2;
    return rows * (int64_t)d <= kFewFloats;
}
LossPlan plan_loss(int64_t n, int64_t V, int32_t d, int32_t k, int dtype, bool grad) {
    LossPlan p{};
    const int64_t b = (int64_t)dtype_bytes(dtype), step = 128 / b;
    p.few = few_rows(n, d, grad);
    if (p.few) {
        p.o_max = sizeof(LossHeader);
        p.o_sum = p.o_max + kFewGroups * kFewRows * 4;
        p.total = p.o_sum + kFewGroups * kFewRows * 4;
        return p;
    }
    p.sweep = dtype != ND_F32 && sweep_width(d) > 0;
    p.dp = p.sweep ? sweep_width(d) : (int32_t)((d + step - 1) / step * step);
    p.blocks = n > 0 ? (n + kTile - 1) / kTile : 1;  // without rows: the header is written all the same
    p.n_pad = (p.blocks * kTile + kTileM - 1) / kTileM * kTileM;
    const int64_t v_tiles = (V + kTileM - 1) / kTileM;
    // two workgroups per compute unit at a time, and all of them with about as many tiles
    const int64_t n_tiles = p.n_pad / kTile, groups = n_tiles < 512 ? 512 / n_tiles : 1;
    p.groups = (int32_t)(groups < v_tiles ? groups : v_tiles);
    int64_t piece_tiles = (int64_t)(kPieceBytes / (size_t)(p.n_pad * kTileM * b));
    if (piece_tiles < 1) piece_tiles = 1;
    if (piece_tiles > 32768) piece_tiles = 32768;
    if (piece_tiles > v_tiles) piece_tiles = v_tiles;
    // Scores are kept for the gradient where rows are long, so that to write and read them takes less than to make them again.
    // Both ways with what comes before the products, us: 2,304 x 57,000 x 1,024 fp16 545 and 674, 512 x 20,000 x 512 bf16 42
    // and 49, 4,096 x 20,000 x 512 232 and 236, but 2,000 x 20,000 x 320 104 and 93; fp32 4,096 x 4,096 x 128 72 and 94,
    // 4,096 x 57,000 x 64 713 and 709.
    p.kept = grad && !p.sweep && v_tiles <= 32768 && p.n_pad * v_tiles * kTileM * 4 <= kKeptBytes &&
             p.dp >= (dtype == ND_F32 ? 128 : 512);
    if (p.kept && dtype == ND_F32) piece_tiles = v_tiles;  // probabilities take the scores' place
    p.piece = piece_tiles * kTileM;
    // The summed dimension is shared out where there are fewer tiles than two per compute unit; one more share than that
    // would take as long as twice as many.  More than 16 shares cost more to join than the second workgroup of a compute
    // unit gives (4,096 x 4,096 x 128 fp32: 16 and 32 shares both 55 us, and 7 and 12 to join), so beyond them it is one
    // (1,000 x 20,000 x 100 fp32: dx 185 us with 16 shares, 60 with 64).
    auto shares = [](int64_t tiles, int64_t most) {
        const int64_t two = tiles < 512 ? 512 / tiles : 1, one = tiles < 16 ? 256 / tiles : 16;
        const int64_t s = two < one ? two : one;
        return (int32_t)(s < most ? s : most);
    };
    p.shares = shares(p.n_pad / kTileM * ((p.dp + kTileN - 1) / kTileN), p.piece / kLeastShare);
    p.dw_shares = shares(piece_tiles * ((p.dp + kTileN - 1) / kTileN), p.blocks * kTile / kLeastShare);
    size_t o = sizeof(LossHeader);
    auto take = [&](size_t bytes) {
        const size_t at = o;
        o += up256(bytes);
        return at;
    };
    p.o_live = take((size_t)p.blocks * 4);
    p.o_weight = take((size_t)p.blocks * 4);
    p.o_bad = take((size_t)p.blocks * 4);
    p.o_row = take((size_t)p.n_pad * 4);
    p.o_count = take((size_t)p.n_pad * 4);
    p.o_gweight = take((size_t)p.n_pad * 4);
    p.o_lse = take((size_t)p.n_pad * 4);
    p.o_labels = take((size_t)p.n_pad * (size_t)k * 4);
    p.o_rows = take((size_t)p.n_pad * (size_t)p.dp * (size_t)b);
    p.o_w = take((size_t)V * (size_t)p.dp * (size_t)b);
    auto take_labels = [&] {
        const size_t slots = (size_t)n * (size_t)k, some = slots > 0 ? slots : 1;
        p.o_label_score = take(some * 4);
        p.o_label_weight = take(some * 4);
        p.o_factor = take((size_t)p.n_pad * 4);
        const size_t tiles = (size_t)group_sum_tiles((int64_t)slots, p.dp, dtype);
        p.label_groups = (int64_t)slots < V ? (int64_t)slots : V;
        p.sort = make_sort_plan((int64_t)slots, V);
        p.o_ctl = take(sizeof(StepCtl));
        for (int i = 0; i < 2; ++i) {
            p.o_keys[i] = take(some * 4);
            p.o_vals[i] = take(some * 4);
        }
        p.o_hist = take(sort_hist_bytes(p.sort));
        p.o_scratch = take(seg_scratch_bytes((int64_t)slots));
        p.o_gkey = take(some * 4);
        p.o_gstart = take((some + 1) * 4);
        p.o_label_row = take((size_t)V * 4);
        p.o_label_sums = take((size_t)p.label_groups * (size_t)p.dp * 4);
        p.o_tile_group = take(tiles * 4);
        p.o_label_parts = take(tiles * 2 * (size_t)p.dp * 4);
    };
    if (p.sweep) {
        // the sweeps run one after the other and share the segments' memory
        size_t held = 0, sums = 0;
        for (int mode = kSweepLse; mode <= (grad ? kSweepDw : kSweepLse); ++mode) {
            const size_t rows = (size_t)sweep_rows(mode, mode == kSweepDw ? V : n, mode == kSweepDw ? n : V, p.dp);
            if (rows > held) held = rows;
            if (mode > kSweepRest && rows > sums) sums = rows;
        }
        p.o_max = take(held * 4);
        p.o_sum = take(held * 4);
        p.o_parts = take(sums * (size_t)p.dp * 4);
        if (grad) take_labels();
        p.total = o;
        return p;
    }
    p.o_max = take((size_t)p.groups * (size_t)p.n_pad * 4);
    p.o_sum = take((size_t)p.groups * (size_t)p.n_pad * 4);
    if (grad) {
        if (dtype != ND_F32) take_labels();
        p.o_probs = take((size_t)p.piece * (size_t)p.n_pad * (size_t)b);
        p.o_scores = p.kept && b < 4 ? take((size_t)(v_tiles * kTileM) * (size_t)p.n_pad * 4) : p.o_probs;
        p.o_parts = take((size_t)p.shares * (size_t)p.n_pad * (size_t)p.dp * 4);
        p.o_dw_parts = p.dw_shares > 1 ? take((size_t)p.dw_shares * (size_t)p.piece * (size_t)p.dp * 4) : 0;
    }
    p.total = o;
    return p;
}

int check_loss_sizes(int64_t n, int64_t V, int32_t d, int32_t k, int dtype) {
    int rc = check_row_type(dtype, d);
    if (rc != ND_OK) return rc;
    if (n < 0 || V < 1 || k < 1) {
        set_error("n must not be negative, V and k at least 1");
        return ND_ERR_BAD_ARGUMENT;
    }
    if (n >= (1ll << 30) || V >= (1ll << 31) || k > ND_MAX_LABELS || n * (int64_t)k >= (1ll << 31)) {
        set_error("fewer than 2^30 rows, 2^31 vertices and 2^31 labels, at most %d labels per row", ND_MAX_LABELS);
        return ND_ERR_TOO_LARGE;
    }
    return ND_OK;
}

struct LossCall {
    const void *x, *w;
    int64_t x_stride, w_stride;
    int dtype;
    int64_t n, V;
    int32_t d, k;
    const int32_t* labels;
    const float* row_weight;
    float *loss, *lse;
    void *dx, *dw;
    int64_t dx_stride, dw_stride;
    bool grad;
};

// The rows under every vertex that is a label, times what they weigh, summed: what labels take off dw.
template <typename T>
int sum_labels(const LossArgs& a, const LossPlan& p, char* ws, const T* rows, SweepParts* parts, hipStream_t stream) {
    const int64_t slots = a.n * a.k;
    StepCtl* ctl = (StepCtl*)(ws + p.o_ctl);
    int32_t *keys = nullptr, *vals = nullptr, *g_key = (int32_t*)(ws + p.o_gkey), *g_start = (int32_t*)(ws + p.o_gstart);
    int rc = sort_pairs(a.labels_of, slots, (int32_t)a.V, p.sort, (int32_t*)(ws + p.o_keys[0]), (int32_t*)(ws + p.o_vals[0]),
                        (int32_t*)(ws + p.o_keys[1]), (int32_t*)(ws + p.o_vals[1]), (uint32_t*)(ws + p.o_hist), ctl, nullptr,
                        1, nullptr, &keys, &vals, stream);
    if (rc == ND_OK) rc = build_groups(keys, slots, ctl, g_key, g_start, (uint32_t*)(ws + p.o_scratch), nullptr, 0, stream);
    if (rc != ND_OK) return rc;
    GroupSum g{};
    g.slots = vals;
    g.start = g_start;
    g.ctl = ctl;
    g.mark_key = g_key;
    g.mark = a.label_row;
    g.n_pairs = slots;
    g.n_groups = g.out_rows = p.label_groups;
    g.out_stride = a.dp;
    g.tile_group = (int32_t*)(ws + p.o_tile_group);
    g.parts = (float*)(ws + p.o_label_parts);
    parts->label_row = a.label_row;
    parts->label_sums = (const float*)(ws + p.o_label_sums);
    return group_sum_floats<T>(rows, a.dp, p.n_pad, a.dp, a.k, a.label_weight, g, (float*)(ws + p.o_label_sums), stream);
}

template <typename T, int VEC, int N>
void launch_few(LossArgs& a, const LossCall& c, hipStream_t stream) {
    int log_lanes = 2;  // four lanes at least, one for each vertex under way
    while (log_lanes < 6 && (VEC << log_lanes) < c.d) ++log_lanes;
    const int64_t per = 4 * (kWave >> log_lanes) * kFewAtOnce, groups = (c.V + per - 1) / per;
    a.groups = (int32_t)(groups < kFewGroups ? groups : kFewGroups);
    hipLaunchKernelGGL((few_kernel<T, VEC, N>), dim3((unsigned)a.groups), dim3(kThreads),
                       (size_t)N * ((c.d + VEC - 1) / VEC * VEC) * 4, stream, a,
                       (const T*)c.x, c.x_stride, (const T*)c.w, c.w_stride, log_lanes);
    hipLaunchKernelGGL(few_finish_kernel<T>, dim3((unsigned)c.n), dim3(kThreads), 0, stream, a, (const T*)c.x, c.x_stride,
                       (const T*)c.w, c.w_stride, (int32_t)N);
}
template <typename T, int VEC>
int run_few(LossArgs& a, const LossCall& c, hipStream_t stream) {
    if (c.n == 1)
        launch_few<T, VEC, 1>(a, c, stream);
    else if (c.n == 2)
        launch_few<T, VEC, 2>(a, c, stream);
    else if (c.n <= 4)
        launch_few<T, VEC, 4>(a, c, stream);
    else
        launch_few<T, VEC, kFewRows>(a, c, stream);
    ND_HIP_CHECK(hipGetLastError());
    return ND_OK;
}

template <typename T>
int run_loss(const LossCall& c, const LossPlan& p, char* ws, hipStream_t stream) {
    LossArgs a{};
    a.n = c.n;
    a.V = c.V;
    a.n_pad = p.n_pad;
    a.d = c.d;
    a.dp = p.dp;
    a.k = c.k;
    a.labels = c.labels;
    a.row_weight = c.row_weight;
    a.loss = c.loss;
    a.lse = c.lse;
    a.header = (LossHeader*)ws;
    a.block_live = (uint32_t*)(ws + p.o_live);
    a.block_weight = (float*)(ws + p.o_weight);
    a.block_bad = (uint32_t*)(ws + p.o_bad);
    a.row_of = (int32_t*)(ws + p.o_row);
    a.count = (float*)(ws + p.o_count);
    a.weight = (float*)(ws + p.o_gweight);
    a.place_lse = (float*)(ws + p.o_lse);
    a.part_max = (float*)(ws + p.o_max);
    a.part_sum = (float*)(ws + p.o_sum);
    a.groups = p.groups;
    a.labels_of = (int32_t*)(ws + p.o_labels);
    a.div_k = make_fastdiv((uint32_t)c.k);
    if (p.few) {
        constexpr int kWide = kChunk / (int)sizeof(T);
        return c.d >= kWide ? run_few<T, kWide>(a, c, stream) : run_few<T, 1>(a, c, stream);
    }
    if (sizeof(T) == 2 && c.grad && c.n > 0) {
        if (c.dw) a.label_row = (int32_t*)(ws + p.o_label_row);
        a.label_score = (float*)(ws + p.o_label_score);
        a.label_weight = (float*)(ws + p.o_label_weight);
        if (p.sweep) a.place_factor = (float*)(ws + p.o_factor);
    }
    T* rows = (T*)(ws + p.o_rows);
    const unsigned blocks = (unsigned)p.blocks;
    const Spread spread = make_spread(p.dp, kChunk / (int)sizeof(T));
    if (blocks > 1) hipLaunchKernelGGL(count_kernel, dim3(blocks), dim3(kTile), 0, stream, a);
    if (p.blocks > kScanBlocks)
        hipLaunchKernelGGL(scan_blocks_kernel<T>, dim3(1), dim3(kScanThreads), 0, stream, a, (int32_t)blocks);
    hipLaunchKernelGGL(place_kernel<T>, dim3(blocks), dim3(kTile), 0, stream, a, (int32_t)blocks);
    hipLaunchKernelGGL(gather_kernel<T>, spread_grid(spread, p.n_pad), dim3(kThreads), 0, stream, a, spread, (const T*)c.x,
                       c.x_stride, rows, c.grad ? (T*)c.dx : nullptr, c.dx_stride);
    const T* w = (const T*)c.w;
    int64_t w_stride = c.w_stride;
    // a stride beyond 2^24 numbers would leave 32 bits within a sweep's unit
    const bool as_it_is = c.d == p.dp && w_stride < (1 << 24) && w_stride * (int64_t)sizeof(T) % kChunk == 0 &&
                          (uintptr_t)w % kChunk == 0;
    if (!as_it_is) {
        T* padded = (T*)(ws + p.o_w);
        hipLaunchKernelGGL(pad_kernel<T>, spread_grid(spread, c.V), dim3(kThreads), 0, stream, w, w_stride, c.V, c.d, p.dp,
                           spread, padded);
        w = padded;
        w_stride = p.dp;
    }
    if constexpr (sizeof(T) == 2) {
        if (a.label_score) {
            const int64_t groups = (c.n * c.k + 127) / 128;
            const dim3 grid((unsigned)(groups < (1 << 20) ? groups : 1 << 20));
            if (p.sweep)
                hipLaunchKernelGGL((label_scores_kernel<T, false>), grid, dim3(kThreads), 0, stream, a, rows, w, w_stride);
            else
                hipLaunchKernelGGL((label_scores_kernel<T, true>), grid, dim3(kThreads), 0, stream, a, rows, w, w_stride);
        }
        if (p.sweep) {
            SweepParts parts{a.part_max, a.part_sum, (float*)(ws + p.o_parts), nullptr, nullptr};
            const int mode = !c.grad ? kSweepLse : c.dx ? kSweepDx : kSweepRest;
            int rc = ND_OK;
            if (c.n > 0) {
                rc = sweep<T>(mode, a, rows, w, w_stride, parts, nullptr, 0, stream);
                if (rc == ND_OK) rc = sweep_finish<T>(mode, a, rows, w, w_stride, parts, (T*)c.dx, c.dx_stride, stream);
            }
            if (rc == ND_OK && c.grad && c.dw && c.n > 0) rc = sum_labels<T>(a, p, ws, rows, &parts, stream);
            if (rc == ND_OK && c.grad && c.dw)
                rc = sweep<T>(kSweepDw, a, rows, w, w_stride, parts, (T*)c.dw, c.dw_stride, stream);
            return rc;
        }
    }
    const Operand<T> ow{w, w_stride, c.V, p.dp}, ox{rows, p.dp, p.n_pad, p.dp};
    if (c.n > 0) {
        hipLaunchKernelGGL(stats_kernel<T>, dim3((unsigned)(p.n_pad / kTile * p.groups)), dim3(kThreads), 0, stream, a, ow, ox,
                           p.kept ? (float*)(ws + p.o_scores) : nullptr);
        hipLaunchKernelGGL(loss_kernel<T>, wave_per(c.n), dim3(kThreads), 0, stream, a, rows, w, w_stride);
    }
    if (c.grad) {
        T* probs = (T*)(ws + p.o_probs);
        float* parts = (float*)(ws + p.o_parts);
        float* dw_parts = (float*)(ws + p.o_dw_parts);
        Labels labels{};
        if constexpr (sizeof(T) == 2)
            if (c.dw && c.n > 0) {
                SweepParts sums{};
                const int rc = sum_labels<T>(a, p, ws, rows, &sums, stream);
                if (rc != ND_OK) return rc;
                labels = {sums.label_row, sums.label_sums};
            }
        const int64_t d_tiles = (p.dp + kTileN - 1) / kTileN, join_columns = (c.d + kJoinWidth - 1) / kJoinWidth;
        for (int64_t v = 0; v < c.V; v += p.piece) {
            const int64_t here = c.V - v < p.piece ? c.V - v : p.piece, tiles = (here + kTileM - 1) / kTileM;
            const Operand<T> op{probs, p.n_pad, tiles * kTileM, (int32_t)p.n_pad};
            const dim3 all((unsigned)(p.n_pad / kTile * tiles));
            if (c.n > 0 && p.kept)
                hipLaunchKernelGGL(kept_kernel<T>, all, dim3(kThreads), 0, stream, a, (const float*)(ws + p.o_scores), v, probs);
            else if (c.n > 0)
                hipLaunchKernelGGL(probs_kernel<T>, all, dim3(kThreads), 0, stream, a, ow, ox, v, probs);
            if (c.dw)
                hipLaunchKernelGGL(dw_kernel<T>, dim3((unsigned)(tiles * d_tiles * p.dw_shares)), dim3(kThreads), 0, stream, a, op,
                                   ox, v, (T*)c.dw, c.dw_stride, dw_parts, p.piece, p.dw_shares, labels);
            if (c.dw && p.dw_shares > 1)
                hipLaunchKernelGGL(dw_join_kernel<T>, wave_per(here * join_columns), dim3(kThreads), 0, stream, a, dw_parts,
                                   p.dw_shares, p.piece, v, here, (T*)c.dw, c.dw_stride, labels);
            if (c.dx && c.n > 0) {
                const int64_t share = (tiles * kTileM / kLeastShare + p.shares - 1) / p.shares * kLeastShare;
                hipLaunchKernelGGL(dx_kernel<T>, dim3((unsigned)(p.n_pad / kTileM * d_tiles * p.shares)), dim3(kThreads), 0, stream,
                                   a, op, ow, v, share, tiles * kTileM, (int)(v == 0), parts);
            }
        }
        if (c.dx && c.n > 0)
            hipLaunchKernelGGL(dx_join_kernel<T>, wave_per(c.n * join_columns), dim3(kThreads), 0, stream, a, parts, p.shares,
                               ow, (T*)c.dx, c.dx_stride);
    }
    ND_HIP_CHECK(hipGetLastError());
    return ND_OK;
}

int softmax_loss(const LossCall& c, void* workspace, size_t workspace_bytes, hipStream_t stream) {
    int rc = check_loss_sizes(c.n, c.V, c.d, c.k, c.dtype);
    if (rc == ND_OK) rc = check_rows("x_dev", c.x, c.n, c.d, c.x_stride, c.dtype);
    if (rc == ND_OK) rc = check_rows("w_dev", c.w, c.V, c.d, c.w_stride, c.dtype);
    if (rc == ND_OK && c.dx) rc = check_rows("dx_dev", c.dx, c.n, c.d, c.dx_stride, c.dtype);
    if (rc == ND_OK && c.dw) rc = check_rows("dw_dev", c.dw, c.V, c.d, c.dw_stride, c.dtype);
    if (rc != ND_OK) return rc;
    if (!workspace || (c.n > 0 && (!c.labels || !c.loss || !c.lse))) {
        set_error("a required pointer is NULL");
        return ND_ERR_NULL_POINTER;
    }
    const LossPlan p = plan_loss(c.n, c.V, c.d, c.k, c.dtype, c.grad);
    if (workspace_bytes < p.total || ((uintptr_t)workspace % 256) != 0) {
        set_error("workspace needs %zu bytes aligned to 256", p.total);
        return ND_ERR_WORKSPACE;
    }
    switch (c.dtype) {
        case ND_F32: return run_loss<float>(c, p, (char*)workspace, stream);
        case ND_BF16: return run_loss<bf16_t>(c, p, (char*)workspace, stream);
        default: return run_loss<f16_t>(c, p, (char*)workspace, stream);
    }
}

}  // namespace
}  // namespace nd

using namespace nd;

extern "C" {

size_t nd_softmax_loss_workspace_bytes(int64_t n, int64_t V, int32_t d, int32_t k, int dtype, int grad) {
    if (check_loss_sizes(n, V, d, k, dtype) != ND_OK) return 0;
    return plan_loss(n, V, d, k, dtype, grad != 0).total;
}

int nd_softmax_loss(const void* x_dev, int64_t x_stride, const void* w_dev, int64_t w_stride, int dtype, int64_t n,
                    int64_t V, int32_t d, const int32_t* labels_dev, int32_t k, float* loss_dev, float* lse_dev,
                    void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    const LossCall c{x_dev, w_dev, x_stride, w_stride, dtype, n, V, d, k, labels_dev, nullptr, loss_dev, lse_dev,
                     nullptr, nullptr, 0, 0, false};
    return softmax_loss(c, workspace_dev, workspace_bytes, (hipStream_t)hip_stream);
}

int nd_softmax_loss_grad(const void* x_dev, int64_t x_stride, const void* w_dev, int64_t w_stride, int dtype, int64_t n,
                         int64_t V, int32_t d, const int32_t* labels_dev, int32_t k, const float* row_weight_dev,
                         float* loss_dev, float* lse_dev, void* dx_dev, int64_t dx_stride, void* dw_dev,
                         int64_t dw_stride, void* workspace_dev, size_t workspace_bytes, void* hip_stream) {
    const LossCall c{x_dev, w_dev, x_stride, w_stride, dtype, n, V, d, k, labels_dev, row_weight_dev, loss_dev, lse_dev,
                     dx_dev, dw_dev, dx_stride, dw_stride, true};
    return softmax_loss(c, workspace_dev, workspace_bytes, (hipStream_t)hip_stream);
}

int nd_softmax_loss_status(const void* workspace_dev, void* hip_stream) {
    if (!workspace_dev) {
        set_error("workspace is NULL");
        return ND_ERR_NULL_POINTER;
    }
    uint32_t word = 0;
    ND_HIP_CHECK(hipMemcpyAsync(&word, workspace_dev, 4, hipMemcpyDeviceToHost, (hipStream_t)hip_stream));
    ND_HIP_CHECK(hipStreamSynchronize((hipStream_t)hip_stream));
    if (word & 1u) {
        set_error("a label was V or more; it was treated as NULL");
        return ND_ERR_BAD_ROOT;
    }
    return ND_OK;
}

}  // extern "C"
