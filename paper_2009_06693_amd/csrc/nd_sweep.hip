#include "nd_sweep.h"

#include <type_traits>

// With h a tile of held rows and p a block of 32 passing rows, a wavefront makes
//
//     S[p][h] = p . h,    P = exp(S - top), 0 where p is a label of h, or g c exp(S - lse),    O[h] += sum_p P[p][h] p
//
// in 32 x 32 x 16 matrix instructions.  S is made with the passing rows as the instruction's rows, so that a lane holds 16
// passing rows of one held row: maxima and sums stay inside the lane, and the rounded P is at once the operand of
// the second product, whose other operand, the passing rows read down their columns, comes from the same tile in LDS
// through transposing reads.
//
// P is rounded to the rows' type for that product, relative to each P: with bf16 dx and dw move by 6.4e-4 and 6.0e-4 of their
// size against weights in 32 bits (8,192 x 57,000 x 128), below their own rounding, and stay 1.66e-3 from 64 bits as they are
// with those.  The remainder would be a third product, half as much work again.  It does not hold for a row's own labels, whose
// P stands against a count: dx leaves them out and gets them back where the segments are joined; dw takes off, for every label,
// what it rounded to and the difference from the count, both in 32 bits.
//
// What bounds it: matrix instructions and vector instructions share a SIMD's issue (an instruction of 32 cycles keeps it for
// 16), and under both the clock falls below 2 GHz.  8,192 x 57,000 x 128 bf16: with dx 250 us and dw 229, 956 and 1,044 TFLOP/s of
// products beside an exponential for every score; forward, 14,250 x 57,000 x 128 fp16, 229 us, 908; 8,192 x 233,000 x 256 1,640 and
// 1,760 us.  dx is 220 us where rows have one label: of ten, two fifths fall into an eighth of the vertices here, and the
// workgroups that sweep those end last.
namespace nd {
namespace {

constexpr int kThreads = 256;
constexpr float kLowest = -1e38f;  // below every maximum, and finite times log2 e

typedef float Acc __attribute__((ext_vector_type(16)));
typedef float Float4 __attribute__((ext_vector_type(4)));
typedef short Short4 __attribute__((ext_vector_type(4)));
typedef uint32_t Word4 __attribute__((ext_vector_type(4)));

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
    static constexpr SweepShape kShape = sweep_shape(MODE, D);
    static constexpr int kThreads = 64 * kShape.waves;
    static constexpr int kWaves = kShape.waves * kShape.per_cu / 4;  // of a SIMD
    static constexpr int kHeld = kShape.held();
    // A block's scores are made while the block before is still being worked on, where there are registers for both
    // (of 256: D / 8 for the held rows, D / 2 for the sums, 16 + 8 per block under way) and no second workgroup to fill in.
    static constexpr bool kAhead = MODE > kSweepRest && D <= 128 && kShape.per_cu == 1;
    static constexpr int kRing = kAhead ? 4 : 2;       // units in LDS
    static constexpr int kSteps = D / 16;              // instructions along a row
    static constexpr int kPieces = D / 8;              // 16-byte pieces of a row
    static constexpr int kUnit = kShape.unit;
    static constexpr int kUnitBytes = kUnit * D * 2;
    static constexpr int kLoads = kUnitBytes / (kThreads * 16);  // pieces that a lane moves per unit
    // kSweepDw: what the passing rows weigh, and signs of two rows in a word
    static constexpr int kFactorBytes = MODE == kSweepDw ? kUnit * 4 + kUnit * 2 : 0;
    static constexpr int kLds = kRing * (kUnitBytes + kFactorBytes);
};

// Byte position of piece c of row r of a unit: pieces change places so that 16 rows' reads of one piece, and 4 rows' reads of
// 64 bytes, fall on different banks.
template <int D>
__device__ __forceinline__ int place(int r, int c) {
    if (D == 64) return (r * 8 + (c ^ ((((r >> 1) & 1) << 2) | ((r >> 2) & 3)))) * 16;
    return (r * (D / 8) + (c ^ (((r & 3) << 2) | ((r >> 2) & 3)))) * 16;
}

// A barrier for what lies in LDS only: loads from memory stay under way across it.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <typename V>
using LdsOf = __attribute__((address_space(3))) V;

struct SweepArgs {
    const void *held, *passing;
    int64_t held_stride, passing_stride;
    SweepParts parts;
    void* out;
    int64_t out_stride;
};

template <typename T, int D, int MODE>
__global__ __attribute__((amdgpu_waves_per_eu(Shape<MODE, D>::kWaves, Shape<MODE, D>::kWaves)))
__launch_bounds__((Shape<MODE, D>::kThreads))
void sweep_kernel(LossArgs a, SweepArgs s) {
    using Sh = Shape<MODE, D>;
    using V8 = typename Eight<T>::V;
    constexpr int HELD = Sh::kHeld, STEPS = Sh::kSteps, THREADS = Sh::kThreads, RING = Sh::kRing, UNIT = Sh::kUnit;
    constexpr bool kSums = MODE > kSweepRest, kOnline = MODE != kSweepDw, kAhead = Sh::kAhead;
    constexpr bool kApart = MODE == kSweepRest || MODE == kSweepDx;  // a row's labels are left out
    // fp16 ends at 2^-24: exponentials are taken times 2^8 and may outgrow the maximum that they are relative to by 2^6
    constexpr float kRaise = std::is_same<T, f16_t>::value ? 8.f : 0.f;
    constexpr float kMost = std::is_same<T, f16_t>::value ? 16384.f : 64.f;  // 2^6 times that
    extern __shared__ __align__(16) char lds[];
    const int lane = lane_id(), wave = (int)wave_uniform((uint32_t)wave_id()), half = lane >> 5, col = lane & 31;
    const int64_t live = a.header->n_live;
    const int64_t held_rows = MODE == kSweepDw ? a.V : live, passing_rows = MODE == kSweepDw ? live : a.V;
    if (held_rows == 0 || passing_rows == 0) return;
    const SweepDeal deal(held_rows, passing_rows, Sh::kShape);
    if ((int64_t)blockIdx.x >= deal.groups) return;
    const T* held = (const T*)s.held;
    const T* passing = (const T*)s.passing;
    char* factors = lds + RING * Sh::kUnitBytes;  // [unit]: exponents of 2, a float per passing row; signs, 16 bits per row
    const float scale = MODE == kSweepDw ? a.header->scale : 1.f;

    // Where a lane reads in a unit: piece 2 k + half of one of a block's 32 rows, and column_at[e][j]: of the rows 8 e + 4
    // half to + 3 of a block of 16, eight bytes in columns 32 j on.  What the kernel adds to them is known when it is
    // compiled.  k and e, j only turn bits over (see place), so that short of registers they are made from one place each.
    typedef LdsOf<char> LdsChar;
    LdsChar* unit_lds = (LdsChar*)lds;
    constexpr bool kTight = D > 128 && kSums;
    constexpr int kScoreAt = kTight ? 1 : STEPS < 8 ? STEPS : 8, kColumnAt = kTight ? 1 : D / 32 < 4 ? D / 32 : 4;
    int32_t score_at[kScoreAt], column_at[kTight ? 1 : 2][kColumnAt];
#pragma unroll
    for (int k = 0; k < kScoreAt; ++k) score_at[k] = place<D>(col, k * 2 + half);
#pragma unroll
    for (int e = 0; e < (kTight ? 1 : 2); ++e)
#pragma unroll
        for (int j = 0; j < kColumnAt; ++j) {
            const int sub = lane & 15, at = j * 32 + ((lane >> 4) & 1) * 16 + (sub & 3) * 4;
            column_at[e][j] = place<D>(e * 8 + half * 4 + (sub >> 2), at / 8) + (at & 4) * 2;
        }

    // behind what an instruction's offset reaches from the front of LDS: the lane's own places, kept in registers
    LdsChar *factor_lds = unit_lds + RING * Sh::kUnitBytes + half * 16,
            *sign_lds = unit_lds + RING * Sh::kUnitBytes + UNIT * 4 + half * 8;
    if (MODE == kSweepDw) asm volatile("" : "+v"(factor_lds), "+v"(sign_lds));

    const int64_t end = deal.first((int64_t)blockIdx.x + 1);
    for (int64_t x = deal.first(blockIdx.x); x < end;) {
        const int64_t tile = x / deal.units;
        const int32_t u0 = (int32_t)(x - tile * deal.units);
        const int32_t u1 = (int32_t)(end - x < deal.units - u0 ? u0 + (end - x) : deal.units);
        const int64_t row0 = tile * HELD + wave * 32;
        x += u1 - u0;

        // ---- passing rows on their way to LDS
        Word4 ahead[Sh::kLoads];
        float factor_ahead[2];
        auto load = [&](int32_t u) {
            // No branches: what is loaded must not be waited for here.  Rows behind the last one are the last one again;
            // gathered rows are padded with zeros to whole units, but no further.
            const int64_t r0 = (int64_t)u * UNIT, left = (MODE == kSweepDw ? deal.units * UNIT : passing_rows) - r0;
            const int64_t from_row = left > 0 ? r0 : 0;
            const uint32_t last = left > UNIT ? UNIT - 1 : left > 0 ? (uint32_t)left - 1u : 0u;
            const char* from = (const char*)(passing + from_row * s.passing_stride);
            const uint32_t row_bytes = (uint32_t)s.passing_stride * 2u;
#pragma unroll
            for (int i = 0; i < Sh::kLoads; ++i) {
                const uint32_t e = (uint32_t)(i * THREADS) + threadIdx.x, r = e / Sh::kPieces;
                ahead[i] = *reinterpret_cast<const Word4*>(from + ((r < last ? r : last) * row_bytes + e % Sh::kPieces * 16u));
            }
            if (MODE == kSweepDw) {
                const int64_t p = from_row + (threadIdx.x & (UNIT - 1));
                factor_ahead[0] = a.place_factor[p];
                factor_ahead[1] = a.weight[p];
            }
        };
        auto keep = [&](int32_t u, int slot) {
#pragma unroll
            for (int i = 0; i < Sh::kLoads; ++i) {
                const int e = i * THREADS + (int)threadIdx.x;
                *reinterpret_cast<Word4*>(lds + slot * Sh::kUnitBytes + place<D>(e / Sh::kPieces, e % Sh::kPieces)) = ahead[i];
            }
            if (MODE == kSweepDw && threadIdx.x < UNIT) {
                // behind the segment's last unit nothing weighs
                // g c exp(s - lse) = sign(g) exp2(s log2 e - (lse log2 e - log2 |g c|))
                char* f = factors + slot * Sh::kFactorBytes;
                reinterpret_cast<float*>(f)[threadIdx.x] = u < u1 ? factor_ahead[0] : INFINITY;
                reinterpret_cast<uint16_t*>(f + UNIT * 4)[threadIdx.x] = factor_ahead[1] < 0.f ? 0x8000 : 0;
            }
        };

        // ---- held rows, as operands
        V8 rows[STEPS];
        {
            int64_t r = row0 + col;
            r = r < held_rows ? r : held_rows - 1;
#pragma unroll
            for (int k = 0; k < STEPS; ++k)
                rows[k] = *reinterpret_cast<const V8*>(held + r * s.held_stride + k * 16 + half * 8);
        }
        // ---- the first label of the lane's held row from the segment's first passing row on, the one after it, and how many
        // of the row's are left from the next one on
        uint32_t label = ~0u, label_after = ~0u;
        int32_t labels_left = 0;
        if (kApart && row0 + col < held_rows) {
            const int32_t* labels = a.labels_of + (row0 + col) * a.k;
            int32_t before = 0;
#pragma unroll 4
            for (int32_t j = 0; j < a.k; ++j) before += (uint32_t)labels[j] < (uint32_t)u0 * UNIT;
            if (before < a.k) label = (uint32_t)labels[before];
            if (before + 1 < a.k) label_after = (uint32_t)labels[before + 1];
            labels_left = a.k - before - 1;
        }
        Acc sums[D / 32];
#pragma unroll
        for (int j = 0; j < D / 32; ++j) sums[j] = Acc{};
        float top = kLowest, top2 = kLowest * kLog2e, total = 0.f;  // maximum, the same in the exponent of 2, sum

        lds_barrier();  // the segment before has read its units
        if (kAhead)  // what the sums read in front of the first block
            for (int e = threadIdx.x * 16; e < Sh::kUnitBytes; e += THREADS * 16)
                *reinterpret_cast<Word4*>(lds + (RING - 1) * Sh::kUnitBytes + e) = Word4{0, 0, 0, 0};
        load(u0);
        keep(u0, 0);
        if (kAhead) {
            load(u0 + 1);
            keep(u0 + 1, 1);
        }
        load(u0 + (kAhead ? 2 : 1));
        lds_barrier();

        // ---- operands from LDS: a piece of 32 passing rows for the scores; 16 passing rows down 32 columns for the sums
        auto row_piece = [&](int slot, int b, int k) {
            const int32_t at = kTight ? score_at[0] ^ ((k & 7) * 32) : score_at[kTight ? 0 : k & 7];
            return *reinterpret_cast<const LdsOf<V8>*>(unit_lds + at + (slot * Sh::kUnitBytes + b * 32 * D * 2 + (k >> 3) * 256));
        };
        auto column_piece = [&](int slot, int b, int i) {
            const int t = i / (D / 32), j = i % (D / 32);
            union {
                V8 v;
                Short4 q[2];
            } p;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int32_t at = kTight ? (column_at[0][0] ^ ((j & 3) * 64 + e * 32)) + e * 8 * D * 2
                                          : column_at[kTight ? 0 : e][kTight ? 0 : j & 3];
                p.q[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<LdsOf<Short4>*>(
                    unit_lds + at + (slot * Sh::kUnitBytes + (b * 32 + t * 16) * D * 2 + (j >> 2) * 256)));
            }
            return p.v;
        };
        // ---- scores of block b of the unit in `slot`
        auto scores = [&](Acc& out, int slot, int b) {
            out = Acc{};
#pragma unroll
            for (int k = 0; k < STEPS; ++k) out = multiply(row_piece(slot, b, k), rows[k], out);
        };
        // ---- sums += rows of the block, weighted
        auto add_rows = [&](const V8 (&weight)[2], int slot, int b) {
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int t = i / (D / 32), j = i % (D / 32);
                sums[j] = multiply(column_piece(slot, b, i), weight[t], sums[j]);
            }
        };
        // ---- both, for two blocks, an instruction of each in turn, and `share(i)`, a STEPS-th of other work, in
        // between; operands are read two turns before they are used
        auto scores_and_sums = [&](Acc& out, int slot, int b, const V8 (&weight)[2], int sum_slot, int sum_b, auto&& share) {
            out = Acc{};
            V8 r[3], c[3];
            r[0] = row_piece(slot, b, 0);
            if (kSums) c[0] = column_piece(sum_slot, sum_b, 0);
            r[1] = row_piece(slot, b, 1);
            if (kSums) c[1] = column_piece(sum_slot, sum_b, 1);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int t = i / (D / 32), j = i % (D / 32);
                if (i + 2 < STEPS) {
                    r[(i + 2) % 3] = row_piece(slot, b, i + 2);
                    if (kSums) c[(i + 2) % 3] = column_piece(sum_slot, sum_b, i + 2);
                }
                out = multiply(r[i % 3], rows[i], out);
                if (kSums) sums[j] = multiply(c[i % 3], weight[t], sums[j]);
                share(i);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        // Units from here on hold rows that do not count: behind the last passing row, or another segment's
        const int32_t masked = u1 == (int32_t)deal.units ? u1 - 1 : u1;
        auto mask = [&](Acc& now, int32_t u, int b) {
            if (u < masked) return;
            const int64_t left = passing_rows - (int64_t)u * UNIT;
            const int32_t rows_left = u >= u1 ? 0 : left < UNIT ? (int32_t)left : UNIT;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (half * 4 >= rows_left - (b * 32 + 8 * (r / 4) + r % 4)) now[r] = -INFINITY;
        };
        // ---- Labels among the block's rows weigh nothing here: what they are in the gradient is put together in 32 bits where
        // the segments are joined.  Few blocks hold one: the others cost a comparison.  The label after the next is on its way
        // (260 us; 277 where each was fetched when the one before it was found).
        auto leave_out = [&](Acc& now, int32_t u, int b) {
            const uint32_t first = (uint32_t)u * UNIT + (uint32_t)b * 32u;
            if (!__ballot(label - first < 32u)) return;
            uint32_t found = 0;
            do {
                if (label - first < 32u) {
                    found |= 1u << (label - first);
                    label = label_after;
                    label_after = ~0u;
                    // the row's last labels_left, without the one that moved up
                    if (--labels_left > 0) label_after = (uint32_t)a.labels_of[(row0 + col + 1) * a.k - labels_left];
                }
            } while (__ballot(label - first < 32u));
            found >>= half * 4;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (found & (1u << (8 * (r / 4) + r % 4))) now[r] = -INFINITY;
        };
        // ---- weights of a block from its scores, share i of them
        constexpr int kShare = kAhead ? 16 / STEPS : 4;
        float part;  // the block's sum
        auto weights_of = [&](const Acc& now, V8 (&weight)[2], int i) {
#pragma unroll
            for (int r = i * kShare; r < (i + 1) * kShare; ++r) {
                float p = exp2_of(fmaf(now[r], kLog2e, -top2));
                asm volatile("" : "+v"(p));  // made in this share
                part = r == 0 ? p : part + p;
                if (kSums) weight[r / 8][r % 8] = (T)p;
            }
        };
        // ---- The maximum moves only where a weight may have outgrown it, as a lane's sum of 16 tells without a comparison each,
        // and for a segment's first block: seldom.  The sums do not hold the block yet.
        auto settle = [&](const Acc& now, V8 (&weight)[2], bool first) {
            if (first || __ballot(!(part <= kMost))) {
                float t = now[0];
#pragma unroll
                for (int r = 1; r < 16; ++r) t = fmaxf(t, now[r]);
                t = fmaxf(top, fmaxf(t, __shfl_xor(t, 32)));
                const float f = exp2_of((top - t) * kLog2e);
                total *= f;
                if (kSums)
#pragma unroll
                    for (int j = 0; j < D / 32; ++j) sums[j] *= f;
                top = t;
                top2 = t * kLog2e - kRaise;
#pragma unroll
                for (int i = 0; i < 16 / kShare; ++i) weights_of(now, weight, i);
            }
            total += part;
        };
        // factors of a share's rows: read a share ahead
        typedef float Few __attribute__((ext_vector_type(kShare)));
        typedef uint32_t Signs __attribute__((ext_vector_type(kShare / 2)));
        Few lse_ahead;
        Signs signs_ahead;
        auto load_factors = [&](int slot, int b, int i) {
            const int r = i * kShare, row = b * 32 + 8 * (r / 4) + r % 4;
            lse_ahead = *reinterpret_cast<const LdsOf<Few>*>(factor_lds + slot * Sh::kFactorBytes + row * 4);
            signs_ahead = *reinterpret_cast<const LdsOf<Signs>*>(sign_lds + slot * Sh::kFactorBytes + row * 2);
        };
        auto dw_weights_of = [&](const Acc& now, V8 (&weight)[2], int slot, int b, int i) {
            const Few lse = lse_ahead;
            const Signs signs = signs_ahead;
            if (i + 1 < 16 / kShare) load_factors(slot, b, i + 1);
#pragma unroll
            for (int e = 0; e < kShare; e += 2) {
                typedef T V2 __attribute__((ext_vector_type(2)));
                const int r = i * kShare + e;
                float p0 = exp2_of(fmaf(now[r], kLog2e, -lse[e])), p1 = exp2_of(fmaf(now[r + 1], kLog2e, -lse[e + 1]));
                asm volatile("" : "+v"(p0), "+v"(p1));
                const V2 p = __builtin_bit_cast(V2, __builtin_bit_cast(uint32_t, V2{(T)p0, (T)p1}) ^ signs[e / 2]);
                weight[r / 8][r % 8] = p[0];
                weight[r / 8][r % 8 + 1] = p[1];
            }
        };

        V8 weight[2][2];  // of the two blocks under way
        Acc score[2];
        weight[1][0] = V8{};
        weight[1][1] = V8{};
        if (kAhead) scores(score[0], 0, 0);
        // one unit; its place in LDS is known when it is compiled
        auto step = [&](int32_t u, auto place_of) {
            constexpr int slot = decltype(place_of)::value;
            constexpr int next = (slot + 1) & (RING - 1), previous = (slot + RING - 1) & (RING - 1);
            keep(u + (kAhead ? 2 : 1), (slot + (kAhead ? 2 : 1)) & (RING - 1));
            load(u + (kAhead ? 3 : 2));
            if (kTight) asm volatile("" : "+v"(score_at[0]), "+v"(column_at[0][0]));  // not all made in front of the loop
#pragma unroll
            for (int b = 0; b < UNIT / 32; ++b) {
                // Ahead: this block's weights, while the next block's scores and the sums over the block before are made
                // (in front of the first block: weights of zero, of a unit that starts as zeros).
                Acc& now = score[kAhead ? b : 0];
                V8(&mine)[2] = weight[kAhead ? b : 0];
                const int next_slot = b == 0 ? slot : next, before_slot = b == 0 ? previous : slot;
                if (!kAhead) scores(now, slot, b);
                if (kTight) __builtin_amdgcn_sched_barrier(0);  // what the steps read of LDS takes turns in the registers left
                if (kOnline) {
                    mask(now, u, b);
                    if (kApart) leave_out(now, u, b);
                    if (kAhead)
                        scores_and_sums(score[b ^ 1], next_slot, b ^ 1, weight[b ^ 1], before_slot, b ^ 1,
                                        [&](int i) { weights_of(now, mine, i); });
                    else
#pragma unroll
                        for (int i = 0; i < 16 / kShare; ++i) weights_of(now, mine, i);
                    settle(now, mine, b == 0 && u == u0);
                } else {
                    load_factors(slot, b, 0);
                    if (kAhead)
                        scores_and_sums(score[b ^ 1], next_slot, b ^ 1, weight[b ^ 1], before_slot, b ^ 1,
                                        [&](int i) { dw_weights_of(now, mine, slot, b, i); });
                    else
#pragma unroll
                        for (int i = 0; i < 16 / kShare; ++i) dw_weights_of(now, mine, slot, b, i);
                }
                if (kSums) asm volatile("" : "+v"(mine[0]), "+v"(mine[1]));  // made here, not where they are used
                if (kTight) __builtin_amdgcn_sched_barrier(0);
                if (!kAhead && kSums) add_rows(mine, slot, b);
            }
            lds_barrier();
        };
        // as many units as there is room for in LDS, whether or not all of them are the segment's: no way out in between
        for (int32_t u = u0; u < u1; u += RING) {
            step(u, std::integral_constant<int, 0>());
            step(u + 1, std::integral_constant<int, 1>());
            if constexpr (RING == 4) {
                step(u + 2, std::integral_constant<int, 2>());
                step(u + 3, std::integral_constant<int, 3>());
            }
        }
        if (kAhead && kSums) add_rows(weight[1], RING - 1, 1);

        // ---- out
        if (kOnline) {
            const int64_t segment = (int64_t)blockIdx.x + tile;
            const float lower = exp2_of(-kRaise);
            const float both = (total + __shfl_xor(total, 32)) * lower;
            const int64_t at = segment * HELD + wave * 32 + col;
            if (half == 0) {
                s.parts.top[at] = top;
                s.parts.sum[at] = both;
            }
            if (kSums)
#pragma unroll
                for (int j = 0; j < D / 32; ++j)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const Float4 v = {sums[j][r * 4], sums[j][r * 4 + 1], sums[j][r * 4 + 2], sums[j][r * 4 + 3]};
                        *reinterpret_cast<Float4*>(s.parts.rows + at * D + j * 32 + r * 8 + half * 4) = v * lower;
                    }
        } else {
            const bool whole = u0 == 0 && u1 == (int32_t)deal.units;
            const float back = 1.f / scale;
            const int64_t segment = (int64_t)blockIdx.x * 2 + (u0 == 0 ? 1 : 0);  // one that ends a tile, one that begins one
            const int64_t v = row0 + col;
            const int32_t labels = whole && v < held_rows ? s.parts.label_row[v] : -1;
            const float* label_sum = s.parts.label_sums + (int64_t)labels * D;
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int e0 = j * 32 + r * 8 + half * 4;
                    const Float4 o = {sums[j][r * 4], sums[j][r * 4 + 1], sums[j][r * 4 + 2], sums[j][r * 4 + 3]};
                    if (!whole) {
                        *reinterpret_cast<Float4*>(s.parts.rows + (segment * HELD + wave * 32 + col) * D + e0) = o;
                    } else if (v < held_rows) {
                        Float4 less = {};
                        if (labels >= 0) less = *reinterpret_cast<const Float4*>(label_sum + e0);
                        T* to = (T*)s.out + v * s.out_stride + e0;
                        Piece<T, 4> q;
#pragma unroll
                        for (int e = 0; e < 4; ++e) q.v[e] = (T)fmaf(o[e], back, -less[e]);
                        if (e0 + 4 <= a.d) {
                            store_piece<T, 4>(to, q);
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (e0 + e < a.d) to[e] = q.v[e];
                        }
                    }
                }
        }
    }
}

// Rows of dw whose tile several workgroups had a part of; all of them where there was nothing to sum.  A workgroup takes 32
// rows of a tile, its lanes four numbers each.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void dw_join_kernel(LossArgs a, SweepParts parts, T* __restrict__ dw, int64_t dw_stride) {
    constexpr int HELD = sweep_shape(kSweepDw, D).held(), kRows = 32, kQuads = D / 4;
    const int64_t live = a.header->n_live;
    const SweepDeal deal(a.V, live, sweep_shape(kSweepDw, D));
    const float back = 1.f / a.header->scale;
    for (int64_t v0 = (int64_t)blockIdx.x * kRows; v0 < a.V; v0 += (int64_t)gridDim.x * kRows) {
        int64_t x0 = 0, g0 = 0, g1 = -1;
        if (live > 0) {
            x0 = v0 / HELD * deal.units;
            g0 = deal.group_of(x0);
            g1 = deal.group_of(x0 + deal.units - 1);
            if (g0 == g1) continue;
        }
        for (int i = threadIdx.x; i < kRows * kQuads; i += kThreads) {
            const int64_t v = v0 + i / kQuads;
            const int e0 = i % kQuads * 4;
            if (v >= a.V) break;
            const int32_t labels = live > 0 ? parts.label_row[v] : -1;
            Float4 sum = {}, less = {};
            if (labels >= 0) less = *reinterpret_cast<const Float4*>(parts.label_sums + (int64_t)labels * D + e0);
            for (int64_t g = g0; g <= g1; ++g) {
                const int64_t segment = g * 2 + (g == g0 && deal.first(g) <= x0 ? 1 : 0);
                sum += *reinterpret_cast<const Float4*>(parts.rows + (segment * HELD + v % HELD) * D + e0);
            }
            Piece<T, 4> q;
#pragma unroll
            for (int e = 0; e < 4; ++e) q.v[e] = (T)fmaf(sum[e], back, -less[e]);
            T* to = dw + v * dw_stride + e0;
            if (e0 + 4 <= a.d) {
                store_piece<T, 4>(to, q);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e0 + e < a.d) to[e] = q.v[e];
            }
        }
    }
}

// lse, loss and dx of the gathered rows and what labels weigh in dw, a wavefront each at a time; a workgroup's are of one tile.
constexpr int kFinishRows = 8;
template <typename T, int D, int MODE>
__global__ __launch_bounds__(kThreads) void finish_kernel(LossArgs a, const T* __restrict__ rows, const T* __restrict__ w,
                                                          int64_t w_stride, SweepParts parts, T* __restrict__ dx,
                                                           int64_t dx_stride) {
    constexpr int HELD = sweep_shape(MODE, D).held();
    constexpr int PER = D / 64;     // numbers of a lane
    constexpr int kAtOnce = 5;      // labels' rows under way
    constexpr bool kApart = MODE != kSweepLse;  // labels are not in the segments' sums
    const int64_t live = a.header->n_live;
    const SweepDeal deal(live, a.V, sweep_shape(MODE, D));
    const int e0 = lane_id() * PER;
    for (int64_t p0 = (int64_t)blockIdx.x * kFinishRows; p0 < live; p0 += (int64_t)gridDim.x * kFinishRows) {
        const int64_t tile = p0 / HELD, x0 = tile * deal.units;
        const int64_t g0 = deal.group_of(x0), g1 = deal.group_of(x0 + deal.units - 1);
        for (int64_t p = p0 + wave_id(); p < p0 + kFinishRows && p < live; p += 4) {
            const int64_t in_tile = p % HELD, row = a.row_of[p];
            const int32_t my_label = lane_id() < a.k ? a.labels_of[p * a.k + lane_id()] : -1;
            const float my_score = kApart && my_label >= 0 ? a.label_score[p * a.k + lane_id()] : 0.f;
            float top = kLowest, sum = 0.f;
            for (int64_t g = g0 + lane_id(); g <= g1; g += kWave) {
                const float t2 = parts.top[(g + tile) * HELD + in_tile], s2 = parts.sum[(g + tile) * HELD + in_tile];
                const float t = fmaxf(top, t2);
                sum = sum * exp2_of((top - t) * kLog2e) + s2 * exp2_of((t2 - t) * kLog2e);
                top = t;
            }
            for (int s = 32; s > 0; s >>= 1) {
                const float t2 = __shfl_xor(top, s), s2 = __shfl_xor(sum, s), t = fmaxf(top, t2);
                sum = sum * exp2_of((top - t) * kLog2e) + s2 * exp2_of((t2 - t) * kLog2e);
                top = t;
            }
            const float c = a.count[p];
            float lse, met;
            LabelTerms terms;
            if constexpr (kApart) {
                terms = label_terms<true>(my_label, my_score, c, top, sum);
                lse = terms.lse;
                met = my_score;
            } else {
                lse = top + logf(sum);
                met = 0.f;
                const Piece<T, PER> x = load_piece<T, PER>(rows + p * D + e0);
                for (int32_t j0 = 0; j0 < a.k; j0 += kAtOnce) {
                    Piece<T, PER> r[kAtOnce];
                    int32_t v[kAtOnce];
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j) {
                        v[j] = j0 + j < a.k ? __builtin_amdgcn_readlane(my_label, j0 + j) : -1;
                        r[j] = Piece<T, PER>{};
                        if (v[j] >= 0) r[j] = load_piece<T, PER>(w + (int64_t)v[j] * w_stride + e0);
                    }
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
                        for (int i = 0; i < PER; ++i)
                            if (v[j] >= 0) met = fmaf((float)x.v[i], (float)r[j].v[i], met);
                }
            }
            for (int s = 32; s > 0; s >>= 1) met += __shfl_xor(met, s);
            if (lane_id() == 0) {
                a.lse[row] = lse;
                a.loss[row] = c * lse - met;
            }
            if constexpr (kApart) {
                // In dw the sweep rounds a label's weight with all others; it is made here to the last bit, so that taking it off
                // again leaves what the label is in 32 bits.
                const float g = a.weight[p], scale = a.header->scale, factor = lse * kLog2e - log2f(fabsf(c * g * scale));
                const float rounded = (float)(T)exp2_of(fmaf(my_score, kLog2e, -factor)) * (1.f / scale);
                if (lane_id() == 0) a.place_factor[p] = factor;
                if (lane_id() < a.k)
                    a.label_weight[p * a.k + lane_id()] = terms.first ? g * terms.rate + (g < 0.f ? -rounded : rounded) : 0.f;
            }
            if constexpr (MODE == kSweepDx) {
                float grad[PER] = {};
#pragma unroll 4
                for (int64_t g = g0; g <= g1; ++g) {
                    const int64_t at = (g + tile) * HELD + in_tile;
                    const float f = exp2_of((parts.top[at] - terms.top) * kLog2e);
                    const Piece<float, PER> v = load_piece<float, PER>(parts.rows + at * D + e0);
#pragma unroll
                    for (int i = 0; i < PER; ++i) grad[i] = fmaf(f, v.v[i], grad[i]);
                }
#pragma unroll
                for (int i = 0; i < PER; ++i) grad[i] *= c / terms.total;
                uint64_t left = __ballot(terms.first);
                while (left) {
                    Piece<T, PER> r[kAtOnce];
                    float rate[kAtOnce];
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j) {
                        r[j] = Piece<T, PER>{};
                        rate[j] = 0.f;
                        if (left) {
                            const int from = __ffsll((unsigned long long)left) - 1;
                            left &= left - 1;
                            rate[j] = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(terms.rate), from));
                            r[j] = load_piece<T, PER>(w + (int64_t)__builtin_amdgcn_readlane(my_label, from) * w_stride + e0);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
                        for (int i = 0; i < PER; ++i) grad[i] = fmaf(-rate[j], (float)r[j].v[i], grad[i]);
                }
                const float g = a.weight[p];
                Piece<T, PER> o;
#pragma unroll
                for (int i = 0; i < PER; ++i) o.v[i] = (T)(g * grad[i]);
                T* to = dx + row * dx_stride + e0;
                if (e0 + PER <= a.d) {
                    store_piece<T, PER>(to, o);
                } else {
#pragma unroll
                    for (int i = 0; i < PER; ++i)
                        if (e0 + i < a.d) to[i] = o.v[i];
                }
            }
        }
    }
}

// A launch holds fewer than 2^32 lanes: workgroups go on to further rows from here on.
inline dim3 groups_for(int64_t rows, int64_t per) {
    const int64_t groups = (rows + per - 1) / per;
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
    hipLaunchKernelGGL((sweep_kernel<T, D, MODE>), dim3(sweep_shape(MODE, D).groups()), dim3(Shape<MODE, D>::kThreads),
                       kLds, stream, a, s);
    ND_HIP_CHECK(hipGetLastError());
    return ND_OK;
}

}  // namespace

int sweep_width(int32_t d) { return d <= 64 ? 64 : d <= 128 ? 128 : d <= 256 ? 256 : 0; }
int64_t sweep_rows(int mode, int64_t held, int64_t passing, int32_t dp) {
    // Fewer rows are dealt out to as many workgroups or fewer.  Segments' numbers: by workgroup and tile (both go up by one at a
    // time), or two of a workgroup.
    const SweepShape shape = sweep_shape(mode, dp);
    const SweepDeal deal(held, passing, shape);
    return (mode == kSweepDw ? 2 * deal.groups : deal.groups + deal.tiles) * shape.held();
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
        if (mode == kSweepLse) return launch_sweep<T, D, kSweepLse>(a, s, stream);
        if (mode == kSweepRest) return launch_sweep<T, D, kSweepRest>(a, s, stream);
        if (mode == kSweepDx) return launch_sweep<T, D, kSweepDx>(a, s, stream);
        const int rc = launch_sweep<T, D, kSweepDw>(a, s, stream);
        if (rc != ND_OK) return rc;
        hipLaunchKernelGGL((dw_join_kernel<T, D>), groups_for(a.V, 32), dim3(kThreads), 0, stream, a, parts, dw,
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
        const dim3 grid = groups_for(a.n, kFinishRows), block(kThreads);
        if (mode == kSweepLse)
            hipLaunchKernelGGL((finish_kernel<T, D, kSweepLse>), grid, block, 0, stream, a, rows, w, w_stride, parts, dx,
                               dx_stride);
        else if (mode == kSweepRest)
            hipLaunchKernelGGL((finish_kernel<T, D, kSweepRest>), grid, block, 0, stream, a, rows, w, w_stride, parts, dx,
                               dx_stride);
        else
            hipLaunchKernelGGL((finish_kernel<T, D, kSweepDx>), grid, block, 0, stream, a, rows, w, w_stride, parts, dx,
                               dx_stride);
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
