// Rows held in registers against rows that pass by in LDS: the softmax loss for rows of at most 256 numbers of a 16-bit
// type, logits and the product that follows them in one kernel, so that no logit and no probability reaches memory.
#pragma once

#include "nd_rowtypes.h"
#include "nd_wave.h"

namespace nd {

constexpr int kSweepLeast = 4;      // units that a workgroup takes at least

enum SweepMode {
    kSweepLse = 0,   // x held, w passes: maximum and sum of exponentials per row of x
    kSweepRest = 1,  // the same over the vertices that are no labels of the row
    kSweepDx = 2,    // the same as that, and the sums of w's rows weighted with the exponentials
    kSweepDw = 3,    // w held, x passes: sums of x's rows weighted with g c p, less what label_weight says of labels
};

// What a workgroup of the sweep in a mode over rows of d numbers is: wavefronts, 32 held rows each; passing rows at a time;
// how many there are, all of them at work at once.
struct SweepShape {
    int waves, unit, per_cu;
    constexpr int held() const { return 32 * waves; }
    constexpr int groups() const { return 256 * per_cu; }
};
constexpr SweepShape sweep_shape(int mode, int d) {
    // Registers leave room for two workgroups where few sums are kept: 14,250 x 57,000 x 128 forward 230 us, 248 with one;
    // over rows of 64 numbers 159 and 187, with dx (8,192 rows of ten labels) 146 and 163.
    if (mode <= kSweepRest) return d > 128 ? SweepShape{8, 64, 1} : SweepShape{8, 64, 2};
    if (mode == kSweepDx && d <= 64) return SweepShape{8, 64, 2};
    // two of these blocks of 32 rows are a unit of the others
    return d > 128 ? SweepShape{8, 32, 1} : SweepShape{8, 64, 1};
}

// How the work, tiles of held rows x units of passing rows, is dealt out: workgroup g takes the units
// [g total / groups, (g + 1) total / groups) of all tiles in a row, so that every one has as many, whatever the number of
// tiles; what it holds of a tile is a segment.
struct SweepDeal {
    int64_t tiles, units, total, groups;
    __host__ __device__ SweepDeal(int64_t held, int64_t passing, SweepShape shape) {
        tiles = (held + shape.held() - 1) / shape.held();
        units = (passing + shape.unit - 1) / shape.unit;
        total = tiles * units;
        groups = total / kSweepLeast;
        if (groups > shape.groups()) groups = shape.groups();
        if (groups < 1) groups = 1;
    }
    __host__ __device__ int64_t first(int64_t g) const { return g * total / groups; }
    // the workgroup that has unit x
    __host__ __device__ int64_t group_of(int64_t x) const {
        int64_t g = x * groups / total;
        while (g + 1 < groups && first(g + 1) <= x) ++g;
        while (g > 0 && first(g) > x) --g;
        return g;
    }
};

// What the kernels of the loss share.  Arrays by place are those of the gathered rows: the rows with labels, in their
// order, one after the other.
struct LossHeader {
    uint32_t status;   // bit 0: a label was V or more
    uint32_t n_live;   // rows with labels
    float scale;       // what probabilities are multiplied by before they are rounded, a power of two
    uint32_t pad[61];
};
static_assert(sizeof(LossHeader) == 256, "one 256-byte block");

struct LossArgs {
    int64_t n, V, n_pad;
    int32_t d, dp, k;
    const int32_t* labels;
    const float* row_weight;
    float *loss, *lse;        // by row
    LossHeader* header;
    uint32_t* block_live;     // per 128 rows: rows with labels,
    float* block_weight;      // the largest weight among them,
    uint32_t* block_bad;      // whether a label is V or more
    int32_t* row_of;          // by place: row
    int32_t* labels_of;       // by place: k labels, -1 where one does not count
    float* count;             // by place: labels that count
    float* weight;            // by place: row weight
    float* place_lse;         // by place
    // Gradients of 16-bit rows (else null), by place and label; labels_of then ascends, what does not count behind it.
    float* label_score;       // the score
    float* label_weight;      // what the label's row is multiplied by when it is taken off, 0 where a label comes again
    float* place_factor;      // sweeps: log2 e lse - log2 |g c scale|, infinite where a place has no row
    float *part_max, *part_sum;  // [groups of vertices][n_pad]
    int32_t groups;
    FastDiv div_k;
    int32_t* label_row;       // dw of 16-bit rows: by vertex, the row of the sums over its labels, or -1 (else null)
};

constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// What labels are in their row's gradient.  held - c p, `held` how often a label comes among the c that count, is a difference
// that the fit takes to 0, far below what rounding p to 16 bits leaves.  So it is made of what does not cancel: with E the
// label's exponential, S the sum of those of all vertices that are no labels and Z = S + sum E,
//
//     held - c p = (held S + held (sum E - E) - (c - held) E) / Z,
//
// the last two terms exactly 0 in a row of one label.
struct LabelTerms {
    float top, total, lse;  // maximum, Z relative to it, log of the sum over all vertices
    float rate;             // held - c p; 0 where the label came before or does not count
    bool first;             // the label counts and did not come before
};
// Lanes are the row's labels in ascending order, -1 behind them; all of them are active.  top, sum: of the exponentials of
// all other vertices (APART), or of all.
template <bool APART>
__device__ __forceinline__ LabelTerms label_terms(int32_t label, float score, float count, float top, float sum) {
    const int lane = lane_id();
    const int32_t before = __shfl_up(label, 1);
    LabelTerms t;
    t.first = label >= 0 && (lane == 0 || before != label);
    const uint64_t labels = __ballot(label >= 0), later = __ballot(t.first) >> lane >> 1;
    const float held = (float)(later ? __ffsll((unsigned long long)later) : __popcll(labels) - lane);
    t.top = top;
    if constexpr (APART) {
        float most = label >= 0 ? score : top;
        for (int s = 32; s > 0; s >>= 1) most = fmaxf(most, __shfl_xor(most, s));
        t.top = fmaxf(top, most);
    }
    const float e = t.first ? exp_of(score - t.top) : 0.f;
    float all = e;
    for (int s = 32; s > 0; s >>= 1) all += __shfl_xor(all, s);
    float rest = APART ? sum * exp_of(top - t.top) : sum - all;
    if (!APART && rest < 0.f) rest = 0.f;
    t.total = APART ? rest + all : sum;
    t.lse = t.top + logf(t.total);
    t.rate = t.first ? (held * rest + (held * (all - e) - (count - held) * e)) / t.total : 0.f;
    return t;
}

// Memory of a sweep's segments.
struct SweepParts {
    float *top, *sum;   // [segment][held rows of a tile]
    float* rows;        // [segment][held rows of a tile][dp]
    // kSweepDw: by vertex, the row of label_sums with the sum of its labels' rows, or -1
    const int32_t* label_row;
    const float* label_sums;
};
int sweep_width(int32_t d);                   // numbers in a padded row, 0: rows are too long
// Held rows of all segments, of as many held and passing rows at most.
int64_t sweep_rows(int mode, int64_t held, int64_t passing, int32_t dp);
template <typename T>
int sweep(int mode, const LossArgs& a, const T* rows, const T* w, int64_t w_stride, const SweepParts& parts, T* dw,
          int64_t dw_stride, hipStream_t stream);
// lse, loss and (dx: not null) dx of the gathered rows, from the segments of the sweep in `mode`.
template <typename T>
int sweep_finish(int mode, const LossArgs& a, const T* rows, const T* w, int64_t w_stride, const SweepParts& parts, T* dx,
                 int64_t dx_stride, hipStream_t stream);

}  // namespace nd
