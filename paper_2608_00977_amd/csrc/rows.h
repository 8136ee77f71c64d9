// Operators on rows of factor tables (rows.hip) and on the probabilities that
// factors give over all items (head.hip).  Internal; the entry points are in
// include/tsid.h.
#pragma once

#include "internal.h"

namespace tsid {

// Takes pieces of a caller's workspace, each 256-byte aligned; with a null
// base it only counts, so that the sizes asked for and the pieces taken come
// from the same code.
struct Carve {
    char *base = nullptr;
    size_t used = 0;
    template <typename T>
    T *take(int64_t count) {
        T *p = base ? reinterpret_cast<T *>(base + used) : nullptr;
        used += ((size_t)(count > 0 ? count : 1) * sizeof(T) + 255) & ~size_t(255);
        return p;
    }
};

// A launch has fewer than 2^32 threads in x: more workgroups than kGridX (of at
// most 512 threads) go on in y, whose last line has some beyond `blocks`.
constexpr int64_t kGridX = int64_t(1) << 22;
inline dim3 grid_of_blocks(int64_t blocks) {
    return blocks <= kGridX ? dim3((unsigned)blocks) : dim3((unsigned)kGridX, (unsigned)((blocks + kGridX - 1) / kGridX));
}
__device__ __forceinline__ int64_t block_of_grid() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// E_INVAL unless ws is 256-byte aligned and holds `needed` bytes (before any launch).
void check_workspace(const void *ws, size_t bytes, size_t needed);

// taken[j] = slots[j], and slots[j] = 0, for j < n (at most 64), each in one step.
void launch_take_slots(int32_t *slots, int32_t *taken, int n, hipStream_t s);

// Rows of a factor table: fp32 or bf16, k per row, ld elements from row to row.
struct Rows {
    void *p;
    int64_t count, ld;
};

// out[t] = scale * F[ids[t]]; id -1 gives zeros, another id outside the table
// zeros and ERR_RANGE.
void launch_lookup(int k, int prec, const Rows &F, const int32_t *ids, float scale, const Rows &out, int32_t *err,
                   hipStream_t s);

// Sums of weighted rows by id: entry e (0 .. entries - 1) adds w[e] times row
// e / per_row of X to the sum of row ids[e].  Used as the gradient of a lookup
// (w null, per_row 1) and for the listed items' part of a table's gradient.
struct SumPlan {
    int64_t entries, n;
    int k;
    bool plain;          // a lookup's gradient: rows of X alone, without weights, exclusions and parts
    // pieces of the workspace
    uint64_t *keys[2];
    uint32_t *vals[2];
    uint32_t *sort_scratch;
    uint32_t *ptr;       // n + 1: first sorted entry of each row
    float *carry[2];     // sums of pieces of long rows, two per piece (two levels)
    bool alt;            // where the sort left its result
    bool scan;           // few entries of a plain sum: no sort, none of these pieces
};
// Entries one piece of a long row's sum takes, and the row length from which
// a row is summed in pieces.
constexpr int kSumPiece = 64;
// Entries, and rows of the table, up to which every row looks through all ids
// instead of a sort and the launches that follow it.  Entries of random ids, us
// (looked through / sorted): 500 into 8,192 rows of 32 12 / 29, 2,048 12 / 33; at
// the limits 2,048 into 65,536 rows of 128 47 / 48, of 8 53 / 41; beyond, 4,096
// into 65,536 83 / 44, 1 into 1 M 331 / 32 (a wave per row).  A row that all
// entries name is one wave's work: 500 entries 35 / 31, 2,048 133 / 35.
constexpr int64_t kScanEntries = 2048, kScanRows = 65536;
void carve_sum(SumPlan &p, Carve &c);
// out[i] = scale * (sum of the entries of i + sum of the parts' rows i), every
// row of out written; parts: n_parts fp32 arrays of n x k, part_stride apart.
// An entry whose id is -1, or whose row of the table is excluded by bias, adds
// nothing; one with another id outside the table neither, and sets ERR_RANGE.
struct SumArgs {
    const int32_t *ids;
    const float *bias;
    int32_t *err;
    Rows X;
    const float *w;
    int32_t per_row;
    const float *parts;
    int32_t n_parts;
    int64_t part_stride;
    float scale;
    Rows out;
};
void launch_sum_rows(SumPlan &p, int prec, const SumArgs &a, hipStream_t s);

// ------------------------------------------------------------------- head
// Scores z_ti = scale h_t . f_i + bias_i of all items for all rows, divided by
// the temperature.
struct Head {
    Rows H, F;
    const float *bias;
    int k, prec;
    double scale, bias_scale;  // both divided by the temperature
};
// A bias below this excludes its item: its row of F is never used.
constexpr float kExcluded = -1e7f;

struct ScoreOut {
    const int32_t *ids;
    int32_t per_row, top;
    float *lse, *logp, *entropy;
    int32_t *top_ids;
    float *top_logp;
};
size_t score_workspace(int64_t T, int64_t n, int k, int prec, int top);
void run_score(const Head &h, const ScoreOut &o, void *ws, size_t bytes, int32_t *err, hipStream_t s);

// dz_ti = (a_t + b_t log p_ti) p_ti + sum_j c_tj [i = id_tj].
struct HeadGrad {
    const int32_t *ids;
    int32_t per_row;
    const float *lse;
    // of log probabilities and entropy
    const float *dlogp, *entropy, *dentropy;
    // of a distillation
    const float *teacher, *dloss;
    float temperature;
    Rows dH, dF;  // p null: not wanted
};
size_t head_grad_workspace(int64_t T, int64_t n, int k, int prec, int per_row);
void run_head_grad(const Head &h, const HeadGrad &g, void *ws, size_t bytes, int32_t *err, hipStream_t s);

struct DistillOut {
    const int32_t *ids;
    int32_t per_row;
    const float *teacher;
    float temperature;
    float *loss, *lse;
};
void run_distill(const Head &h, const DistillOut &o, void *ws, size_t bytes, int32_t *err, hipStream_t s);

}  // namespace tsid
