// Probabilities over all items: z = scale H F^T + bias, p = softmax of each row.
// Scores (log sum, log probabilities of given items, entropy, best items),
// distillation, and the gradients of both in H and F.
//
// No score ever reaches memory.  Both directions stream tiles of one side (Y; 64
// rows in bf16, 32 in fp32) past rows of the other side that stay in registers
// (X), one wave per 32 or 64 of them, and take S = Y X^T, 32 rows of Y at a time,
// with v_mfma_f32_32x32x16_bf16, which leaves lane l with column l % 32 (its own
// row of X) and 16 of the 32 rows of Y (the matrix unit's rows 8 (r / 4) +
// 4 (l / 32) + r % 4, r = 0 .. 15): a row's running maximum and sums are the
// lane's own, without any exchange.
//
// fp32 factors are split into three bf16 parts each (8 + 8 + 8 bits, exact) and
// multiplied part by part, six products for the nine (the other three are below
// 2^-24 of the whole): 96 cycles of a SIMD per 64 scores at k = 128, where
// v_mfma_f32_32x32x2_f32 takes 256.  bf16 factors take 16.
//
// What bounds the passes (one MI355X, k = 128, bf16; counters).  Scores: vector
// work, 74 to 77 % of the cycles (an exponential is four issue slots, and with
// maximum, exponent, sums and entropy a score takes 7.5), beside it the matrix
// unit at 34 to 44 %: 16,384 x 100 k scores in 0.49 ms, 3.4e12 a second.  Few
// rows: the table's read, 256 MB in 42 us.  Gradients: matrix unit 63 % and vector
// work 61 % of the cycles of two waves a SIMD, both sides of 16,384 x 100 k in
// 2.1 ms, 0.8 PFLOP/s of the products that they need and 1.2 of those that they
// make (a weight has two parts), where a large library product reaches 1.3.
//
// Exponentials are base 2: p = 2^(c s - m) with c = |scale| log2 e (a negative
// scale turns the sign of X).
#include <algorithm>
#include <atomic>
#include <cmath>
#include <type_traits>

#include "rows.h"

namespace tsid {

namespace {

constexpr int kThreads = 256;
constexpr double kLog2e = 1.4426950408889634074, kLn2 = 0.69314718055994530942;
// The exponent of an excluded item: below that of any other (a bias of -1e7 at
// temperature 1e-6 is -1.4e13), or blocks of excluded items would be taken for
// better ones.
constexpr float kOff = -1e20f;
// A running maximum before the first item: -5e7 log2 e.  A row whose scores all
// lie below is empty: its sum stays 0, and none of its items may be had, in the
// results and in the gradients alike.
constexpr float kLeast = -7.2134752e7f;
constexpr float kNoRow = 1e25f;  // the log sum of a row that is none, or empty: p = 0 whatever is added to the exponent
constexpr float kPeak = -6.f;    // a gradient's exponent (log2 p) beyond which two bf16 parts are too coarse for it

typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f8 __attribute__((ext_vector_type(8)));
typedef float f16 __attribute__((ext_vector_type(16)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));

// Sizes for rank K and NP bf16 parts per factor: k-steps of the scores, the
// width of a row in LDS (at least one block of 32 coordinates, zeros beyond K)
// and its stride (16 bytes of padding: 16 lanes' 16-byte reads of 16 rows, and
// the transposing reads, fall on distinct banks).
template <int K, int NP>
struct Shape {
    static constexpr int KS = K < 16 ? 1 : K / 16;
    static constexpr int KW = K < 32 ? 32 : K;
    static constexpr int NB = KW / 32;  // coordinate blocks of the gradients
    static constexpr int RS = KW + 8;
    static constexpr int CH = K / 8;    // 16-byte chunks of a row
};

// Eight factors as read: bf16 (NP = 1) or fp32 (NP = 3).
template <int NP>
struct Raw {
    uint4 w[NP == 1 ? 1 : 2];
};
template <int NP>
__device__ __forceinline__ Raw<NP> load_raw(const void *base, int64_t at) {
    Raw<NP> r;
    if constexpr (NP == 1) {
        r.w[0] = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(base) + at);
    } else {
        const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const float *>(base) + at);
        r.w[0] = p[0];
        r.w[1] = p[1];
    }
    return r;
}
template <int NP>
__device__ __forceinline__ Raw<NP> zero_raw() {
    Raw<NP> r;
    for (auto &w : r.w) w = make_uint4(0u, 0u, 0u, 0u);
    return r;
}

// x = part[0] + part[1] + part[2], each rounded to nearest even from what the
// ones before it leave (the differences are exact).
__device__ __forceinline__ void split3(f8 x, b8 (&part)[3]) {
    part[0] = __builtin_convertvector(x, b8);
    x -= __builtin_convertvector(part[0], f8);
    part[1] = __builtin_convertvector(x, b8);
    x -= __builtin_convertvector(part[1], f8);
    part[2] = __builtin_convertvector(x, b8);
}
template <int NP>
__device__ __forceinline__ void parts_of(const Raw<NP> &r, b8 (&part)[NP]) {
    if constexpr (NP == 1) {
        part[0] = __builtin_bit_cast(b8, r.w[0]);
    } else {
        const f4 a = __builtin_bit_cast(f4, r.w[0]), b = __builtin_bit_cast(f4, r.w[1]);
        split3(f8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}, part);
    }
}

// acc += a b over the parts.
template <int NP>
__device__ __forceinline__ f16 product(const b8 (&a)[NP], const b8 (&b)[NP], f16 acc) {
    if constexpr (NP == 3) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[2], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[2], b[0], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1], b[1], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[1], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[1], b[0], acc, 0, 0, 0);
    }
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[0], b[0], acc, 0, 0, 0);
}

// One side of the scores.
struct Side {
    const void *p;
    int64_t count, ld;
    const float *bias;  // of the items, or null
};

// A tile of YT rows of Y in LDS: NP planes of bf16 parts, then an offset per row.
template <int K, int NP, int YT>
struct Tile {
    using S = Shape<K, NP>;
    static constexpr int kPlane = YT * S::RS;
    static constexpr int kPer = (YT * S::CH + kThreads - 1) / kThreads;  // chunks per thread
    static constexpr size_t kBytes = (size_t)NP * kPlane * 2 + YT * 16;
    Raw<NP> raw[kPer];

    static __device__ __forceinline__ bool idle(int q) { return (YT * S::CH) % kThreads != 0 && q >= YT * S::CH; }
    // Rows y0 .. y0 + YT - 1 into registers (the side's last row beyond its end).
    __device__ __forceinline__ void load(const Side &Y, int64_t y0) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int q = threadIdx.x + i * kThreads;
            if (idle(q)) continue;
            const int64_t row = std::min<int64_t>(y0 + q / S::CH, Y.count - 1);
            raw[i] = load_raw<NP>(Y.p, row * Y.ld + (q % S::CH) * 8);
        }
    }
    // ... into LDS; `special`: zeros for rows beyond the side and excluded items.
    __device__ __forceinline__ void store(const Side &Y, int64_t y0, bool special, uint16_t *lds) const {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int q = threadIdx.x + i * kThreads;
            if (idle(q)) continue;
            Raw<NP> r = raw[i];
            if (special) {
                const int64_t row = y0 + q / S::CH;
                if (row >= Y.count || (Y.bias && Y.bias[row] < kExcluded)) r = zero_raw<NP>();
            }
            b8 part[NP];
            parts_of<NP>(r, part);
#pragma unroll
            for (int p = 0; p < NP; ++p)
                *reinterpret_cast<uint4 *>(lds + p * kPlane + (q / S::CH) * S::RS + (q % S::CH) * 8) =
                    __builtin_bit_cast(uint4, part[p]);
        }
    }
};

// What becomes of X's sign: kTurn for a negative scale; kNone (X zero) for scale 0.
enum Turn { kKeep = 0, kTurn = 1, kNone = 2 };

// The rows x0 + l % 32 of X as B operands.
template <int K, int NP>
__device__ __forceinline__ void load_x(const Side &X, int64_t x0, int turn, b8 (&x)[Shape<K, NP>::KS][NP]) {
    const int lane = threadIdx.x & 63;
    const int64_t row = x0 + (lane & 31);
#pragma unroll
    for (int s = 0; s < Shape<K, NP>::KS; ++s) {
        const int c = 16 * s + 8 * (lane >> 5);
        Raw<NP> r = zero_raw<NP>();
        if (turn != kNone && row < X.count && c < K && !(X.bias && X.bias[row] < kExcluded)) r = load_raw<NP>(X.p, row * X.ld + c);
        if (turn == kTurn) {
            const uint32_t f = NP == 1 ? 0x80008000u : 0x80000000u;
            for (auto &w : r.w) w = make_uint4(w.x ^ f, w.y ^ f, w.z ^ f, w.w ^ f);
        }
        parts_of<NP>(r, x[s]);
    }
}

// The row of a tile's 32-row block that the matrix unit's row m is: the four
// rows that a lane's scores r .. r + 3 belong to lie two apart, and with a row
// stride of 4 banks more than a whole number of turns the 16 rows that a
// transposing read takes (four by four) fall on banks of their own.
__device__ __forceinline__ constexpr int block_row(int m) { return (m & 24) | (m & 3) << 1 | (m >> 2 & 1); }
__device__ __forceinline__ constexpr int matrix_row(int row) { return (row & 24) | (row & 1) << 2 | (row >> 1 & 3); }

// Where a tile's row has its offset.
__device__ __forceinline__ int offset_place(int row) { return (row & ~31) | matrix_row(row & 31); }

// S = Y X^T for the 32 rows of Y at `y` in LDS, from acc.
template <int K, int NP, int YT>
__device__ __forceinline__ f16 scores(const uint16_t *y, const b8 (&x)[Shape<K, NP>::KS][NP], f16 acc) {
    using S = Shape<K, NP>;
    const int lane = threadIdx.x & 63;
    const uint16_t *row = y + block_row(lane & 31) * S::RS + 8 * (lane >> 5);
#pragma unroll
    for (int s = 0; s < S::KS; ++s) {
        b8 a[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p)
            a[p] = __builtin_bit_cast(b8, *reinterpret_cast<const uint4 *>(row + p * Tile<K, NP, YT>::kPlane + 16 * s));
        acc = product<NP>(a, x[s], acc);
    }
    return acc;
}

// The matrix unit's row that a lane's r-th score belongs to (without 4 (l / 32)).
__device__ __forceinline__ constexpr int tile_row(int r) { return 8 * (r / 4) + r % 4; }

// A value per row of a block, as its scores lie (off: of the lane's first row;
// kept in the order of the matrix unit's rows).
// Given to scores() to start from, an offset per row of Y costs no arithmetic.
__device__ __forceinline__ f16 per_row(const float *off) {
    f16 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const f4 o = *reinterpret_cast<const f4 *>(off + 8 * q);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[4 * q + j] = o[j];
    }
    return v;
}

// ------------------------------------------------------------------ scores

// Running maximum m (base-2 exponent), s = sum 2^(x - m), e = sum 2^(x - m) (x - m).
struct Stat {
    float m = kLeast, s = 0.f, e = 0.f;
};

__device__ __forceinline__ void merge(Stat &a, const Stat &b) {
    const float m = fmaxf(a.m, b.m), da = a.m - m, db = b.m - m;
    const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
    a.e = (a.s > 0.f ? fmaf(a.s, da, a.e) * fa : 0.f) + (b.s > 0.f ? fmaf(b.s, db, b.e) * fb : 0.f);
    a.s = a.s * fa + b.s * fb;
    a.m = m;
}

// Takes 16 scores; returns the largest exponent.
template <bool ENT>
__device__ __forceinline__ float take(Stat &st, const f16 &acc, float c) {
    float top = acc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = fmaxf(top, acc[r]);
    top *= c;
    const float m = fmaxf(st.m, top), d = st.m - m, f = __builtin_amdgcn_exp2f(d);
    if (ENT) st.e = fmaf(st.s, d, st.e) * f;
    st.s *= f;
    st.m = m;
    float s0 = 0.f, s1 = 0.f, e0 = 0.f, e1 = 0.f;
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
        const float y0 = fmaf(acc[r], c, -st.m), y1 = fmaf(acc[r + 1], c, -st.m);
        const float p0 = __builtin_amdgcn_exp2f(y0), p1 = __builtin_amdgcn_exp2f(y1);
        s0 += p0;
        s1 += p1;
        if (ENT) {
            e0 = fmaf(p0, y0, e0);
            e1 = fmaf(p1, y1, e1);
        }
    }
    st.s += s0 + s1;
    if (ENT) st.e += e0 + e1;
    return top;
}

struct ScoreK {
    Side H, F;
    float c;           // |scale| log2 e
    int turn;
    float bias_c, off;  // a bias, and the offset of an excluded item, in units of the scores s
    int64_t t0;        // first row of this run
    int64_t T;         // rows of this run
    int64_t slice_items;
    int32_t n_slices, n_tiles;
    float4 *part;      // [slice][T]: m, s, e
    float *blkmax;     // [row / 64][item / 32][row % 64]: the largest score of each block of 32 items ([item / 32][T] for few rows)
    int64_t nblk;
    float *sup;        // [T][ngrp]: of each group of 2^g_log blocks, or null
    int32_t g_log;
    int64_t ngrp;
};

// In lanes 0 .. 31 the larger of a lane's a and lane + 32's; in the others the
// same of b, with lane - 32's.
__device__ __forceinline__ float max_halves(float a, float b) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(a), __float_as_uint(b), false, false);
    return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// The slice and row tile of a workgroup: workgroups go to the 8 XCDs in turn,
// so that the row tiles which read a slice of F run on one XCD and share its L2.
__device__ __forceinline__ bool place(int32_t b, int32_t n_slices, int32_t n_tiles, int32_t &slice, int32_t &tile) {
    if (n_slices < 8) {
        slice = b / n_tiles;
        tile = b % n_tiles;
    } else {
        slice = b / 8 / n_tiles * 8 + b % 8;
        tile = b / 8 % n_tiles;
    }
    return slice < n_slices;
}
inline int grid_of(int32_t n_slices, int32_t n_tiles) {
    return n_slices < 8 ? n_slices * n_tiles : (n_slices + 7) / 8 * 8 * n_tiles;
}

// Many rows: four waves of CX * 32 rows each share tiles of F through LDS, three
// tiles deep: while one is worked on, the next is there (its first scores are
// taken already) and the one after it is on its way from memory.  The matrix
// products of 32 items run beside the exponentials of the 32 before them: both
// are in one stretch of code without branches, dealt out in turn.
template <int K, int NP, int CX, int YT, bool BIAS, bool ENT, bool TOP>
__global__ __launch_bounds__(kThreads, 2) void k_score_pass(ScoreK A) {
    using TL = Tile<K, NP, YT>;
    using S = Shape<K, NP>;
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    int32_t slice, tile;
    if (!place(blockIdx.x, A.n_slices, A.n_tiles, slice, tile)) return;
    const int64_t x0 = (int64_t)tile * (4 * CX * 32) + wave * (CX * 32);  // of this run's rows
    const int64_t i0 = slice * A.slice_items, i1 = std::min<int64_t>(i0 + A.slice_items, A.F.count);
    auto buf = [&](int b) { return reinterpret_cast<uint16_t *>(smem + b * TL::kBytes); };
    if constexpr (K < 32) {
        for (size_t j = threadIdx.x; j < 3 * TL::kBytes / 4; j += kThreads) reinterpret_cast<uint32_t *>(smem)[j] = 0u;
        __syncthreads();
    }
    b8 x[CX][S::KS][NP];
    const Side X{A.H.p, A.t0 + A.T, A.H.ld, nullptr};
#pragma unroll
    for (int q = 0; q < CX; ++q) load_x<K, NP>(X, A.t0 + x0 + 32 * q, A.turn, x[q]);
    Stat st[CX];
    float group = kOff;
    TL t;
    auto put = [&](int b, int64_t y0) {
        const bool some = BIAS || y0 + YT > i1;  // of its rows are left out, or have a bias
        t.store(A.F, y0, some, buf(b));
        if (some && threadIdx.x < YT) {
            const int64_t i = y0 + threadIdx.x;
            float o = A.off;
            if (i < i1) {
                o = BIAS ? A.F.bias[i] : 0.f;
                o = o < kExcluded ? A.off : o * A.bias_c;
            }
            reinterpret_cast<float *>(buf(b) + NP * TL::kPlane)[offset_place(threadIdx.x)] = o;
        }
    };
    // the scores of block u of a tile
    auto start = [&](const uint16_t *b, int u, f16 (&acc)[CX], auto offsets) {
        const float *off = reinterpret_cast<const float *>(b + NP * TL::kPlane) + 32 * u + 4 * h;
#pragma unroll
        for (int q = 0; q < CX; ++q)
            acc[q] = scores<K, NP, YT>(b + u * 32 * S::RS, x[q], offsets() ? per_row(off) : f16{});
    };
    // keeps the largest scores of the block at item y
    auto keep = [&](const float (&top)[CX], int64_t y) {
        if constexpr (TOP) {
            // both halves of a wave join; lanes 32 and up then hold the second 32
            // rows (CX = 2), so that the store needs no branch, whose wait would
            // hold up the loads of the tile to come (blkmax has room for a last
            // tile's blocks beyond the items).  A wave's values follow one another.
            const float v = max_halves(top[0], top[CX - 1]);
            const int32_t row = (int32_t)x0 + (CX == 2 ? lane : lane & 31);
            A.blkmax[((int64_t)(row >> 6) * A.nblk + (y >> 5)) * 64 + (row & 63)] = v;
            group = fmaxf(group, v);
        }
    };
    auto keep_group = [&](int64_t end) {  // after whole groups, and after the items
        if constexpr (TOP) {
            if (A.sup && ((end & ((32 << A.g_log) - 1)) == 0 || end >= A.F.count)) {
                const int64_t row = x0 + (CX == 2 ? lane : lane & 31);
                if (row < A.T) A.sup[row * A.ngrp + ((end - 1) >> (5 + A.g_log))] = group;
                group = kOff;
            }
        }
    };
    if (i0 < i1) {
        t.load(A.F, i0);
        put(0, i0);
        t.load(A.F, i0 + YT);
        put(1, i0 + YT);
        __syncthreads();
        using Offsets = std::integral_constant<bool, BIAS>;
        f16 acc[CX];
        start(buf(0), 0, acc, Offsets());
        int cur = 0;
        int64_t y0 = i0;
        for (; BIAS ? y0 < i1 : y0 + YT <= i1; y0 += YT) {
            const int nxt = cur == 2 ? 0 : cur + 1, far = nxt == 2 ? 0 : nxt + 1;
            t.load(A.F, y0 + 2 * YT);
#pragma unroll
            for (int u = 0; u < YT / 32; ++u) {
                f16 next[CX];
                float top[CX];
                start(u + 1 < YT / 32 ? buf(cur) : buf(nxt), u + 1 < YT / 32 ? u + 1 : 0, next, Offsets());
#pragma unroll
                for (int q = 0; q < CX; ++q) top[q] = take<ENT>(st[q], acc[q], A.c);
                constexpr int kProducts = CX * S::KS * (NP == 1 ? 1 : 6), kVector = CX * (ENT ? 76 : 60);
#pragma unroll
                for (int g = 0; g < kProducts; ++g) {
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);  // a matrix product, then its share of vector work
                    __builtin_amdgcn_sched_group_barrier(0x2, (kVector + kProducts - 1) / kProducts, 0);
                }
                keep(top, y0 + 32 * u);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int q = 0; q < CX; ++q) acc[q] = next[q];
            }
            keep_group(y0 + YT);
            put(far, y0 + 2 * YT);
            __syncthreads();
            cur = nxt;
        }
        if (!BIAS && y0 < i1) {  // the items' last, partial tile
            for (int u = 0; u < YT / 32; ++u) {
                float top[CX];
                start(buf(cur), u, acc, std::true_type());
#pragma unroll
                for (int q = 0; q < CX; ++q) top[q] = take<ENT>(st[q], acc[q], A.c);
                keep(top, y0 + 32 * u);
            }
            keep_group(y0 + YT);
        }
    }
#pragma unroll
    for (int q = 0; q < CX; ++q) {
        Stat o{__shfl_xor(st[q].m, 32, 64), __shfl_xor(st[q].s, 32, 64), __shfl_xor(st[q].e, 32, 64)};
        merge(st[q], o);
        const int64_t row = x0 + 32 * q + (lane & 31);
        if (h == 0 && row < A.T) A.part[(int64_t)slice * A.T + row] = make_float4(st[q].m, st[q].s, st[q].e, 0.f);
    }
}

// At most 32 rows: reading F is all there is, so every wave takes blocks of 32
// items of its own straight from memory into the A operand (a row's 128-byte
// lines are read by two to four loads that follow one another).  32 rows are what
// one product takes; against the pass of more rows, us: 32 rows of 1 M items, bf16,
// k = 128 47 / 78, k = 8 18 / 56; fp32, 300 k, k = 128 37 / 64, 17,770, k = 64 14 / 14.
template <int K, int NP, bool ENT>
__global__ __launch_bounds__(kThreads, 2) void k_score_few(ScoreK A) {
    // a wave's items are contiguous, whole groups of blocks where there are groups
    using S = Shape<K, NP>;
    __shared__ float4 join[4][32];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    const int32_t slice = blockIdx.x;
    const int64_t i0 = slice * A.slice_items, i1 = std::min<int64_t>(i0 + A.slice_items, A.F.count);
    b8 x[S::KS][NP];
    load_x<K, NP>(Side{A.H.p, A.t0 + A.T, A.H.ld, nullptr}, A.t0, A.turn, x);
    Stat st;
    float group = kOff;
    const int64_t w0 = i0 + wave * (A.slice_items / 4), w1 = std::min<int64_t>(w0 + A.slice_items / 4, i1);
    for (int64_t y0 = w0; y0 < w1; y0 += 32) {
        const int64_t item = y0 + (lane & 31);
        float o = A.off;
        if (item < i1) {
            o = A.F.bias ? A.F.bias[item] : 0.f;
            o = o < kExcluded ? A.off : o * A.bias_c;
        }
        Raw<NP> raw[S::KS];
#pragma unroll
        for (int s = 0; s < S::KS; ++s) {
            const int c = 16 * s + 8 * h;
            raw[s] = zero_raw<NP>();
            if (o != A.off && c < K) raw[s] = load_raw<NP>(A.F.p, item * A.F.ld + c);
        }
        f16 acc = {};
        if (A.F.bias || y0 + 32 > i1) {
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] = __shfl(o, tile_row(r) + 4 * h, 64);
        }
#pragma unroll
        for (int s = 0; s < S::KS; ++s) {
            b8 a[NP];
            parts_of<NP>(raw[s], a);
            acc = product<NP>(a, x[s], acc);
        }
        const float top = take<ENT>(st, acc, A.c);
        if (A.blkmax) {
            const int64_t blk = y0 >> 5;
            const float v = max_halves(top, top);
            if (lane < A.T) A.blkmax[blk * A.T + lane] = v;
            group = fmaxf(group, v);
            if (A.sup && (((blk + 1) & ((1 << A.g_log) - 1)) == 0 || y0 + 32 >= A.F.count)) {
                if (lane < A.T) A.sup[lane * A.ngrp + (blk >> A.g_log)] = group;
                group = kOff;
            }
        }
    }
    Stat o{__shfl_xor(st.m, 32, 64), __shfl_xor(st.s, 32, 64), __shfl_xor(st.e, 32, 64)};
    merge(st, o);
    if (h == 0) join[wave][lane] = make_float4(st.m, st.s, st.e, 0.f);
    __syncthreads();
    if (threadIdx.x < A.T) {
        Stat all{join[0][lane].x, join[0][lane].y, join[0][lane].z};
        for (int w = 1; w < 4; ++w) merge(all, Stat{join[w][lane].x, join[w][lane].y, join[w][lane].z});
        A.part[(int64_t)slice * A.T + lane] = make_float4(all.m, all.s, all.e, 0.f);
    }
}

// ------------------------------------------------- a row's results

constexpr int kMargin = 8;        // blocks beyond the wanted best items that are looked at
constexpr int kMaxPick = TSID_MAX_TOP + kMargin;
constexpr int kSelCap = kMaxPick * 32;  // candidates chosen from at a time: the items of the picked blocks
constexpr int kMaxGroups = 2048;        // one round of them
static_assert(kMaxGroups <= kSelCap && kMaxPick <= 256, "");

// Larger floats have larger keys, equal ones (both zeros) the same; NaN is below everything.
__device__ __forceinline__ uint32_t order_key(float v) {
    if (!(v == v)) return 0u;
    const uint32_t b = __float_as_uint(v + 0.f);  // -0 + 0 = 0
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t order_key(double v) {
    if (!(v == v)) return 0ull;
    const uint64_t b = __double_as_longlong(v + 0.0);
    return (b >> 63) ? ~b : b | (1ull << 63);
}

struct SelectLds {
    uint32_t best[512];
    uint32_t found, bound;
    uint16_t place[kSelCap];
    int32_t out[kMaxPick];
};

// The `want` (at most kMaxPick) largest of key[0 .. N - 1] (N <= kSelCap), equal
// keys in order of place: thread j < min(want, N) returns the place of the
// j-th, the others -1.  The keys are dealt to 256 shares; of the best upper half
// of each share the want-th largest is a bound that at least `want` keys reach
// (found bit by bit, by one wave: all waves of a large team would wait for one
// another's issue slots).  The keys that reach it, hardly more, are ranked by
// counting.
template <int TEAM>
__device__ int32_t select_largest(const uint64_t *key, int N, int want, SelectLds &L) {
    const int t = threadIdx.x;
    if (want > N) want = N;
    uint32_t best = 0u;
    for (int j = t; j < N; j += TEAM) best = max(best, (uint32_t)(key[j] >> 32));
    L.best[t] = best;
    if (t == 0) L.found = 0u;
    __syncthreads();
    if (t < 64) {
        uint32_t share[4], bound = 0u;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            share[q] = L.best[64 * q + t];
#pragma unroll
            for (int w = 256; w < TEAM; w += 256) share[q] = max(share[q], L.best[w + 64 * q + t]);
        }
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t with = bound | 1u << bit;
            int reach = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) reach += __popcll(__ballot(share[q] >= with));
            if (reach >= want) bound = with;
        }
        if (t == 0) L.bound = bound;
    }
    __syncthreads();
    const uint32_t bound = L.bound;
    for (int j = t; j < N; j += TEAM) {
        if ((uint32_t)(key[j] >> 32) >= bound) L.place[atomicAdd(&L.found, 1u)] = (uint16_t)j;
    }
    __syncthreads();
    const int have = (int)L.found;
    for (int q = t; q < have; q += TEAM) {
        const int32_t p = L.place[q];
        const uint64_t k = key[p];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < have; ++j) {
            const int32_t o = L.place[j];
            rank += key[o] > k || (key[o] == k && o < p);
        }
        if (rank < want) L.out[rank] = p;
    }
    __syncthreads();
    return t < want ? L.out[t] : -1;
}

struct FinishK {
    const float4 *part;
    int32_t n_parts;
    Side H, F;
    double scale, bias_scale;
    int64_t t0, T;
    const int32_t *ids;
    int32_t per_row;
    float *lse, *logp, *entropy;
    const float *teacher;  // distillation: loss from these
    double tau;
    float *loss;
    int32_t top;
    const float *blkmax, *sup;
    int64_t blocks, nblk, ngrp;  // blocks of items; room for them in a row of blkmax
    int32_t g_log, width;  // rows that lie together in blkmax
    int32_t *top_ids;
    float *top_logp;
    int32_t *err;
};

// Eight factors.
__device__ __forceinline__ f8 load8(const float *p) {
    const f4 a = *reinterpret_cast<const f4 *>(p), b = *reinterpret_cast<const f4 *>(p + 4);
    return f8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}
__device__ __forceinline__ f8 load8(const uint16_t *p) {
    return __builtin_convertvector(__builtin_bit_cast(b8, *reinterpret_cast<const uint4 *>(p)), f8);
}

// The value of another lane of the same 16, by a data-parallel move.
template <int CTRL>
__device__ __forceinline__ double across(double v) {
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xF, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xF, 0xF, true);
    return __longlong_as_double((long long)((uint64_t)hi << 32 | lo));
}

// Sum and maximum over a team of TEAM threads.
template <int TEAM>
__device__ __forceinline__ double team_sum(double v, double *red) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if constexpr (TEAM == 64) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
    for (int q = 1; q < TEAM / 64; ++q) v += red[q];
    return v;
}
template <int TEAM>
__device__ __forceinline__ float team_max(float v, double *red) {
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    if constexpr (TEAM == 64) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = (double)v;
    __syncthreads();
    v = (float)red[0];
    for (int q = 1; q < TEAM / 64; ++q) v = fmaxf(v, (float)red[q]);
    return v;
}

// A row's results by one wave (TEAM 64), or by a workgroup where the best items
// are wanted (256 threads; 512 for few rows, which leave the CUs to them: one row
// of 1 M items 68 us instead of 73, 257 rows of 17,770 39 instead of 40; 1,024
// threads took 69 and 53): the slices' sums joined in fp64, the given items'
// scores in fp64 (k / 8 lanes each), and the best items.  The best `top` items
// lie in the `top` blocks of 32 whose maxima are largest (an item outside them
// has `top` better ones), so those blocks and kMargin more, for the rounding of
// the maxima, are scored again in fp64 and ranked by these scores.  The blocks
// are found through groups of blocks in the same way.
template <typename E, int K, int TEAM>
__global__ __launch_bounds__(TEAM == 64 ? kThreads : TEAM) void k_score_finish(FinishK A) {
    constexpr bool TOP = TEAM > 64;
    constexpr int kTeams = TOP ? 1 : kThreads / TEAM;
    constexpr int LN = K / 8, NI = TEAM / LN;  // lanes of an item, items at a time
    __shared__ double red[TEAM / 64];
    const int tid = threadIdx.x % TEAM, sub = tid % LN;
    const int64_t row = (int64_t)blockIdx.x * kTeams + threadIdx.x / TEAM, t = A.t0 + row;
    if (row >= A.T) return;  // whole teams
    const E *F = static_cast<const E *>(A.F.p);
    const f8 hv = load8(static_cast<const E *>(A.H.p) + t * A.H.ld + sub * 8);
    // log sum and entropy
    float m = kLeast;
    for (int q = tid; q < A.n_parts; q += TEAM) m = fmaxf(m, A.part[(int64_t)q * A.T + row].x);
    m = team_max<TEAM>(m, red);
    double s = 0.0, e = 0.0;
    for (int q = tid; q < A.n_parts; q += TEAM) {
        const float4 p = A.part[(int64_t)q * A.T + row];
        if (p.y == 0.f) continue;
        const double d = (double)p.x - (double)m, f = exp2(d);
        s += (double)p.y * f;
        e += ((double)p.z + (double)p.y * d) * f;
    }
    s = team_sum<TEAM>(s, red);
    e = team_sum<TEAM>(e, red);
    const bool empty = s == 0.0;
    const double lse = empty ? -INFINITY : kLn2 * ((double)m + log2(s));
    if (tid == 0) {
        if (A.lse) A.lse[t] = (float)lse;
        if (A.entropy) A.entropy[t] = empty ? 0.f : (float)(kLn2 * (log2(s) - e / s));
    }
    auto usable = [&](int64_t id) { return !empty && id >= 0 && id < A.F.count && !(A.F.bias && A.F.bias[id] < kExcluded); };
    // the score of an item whose factors f the LN lanes hold
    auto score_of = [&](float bias, const f8 &f) {
        double z = 0.0;
#pragma unroll
        for (int c = 0; c < 8; ++c) z = fma((double)hv[c], (double)f[c], z);
        if constexpr (LN >= 2) z += across<0xB1>(z);    // lanes i ^ 1
        if constexpr (LN >= 4) z += across<0x4E>(z);    // i ^ 2
        if constexpr (LN >= 8) z += across<0x141>(z);   // 7 - i of each 8
        if constexpr (LN >= 16) z += across<0x140>(z);  // 15 - i of each 16
        return z * A.scale + (double)bias * A.bias_scale;
    };
    const int32_t *ids = A.ids ? A.ids + t * A.per_row : nullptr;
    constexpr int NP = sizeof(E) == 2 ? 1 : 3;
    auto eight = [](const Raw<NP> &r) {
        if constexpr (NP == 1) return __builtin_convertvector(__builtin_bit_cast(b8, r.w[0]), f8);
        else return load8(reinterpret_cast<const float *>(r.w));
    };
    // an item's row and bias, whatever they are, so that one does not wait for
    // the other; -inf for what is no item, 0 without a bias
    auto row_of = [&](int64_t id, float &bias) {
        const bool in = id >= 0 && id < A.F.count;
        const int64_t at = in ? id : 0;
        bias = A.F.bias ? A.F.bias[at] : 0.f;
        if (!in) bias = -INFINITY;
        return load_raw<NP>(F, at * A.F.ld + sub * 8);
    };
    // visit(j, id, usable, score) for the listed items, by the LN lanes of each
    auto listed = [&](auto visit) {
        if (A.F.count <= 0) {
            for (int j = tid / LN; j < A.per_row; j += NI) visit(j, (int64_t)ids[j], false, 0.0);
            return;
        }
        constexpr int U = 4;
        for (int base = 0; base < A.per_row; base += NI * U) {
            const int j0 = base + tid / LN;
            Raw<NP> r[U];
            int64_t id[U];
            float bias[U];
#pragma unroll
            for (int u = 0; u < U; ++u) id[u] = j0 + u * NI < A.per_row ? ids[j0 + u * NI] : -1;
#pragma unroll
            for (int u = 0; u < U; ++u) r[u] = row_of(id[u], bias[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (base + u * NI >= A.per_row) break;
                const bool use = !empty && bias[u] >= kExcluded;
                const double z = score_of(use ? bias[u] : 0.f, eight(r[u]));
                if (j0 + u * NI < A.per_row) visit(j0 + u * NI, id[u], use, z);
            }
        }
    };
    if (A.logp) {
        listed([&](int j, int64_t id, bool use, double z) {
            float v = 0.f;
            if (use) v = (float)(z - lse);
            else if (id >= 0 && id < A.F.count) v = -INFINITY;
            else if (id != -1) A.err[ERR_RANGE] = 1;
            if (sub == 0) A.logp[t * A.per_row + j] = v;
        });
    }
    if (A.teacher) {
        const float *tl = A.teacher + t * A.per_row;
        float tm = -INFINITY;
        for (int j = tid; j < A.per_row; j += TEAM) {
            const int32_t id = ids[j];
            if (usable(id)) tm = fmaxf(tm, tl[j]);
            else if (id < -1 || id >= A.F.count) A.err[ERR_RANGE] = 1;
        }
        tm = team_max<TEAM>(tm, red);
        double w_sum = 0.0, a_sum = 0.0;
        if (tm > -INFINITY) {
            listed([&](int j, int64_t, bool use, double z) {
                const double lw = ((double)tl[j] - (double)tm) / A.tau, w = use ? exp(lw) : 0.0;
                if (sub == 0 && w != 0.0) {  // a NaN logit reaches the loss
                    w_sum += w;
                    a_sum += w * (lw - (z - lse));
                }
            });
        }
        w_sum = team_sum<TEAM>(w_sum, red);
        a_sum = team_sum<TEAM>(a_sum, red);
        if (tid == 0) A.loss[t] = w_sum == 0.0 ? 0.f : (float)(A.tau * A.tau * (a_sum / w_sum - log(w_sum)));
    }
    if constexpr (TOP) {
        __shared__ uint64_t cand[kSelCap];
        __shared__ int32_t pick[2][kMaxPick];
        __shared__ SelectLds L;
        // the `want` largest of `total` candidates get(j, value, payload), equal
        // ones in order of payload, best first, to out
        auto choose = [&](int64_t total, int want, int32_t *out, auto get) {
            int have = 0;
            int64_t next = 0;
            do {
                const int n_new = (int)std::min<int64_t>(kSelCap - have, total - next);
                for (int j = tid; j < n_new; j += TEAM) {
                    float v;
                    int32_t p;
                    get(next + j, v, p);
                    cand[have + j] = (uint64_t)order_key(v) << 32 | (uint32_t)~p;
                }
                __syncthreads();
                next += n_new;
                const int32_t place = select_largest<TEAM>(cand, have + n_new, want, L);
                have = std::min(have + n_new, want);
                const uint64_t c = place >= 0 ? cand[place] : 0;
                __syncthreads();
                if (place >= 0) {  // the front of the next round
                    cand[tid] = c;
                    out[tid] = (int32_t)~(uint32_t)c;
                }
                __syncthreads();
            } while (next < total);
            return have;
        };
        const int want = A.top + kMargin;
        int got;
        const float *maxima = A.blkmax + row / A.width * A.nblk * A.width + row % A.width;
        if (A.sup) {
            const float *sup = A.sup + row * A.ngrp;
            const int groups = choose(A.ngrp, want, pick[0], [&](int64_t j, float &v, int32_t &p) {
                v = sup[j];
                p = (int32_t)j;
            });
            got = choose((int64_t)groups << A.g_log, want, pick[1], [&](int64_t j, float &v, int32_t &p) {
                const int64_t b = ((int64_t)pick[0][j >> A.g_log] << A.g_log) + (j & ((1 << A.g_log) - 1));
                v = b < A.blocks ? maxima[b * A.width] : -INFINITY;
                p = (int32_t)b;
            });
        } else {
            got = choose(A.blocks, want, pick[1], [&](int64_t j, float &v, int32_t &p) {
                v = maxima[j * A.width];
                p = (int32_t)j;
            });
        }
        // their items, best first
        int32_t b0 = 0;
        int rank = 0;
        if (tid < got) {
            b0 = pick[1][tid];
            for (int j = 0; j < got; ++j) rank += pick[1][j] < b0;
        }
        __syncthreads();
        if (tid < got) pick[0][rank] = b0;  // ascending, for the ties
        __syncthreads();
        constexpr int U = 8;  // items of a lane group in flight
        for (int j0 = tid / LN; j0 < got * 32; j0 += NI * U) {
            Raw<NP> r[U];
            float bias[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + u * NI;
                r[u] = row_of(j < got * 32 ? (int64_t)pick[0][j >> 5] * 32 + (j & 31) : -1, bias[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + u * NI;
                const bool use = !empty && bias[u] >= kExcluded;
                const double z = score_of(use ? bias[u] : 0.f, eight(r[u]));
                if (sub == 0 && j < got * 32) cand[j] = use ? order_key(z) : 0ull;
            }
        }
        __syncthreads();
        const int32_t place = select_largest<TEAM>(cand, got * 32, A.top, L);
        if (tid < A.top) {
            int32_t id = -1;
            float lp = -INFINITY;
            const uint64_t kv = place >= 0 ? cand[place] : 0ull;
            if (kv != 0ull) {
                id = pick[0][place >> 5] * 32 + (place & 31);
                const double z = __longlong_as_double((long long)((kv >> 63) ? kv & ~(1ull << 63) : ~kv));
                lp = (float)(z - lse);
            }
            A.top_ids[t * A.top + tid] = id;
            A.top_logp[t * A.top + tid] = lp;
        }
    }
}

// ------------------------------------------------------------- gradients

// What a row's gradient in the scores needs (see HeadGrad): x = log2 of the
// sum, y = a, z = b ln 2, corrected for x being rounded; and the weights of its
// listed items.  One wave per row.
__global__ __launch_bounds__(kThreads) void k_head_coef(HeadGrad G, int64_t T, int64_t n, const float *bias,
                                                        float4 *coef, float *w, int32_t *err) {
    const int64_t t = block_of_grid() * 4 + (threadIdx.x >> 6);
    if (t >= T) return;
    const int lane = threadIdx.x & 63;
    const int32_t *ids = G.ids ? G.ids + t * G.per_row : nullptr;
    const float lse = G.lse[t];
    const bool empty = lse < -1e29f;
    auto usable = [&](int32_t id) {
        const bool in = id >= 0 && id < n;
        if (!in && id != -1) err[ERR_RANGE] = 1;
        return in && !empty && !(bias && bias[id] < kExcluded);
    };
    auto wave_sum = [](double v) {
        for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
        return v;
    };
    double a = 0.0, b = 0.0;
    if (G.teacher) {
        const float *tl = G.teacher + t * G.per_row;
        const double tau = G.temperature;
        float tm = -INFINITY;
        for (int j = lane; j < G.per_row; j += 64)
            if (usable(ids[j])) tm = fmaxf(tm, tl[j]);
        for (int off = 32; off > 0; off >>= 1) tm = fmaxf(tm, __shfl_xor(tm, off, 64));
        double sum = 0.0;
        for (int j = lane; j < G.per_row; j += 64)
            if (usable(ids[j])) sum += exp(((double)tl[j] - (double)tm) / tau);
        sum = wave_sum(sum);
        const bool some = tm > -INFINITY;
        const double u = some ? (double)G.dloss[t] * tau * tau : 0.0;
        a = u;
        for (int j = lane; j < G.per_row; j += 64)
            w[t * G.per_row + j] =
                some && usable(ids[j]) ? (float)(-u * exp(((double)tl[j] - (double)tm) / tau) / sum) : 0.f;
    } else {
        double sum = 0.0;
        for (int j = lane; j < G.per_row; j += 64) {
            const float v = usable(ids[j]) ? G.dlogp[t * G.per_row + j] : 0.f;
            w[t * G.per_row + j] = v;
            sum += (double)v;
        }
        sum = wave_sum(sum);
        b = G.dentropy && !empty ? -(double)G.dentropy[t] : 0.0;
        a = -sum + (b != 0.0 ? b * (double)G.entropy[t] : 0.0);
    }
    if (lane == 0) {
        const double l2 = (double)lse * kLog2e;
        const float l2f = (float)l2;
        const double d = (double)l2f - l2, f = exp2(d);  // log2 p = (c s - l2f) + d
        coef[t] = empty ? make_float4(kNoRow, 0.f, 0.f, 0.f)
                        : make_float4(l2f, (float)(f * (a + b * kLn2 * d)), (float)(f * b * kLn2), 0.f);
    }
}

struct GradK {
    Side X, Y;
    float c;
    int turn;
    float bias_c;
    float unit;        // of the offsets per row of Y: 1 / c where the scores start from them (bf16), else 1
    const float4 *coef;
    int64_t slice_rows;
    int32_t n_slices, n_tiles;
    float *part;       // [slice][rows of X][K]
    // the listed items' part of the items' gradient, added in the pass (per_row 0: not here)
    const int32_t *ids;
    const float *w;
    int32_t per_row;
    // the items' gradient itself, where one slice holds all of it (else null)
    void *out;
    int64_t ldo;
    float scale;
};

// Ends a workgroup's sums of 128 items: adds the listed items' part, if it is
// added here, and stores the sums, or where they are whole the gradient.  Of the
// entries of its rows y (a slice), w h_y to the item that the entry lists.  The
// sums go through LDS.  Entries are looked through 1,024 at a time (512 at k =
// 128, where two workgroups share a CU's LDS); those of these items are listed
// in order, dealt to eight teams of 32 lanes by their item, and added by them in
// order, four rows in flight.
constexpr int listed_at_once(int K) { return K >= 128 ? 512 : 1024; }
constexpr size_t listed_lds(int K) { return 128 * (size_t)K * 4 + (size_t)listed_at_once(K) * (12 + 8 * 2); }

template <int K, int NP, int NB>
__device__ __forceinline__ void finish_items(const GradK &A, const f16 (&acc)[NB], int64_t x0, int64_t i0, int64_t i1,
                                           int32_t slice, unsigned char *smem, uint32_t *wave_count) {
    constexpr int kListed = listed_at_once(K), P = kListed / kThreads;
    float *sum = reinterpret_cast<float *>(smem);  // [128][K]
    int32_t *item = reinterpret_cast<int32_t *>(sum + 128 * K);
    uint32_t *row = reinterpret_cast<uint32_t *>(item + kListed);
    float *weight = reinterpret_cast<float *>(row + kListed);
    uint16_t *mine = reinterpret_cast<uint16_t *>(weight + kListed);  // [8][kListed]
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, h = lane >> 5;
    __syncthreads();  // the tiles of Y are done with
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
        const int c = nb * 16 + (lane >> 4 & 1) * (NB * 16) + (lane & 15);
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (c < K) sum[(wave * 32 + 8 * (r / 4) + r % 4 + 4 * h) * K + c] = acc[nb][r];
    }
    const int team = tid >> 5, tl = tid & 31, c = 4 * tl;
    const uint64_t below = (uint64_t(1) << lane) - 1;
    const int64_t e_end = std::min<int64_t>(i1, A.Y.count) * A.per_row;
    for (int64_t e0 = i0 * A.per_row; e0 < e_end; e0 += kListed) {
        int64_t local[P];
        float w[P];
        uint32_t at = 0, hits = 0, count = 0;
#pragma unroll
        for (int q = 0; q < P; ++q) {
            const int64_t e = e0 + P * tid + q;
            local[q] = e < e_end ? (int64_t)A.ids[e] - x0 : -1;
        }
#pragma unroll
        for (int q = 0; q < P; ++q) {
            w[q] = local[q] >= 0 && local[q] < 128 ? A.w[e0 + P * tid + q] : 0.f;  // 0: also an entry that is no item's
            const uint64_t hit = __ballot(w[q] != 0.f);
            at += (uint32_t)__popcll(hit & below);
            hits += (uint32_t)__popcll(hit);
        }
        if (lane == 0) wave_count[wave] = hits;
        __syncthreads();
        for (int v = 0; v < 4; ++v) {
            if (v < wave) at += wave_count[v];
            count += wave_count[v];
        }
#pragma unroll
        for (int q = 0; q < P; ++q) {
            if (w[q] != 0.f) {
                item[at] = (int32_t)local[q];
                row[at] = (uint32_t)(e0 + P * tid + q) / (uint32_t)A.per_row;
                weight[at] = w[q];
                ++at;
            }
        }
        __syncthreads();
        uint32_t n_mine = 0;
        for (uint32_t j0 = 0; j0 < count; j0 += 32) {
            const uint32_t j = j0 + tl;
            const uint64_t b = __ballot(j < count && (item[j < count ? j : 0] & 7) == team);
            const uint32_t half = (uint32_t)(b >> (32 * h));
            if (half >> tl & 1u) mine[team * kListed + n_mine + __popc(half & ((1u << tl) - 1u))] = (uint16_t)j;
            n_mine += __popc(half);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (c < K) {
            for (uint32_t j = 0; j < n_mine; j += 4) {
                f4 y[4];
                uint32_t m[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    m[q] = mine[team * kListed + std::min<uint32_t>(j + q, n_mine - 1)];
                    const int64_t from = (int64_t)row[m[q]] * A.Y.ld + c;
                    if constexpr (NP == 1) {
                        y[q] = __builtin_convertvector(
                            __builtin_bit_cast(b4, *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(A.Y.p) + from)), f4);
                    } else {
                        y[q] = *reinterpret_cast<const f4 *>(static_cast<const float *>(A.Y.p) + from);
                    }
                }
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (j + q < n_mine) {
                        f4 *s = reinterpret_cast<f4 *>(sum + item[m[q]] * K + c);
                        *s += weight[m[q]] * y[q];
                    }
            }
        }
        __syncthreads();  // before the list is written anew
    }
    __syncthreads();
    for (int j = tid; j < 128 * K / 4; j += kThreads) {
        const int64_t x = x0 + j / (K / 4);
        if (x >= A.X.count) continue;
        const f4 v = reinterpret_cast<const f4 *>(sum)[j];
        const int at = j % (K / 4) * 4;
        if (!A.out) {
            *reinterpret_cast<f4 *>(A.part + ((int64_t)slice * A.X.count + x) * K + at) = v;
        } else if constexpr (NP == 1) {
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(A.out) + x * A.ldo + at) =
                __builtin_bit_cast(uint2, __builtin_convertvector(v * A.scale, b4));
        } else {
            *reinterpret_cast<f4 *>(static_cast<float *>(A.out) + x * A.ldo + at) = v * A.scale;
        }
    }
}

// part[slice][x] = sum over the slice's rows y of g(x, y) y, with
// g = p a + p log2 p b (ITEMS: a and b of the row y; else of the row x, where a
// alone is left to the sum's end).  The scores leave 16 rows of Y in a lane,
// eight at a time the A operand of the second product (its k index counts rows
// of Y in the order the scores left them); the B operand is a column of the
// same rows of the tile, by transposing LDS reads (ds_read_b64_tr_b16).
//
// g is split as fp32 factors are: no product takes it in fewer bits than it has.
// fp32 factors: three parts.  bf16: two, which leave 2^-16 of a term at most, and
// a third in a product of its own in blocks of 32 x 32 with a p over 2^-6: what
// is left out is then below 2^-22 of the row's weight whatever p is, as fp32's
// own roundings are, also where the sum and the listed part nearly cancel (a row
// sure of its item, equal rows of F).  The second part costs half as many matrix
// products again, with the same reads of LDS.
template <int K, int NP, int YT, bool ITEMS, bool ENT>
__device__ __forceinline__ void grad_pass(const GradK &A, int32_t block, unsigned char *smem, uint32_t *wave_count) {
    using S = Shape<K, NP>;
    using TL = Tile<K, NP, YT>;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
    int32_t slice, tile;
    if (!place(block, A.n_slices, A.n_tiles, slice, tile)) return;
    const int64_t x0 = (int64_t)tile * 128 + wave * 32, xr = x0 + (lane & 31);
    const int64_t i0 = slice * A.slice_rows, i1 = std::min<int64_t>(i0 + A.slice_rows, A.Y.count);
    auto buf = [&](int b) { return reinterpret_cast<uint16_t *>(smem + b * TL::kBytes); };
    if constexpr (K < 32) {
        for (size_t j = threadIdx.x; j < 3 * TL::kBytes / 4; j += kThreads) reinterpret_cast<uint32_t *>(smem)[j] = 0u;
        __syncthreads();
    }
    b8 x[S::KS][NP];
    load_x<K, NP>(A.X, x0, A.turn, x);
    // the lane's own part of the exponent's offset, and of the gradient; a row
    // beyond the side has no probability (else its wave took it for a large one)
    float own_off = kOff, own_a = 0.f, own_b = 0.f;
    if (xr < A.X.count) {
        if constexpr (ITEMS) {
            own_off = A.X.bias ? A.X.bias[xr] : 0.f;
            own_off = own_off < kExcluded ? kOff : own_off * A.bias_c;
        } else {
            const float4 q = A.coef[xr];
            own_off = -q.x;
            own_a = q.y;
            own_b = q.z;
        }
    }
    f16 acc[S::NB] = {};
    TL t;
    // a row of Y: the offset; ITEMS: its a and b
    auto put = [&](uint16_t *b, int64_t y0) {
        t.store(A.Y, y0, (!ITEMS && A.Y.bias) || y0 + YT > A.Y.count, b);
        if (threadIdx.x < YT) {
            const int64_t i = y0 + threadIdx.x;
            float *o = reinterpret_cast<float *>(b + NP * TL::kPlane) + offset_place(threadIdx.x);
            if constexpr (ITEMS) {
                float4 q = make_float4(kNoRow, 0.f, 0.f, 0.f);
                if (i < i1) q = A.coef[i];
                o[0] = -q.x * A.unit;
                o[YT] = q.y;
                o[2 * YT] = q.z;
            } else {
                float v = kOff;
                if (i < i1) {
                    v = A.Y.bias ? A.Y.bias[i] : 0.f;
                    v = v < kExcluded ? kOff : v * A.bias_c;
                }
                o[0] = v * A.unit;
            }
        }
    };
    const int grp = lane >> 4, gi = lane & 15;
    auto offsets = [&](const uint16_t *b, int u) {
        return reinterpret_cast<const float *>(b + NP * TL::kPlane) + 32 * u + 4 * h;
    };
    // the scores of block u of a tile; bf16: from the offsets.  fp32: those are
    // added to the exponents, so that no sum is rounded at their size.
    auto start = [&](const uint16_t *b, int u) {
        return scores<K, NP, YT>(b + u * 32 * S::RS, x, NP == 1 ? per_row(offsets(b, u)) : f16{});
    };
    // ... their g, in the parts that the second product takes, or (bf16, `rest`)
    // what those leave as the first of them; returns the largest exponent
    constexpr int GP = NP == 1 ? 2 : NP;
    auto weights = [&](const f16 &s, const float *off, b8 (&ga)[2][GP], auto rest) {
        float peak = kOff;
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
            f8 g;
#pragma unroll
            for (int q = 2 * h2; q < 2 * h2 + 2; ++q) {
                f4 o = {}, ya = {}, yb = {};
                if constexpr (NP != 1) o = *reinterpret_cast<const f4 *>(off + 8 * q);
                if constexpr (ITEMS) {
                    ya = *reinterpret_cast<const f4 *>(off + YT + 8 * q);
                    if constexpr (ENT) yb = *reinterpret_cast<const f4 *>(off + 2 * YT + 8 * q);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float e = fmaf(s[4 * q + j], A.c, NP == 1 ? own_off : o[j] + own_off);
                    const float p = __builtin_amdgcn_exp2f(e);
                    if constexpr (NP == 1) peak = fmaxf(peak, e);
                    if constexpr (ITEMS) g[4 * (q & 1) + j] = p * (ENT ? fmaf(e, yb[j], ya[j]) : ya[j]);
                    else g[4 * (q & 1) + j] = ENT ? p * fmaf(e, own_b, own_a) : p;
                }
            }
            if constexpr (NP == 1) {
                ga[h2][0] = __builtin_convertvector(g, b8);
                g -= __builtin_convertvector(ga[h2][0], f8);
                ga[h2][1] = __builtin_convertvector(g, b8);
                if constexpr (rest()) ga[h2][0] = __builtin_convertvector(g - __builtin_convertvector(ga[h2][1], f8), b8);
            } else {
                split3(g, ga[h2]);
            }
        }
        return peak;
    };
    // acc += g (rest: its first part) times the 32 rows at yt
    auto products = [&](const uint16_t *yt, const b8 (&ga)[2][GP], auto rest) {
#pragma unroll
        for (int h2 = 0; h2 < 2; ++h2) {
#pragma unroll
            for (int nb = 0; nb < S::NB; ++nb) {
                // in each group of 16 lanes, lane i receives element i % 4 of
                // the 8-byte pieces of lanes i / 4, 4 + i / 4, ...: lane 4 j + q
                // points at row j, coordinates 4 q .. 4 q + 3 (the two groups of a
                // half wave half a row apart, 32 banks at k = 128)
                const uint16_t *src = yt + (16 * h2 + 2 * (gi >> 2) + h) * S::RS + nb * 16 + (grp & 1) * (S::KW / 2) + 4 * (gi & 3);
                b8 yb[NP];
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const uint16_t *at = src + p * TL::kPlane;
                    const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                                   (__attribute__((address_space(3))) s4 *)(at)));
                    const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                                   (__attribute__((address_space(3))) s4 *)(at + 8 * S::RS)));
                    yb[p] = __builtin_bit_cast(b8, make_uint4(lo.x, lo.y, hi.x, hi.y));
                }
                if constexpr (NP == 1) {
                    if constexpr (!rest()) acc[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ga[h2][1], yb[0], acc[nb], 0, 0, 0);
                    acc[nb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ga[h2][0], yb[0], acc[nb], 0, 0, 0);
                } else {
                    acc[nb] = product<NP>(ga[h2], yb, acc[nb]);
                }
            }
        }
    };
    if (i0 < i1) {  // nothing to read of an empty side
        t.load(A.Y, i0);
        put(buf(0), i0);
        t.load(A.Y, i0 + YT);
        put(buf(1), i0 + YT);
        __syncthreads();
        f16 s = start(buf(0), 0);
        int cur = 0;
        for (int64_t y0 = i0; y0 < i1; y0 += YT) {
            const int nxt = cur == 2 ? 0 : cur + 1, far = nxt == 2 ? 0 : nxt + 1;
            t.load(A.Y, y0 + 2 * YT);
#pragma unroll
            for (int u = 0; u < YT / 32; ++u) {
                b8 ga[2][GP];
                const f16 next = start(u + 1 < YT / 32 ? buf(cur) : buf(nxt), u + 1 < YT / 32 ? u + 1 : 0);
                const float peak = weights(s, offsets(buf(cur), u), ga, std::false_type());
                products(buf(cur) + u * 32 * S::RS, ga, std::false_type());
                if (NP == 1 && __any(peak > kPeak)) {
                    weights(s, offsets(buf(cur), u), ga, std::true_type());
                    products(buf(cur) + u * 32 * S::RS, ga, std::true_type());
                }
                __builtin_amdgcn_sched_barrier(0);  // else reads of many blocks ahead spill
                s = next;
            }
            put(buf(far), y0 + 2 * YT);
            __syncthreads();
            cur = nxt;
        }
    }
    if constexpr (ITEMS) {
        if (A.per_row > 0 || A.out) {
            finish_items<K, NP>(A, acc, (int64_t)tile * 128, i0, i1, slice, smem, wave_count);
            return;
        }
    }
#pragma unroll
    for (int nb = 0; nb < S::NB; ++nb) {
        const int c = nb * 16 + (grp & 1) * (S::KW / 2) + gi;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int64_t row = x0 + tile_row(r) + 4 * h;
            if (row < A.X.count && c < K) A.part[((int64_t)slice * A.X.count + row) * K + c] = acc[nb][r];
        }
    }
}

// Both gradients in one launch: the first `h_blocks` workgroups (a multiple of
// 8, for place()) take the rows' gradients, the others the items'.
template <int K, int NP, int YT, bool ENT>
__global__ __launch_bounds__(kThreads, 2) void k_grad_pass(GradK rows, GradK items, int32_t h_blocks) {
    extern __shared__ __align__(16) unsigned char smem[];
    __shared__ uint32_t wave_count[4];
    const int64_t block = block_of_grid();  // below 2^26
    if (block < h_blocks) grad_pass<K, NP, YT, false, ENT>(rows, (int32_t)block, smem, wave_count);
    else if (items.n_tiles) grad_pass<K, NP, YT, true, ENT>(items, (int32_t)block - h_blocks, smem, wave_count);
}

// out[t] = scale (a_t * sum of the parts + sum_j w_tj F[id_tj]) (a_t in the
// parts already: coef null); K / 8 lanes a row, four listed items in flight.
template <typename E, int K>
__global__ __launch_bounds__(kThreads) void k_grad_rows(const float *part, int32_t n_parts, int64_t T,
                                                        const float4 *coef, const int32_t *ids, const float *w,
                                                        int32_t per_row, const E *F, int64_t ldf, float scale, E *out,
                                                        int64_t ldo) {
    constexpr int LN = K / 8, U = 4;
    const int64_t t = (block_of_grid() * kThreads + threadIdx.x) / LN;
    const int c = (int)(threadIdx.x % LN) * 8;
    if (t >= T) return;
    f8 sum = {}, more = {};
#pragma unroll 4
    for (int32_t p = 0; p < n_parts; ++p) sum += load8(part + ((int64_t)p * T + t) * K + c);
    if (coef) sum *= coef[t].y;
    for (int32_t q = 0; q < per_row; q += U) {
        float v[U];
        f8 f[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = q + u < per_row ? w[t * per_row + q + u] : 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            f[u] = f8{};
            if (v[u] != 0.f) f[u] = load8(F + (int64_t)ids[t * per_row + q + u] * ldf + c);  // 0: also no item's entry
        }
#pragma unroll
        for (int u = 0; u < U; ++u) more += v[u] * f[u];
    }
    sum = (sum + more) * scale;
    if constexpr (sizeof(E) == 4) {
        *reinterpret_cast<f4 *>(out + t * ldo + c) = f4{sum[0], sum[1], sum[2], sum[3]};
        *reinterpret_cast<f4 *>(out + t * ldo + c + 4) = f4{sum[4], sum[5], sum[6], sum[7]};
    } else {
        *reinterpret_cast<uint4 *>(out + t * ldo + c) = __builtin_bit_cast(uint4, __builtin_convertvector(sum, b8));
    }
}

// ------------------------------------------------------------- host side

constexpr int kCus = 256;
constexpr int64_t kSlots = 2 * kCus;  // workgroups of a pass at a time

// How a streamed side of `rows` rows is cut: `tiles` workgroups per slice, of
// which two fit a CU; slices of whole units, a multiple of the 8 XCDs from 8
// on.  Chosen from up to 8 and from whole rounds by the time it takes: rounds of workgroups, each its slice and a
// start that takes as long as about 400 rows, the last round's uneven end, and `slice_cost`, what a
// slice's sums cost to write and add, in rows.
void slices_of(int64_t rows, int64_t tiles, int64_t unit, double slice_cost, int32_t &n_slices, int64_t &slice_rows) {
    double best = 0.0;
    n_slices = 1;
    slice_rows = unit;
    tiles = std::max<int64_t>(1, tiles);  // an empty side
    auto look = [&](int64_t ns) {
        if (ns >= 8) ns = ns / 8 * 8;
        const int64_t each = std::max<int64_t>(unit, ((rows + ns - 1) / ns + unit - 1) / unit * unit);
        const int64_t used = std::max<int64_t>(1, (rows + each - 1) / each);
        const double rounds = (double)((used * tiles + kSlots - 1) / kSlots);
        const double cost = (rounds + 0.15) * ((double)each + 400.0) + (double)used * slice_cost;
        if (best == 0.0 || cost < best) {
            best = cost;
            n_slices = (int32_t)used;
            slice_rows = each;
        }
    };
    for (int64_t ns = 1; ns <= 8; ++ns) look(ns);
    for (int64_t r = 1; r <= 8; ++r)  // whole rounds
        if (kSlots * r / tiles > 8) look(kSlots * r / tiles);
}

struct ScorePlan {
    bool few;
    int64_t chunk;        // rows of a run
    int64_t nblk, padded, ngrp;  // padded: rows with room in blkmax
    int32_t g_log;
    int32_t n_slices, n_tiles, cx;
    int64_t slice_items;
    float4 *part;
    float *blkmax, *sup;
};

// Rows of a run at most: 512 threads a row stay below the 2^32 of a launch.
constexpr int64_t kRunRows = int64_t(1) << 22;

ScorePlan plan_score(int64_t T, int64_t n, int prec, int top, Carve &c) {
    ScorePlan p{};
    p.nblk = (n + 63) / 64 * 2;
    p.few = T <= 32;
    p.chunk = std::min(T, kRunRows);
    if (top > 0) {  // at most 1 GiB of block maxima at a time, but of 256 rows at least (more from 33 M items on)
        const int64_t most = std::max<int64_t>(256, (int64_t(1) << 28) / std::max<int64_t>(p.nblk, 1) / 256 * 256);
        p.chunk = std::min(p.chunk, most);
    }
    p.cx = prec == TSID_BF16 ? 2 : 1;
    if (top > 0)
        while (p.g_log < 6 && p.nblk > (int64_t)kMaxGroups << p.g_log) ++p.g_log;
    const int64_t G = int64_t(1) << p.g_log;  // blocks of a group
    p.ngrp = (p.nblk + G - 1) / G;
    p.padded = T;
    if (p.few) {
        p.n_tiles = 1;
        slices_of(n, 1, 128 * G, 0.0, p.n_slices, p.slice_items);
    } else {
        const int64_t rows = 128 * p.cx;
        p.n_tiles = (int32_t)((p.chunk + rows - 1) / rows);
        p.padded = p.n_tiles * rows;
        slices_of(n, p.n_tiles, std::max<int64_t>(64, 32 * G), 0.5, p.n_slices, p.slice_items);
    }
    p.part = c.take<float4>((int64_t)p.n_slices * p.chunk);
    if (top > 0) {
        p.blkmax = c.take<float>(p.nblk * p.padded);
        if (p.g_log > 0) p.sup = c.take<float>(p.ngrp * p.chunk);
    }
    return p;
}

// Lets a kernel take `lds` bytes of dynamic LDS; `done`: a bit per device.
void allow_lds(const void *kernel, size_t lds, std::atomic<uint64_t> &done) {
    int device = 0;
    TSID_HIP(hipGetDevice(&device));
    const uint64_t bit = uint64_t(1) << (device & 63);
    if (done.load() & bit) return;
    TSID_HIP(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    done.fetch_or(bit);
}

// 64 rows per wave in bf16: two sets of products share each read of F's tile
// (2,048 x 1 M, k = 128: 555 us; 32 rows: 647 us).  Tiles of 64 rows of F, also
// where the blocks' maxima are kept: at k = 128 a dozen registers spill then, and
// still 2,048 x 1 M with entropy and the best 20 takes 920 us, in tiles of 32 rows,
// which do not spill, 1,005 (k = 64: 630 and 730, k = 8: 512 and 570; 16,384 x
// 100 k at k = 128 1,280 and 1,315, with a bias 1,487 and 1,432).  fp32: 32 rows and
// tiles of 32, three parts each.
template <int K, int NP, bool BIAS, bool ENT, bool TOP>
void launch_score_pass(const ScoreK &a, hipStream_t s) {
    constexpr int CX = NP == 1 ? 2 : 1, YT = NP == 1 ? 64 : 32;
    constexpr size_t lds = 3 * Tile<K, NP, YT>::kBytes;
    auto *pass = &k_score_pass<K, NP, CX, YT, BIAS, ENT, TOP>;
    if (lds > 64 * 1024) {  // more dynamic LDS than the default limit: said once per kernel and device
        static std::atomic<uint64_t> done;
        allow_lds(reinterpret_cast<const void *>(pass), lds, done);
    }
    pass<<<grid_of(a.n_slices, a.n_tiles), kThreads, lds, s>>>(a);
}

template <int K, int NP, bool ENT>
void launch_score(const ScoreK &a, const ScorePlan &p, hipStream_t s) {
    if (p.few) {
        k_score_few<K, NP, ENT><<<p.n_slices, kThreads, 0, s>>>(a);
    } else {
        const bool bias = a.F.bias != nullptr;
        if (a.blkmax) bias ? launch_score_pass<K, NP, true, ENT, true>(a, s) : launch_score_pass<K, NP, false, ENT, true>(a, s);
        else bias ? launch_score_pass<K, NP, true, ENT, false>(a, s) : launch_score_pass<K, NP, false, ENT, false>(a, s);
    }
    TSID_HIP(hipGetLastError());
}

template <int K, int NP, bool ENT>
void launch_grad(const GradK &rows, const GradK &items, hipStream_t s) {
    constexpr int YT = NP == 1 ? 64 : 32;
    constexpr size_t tiles = 3 * Tile<K, NP, YT>::kBytes, most = std::max(tiles, listed_lds(K));
    const size_t lds = items.n_tiles && (items.per_row > 0 || items.out) ? most : tiles;
    auto *pass = &k_grad_pass<K, NP, YT, ENT>;
    if (most > 64 * 1024) {
        static std::atomic<uint64_t> done;
        allow_lds(reinterpret_cast<const void *>(pass), most, done);
    }
    const int h_blocks = rows.n_tiles ? (grid_of(rows.n_slices, rows.n_tiles) + 7) / 8 * 8 : 0;
    const int f_blocks = items.n_tiles ? grid_of(items.n_slices, items.n_tiles) : 0;
    pass<<<grid_of_blocks((int64_t)h_blocks + f_blocks), kThreads, lds, s>>>(rows, items, h_blocks);
    TSID_HIP(hipGetLastError());
}

// f.template operator()<K, NP>() for the rank and precision at hand.
template <typename Fn>
void for_rank(int k, int prec, Fn &&f) {
    auto np = [&](auto kk) {
        if (prec == TSID_BF16) f(kk, std::integral_constant<int, 1>());
        else f(kk, std::integral_constant<int, 3>());
    };
    switch (k) {
        case 8: np(std::integral_constant<int, 8>()); break;
        case 16: np(std::integral_constant<int, 16>()); break;
        case 32: np(std::integral_constant<int, 32>()); break;
        case 64: np(std::integral_constant<int, 64>()); break;
        case 128: np(std::integral_constant<int, 128>()); break;
        default: fail(TSID_E_INVAL, "unsupported rank");
    }
}

Side side_of(const Rows &r, const float *bias) { return Side{r.p, r.count, r.ld, bias}; }

// c and the sign of the scores; scale 0 is X = 0 and c = 1.
void exponent_of(const Head &h, float &c, int &turn) {
    c = h.scale == 0.0 ? 1.f : (float)(std::fabs(h.scale) * kLog2e);
    turn = h.scale == 0.0 ? kNone : h.scale < 0.0 ? kTurn : kKeep;
}

// The pass over all items and the rows' results, a run of rows at a time.
void score_rows(const Head &h, const ScorePlan &p, FinishK f, bool entropy, hipStream_t s) {
    ScoreK a{};
    a.H = side_of(h.H, nullptr);
    a.F = side_of(h.F, h.bias);
    exponent_of(h, a.c, a.turn);
    a.bias_c = (float)(h.bias_scale * kLog2e / (double)a.c);
    a.off = kOff / a.c;
    a.slice_items = p.slice_items;
    a.n_slices = p.n_slices;
    a.part = p.part;
    a.blkmax = p.blkmax;
    a.sup = p.sup;
    a.nblk = p.nblk;
    f.width = p.few ? (int32_t)h.H.count : 64;
    a.g_log = f.g_log = p.g_log;
    a.ngrp = p.ngrp;
    f.part = p.part;
    f.n_parts = p.n_slices;
    f.H = a.H;
    f.F = a.F;
    f.scale = h.scale;
    f.bias_scale = h.bias_scale;
    f.blkmax = p.blkmax;
    f.sup = p.sup;
    f.blocks = (h.F.count + 31) / 32;
    f.nblk = p.nblk;
    f.ngrp = p.ngrp;
    for (int64_t t0 = 0; t0 < h.H.count; t0 += p.chunk) {
        a.t0 = f.t0 = t0;
        a.T = f.T = std::min<int64_t>(p.chunk, h.H.count - t0);
        a.n_tiles = (int32_t)((a.T + 128 * p.cx - 1) / (128 * p.cx));
        for_rank(h.k, h.prec, [&](auto kk, auto np) {
            if (entropy) launch_score<kk(), np(), true>(a, p, s);
            else launch_score<kk(), np(), false>(a, p, s);
        });
        for_rank(h.k, h.prec, [&](auto kk, auto np) {
            using E = std::conditional_t<np() == 1, uint16_t, float>;
            if (f.top <= 0) k_score_finish<E, kk(), 64><<<ceil_div(a.T, kThreads / 64), kThreads, 0, s>>>(f);
            else if (a.T > 2 * kCus) k_score_finish<E, kk(), 256><<<(unsigned)a.T, 256, 0, s>>>(f);
            else k_score_finish<E, kk(), 512><<<(unsigned)a.T, 512, 0, s>>>(f);
        });
        TSID_HIP(hipGetLastError());
    }
}

struct GradPlan {
    int32_t h_slices, h_tiles, f_slices, f_tiles;
    int64_t h_rows, f_rows;
    float4 *coef;
    float *w, *h_part, *f_part;
    bool in_pass;  // the listed items' part of dF is added in the pass
    SumPlan sum;
};

// Ids that the workgroups of the items' gradient look through at most for the
// listed items' part, all slots of the device together, taken or not (with few
// workgroups each looks through more); beyond, the entries are sorted, which
// costs seven more launches.  dF in the pass / with the sort, us: 4,096 rows, 20
// listed of 8,192 items (5.2 M) 90 / 112, 50 listed (13 M) 125 / 124, 100 listed
// (26 M) 180 / 147; 2,048 rows, 10 listed of 100 k (16 M) 266 / 260; 256 rows, 8
// listed of 1 M (16 M) 216 / 277; 1,000 rows, 100 listed of 20 k (17 M, 157
// workgroups a slice) 96 / 70; 512 rows, 1,000 listed of 2,000 (33 M, 16) 241 / 99.
constexpr int64_t kInPass = int64_t(1) << 24;

GradPlan plan_grad(int64_t T, int64_t n, int k, int prec, int n_ids, Carve &c) {
    GradPlan p{};
    p.h_tiles = (int32_t)((T + 127) / 128);
    p.f_tiles = (int32_t)((n + 127) / 128);
    // a slice's part of the sums, 8 k bytes a row of X written and read, at 4
    // bytes a ns, against 30 ns a streamed row (128 ns in fp32) for a workgroup
    const double per_row = 2e-3 * k / (prec == TSID_BF16 ? 30.0 : 128.0);
    slices_of(n, p.h_tiles, 64, per_row * (double)T, p.h_slices, p.h_rows);
    slices_of(T, p.f_tiles, 64, per_row * (double)n, p.f_slices, p.f_rows);
    p.coef = c.take<float4>(T);
    p.w = c.take<float>(T * n_ids);
    p.h_part = c.take<float>((int64_t)p.h_slices * T * k);
    const int64_t listed = T * n_ids;
    p.in_pass = listed > 0 && std::max(p.f_tiles * listed, kSlots * ((listed + p.f_slices - 1) / p.f_slices)) <= kInPass;
    p.sum.entries = p.in_pass ? 0 : listed;
    p.f_part = c.take<float>(p.f_slices == 1 && p.sum.entries == 0 ? 0 : (int64_t)p.f_slices * n * k);
    p.sum.n = n;
    p.sum.k = k;
    carve_sum(p.sum, c);
    return p;
}

}  // namespace

size_t score_workspace(int64_t T, int64_t n, int k, int prec, int top) {
    Carve c;
    plan_score(T, n, prec, top, c);
    return c.used;
}

void run_score(const Head &h, const ScoreOut &o, void *ws, size_t bytes, int32_t *err, hipStream_t s) {
    Carve c{static_cast<char *>(ws)};
    const ScorePlan p = plan_score(h.H.count, h.F.count, h.prec, o.top, c);
    check_workspace(ws, bytes, c.used);
    if (h.H.count <= 0) return;
    FinishK f{};
    f.ids = o.ids;
    f.per_row = o.per_row;
    f.lse = o.lse;
    f.logp = o.logp;
    f.entropy = o.entropy;
    f.top = o.top;
    f.top_ids = o.top_ids;
    f.top_logp = o.top_logp;
    f.err = err;
    score_rows(h, p, f, o.entropy != nullptr, s);
}

void run_distill(const Head &h, const DistillOut &o, void *ws, size_t bytes, int32_t *err, hipStream_t s) {
    Carve c{static_cast<char *>(ws)};
    const ScorePlan p = plan_score(h.H.count, h.F.count, h.prec, 0, c);
    check_workspace(ws, bytes, c.used);
    if (h.H.count <= 0) return;
    FinishK f{};
    f.ids = o.ids;
    f.per_row = o.per_row;
    f.lse = o.lse;
    f.teacher = o.teacher;
    f.tau = o.temperature;
    f.loss = o.loss;
    f.err = err;
    score_rows(h, p, f, false, s);
}

size_t head_grad_workspace(int64_t T, int64_t n, int k, int prec, int per_row) {
    Carve c;
    plan_grad(T, n, k, prec, per_row, c);
    return c.used;
}

void run_head_grad(const Head &h, const HeadGrad &g, void *ws, size_t bytes, int32_t *err, hipStream_t s) {
    const int64_t T = h.H.count, n = h.F.count;
    Carve c{static_cast<char *>(ws)};
    GradPlan p = plan_grad(T, n, h.k, h.prec, g.per_row, c);
    check_workspace(ws, bytes, c.used);
    const bool ent = g.dentropy != nullptr;
    if (T > 0) {
        k_head_coef<<<grid_of_blocks(ceil_div(T, 4)), kThreads, 0, s>>>(g, T, n, h.bias, p.coef, p.w, err);
        TSID_HIP(hipGetLastError());
    }
    GradK a{};
    exponent_of(h, a.c, a.turn);
    a.unit = h.prec == TSID_BF16 ? 1.f / a.c : 1.f;
    a.bias_c = (float)(h.bias_scale * kLog2e);
    a.coef = p.coef;
    GradK b = a;
    const bool want_h = g.dH.p && T > 0, want_f = g.dF.p && n > 0;
    if (want_h) {
        a.X = side_of(h.H, nullptr);
        a.Y = side_of(h.F, h.bias);
        a.slice_rows = p.h_rows;
        a.n_slices = p.h_slices;
        a.n_tiles = p.h_tiles;
        a.part = p.h_part;
    }
    if (want_f && T > 0) {
        b.X = side_of(h.F, h.bias);
        b.Y = side_of(h.H, nullptr);
        b.slice_rows = p.f_rows;
        b.n_slices = p.f_slices;
        b.n_tiles = p.f_tiles;
        b.part = p.f_part;
        if (p.in_pass) {
            b.ids = g.ids;
            b.w = p.w;
            b.per_row = g.per_row;
        }
        if (p.f_slices == 1 && p.sum.entries == 0) {  // one slice, and nothing to add: no sums in memory
            b.out = g.dF.p;
            b.ldo = g.dF.ld;
            b.scale = (float)h.scale;
        }
    }
    if (a.n_tiles || b.n_tiles)
        for_rank(h.k, h.prec, [&](auto kk, auto np) {
            if (ent) launch_grad<kk(), np(), true>(a, b, s);
            else launch_grad<kk(), np(), false>(a, b, s);
        });
    if (want_h) {
        const float4 *coef = ent ? nullptr : p.coef;
        for_rank(h.k, h.prec, [&](auto kk, auto np) {
            using E = std::conditional_t<np() == 1, uint16_t, float>;
            k_grad_rows<E, kk()><<<grid_of_blocks(ceil_div(T * (kk() / 8), kThreads)), kThreads, 0, s>>>(
                p.h_part, p.h_slices, T, coef, g.ids, p.w, g.per_row, static_cast<const E *>(h.F.p), h.F.ld, (float)h.scale,
                static_cast<E *>(g.dH.p), g.dH.ld);
        });
        TSID_HIP(hipGetLastError());
    }
    if (want_f && !b.out) {
        SumArgs sa{};
        sa.ids = g.ids;
        sa.bias = h.bias;
        sa.err = err;
        sa.X = h.H;
        sa.w = p.w;
        sa.per_row = std::max(1, g.per_row);
        sa.parts = p.f_part;
        sa.n_parts = T > 0 ? p.f_slices : 0;
        sa.part_stride = n * h.k;
        sa.scale = (float)h.scale;
        sa.out = g.dF;
        launch_sum_rows(p.sum, h.prec, sa, s);
    }
}

}  // namespace tsid
