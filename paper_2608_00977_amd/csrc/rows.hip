// Rows of a factor table by id, scaled, and the gradient of that lookup: the
// sum of the gradients of equal ids.
//
// Both move memory and little else.  A row of k factors is handled by k / 8
// lanes, eight factors each (one 16-byte access in bf16, two in fp32).
//
// The gradient sorts the entries by id (stable, so equal ids keep their
// order), and every row of the table is then written once by the lanes that
// own it, zeros included: no atomics, no clearing pass, the same bits every
// time.  Ids are popular by a power law, so one row may own a large share of
// the entries: rows of more than kSumPiece entries are summed in pieces.  Piece
// q holds the sorted entries 64 q .. 64 q + 63; at most two long rows reach
// into it (a third would lie inside it and be no longer than it), so it leaves
// at most two partial sums, and the row adds its pieces in order.  The same
// once more over the pieces' sums, 64 at a time, where the entries are many.
// Few entries are not sorted at all (k_sum_scan).
//
// Measured (one MI355X): 1,000,003 rows of 128 fp32 by popular ids in 188 us, 5.4
// TB/s of the 1.02 GB that no repeated row is counted in (a copy moves 4.7).  2 M
// bf16 rows of 128 into 1 M in 388 to 394 us against a floor of 162: the sort takes
// 139, the pieces of the long rows (55 % of the entries) 83, the rows 170, whose chain
// of pointer, entry and row is latency more than bandwidth.
#include <algorithm>

#include "rows.h"

namespace tsid {

namespace {

constexpr int kThreads = 256;
typedef float f8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f8 load8(const float *p) {
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    return f8{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
}
__device__ __forceinline__ f8 load8(const uint16_t *p) {
    return __builtin_convertvector(__builtin_bit_cast(b8, *reinterpret_cast<const uint4 *>(p)), f8);
}
__device__ __forceinline__ void store8(float *p, f8 v) {
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void store8(uint16_t *p, f8 v) {  // round to nearest even
    *reinterpret_cast<uint4 *>(p) = __builtin_bit_cast(uint4, __builtin_convertvector(v, b8));
}

// Four rows of each group of lanes in flight: the gathers' latency, not their
// number, bounds a lookup otherwise.
constexpr int kLookupRows = 4;

template <typename E>
__global__ __launch_bounds__(kThreads) void k_lookup(const E *F, int64_t n, int64_t ldf, const int32_t *ids,
                                                     int64_t count, float scale, E *out, int64_t ldo, int lanes_log,
                                                     int32_t *err) {
    const int64_t g = (block_of_grid() * kThreads + threadIdx.x) >> lanes_log;
    const int64_t groups = ((int64_t)gridDim.y * gridDim.x * kThreads) >> lanes_log;
    const int c = (threadIdx.x & ((1 << lanes_log) - 1)) * 8;
    bool bad = false;
    f8 v[kLookupRows];
#pragma unroll
    for (int x = 0; x < kLookupRows; ++x) {
        const int64_t t = g + x * groups;
        const int32_t id = t < count ? ids[t] : -1;
        const bool in = id >= 0 && id < n;
        bad |= !in && id != -1;
        v[x] = f8{};
        if (in) v[x] = load8(F + (int64_t)id * ldf + c);
    }
#pragma unroll
    for (int x = 0; x < kLookupRows; ++x) {
        const int64_t t = g + x * groups;
        if (t < count) store8(out + t * ldo + c, v[x] * scale);
    }
    if (bad) err[ERR_RANGE] = 1;
}

__global__ void k_take_slots(int32_t *slots, int32_t *taken, int n) {
    if ((int)threadIdx.x < n) taken[threadIdx.x] = atomicExch(slots + threadIdx.x, 0);
}

// key = id (n for an entry that adds nothing), value = entry.
__global__ __launch_bounds__(kThreads) void k_sum_keys(const int32_t *ids, int64_t entries, int64_t n,
                                                       const float *bias, uint64_t *keys, uint32_t *vals,
                                                       uint32_t *ctl, int ctl_n, int32_t *err) {
    const int64_t id0 = (int64_t)blockIdx.x * kThreads + threadIdx.x, step = (int64_t)gridDim.x * kThreads;
    for (int64_t j = id0; j < ctl_n; j += step) ctl[j] = 0u;
    bool bad = false;
    for (int64_t e = id0; e < entries; e += step) {
        const int32_t id = ids[e];
        bool in = id >= 0 && id < n;
        bad |= !in && id != -1;
        if (in && bias && bias[id] < kExcluded) in = false;
        keys[e] = in ? (uint64_t)(uint32_t)id : (uint64_t)n;
        vals[e] = (uint32_t)e;
    }
    if (bad) err[ERR_RANGE] = 1;
}

// ptr[x] = first position whose key >= x, for x in [0, n].
__global__ __launch_bounds__(kThreads) void k_sum_ptr(const uint64_t *keys, int64_t entries, int64_t n,
                                                      uint32_t *ptr) {
    const int64_t x = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (x > n) return;
    int64_t lo = 0, hi = entries;
    while (lo < hi) {
        const int64_t mid = lo + ((hi - lo) >> 1);
        if (keys[mid] < (uint64_t)x) lo = mid + 1;
        else hi = mid;
    }
    ptr[x] = (uint32_t)lo;
}

struct SumK {
    const uint64_t *keys;
    const uint32_t *vals, *ptr;
    int64_t entries, n;
    const float *w;
    uint32_t per_row;
    int64_t ldx;
    int lanes_log;  // lanes of a row: k / 8
    float *carry0, *carry1;
    int two_levels;
    const float *parts;
    int32_t n_parts;
    int64_t part_stride;
    float scale;
    int64_t ldo;
};

// The entry at place e of the sorted list.
__device__ __forceinline__ uint32_t source_row(const SumK &A, uint32_t val) {
    return A.per_row == 1 ? val : val / A.per_row;
}

// Sum of the sorted entries e0 .. e1 - 1 in order, U rows in flight.
template <int U, typename E>
__device__ __forceinline__ f8 sum_entries(const SumK &A, const E *X, uint32_t e0, uint32_t e1, int c) {
    f8 sum = f8{};
    for (uint32_t e = e0; e < e1; e += U) {
        uint32_t val[U];
        f8 v[U];
        float w[U];
#pragma unroll
        for (int x = 0; x < U; ++x) val[x] = A.vals[e + x < e1 ? e + x : e0];
#pragma unroll
        for (int x = 0; x < U; ++x) {
            w[x] = A.w ? A.w[val[x]] : 1.f;
            v[x] = load8(X + (int64_t)source_row(A, val[x]) * A.ldx + c);
        }
#pragma unroll
        for (int x = 0; x < U; ++x)
            if (e + x < e1) sum += w[x] * v[x];
    }
    return sum;
}

// The value of the lane `off` lanes away (a power of two), eight at a time.
__device__ __forceinline__ f8 other_lanes(f8 v, int off) {
    f8 o;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = __shfl_xor(v[j], off, 64);
    return o;
}

// The partial sums that a piece of kSumPiece consecutive units (entries, or
// the pieces of the level below) leaves for the long rows that reach into it:
// [0] of the row at its first entry, [1] of the row at its last, if another.
// Four lane groups take a quarter of the piece each, in order, since one would
// wait for 64 rows after one another.
template <typename E, int LEVEL>
__global__ __launch_bounds__(kThreads) void k_sum_pieces(SumK A, const E *X, int64_t pieces) {
    const int64_t g = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> A.lanes_log, q = g >> 2;
    if (q >= pieces) return;  // whole pieces leave together
    constexpr int64_t kSpan = LEVEL == 0 ? kSumPiece : kSumPiece * kSumPiece;  // entries of a piece
    const int lanes = 1 << A.lanes_log, part = (int)(g & 3);
    const int c = (threadIdx.x & (lanes - 1)) * 8, k = 8 << A.lanes_log;
    const int64_t first = q * kSpan, last = (first + kSpan < A.entries ? first + kSpan : A.entries) - 1;
    const uint64_t r0 = A.keys[first], r1 = A.keys[last];
    float *out = (LEVEL == 0 ? A.carry0 : A.carry1) + q * 2 * k + c;
    for (int slot = 0; slot < 2; ++slot) {
        const uint64_t r = slot ? r1 : r0;
        if (r >= (uint64_t)A.n || (slot && r1 == r0)) continue;
        const int64_t a = A.ptr[r], b = A.ptr[r + 1];
        if (b - a <= kSpan) continue;
        int64_t e0 = a > first ? a : first, e1 = b < last + 1 ? b : last + 1;
        f8 sum = f8{};
        if constexpr (LEVEL == 0) {
            const int64_t quarter = (e1 - e0 + 3) / 4;
            const int64_t s0 = e0 + part * quarter < e1 ? e0 + part * quarter : e1;
            const int64_t s1 = s0 + quarter < e1 ? s0 + quarter : e1;
            sum = sum_entries<8>(A, X, (uint32_t)s0, (uint32_t)s1, c);
        } else {
            const int64_t p0 = e0 / kSumPiece, p1 = (e1 + kSumPiece - 1) / kSumPiece, quarter = (p1 - p0 + 3) / 4;
            const int64_t s1 = p0 + (part + 1) * quarter < p1 ? p0 + (part + 1) * quarter : p1;
#pragma unroll 4
            for (int64_t p = p0 + part * quarter; p < s1; ++p)
                sum += load8(A.carry0 + (p * 2 + (a > p * kSumPiece ? 1 : 0)) * k + c);
        }
        sum += other_lanes(sum, lanes);
        sum += other_lanes(sum, 2 * lanes);
        if (part == 0) store8(out + slot * k, sum);
    }
}

// The parts' sums of row i.
__device__ __forceinline__ f8 sum_parts(const SumK &A, int64_t i, int c, int k) {
    f8 sum = f8{};
#pragma unroll 4
    for (int32_t p = 0; p < A.n_parts; ++p) sum += load8(A.parts + p * A.part_stride + i * k + c);
    return sum;
}

// One row per lane group: a wave waits for the longest of its rows, so that two
// rows each, with their first entries loaded ahead, are no faster where most rows
// have no entry either (25 k entries into 100 k rows of 128: 58 us both ways).
template <typename E>
__global__ __launch_bounds__(kThreads) void k_sum_rows(SumK A, const E *X, E *out) {
    const int64_t i = (block_of_grid() * kThreads + threadIdx.x) >> A.lanes_log;
    if (i >= A.n) return;
    const int c = (threadIdx.x & ((1 << A.lanes_log) - 1)) * 8, k = 8 << A.lanes_log;
    const uint32_t a = A.entries ? A.ptr[i] : 0u, b = A.entries ? A.ptr[i + 1] : 0u;
    f8 sum = sum_parts(A, i, c, k);
    if (b - a > (uint32_t)kSumPiece) {
        const bool two = A.two_levels && b - a > (uint32_t)(kSumPiece * kSumPiece);
        const float *carry = two ? A.carry1 : A.carry0;
        const int64_t span = two ? kSumPiece * kSumPiece : kSumPiece;
        f8 more = f8{};
#pragma unroll 4
        for (int64_t p = a / span; p < (b + span - 1) / span; ++p)
            more += load8(carry + (p * 2 + (a > p * span ? 1 : 0)) * k + c);
        sum += more;
    } else if (b > a) {
        sum += sum_entries<4>(A, X, a, b, c);
    }
    store8(out + i * A.ldo + c, sum * A.scale);
}

// A lookup's gradient without a sort: a wave per row of the table reads the ids of
// all entries, 64 at a time, and its lane groups take the matching ones in
// turn.  Few entries and rows only (kScanEntries, kScanRows).
template <typename E>
__global__ __launch_bounds__(kThreads) void k_sum_scan(const int32_t *ids, int64_t entries, const E *X, int64_t ldx,
                                                       float scale, E *out, int64_t n, int64_t ldo, int lanes_log,
                                                       int32_t *err) {
    const int64_t i = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6);
    if (i >= n) return;
    const int lane = threadIdx.x & 63, lanes = 1 << lanes_log, groups = 64 >> lanes_log, grp = lane >> lanes_log;
    const int c = (lane & (lanes - 1)) * 8;
    f8 sum = f8{};
    bool bad = false;
    int turn = 0;  // of the groups
    for (int64_t e0 = 0; e0 < entries; e0 += 256) {
        int32_t id[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int64_t e = e0 + 64 * x + lane;
            id[x] = e < entries ? ids[e] : -1;
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            bad |= id[x] < -1 || id[x] >= n;
            uint64_t match = __ballot(id[x] == (int32_t)i);
            while (match) {  // `groups` matches at a time
                uint32_t mine = ~0u;
                for (int g = 0; g < groups && match; ++g) {
                    const uint32_t e = (uint32_t)(e0 + 64 * x) + (uint32_t)__builtin_ctzll(match);
                    match &= match - 1;
                    if (((turn + g) & (groups - 1)) == grp) mine = e;
                }
                turn += 1;
                if (mine != ~0u) sum += load8(X + (int64_t)mine * ldx + c);
            }
        }
    }
    if (bad && i == 0) err[ERR_RANGE] = 1;
    for (int off = lanes; off < 64; off <<= 1) sum += other_lanes(sum, off);
    if (grp == 0) store8(out + i * ldo + c, sum * scale);
}

int lanes_log_of(int k) {
    switch (k) {
        case 8: return 0;
        case 16: return 1;
        case 32: return 2;
        case 64: return 3;
        case 128: return 4;
        default: fail(TSID_E_INVAL, "unsupported rank");
    }
}

int64_t pieces_of(int64_t entries, int64_t span) { return (entries + span - 1) / span; }

template <typename E>
void sum_rows(const SumPlan &p, const SumArgs &a, hipStream_t s) {
    const E *X = static_cast<const E *>(a.X.p);
    E *out = static_cast<E *>(a.out.p);
    if (p.scan) {
        k_sum_scan<E><<<ceil_div(p.n, kThreads / 64), kThreads, 0, s>>>(
            a.ids, p.entries, X, a.X.ld, a.scale, out, p.n, a.out.ld, lanes_log_of(p.k), a.err);
        TSID_HIP(hipGetLastError());
        return;
    }
    SumK A{};
    A.keys = p.keys[p.alt];
    A.vals = p.vals[p.alt];
    A.ptr = p.ptr;
    A.entries = p.entries;
    A.n = p.n;
    A.w = a.w;
    A.per_row = (uint32_t)a.per_row;
    A.ldx = a.X.ld;
    A.lanes_log = lanes_log_of(p.k);
    A.carry0 = p.carry[0];
    A.carry1 = p.carry[1];
    A.two_levels = p.entries > kSumPiece * kSumPiece;
    A.parts = a.parts;
    A.n_parts = a.n_parts;
    A.part_stride = a.part_stride;
    A.scale = a.scale;
    A.ldo = a.out.ld;
    if (p.entries > kSumPiece) {
        const int64_t n0 = pieces_of(p.entries, kSumPiece);
        k_sum_pieces<E, 0><<<ceil_div(n0 << (A.lanes_log + 2), kThreads), kThreads, 0, s>>>(A, X, n0);
        TSID_HIP(hipGetLastError());
    }
    if (A.two_levels) {
        const int64_t n1 = pieces_of(p.entries, kSumPiece * kSumPiece);
        k_sum_pieces<E, 1><<<ceil_div(n1 << (A.lanes_log + 2), kThreads), kThreads, 0, s>>>(A, X, n1);
        TSID_HIP(hipGetLastError());
    }
    k_sum_rows<E><<<grid_of_blocks(ceil_div(p.n << A.lanes_log, kThreads)), kThreads, 0, s>>>(A, X, out);
    TSID_HIP(hipGetLastError());
}

}  // namespace

void launch_lookup(int k, int prec, const Rows &F, const int32_t *ids, float scale, const Rows &out, int32_t *err,
                   hipStream_t s) {
    if (out.count <= 0) return;
    const int lg = lanes_log_of(k);
    const dim3 blocks = grid_of_blocks(ceil_div(((out.count + kLookupRows - 1) / kLookupRows) << lg, kThreads));
    if (prec == TSID_BF16)
        k_lookup<uint16_t><<<blocks, kThreads, 0, s>>>(static_cast<const uint16_t *>(F.p), F.count, F.ld, ids,
                                                       out.count, scale, static_cast<uint16_t *>(out.p), out.ld, lg,
                                                       err);
    else
        k_lookup<float><<<blocks, kThreads, 0, s>>>(static_cast<const float *>(F.p), F.count, F.ld, ids, out.count,
                                                    scale, static_cast<float *>(out.p), out.ld, lg, err);
    TSID_HIP(hipGetLastError());
}

void launch_take_slots(int32_t *slots, int32_t *taken, int n, hipStream_t s) {
    k_take_slots<<<1, 64, 0, s>>>(slots, taken, n);
    TSID_HIP(hipGetLastError());
}

void check_workspace(const void *ws, size_t bytes, size_t needed) {
    if (!ws || reinterpret_cast<uintptr_t>(ws) % 256 != 0)
        fail(TSID_E_INVAL, "the workspace must be 256-byte aligned device memory");
    if (bytes < needed)
        fail(TSID_E_INVAL, "the workspace has " + std::to_string(bytes) + " bytes of " + std::to_string(needed));
}

void carve_sum(SumPlan &p, Carve &c) {
    p.scan = p.plain && p.entries > 0 && p.n > 0 && p.entries <= kScanEntries && p.n <= kScanRows;
    if (p.scan) {
        c.take<uint32_t>(1);  // a size of 0 says that the arguments are wrong
        return;
    }
    for (int x = 0; x < 2; ++x) {
        p.keys[x] = c.take<uint64_t>(p.entries);
        p.vals[x] = c.take<uint32_t>(p.entries);
    }
    p.sort_scratch = c.take<uint32_t>((int64_t)radix_scratch_elems(p.entries));
    p.ptr = c.take<uint32_t>(p.n + 1);
    p.carry[0] = c.take<float>(pieces_of(p.entries, kSumPiece) * 2 * p.k);
    p.carry[1] = c.take<float>(pieces_of(p.entries, kSumPiece * kSumPiece) * 2 * p.k);
    p.alt = false;
}

static void sum_sort(SumPlan &p, const int32_t *ids, const float *bias, int32_t *err, hipStream_t s) {
    if (p.entries <= 0) return;
    const int blocks = (int)std::min<int64_t>(ceil_div(p.entries, kThreads), 2048);
    k_sum_keys<<<blocks, kThreads, 0, s>>>(ids, p.entries, p.n, bias, p.keys[0], p.vals[0], p.sort_scratch,
                                           radix_ctl_elems(), err);
    TSID_HIP(hipGetLastError());
    p.alt = radix_sort(p.keys[0], p.vals[0], p.keys[1], p.vals[1], p.entries, 0, bits_for(p.n + 1), p.sort_scratch, s,
                       {}, true);
    k_sum_ptr<<<ceil_div(p.n + 1, kThreads), kThreads, 0, s>>>(p.keys[p.alt], p.entries, p.n, p.ptr);
    TSID_HIP(hipGetLastError());
}

void launch_sum_rows(SumPlan &p, int prec, const SumArgs &a, hipStream_t s) {
    if (!p.scan) sum_sort(p, a.ids, a.bias, a.err, s);  // reports the ids of an empty table too
    if (p.n <= 0) return;
    if (prec == TSID_BF16) sum_rows<uint16_t>(p, a, s);
    else sum_rows<float>(p, a, s);
}

}  // namespace tsid
