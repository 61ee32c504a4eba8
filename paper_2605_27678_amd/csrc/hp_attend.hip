// Attention of packed query rows to packed states: row r sees the states lo(r) .. hi(r) - 1.
//     s = scale q k^T,  p = exp(s - m) / sum,  out = p v
// in one pass over the states with a running maximum m and sum, and backward, with P = exp(s - lse) and
// delta = sum over channels of dout out,
//     dv = P^T dout,  dS = P (dout v^T - delta),  dq = scale dS k,  dk = scale dS^T q.
//
// The query heads that share a state head are rows of one matrix: its row M = row * group + head of the group, so a
// tile of states serves all of them, and their gradients add up in the accumulators.
//
// Every product is v_mfma_f32_32x32x16_bf16, or eight v_mfma_f32_32x32x2_f32 over the same 16 values for binary32, and
// is laid out so that no intermediate leaves the registers.  For such a product lane l holds, of the left operand, row
// l % 32, of the right one column l % 32, and of the result column l % 32 and rows 8b + 4(l / 32) + t (b, t < 4).  With the
// states on the left, S^T = K Q^T, each lane has scores of one query row, so maxima and sums are taken within the lane and
// its partner l ^ 32; and the rows that a lane holds of P^T are, taken eight at a time, the 8 of 16 inner values that it
// has to hold of the right operand of the next product, out^T = V^T P^T, if V^T is read with its keys in that order.  That
// left operand comes from V as it lies in memory, by the transposing LDS load (four keys of one channel in a lane).
//
// In bf16 two values on the way are rounded to 16 bits besides the results: P, as an operand of V^T P^T and P^T dout, and dS,
// as one of dS k and dS^T q (statistics, sums and accumulators are binary32, and in binary32 nothing is rounded).  The
// matrix units take 16-bit operands; a second one for what the first leaves out would make three products of the forward's
// two.  Measured against 64 bits the results are 0.0020 to 0.0024 of their size off, 0.0017 if they alone were rounded.
//
// A row must not feel what it does not see, and 0 * inf is NaN: scores are masked by selection, and where a tile of
// states that not all rows of a wave see holds an infinity or NaN, the workgroup begins again in a function of its own,
// which makes the products of such tiles value by value (careful_product).  Beside the loop that is there for speed, that
// code cost it registers, and loads from scratch memory wait for the tiles on their way.
//
// What bounds it.  A wave reads 1 KiB of LDS for each product of 32 x 32 x 16, which takes LDS as long (at 128 bytes a cycle)
// as the matrix units: both, and the exponentials, are busy for 30 to 45 % of the time each, and only waves at different
// places overlap them - two a SIMD, which is what registers allow.  Heads of 128 in bf16 on an MI355X, counting what is seen:
// forward 1.0 PFLOP/s (8192 rows of 32 heads, 4032 states each: 0.54 ms) and 0.92 (16384 rows of 10 heads against up to 40139:
// 1.85 ms); dq 0.6 ms and dk, dv 1.3 ms of 2.16 for 8192 rows of 32 heads against up to 5760 states (8192^3 by the library:
// 1.18 PFLOP/s).  Single tokens are bound by memory: 64 rows of 64 heads against 576 to 6404 states 4.8 TB/s (a large copy:
// 5.2).  Tried and left: 64-row tiles in one loop with the other block's exponentials among the products (the backward of
// states spills: 4.7 ms), raised priority for the waves in a product (no change).
#include <cfloat>
#include <climits>
#include <cmath>
#include <type_traits>

#include "hp_device.hpp"
#include "hp_meet.hpp"
#include "hp_operators.h"

#pragma clang fp contract(fast)

namespace {

using namespace hp;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kBlock = 256, kWaves = kBlock / kWave;
constexpr int kTileM = 32 * kWaves;                 // query rows (times group) of a workgroup
constexpr int kStepKeys = 32 * kWaves;              // states that a workgroup of the single-token kernel takes at a time

typedef float Acc __attribute__((ext_vector_type(16)));
template <class T> using Frag = Vec<T, 8>;

// Whether a pass met what only the careful one takes right.
__device__ __forceinline__ bool again(const int *bad) {
    return __builtin_amdgcn_readfirstlane(read_together(bad, [] { __syncthreads(); })) != 0;
}

// Division of numbers below 2^30 by one that a launch keeps.
struct Divisor {
    uint32_t by, factor, shift;
    __device__ __forceinline__ int operator()(int n) const { return (int)(__umulhi(2u * (uint32_t)n, factor) >> shift); }
};

struct Attend {
    int64_t rows, keys;
    int32_t heads_q, heads_k, group, dim, splits, m_total;
    Divisor by_group;
    float scale, scale2;                            // scale2: for exponents of two
    hp_heads_t q, k, v, out, dout, dq, dk, dv;
    const int32_t *ranges;
    float *lse;
    float *part, *part_lse;                         // [splits][rows * heads_q][dim], [splits][rows * heads_q]
    float *info;                                    // [heads_k][m_lines / tile][4][tile]: lse2, delta, first and end of what a row M sees
    int4 *bounds;                                   // of each 32 rows M
    int32_t m_lines, reserved;                      // rows M, filled up to whole workgroups
    float *part_k, *part_v;                         // [splits][keys * heads_k][dim]
};

__device__ __forceinline__ Acc mma(const Frag<__bf16> &a, const Frag<__bf16> &b, const Acc &c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ Acc mma(const Frag<float> &a, const Frag<float> &b, Acc c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
}

// A tile of states or query rows in LDS: rows of DP elements, one behind the other as the loads that write LDS directly
// leave them, the 16-byte pieces of each row turned among themselves.  Operands take one piece of 8 neighbouring rows, or
// two pieces of 4, at a time: turned, these lie in different banks.
template <class T, int DP> struct Tile {
    static constexpr int kPiece = 16 / (int)sizeof(T), kPieces = DP / kPiece;
    static __device__ __forceinline__ int turn(int row) {              // the same for rows 16 apart
        if constexpr (kPieces == 8) return (row & 6) | ((row >> 3) & 1);
        else if constexpr (kPieces == 12) return (row >> 2) & 3;
        else if constexpr (kPieces == 24) return (row >> 1) & 7;
        else return ((row << 1) & 14) | ((row >> 3) & 1);
    }
    static constexpr bool kRolls = kPieces == 12 || kPieces == 24;     // no power of two: turned round, not exchanged
    static __device__ __forceinline__ int slot_of(int row, int piece) {
        if constexpr (kRolls) {
            const int at = piece + turn(row);
            return at >= kPieces ? at - kPieces : at;
        } else return piece ^ turn(row);
    }
    static __device__ __forceinline__ int piece_of(int row, int slot) {
        if constexpr (kRolls) {
            const int at = slot - turn(row);
            return at < 0 ? at + kPieces : at;
        } else return slot ^ turn(row);
    }
    static __device__ __forceinline__ int offset(int row, int piece) { return row * DP + slot_of(row, piece) * kPiece; }
    static __device__ __forceinline__ float value(const T *tile, int row, int channel) {
        return (float)tile[offset(row, channel / kPiece) + channel % kPiece];
    }
};

// Row `row` of a tile, channels 16s + 8(l / 32) and on: an operand whose inner index is the channel.
template <class T, int DP> __device__ __forceinline__ Frag<T> row_frag(const T *tile, int row, int s, int half) {
    typedef Vec<T, 16 / (int)sizeof(T)> Piece;
    if constexpr (sizeof(T) == 2) {
        return *(const Piece *)(tile + Tile<T, DP>::offset(row, 2 * s + half));
    } else {
        const Piece a = *(const Piece *)(tile + Tile<T, DP>::offset(row, 4 * s + 2 * half)), b = *(const Piece *)(tile + Tile<T, DP>::offset(row, 4 * s + 2 * half + 1));
        return Frag<T>{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    }
}

// Rows 16 ks + 4(l / 32) + {0..3} and 8 more of a tile, at channel 32 db + l % 32: a left operand whose inner index is
// the tile's row, in the order in which a lane holds the rows of a result.
template <class T, int DP> __device__ __forceinline__ Frag<T> column_frag(const T *tile, int ks, int db, int lane) {
    if constexpr (sizeof(T) == 2) {
        typedef short Quad __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) Quad *Lds;
        // 16 lanes together take 16 channels of four rows, four of them each, and get four rows of one
        const int i = lane % 16, row = 4 * (lane / 32) + i / 4, piece = 4 * db + 2 * ((lane / 16) % 2) + (i % 4) / 2;
        union {
            Quad q[2];
            Frag<T> f;
        } u;
        u.q[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(tile + Tile<T, DP>::offset(row, piece) + 16 * ks * DP + 4 * (i % 2)));
        u.q[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(tile + Tile<T, DP>::offset(row + 8, piece) + 16 * ks * DP + 4 * (i % 2)));
        return u.f;
    } else {
        Frag<T> f;
        const int channel = 32 * db + lane % 32;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = 4 * (lane / 32) + 8 * (j / 4) + j % 4;
            f[j] = tile[Tile<T, DP>::offset(row, channel / 4) + 16 * ks * DP + channel % 4];
        }
        return f;
    }
}

// Tells the scheduler how the code before this goes: `ahead` LDS reads, then `products` matrix instructions with the
// remaining reads between them, `each` after every one.  Left to itself it reads one operand, waits and multiplies.
template <int READS, int PRODUCTS, int AHEAD, int EACH> __device__ __forceinline__ void stream() {
    constexpr int kProduct = 0x8, kRead = 0x100;
    __builtin_amdgcn_sched_group_barrier(kRead, AHEAD < READS ? AHEAD : READS, 0);
#pragma unroll
    for (int n = 0; n < PRODUCTS; ++n) {
        __builtin_amdgcn_sched_group_barrier(kProduct, 1, 0);
        if (AHEAD + n * EACH < READS) __builtin_amdgcn_sched_group_barrier(kRead, EACH, 0);
    }
}

// Eight of a result's rows as the right operand of the next product.
template <class T> __device__ __forceinline__ Frag<T> result_frag(const Acc &r, int eighths) {
    Frag<T> f;
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (T)r[8 * eighths + j];          // rounded to nearest even for bf16
    return f;
}

__device__ __forceinline__ int result_row(int i, int half) { return 8 * (i / 4) + 4 * half + i % 4; }

// The values of lanes l % 32 and l % 32 + 32.
__device__ __forceinline__ float2 both_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Whether any of the tile's values is an infinity or NaN, as far as this lane looks.
template <class T, int DP, int ROWS, int THREADS = kBlock> __device__ __forceinline__ bool not_finite(const T *tile, int tid) {
    typedef uint32_t Piece __attribute__((ext_vector_type(4)));
    bool bad = false;
    for (int e = tid; e < ROWS * Tile<T, DP>::kPieces; e += THREADS) {
        const Piece v = *(const Piece *)(tile + e * Tile<T, DP>::kPiece);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (sizeof(T) == 2) bad |= (v[j] & 0x7f80u) == 0x7f80u || (v[j] & 0x7f800000u) == 0x7f800000u;
            else bad |= (v[j] & 0x7f800000u) == 0x7f800000u;
        }
    }
    return bad;
}

// acc^T += tile^T p^T over 32 rows of a tile that p holds (from `row0`), leaving out what is not seen: for values there
// that are not finite, which a product would carry into every row.
template <class T, int DP, int DB, class Seen>
__device__ __forceinline__ void careful_product(Acc (&acc)[DB], const Acc &p, const T *tile, int row0, int half, const Seen &seen) {
    for (int j = 0; j < 32; ++j) {
        float own = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) own = i == 4 * (j / 8) + j % 4 ? p[i] : own;
        const float2 two = both_halves(own);
        const float w = (j / 4) % 2 ? two.y : two.x;
        if (!seen(j)) continue;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[db][i] += w * Tile<T, DP>::value(tile, row0 + j, 32 * db + result_row(i, half));
    }
}

// Brings tiles of ROWS rows from memory to LDS.  Where rows are whole aligned pieces (EXACT) the loads write LDS
// themselves, from a buffer that begins at the tile's first row, and what lies behind its rows or channels is out of the
// buffer's bounds and comes as zeros; the caller waits (arrived()) before the barrier behind which the tile is read.
// Other rows pass through registers at once.
constexpr uint32_t kOutside = 0x80000000u;
constexpr int but(int loads) { return (loads & 15) | 0x0f70 | (loads >> 4) << 14; }            // s_waitcnt vmcnt(loads)
__device__ __forceinline__ void arrived() { __builtin_amdgcn_s_waitcnt(but(0)); }
// All loads of this wave but those of the last `tiles` tiles, of which it makes EACH a tile.
template <int EACH> __device__ __forceinline__ void arrived_but(int tiles) {
    if (tiles <= 0) __builtin_amdgcn_s_waitcnt(but(0));
    else if (tiles == 1) __builtin_amdgcn_s_waitcnt(but(under_way(EACH, 1)));
    else __builtin_amdgcn_s_waitcnt(but(under_way(EACH, 2)));
}

template <class T, int DP, int ROWS, int THREADS, bool EXACT> struct Loader {
    typedef Tile<T, DP> L;
    static constexpr int kAll = ROWS * L::kPieces, kEach = (kAll + THREADS - 1) / THREADS;
    static_assert(kAll % kWave == 0, "every wave loads whole or not");
    static constexpr int kMost = loads_of_wave(kAll, THREADS, 0), kLeast = loads_of_wave(kAll, THREADS, THREADS / kWave - 1);
    // whether the lane's wave has pieces in round n
    static __device__ __forceinline__ bool loads(int n, int tid) { return (n + 1) * THREADS <= kAll || __builtin_amdgcn_readfirstlane(n * THREADS + tid) < kAll; }
    static __device__ __forceinline__ void piece(T *tile, int n, const T *p, int valid, int tid) {
        *(Vec<T, L::kPiece> *)(tile + (n * THREADS + tid) * L::kPiece) = load<L::kPiece>(p, valid);
    }
    static __device__ __forceinline__ void direct(T *tile, int n, const __amdgpu_buffer_rsrc_t &from, uint32_t offset, int tid) {
        // a wave writes 64 pieces in a row
        __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void *)(tile + (n * THREADS + __builtin_amdgcn_readfirstlane(tid / kWave * kWave)) * L::kPiece),
                                                 16, (int)offset, 0, 0, 0);
    }
    static __device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer(const void *base) {
        return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, 0x7fffffff, 0x00020000);
    }
    uint32_t offsets[EXACT ? kEach : 1];

    // Tiles of consecutive rows of one head.
    __device__ __forceinline__ void plan(int64_t row_stride, int dim, int tid) {
        if constexpr (EXACT)
#pragma unroll
            for (int n = 0; n < kEach; ++n) {
                const int e = n * THREADS + tid, row = e / L::kPieces, c = L::piece_of(row, e % L::kPieces);
                offsets[n] = c * L::kPiece < dim ? (uint32_t)(row * row_stride * sizeof(T)) + c * 16 : kOutside;
            }
    }
    // first: the tile's first row; left: rows from there on that are there
    __device__ __forceinline__ void fetch(T *tile, const T *first, int64_t row_stride, int left, int dim, int tid) const {
        if constexpr (EXACT) {
            const auto from = buffer(first);
#pragma unroll
            for (int n = 0; n < kEach; ++n)
                if (loads(n, tid)) direct(tile, n, from, (n * THREADS + tid) / L::kPieces < left ? offsets[n] : kOutside, tid);
        } else {
#pragma unroll
            for (int n = 0; n < kEach; ++n) {
                if (!loads(n, tid)) continue;
                const int e = n * THREADS + tid, row = e / L::kPieces, c = L::piece_of(row, e % L::kPieces);
                piece(tile, n, first + row * row_stride + c * L::kPiece, row < left ? dim - c * L::kPiece : 0, tid);
            }
        }
    }
    // Rows M of the matrix that a state head's query heads make.  Where a tile is whole query rows, as for every group that
    // is a power of two, its places are the same for all tiles; otherwise each tile's are worked out for it.
    static __device__ __forceinline__ bool regular(const Divisor &group) { return group.by <= ROWS && ROWS % group.by == 0; }
    __device__ __forceinline__ void plan_m(const hp_heads_t &x, const Divisor &group, int dim, int tid) {
        if constexpr (EXACT)
#pragma unroll
            for (int n = 0; n < kEach; ++n) {
                const int e = n * THREADS + tid, r = e / L::kPieces, c = L::piece_of(r, e % L::kPieces), row = group(r), head = r - row * (int)group.by;
                offsets[n] = c * L::kPiece < dim ? (uint32_t)((row * (int)x.row_stride + head * (int)x.head_stride) * (int)sizeof(T)) + c * 16 : kOutside;
            }
    }
    __device__ __forceinline__ void fetch_m(T *tile, const hp_heads_t &x, int m0, int m_total, const Divisor &group, int head0, int dim, int tid) const {
        const int row0 = __builtin_amdgcn_readfirstlane(group(m0));
        const T *first = (const T *)x.data + row0 * x.row_stride + (int64_t)head0 * x.head_stride;
        const auto from = buffer(first);
        if (EXACT && regular(group)) {
#pragma unroll
            for (int n = 0; n < kEach; ++n)
                if (loads(n, tid)) direct(tile, n, from, (n * THREADS + tid) / L::kPieces < m_total - m0 ? offsets[EXACT ? n : 0] : kOutside, tid);
            return;
        }
#pragma unroll
        for (int n = 0; n < kEach; ++n) {
            if (!loads(n, tid)) continue;
            const int e = n * THREADS + tid, r = e / L::kPieces, c = L::piece_of(r, e % L::kPieces), m = m0 + r;
            const int row = group(m), head = m - row * (int)group.by;
            if constexpr (EXACT) {
                const uint32_t at = (uint32_t)(((row - row0) * (int)x.row_stride + head * (int)x.head_stride) * (int)sizeof(T)) + c * 16;
                direct(tile, n, from, m < m_total && c * L::kPiece < dim ? at : kOutside, tid);
            } else {
                const int64_t at = (row - row0) * x.row_stride + head * x.head_stride + c * L::kPiece;
                piece(tile, n, first + at, m < m_total ? dim - c * L::kPiece : 0, tid);
            }
        }
    }
};

// What one query row sees.
struct Range {
    int lo, hi;
    __device__ __forceinline__ bool empty() const { return lo >= hi; }
    __device__ __forceinline__ bool has(int key) const { return key >= lo && key < hi; }
};
__device__ __forceinline__ Range range_of(const Attend &p, int64_t row) {
    Range r{0, (int)p.keys};
    if (p.ranges) {
        r.lo = max(p.ranges[2 * row], 0);
        r.hi = min(p.ranges[2 * row + 1], (int)p.keys);
    }
    if (r.lo >= r.hi) r.lo = r.hi = 0;
    return r;
}

// first .. end: what any of some rows sees; all .. all_end: what all of them see (rows that see nothing count for neither).
struct Bounds {
    int first, end, all, all_end;
    __device__ __forceinline__ void add(const Bounds &o) {
        first = min(first, o.first), end = max(end, o.end), all = max(all, o.all), all_end = min(all_end, o.all_end);
    }
    __device__ __forceinline__ bool meets(int a, int b) const { return a < end && b > first; }
    __device__ __forceinline__ bool covers(int a, int b) const { return a >= all && b <= all_end; }
};
__device__ __forceinline__ Bounds bounds_of(const Range &r, bool counts) {
    return counts && !r.empty() ? Bounds{r.lo, r.hi, r.lo, r.hi} : Bounds{INT_MAX, INT_MIN, INT_MIN, INT_MAX};
}
__device__ __forceinline__ Bounds over_columns(Bounds b) {              // of the 32 rows of a wave
#pragma unroll
    for (int d = 16; d; d /= 2) b.add(Bounds{__shfl_xor(b.first, d), __shfl_xor(b.end, d), __shfl_xor(b.all, d), __shfl_xor(b.all_end, d)});
    return Bounds{__builtin_amdgcn_readfirstlane(b.first), __builtin_amdgcn_readfirstlane(b.end),
                  __builtin_amdgcn_readfirstlane(b.all), __builtin_amdgcn_readfirstlane(b.all_end)};
}
__device__ __forceinline__ Bounds over_waves(const Bounds &mine, Bounds *slots, int wave, int lane) {
    if (lane == 0) slots[wave] = mine;
    __syncthreads();
    Bounds b = slots[0];
    for (int w = 1; w < kWaves; ++w) b.add(slots[w]);
    return Bounds{__builtin_amdgcn_readfirstlane(b.first), __builtin_amdgcn_readfirstlane(b.end),
                  __builtin_amdgcn_readfirstlane(b.all), __builtin_amdgcn_readfirstlane(b.all_end)};
}

// A lane's place: its column of the wave's 32 rows M.
struct Place {
    int m, row, head;
    bool valid;
};
__device__ __forceinline__ Place place_of(const Attend &p, int m, int state_head) {
    Place at;
    at.valid = m < p.m_total;
    at.m = at.valid ? m : p.m_total - 1;
    at.row = p.by_group(at.m);
    at.head = state_head * p.group + (at.m - at.row * p.group);
    return at;
}
template <class T> __device__ __forceinline__ T *address(const hp_heads_t &t, int64_t row, int head) {
    return (T *)t.data + row * t.row_stride + (int64_t)head * t.head_stride;
}

// The running maximum, sum and product of one query row in a lane and its partner.  `top` is a maximum of s * scale2
// that lags: it is raised when a score passes it by 2^8, so that most tiles leave the product as it is.
struct Running {
    float top = -INFINITY, sum = 0.0f;
};
constexpr float kLag = 8.0f;

// Scores (unscaled) of NB blocks of 32 states -> exponentials, with the statistics and the product so far brought up.
template <int NB, int DB> __device__ __forceinline__ void soften(Running &run, Acc (&s)[NB], Acc (&acc)[DB], float scale2) {
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
    const float2 two = both_halves(top);
    top = fmaxf(two.x, two.y) * scale2;
    const bool grows = top > run.top + kLag;
    if (__any(grows)) {
        const float next = grows ? top : run.top;
        const float keep = grows ? __builtin_amdgcn_exp2f(run.top - next) : 1.0f;
        run.top = next;
        run.sum *= keep;
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[db][i] *= keep;
    }
    const float base = run.top == -INFINITY ? 0.0f : run.top;
    float sum = 0.0f;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[b][i] = __builtin_amdgcn_exp2f(s[b][i] * scale2 - base);
            sum += s[b][i];
        }
    run.sum += sum;
}

// Writes a lane's part of a result^T: column l % 32 is one row of `to`.
template <class T, int DB> __device__ __forceinline__ void store_result(T *to, const Acc (&acc)[DB], float scale, int dim, int half) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            Vec<T, 4> v;
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] = (T)(acc[db][4 * b + t] * scale);
            const int d = 32 * db + 8 * b + 4 * half;
            store<4>(to + d, v, dim - d);
        }
}

template <class T, int DP> constexpr int kTileRows = DP * sizeof(T) <= 256 ? 64 : 32;

// Tiles in LDS, two in turn: while one is worked on the next is on its way.
template <class T, int DP, int ROWS, int STAGES = 2> struct Tiles {
    __attribute__((aligned(16))) T a[STAGES][ROWS * DP];
    __attribute__((aligned(16))) T b[STAGES][ROWS * DP];
};

template <class T, int DP> struct QueryLds {
    Tiles<T, DP, kTileRows<T, DP>> tiles;            // states k and v
    Bounds slots[kWaves];
    int bad;
};

// One after the other, with the stage as a constant: addresses in LDS are then one register and a number.
// (Not where that makes more of them than there are registers: beyond 64 KiB.)
template <int STAGES = 2, class Step> __device__ __forceinline__ void in_turn(int begin, int end, const Step &step) {
    if constexpr (STAGES == 2) {
        for (int tile = begin; tile < end; tile += 2) {
            step(tile, std::integral_constant<int, 0>());
            if (tile + 1 < end) step(tile + 1, std::integral_constant<int, 1>());
        }
    } else {
        for (int tile = begin, stage = 0; tile < end; ++tile, stage = stage + 1 < STAGES ? stage + 1 : 0) step(tile, stage);
    }
}

template <class T, int DP> __device__ void forward_careful(const Attend *p, QueryLds<T, DP> *lds);

// One workgroup: 128 rows M against a part of what they see.
template <class T, int DP, bool EXACT, bool CAREFUL> __device__ __forceinline__ void forward_block(const Attend &p, QueryLds<T, DP> &lds) {
    constexpr int NK = kTileRows<T, DP>, NB = NK / 32, DB = DP / 32, DS = DP / 16;
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = tid / kWave, half = lane / 32, col = lane % 32;
    const int state_head = (int)blockIdx.y, split = (int)blockIdx.z;
    // later rows tend to see more: they begin first
    const Place at = place_of(p, ((int)gridDim.x - 1 - (int)blockIdx.x) * kTileM + 32 * wave + col, state_head);
    const Range see = range_of(p, at.row);
    const Bounds own = over_columns(bounds_of(see, at.valid));
    if (tid == 0) lds.bad = 0;
    const Bounds any = over_waves(own, lds.slots, wave, lane);
    Frag<T> q[DS];
#pragma unroll
    for (int s = 0; s < DS; ++s) {
        const int d = 16 * s + 8 * half;
        q[s] = load<8>(address<const T>(p.q, at.row, at.head) + d, p.dim - d);
    }
    Running run;
    Acc acc[DB] = {};
    const int tiles = any.end > any.first ? (any.end - any.first + NK - 1) / NK : 0;
    const int begin = (int)((int64_t)tiles * split / p.splits), end = (int)((int64_t)tiles * (split + 1) / p.splits);
    Loader<T, DP, NK, kBlock, EXACT> ks, vs;
    ks.plan(p.k.row_stride, p.dim, tid);
    vs.plan(p.v.row_stride, p.dim, tid);
    const auto fetch = [&](int tile, int stage) {
        const int key0 = any.first + tile * NK;
        ks.fetch(lds.tiles.a[stage], address<const T>(p.k, key0, state_head), p.k.row_stride, any.end - key0, p.dim, tid);
        vs.fetch(lds.tiles.b[stage], address<const T>(p.v, key0, state_head), p.v.row_stride, any.end - key0, p.dim, tid);
    };
    if (begin < end) fetch(begin, 0);
    in_turn(begin, end, [&](int tile, auto stage) {
        const int key0 = any.first + tile * NK;
        const T *k_tile = lds.tiles.a[stage], *v_tile = lds.tiles.b[stage];
        arrived();
        __syncthreads();                             // this tile is there, and the last one's readers are done
        if (tile + 1 < end) fetch(tile + 1, 1 - stage);
        if (!CAREFUL && !any.covers(key0, key0 + NK) && not_finite<T, DP, NK>(v_tile, tid)) lds.bad = 1;
        if (!own.meets(key0, key0 + NK)) return;
        Acc s[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b] = Acc{};
#pragma unroll
        for (int d = 0; d < DS; ++d)
#pragma unroll
            for (int b = 0; b < NB; ++b) s[b] = mma(row_frag<T, DP>(k_tile, 32 * b + col, d, half), q[d], s[b]);
        if constexpr (sizeof(T) == 2) stream<NB * DS, NB * DS, 6, 1>();
        const bool whole = own.covers(key0, key0 + NK);
        if (!whole)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[b][i] = see.has(key0 + 32 * b + result_row(i, half)) ? s[b][i] : -INFINITY;
        soften(run, s, acc, p.scale2);
        if (CAREFUL && !whole) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
                careful_product<T, DP, DB>(acc, s[b], v_tile, 32 * b, half, [&](int j) { return see.has(key0 + 32 * b + j); });
            return;
        }
#pragma unroll
        for (int k = 0; k < 2 * NB; ++k) {
            const Frag<T> w = result_frag<T>(s[k / 2], k % 2);
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = mma(column_frag<T, DP>(v_tile, k, db, lane), w, acc[db]);
        }
        if constexpr (sizeof(T) == 2) stream<4 * NB * DB, 2 * NB * DB, 6, 2>();
    });
    if constexpr (!CAREFUL)
        if (again(&lds.bad)) return forward_careful<T, DP>((const Attend *)__builtin_amdgcn_kernarg_segment_ptr(), &lds);
    const float2 two = both_halves(run.sum);
    const float sum = two.x + two.y;
    const bool none = see.empty() || sum == 0.0f;
    if (none)
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = Acc{};
    const float inv = none ? 0.0f : 1.0f / sum, lse2 = none ? -INFINITY : run.top + __builtin_amdgcn_logf(sum);
    if (!at.valid) return;
    const int64_t out_row = (int64_t)at.row * p.heads_q + at.head;
    if (p.splits > 1) {
        const int64_t n = p.rows * p.heads_q;
        store_result(p.part + (split * n + out_row) * p.dim, acc, inv, p.dim, half);
        if (half == 0) p.part_lse[split * n + out_row] = lse2;
        return;
    }
    store_result(address<T>(p.out, at.row, at.head), acc, inv, p.dim, half);
    if (p.lse && half == 0) p.lse[out_row] = lse2 * kLn2;
}

template <class T, int DP> __device__ __attribute__((noinline)) void forward_careful(const Attend *at, QueryLds<T, DP> *lds) {
    const Attend p = *at;
    forward_block<T, DP, false, true>(p, *lds);
}

template <class T, int DP, bool EXACT> __global__ __launch_bounds__(kBlock, DP * sizeof(T) <= 256 ? 2 : 1) void attend_forward_kernel(Attend p) {
    __shared__ QueryLds<T, DP> lds;
    forward_block<T, DP, EXACT, false>(p, lds);
}

// One workgroup: up to 32 heads of one row against a part of what the row sees.  The waves take 32 states each on their
// own, without waiting for one another, and join at the end.
// Waves of a workgroup, and tiles that each has on their way or in work: as LDS has room for.
template <class T, int DP> constexpr int kStepWaves = DP * sizeof(T) <= 512 ? 4 : 2;
template <class T, int DP> constexpr int kStepStages = DP * sizeof(T) <= 128 ? 2 : 1;

template <class T, int DP, bool EXACT> __global__ __launch_bounds__((kStepWaves<T, DP> * kWave)) void attend_step_kernel(Attend p) {
    constexpr int kWaves = kStepWaves<T, DP>, kStages = kStepStages<T, DP>, DB = DP / 32, DS = DP / 16;
    __shared__ __attribute__((aligned(16))) T tiles[kWaves][kStages][2][32 * DP];
    __shared__ float tops[kWaves][32], sums[kWaves][32];
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), half = lane / 32, col = lane % 32;
    const int64_t row = blockIdx.x;
    const int parts = (p.group + 31) / 32, state_head = (int)blockIdx.y / parts, first_head = ((int)blockIdx.y % parts) * 32;
    const int split = (int)blockIdx.z;
    const int heads = min(p.group - first_head, 32), head0 = state_head * p.group + first_head;
    const Range see = range_of(p, row);
    Frag<T> q[DS];
#pragma unroll
    for (int s = 0; s < DS; ++s) {
        const int d = 16 * s + 8 * half;
        q[s] = load<8>(address<const T>(p.q, row, head0 + min(col, heads - 1)) + d, p.dim - d);
    }
    Running run;
    Acc acc[DB] = {};
    const int n_tiles = (see.hi - see.lo + 31) / 32;
    const int begin = (int)((int64_t)n_tiles * split / p.splits), end = (int)((int64_t)n_tiles * (split + 1) / p.splits);
    Loader<T, DP, 32, kWave, EXACT> ks, vs;
    ks.plan(p.k.row_stride, p.dim, lane);
    vs.plan(p.v.row_stride, p.dim, lane);
    auto fetch = [&](int tile, int stage) {
        const int key0 = see.lo + tile * 32;
        ks.fetch(tiles[wave][stage][0], address<const T>(p.k, key0, state_head), p.k.row_stride, see.hi - key0, p.dim, lane);
        vs.fetch(tiles[wave][stage][1], address<const T>(p.v, key0, state_head), p.v.row_stride, see.hi - key0, p.dim, lane);
    };
    // a wave's tiles are its own: no barriers, only its own loads to wait for and its own reads to finish
    auto settle = [] {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    int stage = 0;
    if (begin + wave < end) fetch(begin + wave, 0);
    for (int tile = begin + wave; tile < end; tile += kWaves) {
        const int key0 = see.lo + tile * 32;
        const T *k_tile = tiles[wave][stage][0], *v_tile = tiles[wave][stage][1];
        arrived();
        settle();
        if (kStages > 1 && tile + kWaves < end) fetch(tile + kWaves, stage ^ 1);
        Acc s[1] = {};
#pragma unroll
        for (int d = 0; d < DS; ++d) s[0] = mma(row_frag<T, DP>(k_tile, col, d, half), q[d], s[0]);
        if (key0 + 32 > see.hi)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[0][i] = key0 + result_row(i, half) < see.hi ? s[0][i] : -INFINITY;
        soften(run, s, acc, p.scale2);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const Frag<T> w = result_frag<T>(s[0], k);
#pragma unroll
            for (int db = 0; db < DB; ++db) acc[db] = mma(column_frag<T, DP>(v_tile, k, db, lane), w, acc[db]);
        }
        __builtin_amdgcn_s_waitcnt(0xc07f);          // lgkmcnt(0): nothing of this tile is still to be read
        settle();
        if (kStages == 1 && tile + kWaves < end) fetch(tile + kWaves, 0);
        stage = (stage + 1) % kStages;
    }
    // join the waves: statistics through LDS, then the products, 32 channels at a time, in the tiles' place
    const float2 two = both_halves(run.sum);
    if (half == 0) {
        tops[wave][col] = run.top;
        sums[wave][col] = two.x + two.y;
    }
    __syncthreads();
    float top = -INFINITY;
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, tops[w][col]);
    float sum = 0.0f;
    // a wave without a maximum has seen nothing, or NaN alone
    const auto weight = [&](float t) { return t == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(t - top); };
    for (int w = 0; w < kWaves; ++w) sum += sums[w][col] * weight(tops[w][col]);
    const float share = sum == 0.0f ? 0.0f : weight(run.top) / sum;
    const float lse2 = sum == 0.0f ? -INFINITY : top + __builtin_amdgcn_logf(sum);
    float *join = (float *)&tiles[0][0][0][0];                     // [wave][32 heads][36]
    static_assert(sizeof(tiles) >= sizeof(float) * kWaves * 32 * 36, "room for the join");
    const int64_t n = p.rows * p.heads_q, out_row = row * p.heads_q + head0;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
        __syncthreads();
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            Vec<float, 4> v;
#pragma unroll
            for (int t = 0; t < 4; ++t) v[t] = acc[db][4 * b + t] * share;
            *(Vec<float, 4> *)(join + (wave * 32 + col) * 36 + 8 * b + 4 * half) = v;
        }
        __syncthreads();
        const int d0 = (tid % 8) * 4, d = 32 * db + d0;
        for (int m = tid / 8; m < heads; m += kWaves * kWave / 8) {
            Vec<float, 4> v = {};
            for (int w = 0; w < kWaves; ++w) v += *(const Vec<float, 4> *)(join + (w * 32 + m) * 36 + d0);
            if (p.splits > 1) {
                store<4>(p.part + (split * n + out_row + m) * p.dim + d, v, p.dim - d);
            } else {
                Vec<T, 4> o;
#pragma unroll
                for (int t = 0; t < 4; ++t) o[t] = (T)v[t];
                store<4>(address<T>(p.out, row, head0 + m) + d, o, p.dim - d);
            }
        }
    }
    if (wave == 0 && half == 0 && col < heads) {
        if (p.splits > 1) p.part_lse[split * n + out_row + col] = lse2;
        else if (p.lse) p.lse[out_row + col] = lse2 * kLn2;
    }
}

// Joins the parts of each row and head: the lanes of a wave hold a part's statistics each (there are at most 64).  Many
// parts are a workgroup's, its waves take every fourth: one wave going through them one behind the other took 45 us of the
// 54 for one token against 8000 states in 62 parts.  Few are a wave's: 49200 rows and heads of two parts 19 us, with
// a workgroup each 48.
constexpr int kMostParts = kWave, kFewParts = 8;
template <class T> __global__ __launch_bounds__(kBlock) void attend_join_kernel(Attend p) {
    __shared__ __attribute__((aligned(16))) float half_done[kWaves][HP_ATTEND_MAX_DIM];
    const int lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave;
    const bool few = p.splits <= kFewParts;
    const int64_t n = p.rows * p.heads_q, at = few ? (int64_t)blockIdx.x * kWaves + wave : blockIdx.x;
    if (at >= n) return;                                            // whole waves, and only where each works by itself
    const int64_t row = at / p.heads_q;
    const int head = (int)(at - row * p.heads_q);
    const float lse2 = lane < p.splits ? p.part_lse[lane * n + at] : -INFINITY;
    float top = lse2;
#pragma unroll
    for (int d = kWave / 2; d; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float mine = lse2 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(lse2 - top);      // nothing seen in this part; NaN stays
    const float sum = wave_sum(mine);
    Vec<float, 4> acc = {};
    const int d = 4 * lane;
#pragma unroll 4
    for (int s = few ? 0 : wave; s < p.splits; s += few ? 1 : kWaves) {
        const float w = __shfl(mine, s);
        const Vec<float, 4> part = load<4>(p.part + (s * n + at) * p.dim + d, p.dim - d);
        if (w != 0.0f) acc += w * part;
    }
    if (!few) {
        *(Vec<float, 4> *)&half_done[wave][d] = acc;
        __syncthreads();
        if (wave) return;
        for (int w = 1; w < kWaves; ++w) acc += *(const Vec<float, 4> *)&half_done[w][d];
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    Vec<T, 4> o;
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = (T)(acc[t] * inv);
    store<4>(address<T>(p.out, row, head) + d, o, p.dim - d);
    if (p.lse && lane == 0) p.lse[at] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// Whether a lane keeps its own rows' operands in registers, or takes them from memory (the L2 cache) for every tile:
// the accumulators leave room for 16 KiB of one operand a wave at most.
template <class T, int DP> constexpr bool kHoldQuery = DP * sizeof(T) <= 512;
template <class T, int DP> constexpr bool kHoldState = DP * sizeof(T) <= 256;

template <class T, int DP> __device__ void dq_careful(const Attend *p, QueryLds<T, DP> *lds);

// dq of 128 rows M over a part of what they see; on the way, what the other kernel has to know of the rows.
template <class T, int DP, bool EXACT, bool CAREFUL> __device__ __forceinline__ void dq_block(const Attend &p, QueryLds<T, DP> &lds) {
    constexpr int NK = kTileRows<T, DP>, NB = NK / 32, DB = DP / 32, DS = DP / 16;
    constexpr bool kHold = kHoldQuery<T, DP>;
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = tid / kWave, half = lane / 32, col = lane % 32;
    const int state_head = (int)blockIdx.y, split = (int)blockIdx.z;
    const int tile_m = (int)gridDim.x - 1 - (int)blockIdx.x, line = tile_m * kTileM + 32 * wave + col;
    const Place at = place_of(p, line, state_head);
    const Range see = range_of(p, at.row);
    const Bounds own = over_columns(bounds_of(see, at.valid));
    if (tid == 0) lds.bad = 0;
    const Bounds any = over_waves(own, lds.slots, wave, lane);
    const T *q_at = address<const T>(p.q, at.row, at.head), *do_at = address<const T>(p.dout, at.row, at.head);
    const auto frag = [&](const T *from, int s) {
        const int d = 16 * s + 8 * half;
        return load<8>(from + d, p.dim - d);
    };
    Frag<T> q[kHold ? DS : 1], dout[kHold ? DS : 1];
    float delta = 0.0f;
#pragma unroll
    for (int s = 0; s < DS; ++s) {
        const Frag<T> g = frag(do_at, s), o = frag(address<const T>(p.out, at.row, at.head), s);
        if constexpr (kHold) {
            q[s] = frag(q_at, s);
            dout[s] = g;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) delta += (float)g[j] * (float)o[j];
    }
    const float2 two = both_halves(delta);
    delta = two.x + two.y;
    const int64_t out_row = (int64_t)at.row * p.heads_q + at.head;
    const float lse2 = p.lse[out_row] * kLog2e;
    if (!CAREFUL && split == 0) {
        if (half == 0) {
            // rows that are not there see nothing
            float *to = p.info + 4 * ((int64_t)state_head * p.m_lines + line / NK * NK) + line % NK;
            to[0] = lse2;
            to[NK] = delta;
            ((int *)to)[2 * NK] = at.valid ? see.lo : 0;
            ((int *)to)[3 * NK] = at.valid ? see.hi : 0;
        }
        // rows that see nothing, or are not there, keep the states' kernel from taking 32 rows for unmasked
        const bool all = __all(at.valid && !see.empty());
        if (state_head == 0 && lane == 0)
            p.bounds[tile_m * kWaves + wave] = make_int4(own.first, own.end, all ? own.all : INT_MAX, all ? own.all_end : INT_MIN);
    }
    Acc acc[DB] = {};
    const int tiles = any.end > any.first ? (any.end - any.first + NK - 1) / NK : 0;
    const int begin = (int)((int64_t)tiles * split / p.splits), end = (int)((int64_t)tiles * (split + 1) / p.splits);
    Loader<T, DP, NK, kBlock, EXACT> ks, vs;
    ks.plan(p.k.row_stride, p.dim, tid);
    vs.plan(p.v.row_stride, p.dim, tid);
    const auto fetch = [&](int tile, int stage) {
        const int key0 = any.first + tile * NK;
        ks.fetch(lds.tiles.a[stage], address<const T>(p.k, key0, state_head), p.k.row_stride, any.end - key0, p.dim, tid);
        vs.fetch(lds.tiles.b[stage], address<const T>(p.v, key0, state_head), p.v.row_stride, any.end - key0, p.dim, tid);
    };
    if (begin < end) fetch(begin, 0);
    in_turn(begin, end, [&](int tile, auto stage) {
        const int key0 = any.first + tile * NK;
        const T *k_tile = lds.tiles.a[stage], *v_tile = lds.tiles.b[stage];
        arrived();
        __syncthreads();
        if (tile + 1 < end) fetch(tile + 1, 1 - stage);
        if (!CAREFUL && !any.covers(key0, key0 + NK) && not_finite<T, DP, NK>(k_tile, tid)) lds.bad = 1;
        if (!own.meets(key0, key0 + NK)) return;
        const bool whole = own.covers(key0, key0 + NK);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            Acc s = {}, dp = {};
#pragma unroll
            for (int d = 0; d < DS; ++d) {
                s = mma(row_frag<T, DP>(k_tile, 32 * b + col, d, half), kHold ? q[kHold ? d : 0] : frag(q_at, d), s);
                dp = mma(row_frag<T, DP>(v_tile, 32 * b + col, d, half), kHold ? dout[kHold ? d : 0] : frag(do_at, d), dp);
            }
            if constexpr (sizeof(T) == 2) stream<2 * DS, 2 * DS, 6, 1>();
#pragma unroll
            for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i] * p.scale2 - lse2) * (dp[i] - delta);
            if (!whole)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = see.has(key0 + 32 * b + result_row(i, half)) ? s[i] : 0.0f;
            if (CAREFUL && !whole) {
                careful_product<T, DP, DB>(acc, s, k_tile, 32 * b, half, [&](int j) { return see.has(key0 + 32 * b + j); });
                continue;
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const Frag<T> w = result_frag<T>(s, k);
#pragma unroll
                for (int db = 0; db < DB; ++db) acc[db] = mma(column_frag<T, DP>(k_tile, 2 * b + k, db, lane), w, acc[db]);
            }
            if constexpr (sizeof(T) == 2) stream<4 * DB, 2 * DB, 6, 2>();
        }
    });
    if constexpr (!CAREFUL)
        if (again(&lds.bad)) return dq_careful<T, DP>((const Attend *)__builtin_amdgcn_kernarg_segment_ptr(), &lds);
    if (!at.valid) return;
    if (see.empty())
#pragma unroll
        for (int db = 0; db < DB; ++db) acc[db] = Acc{};
    if (p.splits > 1) store_result(p.part + (split * p.rows * p.heads_q + out_row) * p.dim, acc, p.scale, p.dim, half);
    else store_result(address<T>(p.dq, at.row, at.head), acc, p.scale, p.dim, half);
}

template <class T, int DP> __device__ __attribute__((noinline)) void dq_careful(const Attend *at, QueryLds<T, DP> *lds) {
    const Attend p = *at;
    dq_block<T, DP, false, true>(p, *lds);
}

template <class T, int DP, bool EXACT> __global__ __launch_bounds__(kBlock, DP * sizeof(T) <= 256 ? 2 : 1) void attend_dq_kernel(Attend p) {
    __shared__ QueryLds<T, DP> lds;
    dq_block<T, DP, EXACT, false>(p, lds);
}

// dk and dv of some states over a part of the rows that see them: the same products with the roles exchanged, rows M in
// LDS a tile at a time, lanes that hold the states.  In bf16 two waves share 32 states, one for dv and one for dk: each
// makes the weights for itself (five products instead of four), but holds one result, so that two waves fit a SIMD and
// one's exponentials and LDS reads run beside the other's products.  Binary32 is bound by its products: four, in one wave.
template <class T> constexpr bool kPairs = sizeof(T) == 2;
template <class T, int DP> constexpr int kStateWaves = kPairs<T> && DP > 128 ? 2 : 4;           // that share out a workgroup's states
template <class T, int DP> constexpr int kStateBlock = 32 * kStateWaves<T, DP>;
template <class T, int DP> constexpr int kStateThreads = kStateWaves<T, DP> * kWave * (kPairs<T> ? 2 : 1);

enum { kPartBoth, kPartDk, kPartDv };

// A workgroup's registers leave a compute unit no second one that would work while this one waits: its tiles are
// asked for three ahead.  What that gains is known for heads of 97 to 128 in bf16 (2.50 -> 2.25 ms of a training microbatch).
// As compiled, the loop for dk in bf16 up to 96, both in bf16 from 129 on and that of binary32 from 65 to 128 wait for all loads
// before each barrier - other loads, of the states' operands, stand among those of the tiles -, so that one tile overlaps there.
template <class T, int DP> constexpr int kStateStages = kTileRows<T, DP> * DP * sizeof(T) <= 16384 ? 4 : 2;
template <class T, int DP> struct StateLds {
    Tiles<T, DP, kTileRows<T, DP>, kStateStages<T, DP>> tiles;                // rows M of q and dout
    __attribute__((aligned(16))) float info[kStateStages<T, DP>][256];        // of the rows: lse2, delta, first, end, one behind the other
    int bad, first_tile, last_tile;
};

template <class T, int DP> __device__ void dkv_careful(const Attend *p, StateLds<T, DP> *lds);

template <class T, int DP, bool EXACT, bool CAREFUL> __device__ __forceinline__ void dkv_block(const Attend &p, StateLds<T, DP> &lds) {
    constexpr int NM = kTileRows<T, DP>, NB = NM / 32, DB = DP / 32, DS = DP / 16, kThreads = kStateThreads<T, DP>, kStates = kStateBlock<T, DP>;
    constexpr bool kHold = kHoldState<T, DP>, kTwo = !kPairs<T>;
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), half = lane / 32, col = lane % 32;
    const int state_head = (int)blockIdx.y, split = (int)blockIdx.z;
    const int block0 = (int)blockIdx.x * kStates, block_end = min(block0 + kStates, (int)p.keys);
    const bool makes_dk = kTwo || wave >= kStateWaves<T, DP>;                // or dv, or both
    const int key0 = block0 + 32 * (wave % kStateWaves<T, DP>), key = key0 + col;
    const bool valid = key < p.keys;
    const T *k_at = address<const T>(p.k, valid ? key : p.keys - 1, state_head), *v_at = address<const T>(p.v, valid ? key : p.keys - 1, state_head);
    const auto frag = [&](const T *from, int s) {
        const int d = 16 * s + 8 * half;
        return load<8>(from + d, valid ? p.dim - d : 0);
    };
    Acc acc[DB] = {}, dv[kTwo ? DB : 1] = {};                                // dk or dv; dk and dv
    // the first and last tile of rows M that see any of the block's states
    const int m_tiles = (p.m_total + NM - 1) / NM;
    const auto bounds_at = [&](int t) {
        // written by the kernel before: as constant memory it is read without a place in the queue of the tiles
        typedef __attribute__((address_space(4))) const Vec<int, 4> *Constant;
        const Constant at = (Constant)(uintptr_t)p.bounds;
        const Vec<int, 4> one = at[t * NB];
        int4 b = make_int4(one[0], one[1], one[2], one[3]);
        if (NB > 1 && (t * NB + 1) * 32 < p.m_total) {
            const Vec<int, 4> two = at[t * NB + 1];
            b = make_int4(min(b.x, two[0]), max(b.y, two[1]), max(b.z, two[2]), min(b.w, two[3]));
        } else if (NB > 1) {
            b.z = INT_MAX, b.w = INT_MIN;                // rows that are not there see nothing
        }
        return b;
    };
    if (tid == 0) {
        lds.first_tile = INT_MAX;
        lds.last_tile = -1;
        lds.bad = 0;
    }
    __syncthreads();
    int first = INT_MAX, last = -1;
    for (int t = tid; t < m_tiles; t += kThreads) {
        const int4 b = bounds_at(t);
        if (block0 < b.y && block_end > b.x) {
            first = min(first, t);
            last = max(last, t);
        }
    }
    if (last >= 0) {
        atomicMin(&lds.first_tile, first);
        atomicMax(&lds.last_tile, last);
    }
    __syncthreads();
    first = __builtin_amdgcn_readfirstlane(lds.first_tile);
    last = __builtin_amdgcn_readfirstlane(lds.last_tile);
    const int count = last >= 0 ? last + 1 - first : 0;
    const int begin = last >= 0 ? first + (int)((int64_t)count * split / p.splits) : 0, end = last >= 0 ? first + (int)((int64_t)count * (split + 1) / p.splits) : 0;
    typedef Loader<T, DP, NM, kThreads, EXACT> Load;
    Load qs, dos;
    qs.plan_m(p.q, p.by_group, p.dim, tid);
    dos.plan_m(p.dout, p.by_group, p.dim, tid);
    int4 next_b = {};
    const auto fetch = [&](int t, int stage) {
        if (wave == 0) {                                 // 4 NM numbers, 16 bytes a lane
            const float *from = p.info + 4 * ((int64_t)state_head * p.m_lines + (int64_t)t * NM);
            if constexpr (CAREFUL) {
                if (lane < NM) *(Vec<float, 4> *)&lds.info[stage][4 * lane] = *(const Vec<float, 4> *)(from + 4 * lane);
            } else {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(Load::buffer(from), (__attribute__((address_space(3))) void *)lds.info[stage], 16,
                                                         (int)(lane < NM ? 16u * lane : kOutside), 0, 0, 0);
            }
        }
        qs.fetch_m(lds.tiles.a[stage], p.q, t * NM, p.m_total, p.by_group, state_head * p.group, p.dim, tid);
        dos.fetch_m(lds.tiles.b[stage], p.dout, t * NM, p.m_total, p.by_group, state_head * p.group, p.dim, tid);
    };
    // A loop for each part: the waves of one make as many turns, and so meet as many barriers, as those of the other.
    const auto work = [&](auto part) {
    constexpr bool kDv = part != kPartDk, kDk = part != kPartDv;
    Frag<T> k[kHold ? DS : 1], v[kHold && kDk ? DS : 1];
    if constexpr (kHold)
#pragma unroll
        for (int s = 0; s < DS; ++s) {
            k[s] = frag(k_at, s);
            if constexpr (kDk) v[s] = frag(v_at, s);
        }
    constexpr int kStages = CAREFUL ? 2 : kStateStages<T, DP>;
    if (begin < end) next_b = bounds_at(begin);
    for (int n = 0; n < kStages - 1; ++n)
        if (begin + n < end) fetch(begin + n, n);
    in_turn<kStages>(begin, end, [&](int tile, auto stage) {
        const T *q_tile = lds.tiles.a[stage], *do_tile = lds.tiles.b[stage];
        const float *info = lds.info[stage];
        const int4 b = next_b;
        const bool whole = key0 >= b.z && key0 + 32 <= b.w, meets = key0 < b.y && key0 + 32 > b.x;
        if constexpr (!EXACT || kStages == 2) arrived();
        else if (wave == 0) arrived_but<2 * Load::kMost + 1>(min(end - tile, kStages - 1) - 1);      // the rows' numbers too
        else if (Load::loads(Load::kEach - 1, tid)) arrived_but<2 * Load::kMost>(min(end - tile, kStages - 1) - 1);
        else arrived_but<2 * Load::kLeast>(min(end - tile, kStages - 1) - 1);
        __syncthreads();
        if (tile + 1 < end) next_b = bounds_at(tile + 1);
        if (tile + kStages - 1 < end) fetch(tile + kStages - 1, (stage + kStages - 1) % kStages);
        if (!CAREFUL && !(block0 >= b.z && block0 + kStates <= b.w)) {
            const bool one = not_finite<T, DP, NM, kThreads>(q_tile, tid), other = not_finite<T, DP, NM, kThreads>(do_tile, tid);
            if (one || other) lds.bad = 1;
        }
        if (!meets) return;
        const auto sees = [&](int row) { return key >= ((const int *)info)[2 * NM + row] && key < ((const int *)info)[3 * NM + row]; };
#pragma unroll
        for (int mb = 0; mb < NB; ++mb) {
            Acc s = {}, dp = {};
#pragma unroll
            for (int d = 0; d < DS; ++d) s = mma(row_frag<T, DP>(q_tile, 32 * mb + col, d, half), kHold ? k[kHold ? d : 0] : frag(k_at, d), s);
            if constexpr (kDk)
#pragma unroll
                for (int d = 0; d < DS; ++d) dp = mma(row_frag<T, DP>(do_tile, 32 * mb + col, d, half), kHold ? v[kHold ? d : 0] : frag(v_at, d), dp);
            if constexpr (sizeof(T) == 2) stream<kDk ? 2 * DS : DS, kDk ? 2 * DS : DS, 6, 1>();
#pragma unroll
            for (int b4 = 0; b4 < 4; ++b4) {
                const Vec<float, 4> lse2 = *(const Vec<float, 4> *)(info + 32 * mb + 8 * b4 + 4 * half);
#pragma unroll
                for (int t = 0; t < 4; ++t) s[4 * b4 + t] = __builtin_amdgcn_exp2f(s[4 * b4 + t] * p.scale2 - lse2[t]);
            }
            if constexpr (kDk)
#pragma unroll
                for (int b4 = 0; b4 < 4; ++b4) {
                    const Vec<float, 4> delta = *(const Vec<float, 4> *)(info + NM + 32 * mb + 8 * b4 + 4 * half);
#pragma unroll
                    for (int t = 0; t < 4; ++t) dp[4 * b4 + t] = s[4 * b4 + t] * (dp[4 * b4 + t] - delta[t]);
                }
            if (!whole)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const bool seen = sees(32 * mb + result_row(i, half));
                    if constexpr (kDv) s[i] = seen ? s[i] : 0.0f;
                    if constexpr (kDk) dp[i] = seen ? dp[i] : 0.0f;
                }
            const auto add = [&](auto &to, const Acc &x, const T *tile) {
                if (CAREFUL && !whole) {
                    careful_product<T, DP>(to, x, tile, 32 * mb, half, [&](int j) { return sees(32 * mb + j); });
                    return;
                }
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    const Frag<T> w = result_frag<T>(x, m);
#pragma unroll
                    for (int db = 0; db < DB; ++db) to[db] = mma(column_frag<T, DP>(tile, 2 * mb + m, db, lane), w, to[db]);
                }
                if constexpr (sizeof(T) == 2) stream<4 * DB, 2 * DB, 6, 2>();
            };
            if constexpr (kDv && kDk) add(dv, s, do_tile);
            else if constexpr (kDv) add(acc, s, do_tile);
            if constexpr (kDk) add(acc, dp, q_tile);
        }
    });
    };
    if constexpr (kTwo) work(std::integral_constant<int, kPartBoth>());
    else if (makes_dk) work(std::integral_constant<int, kPartDk>());
    else work(std::integral_constant<int, kPartDv>());
    if constexpr (!CAREFUL)
        if (again(&lds.bad)) return dkv_careful<T, DP>((const Attend *)__builtin_amdgcn_kernarg_segment_ptr(), &lds);
    if (!valid) return;
    const auto leave = [&](const auto &x, const hp_heads_t &to, float *part, float scale) {
        if (p.splits > 1) store_result(part + ((split * p.keys + key) * p.heads_k + state_head) * p.dim, x, scale, p.dim, half);
        else store_result(address<T>(to, key, state_head), x, scale, p.dim, half);
    };
    if constexpr (kTwo) {
        leave(acc, p.dk, p.part_k, p.scale);
        leave(dv, p.dv, p.part_v, 1.0f);
    } else if (makes_dk) {
        leave(acc, p.dk, p.part_k, p.scale);
    } else {
        leave(acc, p.dv, p.part_v, 1.0f);
    }
}

template <class T, int DP> __device__ __attribute__((noinline)) void dkv_careful(const Attend *at, StateLds<T, DP> *lds) {
    const Attend p = *at;
    dkv_block<T, DP, false, true>(p, *lds);
}

template <class T, int DP, bool EXACT> __global__ __launch_bounds__((kStateThreads<T, DP>)) void attend_dkv_kernel(Attend p) {
    __shared__ StateLds<T, DP> lds;
    dkv_block<T, DP, EXACT, false>(p, lds);
}

// Adds parts [splits][rows * heads][dim] up, in order: a wave a row and head.
template <class T> __global__ __launch_bounds__(kBlock) void attend_sum_kernel(const float *part, int splits, int64_t rows, int heads, int dim, hp_heads_t out) {
    const int64_t n = rows * heads, at = (int64_t)blockIdx.x * kWaves + threadIdx.x / kWave;
    const int d = 4 * ((int)threadIdx.x % kWave);
    if (at >= n || d >= dim) return;
    const int64_t row = at / heads;
    Vec<float, 4> acc = {};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) acc += load<4>(part + (s * n + at) * dim + d, dim - d);
    Vec<T, 4> o;
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = (T)acc[t];
    store<4>(address<T>(out, row, (int)(at - row * heads)) + d, o, dim - d);
}

// ---- host ------------------------------------------------------------------------------------------------------

// Parts of the long axis: until the launch has about `want` workgroups, none with less than `least` of `length`.
int32_t parts_of(int64_t blocks, int64_t want, int64_t length, int64_t least, int64_t most) {
    int64_t n = (want + blocks - 1) / blocks;
    const int64_t by_length = length / least;
    n = n < by_length ? n : by_length;
    n = n < most ? n : most;
    return (int32_t)(n < 1 ? 1 : n);
}

struct Plan {
    int64_t blocks_m, blocks_k;                     // of 128 rows M, of the states that a workgroup takes
    int32_t splits, splits_dq, splits_dkv, splits_step;
};

Plan plan_of(const hp_attend_args_t &a) {
    Plan n;
    const int64_t group = a.heads_q / a.heads_k, m = a.rows * group;
    n.blocks_m = (m + kTileM - 1) / kTileM;
    const int64_t states = a.dtype == HP_F32 || a.dim <= 128 ? 128 : 64;
    n.blocks_k = (a.keys + states - 1) / states;
    const int64_t one = n.blocks_m * a.heads_k > 0 ? n.blocks_m * a.heads_k : 1, two = n.blocks_k * a.heads_k > 0 ? n.blocks_k * a.heads_k : 1;
    // 256 rows of 32 heads against 4032 states: 42 us with 256 workgroups, 44 with 512, 57 with 1024; 512 rows of 10 heads
    // against 40139: 162, 166, 151; 2048 against 4032: 137, 137, 200.
    n.splits = parts_of(one, 2 * kComputeUnits, a.keys, 256, 32);
    n.splits_dq = parts_of(one, kComputeUnits, a.keys, 256, 32);
    // States early in a sequence are seen by more rows than late ones: workgroups enough to even that out (8192 rows of 32
    // heads against 5760 states, forward and backward: 2.56 ms with 256, 2.28 with 1024, 2.25 with 1280, 2.31 with 3000).
    n.splits_dkv = parts_of(two, 5 * kComputeUnits, m, 256, 32);
    const int64_t each = a.rows * a.heads_k * ((group + 31) / 32);
    // Few rows: as many workgroups as run at once (8 rows of 8 state heads against 3000 states: 24 us with 512, 33 with
    // 2048).  More rows: several times that, so that requests of unequal lengths even out (64 rows of 8 heads against 576 to
    // 6404 states: 191 us with 2048; of equal ones it costs 4 %, 173 to 180).
    n.splits_step = parts_of(each > 0 ? each : 1, each <= kComputeUnits / 2 ? 2 * kComputeUnits : 8 * kComputeUnits, a.keys, kStepKeys, kMostParts);
    return n;
}

int64_t align16(int64_t n) { return (n + 15) / 16 * 16; }

int64_t info_bytes(const hp_attend_args_t &a, const Plan &n) { return 16 * a.heads_k * n.blocks_m * kTileM; }

int64_t workspace_of(const hp_attend_args_t &a, int call) {
    const Plan n = plan_of(a);
    const int64_t outs = a.rows * a.heads_q, states = a.keys * a.heads_k;
    if (call == HP_ATTEND_BACKWARD) {
        const int64_t parts = 4 * a.dim * (n.splits_dq > 1 ? n.splits_dq * outs : 0), parts_kv = 4 * a.dim * (n.splits_dkv > 1 ? 2 * n.splits_dkv * states : 0);
        return info_bytes(a, n) + align16(16 * n.blocks_m * kWaves) + (parts > parts_kv ? parts : parts_kv);
    }
    const int32_t splits = call == HP_ATTEND_STEP ? n.splits_step : n.splits;
    return splits > 1 ? align16(4 * splits * outs) + 4 * splits * outs * a.dim : 0;
}

bool misaligned(const void *p, int to) { return (uintptr_t)p % to != 0; }

int check_sizes(const hp_attend_args_t *a, int call) {
    if (!a) return HP_EINVAL;
    if (a->dtype != HP_BF16 && a->dtype != HP_F32) return HP_EINVAL;
    if (a->dim < 1 || a->dim > HP_ATTEND_MAX_DIM || a->heads_k < 1 || a->heads_q < 1) return HP_EINVAL;
    if (a->heads_q % a->heads_k || a->heads_q > 16384) return HP_ELAYOUT;
    if (a->rows < 0 || a->keys < 0) return HP_EINVAL;
    // rows M, states and lanes of a launch are counted in 32 bits, with tiles to spare
    if (a->rows > ((1 << 30) - 1024) / (a->heads_q / a->heads_k) || a->keys > INT_MAX - 1024) return HP_ELAYOUT;
    // the backward of states has 4 lanes a state in bf16 (in binary32 2)
    if (call == HP_ATTEND_BACKWARD && a->dtype == HP_BF16 && a->keys > (1 << 30) - 1024) return HP_ELAYOUT;
    // single tokens have 256 lanes a row
    if (call == HP_ATTEND_STEP && a->rows > 1 << 23) return HP_ELAYOUT;
    return HP_OK;
}

int check(const hp_attend_args_t *a, int call) {
    if (const int rc = check_sizes(a, call)) return rc;
    if (!(a->scale > 0) || !std::isfinite(a->scale) || !std::isfinite(a->scale * kLog2e)) return HP_EINVAL;
    const int size = a->dtype == HP_BF16 ? 2 : 4;
    const bool back = call == HP_ATTEND_BACKWARD;
    for (const hp_heads_t *t : {&a->q, &a->out, &a->dout, &a->dq}) {
        if (!back && (t == &a->dout || t == &a->dq)) continue;
        if (a->rows > 0 && !t->data) return HP_EINVAL;
        if (misaligned(t->data, size)) return HP_EALIGN;
    }
    for (const hp_heads_t *t : {&a->k, &a->v, &a->dk, &a->dv}) {
        if (!back && (t == &a->dk || t == &a->dv)) continue;
        if (a->keys > 0 && !t->data) return HP_EINVAL;
        if (misaligned(t->data, size)) return HP_EALIGN;
    }
    if (back && a->rows > 0 && !a->lse) return HP_EINVAL;
    if (misaligned(a->ranges, 4) || misaligned(a->lse, 4) || misaligned(a->workspace, 16)) return HP_EALIGN;
    const int64_t need = a->rows > 0 || back ? workspace_of(*a, call) : 0;
    if (need > 0 && (!a->workspace || a->workspace_bytes < need)) return HP_EINVAL;
    return HP_OK;
}

// n / by = (2n * factor) >> (32 + shift) for n < 2^30, with factor = ceil(2^(31 + shift) / by) and 2^shift the least power of
// two that is not below by / 2: what the ceiling adds to the quotient is less than n / 2^(31 + shift) <= 1 / by.
Divisor divisor(uint32_t by) {
    uint32_t shift = 0;
    while (((uint64_t)2 << shift) < by) ++shift;
    return Divisor{by, (uint32_t)((((uint64_t)1 << (31 + shift)) + by - 1) / by), shift};
}

Attend params_of(const hp_attend_args_t &a) {
    Attend p{};
    p.rows = a.rows, p.keys = a.keys;
    p.heads_q = a.heads_q, p.heads_k = a.heads_k, p.group = a.heads_q / a.heads_k, p.dim = a.dim;
    p.splits = 1, p.m_total = (int32_t)(a.rows * p.group);
    p.by_group = divisor((uint32_t)p.group);
    p.scale = a.scale, p.scale2 = a.scale * kLog2e;
    p.q = a.q, p.k = a.k, p.v = a.v, p.out = a.out, p.dout = a.dout, p.dq = a.dq, p.dk = a.dk, p.dv = a.dv;
    p.ranges = a.ranges, p.lse = a.lse;
    return p;
}

bool failed() { return hip_failed(hipGetLastError()); }

enum Kernel { kForward, kStep, kDq, kDkv };

// Whether a tensor's rows are whole aligned 16-byte pieces, and a tile of 64 of them (each with its heads) lies within
// the reach of a buffer's 32-bit offsets.
bool exact(const hp_heads_t &t, int size, int32_t dim, int32_t heads) {
    const int64_t piece = 16 / size;
    if (dim % piece || misaligned(t.data, 16) || t.row_stride % piece || t.head_stride % piece || t.row_stride < 0 || t.head_stride < 0) return false;
    const int64_t most = ((int64_t)1 << 29) / size;      // rows and heads together: less than 2^31 bytes
    return t.row_stride <= most / 64 && t.head_stride <= most / heads;
}

template <class T, int DP, bool EXACT> void launch(Kernel what, const Attend &p, const dim3 &grid, hipStream_t s) {
    if (what == kForward) attend_forward_kernel<T, DP, EXACT><<<grid, kBlock, 0, s>>>(p);
    else if (what == kStep) attend_step_kernel<T, DP, EXACT><<<grid, kStepWaves<T, DP> * kWave, 0, s>>>(p);
    else if (what == kDq) attend_dq_kernel<T, DP, EXACT><<<grid, kBlock, 0, s>>>(p);
    else attend_dkv_kernel<T, DP, EXACT><<<grid, kStateThreads<T, DP>, 0, s>>>(p);
}

template <class T, int DP> void launch(Kernel what, const Attend &p, const dim3 &grid, hipStream_t s) {
    static_assert(kStateBlock<T, DP> == (sizeof(T) == 4 || DP <= 128 ? 128 : 64), "as plan_of() counts");
    const int size = sizeof(T);
    const bool whole = what == kDkv ? exact(p.q, size, p.dim, p.group) && exact(p.dout, size, p.dim, p.group) : exact(p.k, size, p.dim, 1) && exact(p.v, size, p.dim, 1);
    if (whole) launch<T, DP, true>(what, p, grid, s);
    else launch<T, DP, false>(what, p, grid, s);
}

template <class T> void launch(Kernel what, const Attend &p, const dim3 &grid, hipStream_t s) {
    if (p.dim <= 64) launch<T, 64>(what, p, grid, s);
    else if (p.dim <= 96) launch<T, 96>(what, p, grid, s);
    else if (p.dim <= 128) launch<T, 128>(what, p, grid, s);
    else launch<T, 256>(what, p, grid, s);
}

void launch(Kernel what, int dtype, const Attend &p, const dim3 &grid, hipStream_t s) {
    if (dtype == HP_BF16) launch<__bf16>(what, p, grid, s);
    else launch<float>(what, p, grid, s);
}

// Forward in either shape: the launch, and the join of the parts.
int forward(const hp_attend_args_t &a, Kernel what, const dim3 &grid, hipStream_t s) {
    Attend p = params_of(a);
    p.splits = (int32_t)grid.z;
    if (p.splits > 1) {
        p.part_lse = (float *)a.workspace;
        p.part = (float *)((char *)a.workspace + align16(4 * p.splits * p.rows * p.heads_q));
    }
    launch(what, a.dtype, p, grid, s);
    if (failed()) return HP_EHIP;
    if (p.splits > 1) {
        const int64_t items = p.rows * p.heads_q;
        const uint32_t blocks = (uint32_t)(p.splits <= kFewParts ? (items + kWaves - 1) / kWaves : items);
        if (a.dtype == HP_BF16) attend_join_kernel<__bf16><<<blocks, kBlock, 0, s>>>(p);
        else attend_join_kernel<float><<<blocks, kBlock, 0, s>>>(p);
        if (failed()) return HP_EHIP;
    }
    return HP_OK;
}

int add_up(const float *part, int splits, int dtype, int64_t rows, int heads, int dim, const hp_heads_t &out, hipStream_t s) {
    const uint32_t blocks = (uint32_t)((rows * heads + kWaves - 1) / kWaves);
    if (dtype == HP_BF16) attend_sum_kernel<__bf16><<<blocks, kBlock, 0, s>>>(part, splits, rows, heads, dim, out);
    else attend_sum_kernel<float><<<blocks, kBlock, 0, s>>>(part, splits, rows, heads, dim, out);
    return failed() ? HP_EHIP : HP_OK;
}

}  // namespace

extern "C" {

int64_t hp_cross_attend_workspace(const hp_attend_args_t *a, int32_t call) {
    if (const int rc = check_sizes(a, call)) return rc;
    if (call < HP_ATTEND_FORWARD || call > HP_ATTEND_BACKWARD) return HP_EINVAL;
    return workspace_of(*a, call);
}

int hp_cross_attend(const hp_attend_args_t *a, void *stream) {
    if (const int rc = check(a, HP_ATTEND_FORWARD)) return rc;
    if (a->rows == 0) return HP_OK;
    const Plan n = plan_of(*a);
    return forward(*a, kForward, dim3((uint32_t)n.blocks_m, (uint32_t)a->heads_k, (uint32_t)n.splits), (hipStream_t)stream);
}

int hp_cross_attend_step(const hp_attend_args_t *a, void *stream) {
    if (const int rc = check(a, HP_ATTEND_STEP)) return rc;
    if (a->rows == 0) return HP_OK;
    const Plan n = plan_of(*a);
    const int32_t parts = (a->heads_q / a->heads_k + 31) / 32;
    return forward(*a, kStep, dim3((uint32_t)a->rows, (uint32_t)(a->heads_k * parts), (uint32_t)n.splits_step), (hipStream_t)stream);
}

int hp_cross_attend_backward(const hp_attend_args_t *a, void *stream) {
    if (const int rc = check(a, HP_ATTEND_BACKWARD)) return rc;
    const Plan n = plan_of(*a);
    const hipStream_t s = (hipStream_t)stream;
    Attend p = params_of(*a);
    char *ws = (char *)a->workspace;
    p.info = (float *)ws;
    p.m_lines = (int32_t)(n.blocks_m * kTileM);
    p.bounds = (int4 *)(ws + info_bytes(*a, n));
    float *parts = (float *)(ws + info_bytes(*a, n) + align16(16 * n.blocks_m * kWaves));
    if (a->rows > 0) {
        p.splits = n.splits_dq;
        p.part = parts;
        launch(kDq, a->dtype, p, dim3((uint32_t)n.blocks_m, (uint32_t)a->heads_k, (uint32_t)p.splits), s);
        if (failed()) return HP_EHIP;
        if (p.splits > 1)
            if (const int rc = add_up(parts, p.splits, a->dtype, a->rows, a->heads_q, a->dim, a->dq, s)) return rc;
    }
    if (a->keys > 0) {
        p.splits = n.splits_dkv;
        p.part_k = parts;                            // what dq's parts were is read by now: the stream is in order
        p.part_v = parts + (int64_t)p.splits * a->keys * a->heads_k * a->dim;
        launch(kDkv, a->dtype, p, dim3((uint32_t)n.blocks_k, (uint32_t)a->heads_k, (uint32_t)p.splits), s);
        if (failed()) return HP_EHIP;
        if (p.splits > 1) {
            if (const int rc = add_up(p.part_k, p.splits, a->dtype, a->keys, a->heads_k, a->dim, a->dk, s)) return rc;
            if (const int rc = add_up(p.part_v, p.splits, a->dtype, a->keys, a->heads_k, a->dim, a->dv, s)) return rc;
        }
    }
    return HP_OK;
}

}  // extern "C"
