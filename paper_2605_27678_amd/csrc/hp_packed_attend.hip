// Attention of single tokens to states held in 4 bits: row r sees the states lo(r) .. hi(r) - 1, and with a group's
// value = low + step * code,
//     s_j = scale sum_g (step_jg sum_c q_c code_jc + low_jg sum_c q_c),  p_j = exp(s_j - m) / sum,
//     out_c = sum_j (p_j step_jg) code_jc + sum_j p_j low_jg              (g the group of channel c)
// in one pass with a running maximum m and sum.  The codes go into the matrix units as they are (hp_packed.hpp).
//
// A wave takes 64 states at a time by itself.  S^T = K Q^T, so that a lane has scores of one head, four states of each 16.
// A word of codes is a lane's 8 channels of one state, an operand as it is.  The steps go over a group's 16 x 16 results
// before they add up: each lane reads those of one state, and a multiplication takes them from whichever lane of its row has
// them.  (Read from LDS by every lane that needs them they were 32 of 56 LDS reads of 16 bytes, and 120 us for 64 requests of
// 576 to 6404 states.)  out^T = V^T P^T has the states as inner values: the transposing LDS load brings a lane 16 states of one
// channel, in the order in which it has their weights, so that no weight leaves its lane; the weights, times the group's
// steps, are rounded to bfloat16 (three such numbers in binary32).  What the codes' lift puts into a product, and 8 more so
// that codes lie around zero and cancel little, is taken off by a product with -24 throughout, from the very same rounded
// weights (in binary32 they lie there as they are); 8 sum p step + sum p low come from one more product.
//
// A state and head are 5 bits a channel of k and of v, each read once, so memory bounds it: 288 MB of 64 requests are 56 us at
// the rate of a large copy.  It takes 72, and 5 more for the join, which with the same loads without the computing are 63: most
// of the computing hides where three waves share a SIMD.  Heads of 256 leave it one or two: 46 us for 110 MB (a copy 21), 31
// without the computing; heads of 129 to 224 have as many registers, LDS and loads (of 160, 69 MB: 42).
// Where rows are short, what begins and ends them counts: 30 requests of 1 to 2305 states, 16 heads of 72, 53 MB (a copy
// 10) take 32 us in bfloat16, 38 in binary32 (21 without the computing); per added MB they take no more than a copy, and 1.7
// times as much.
// Sets of heads side by side in a product's columns (few heads share a state head) took a quarter less arithmetic and no
// less time; rings of three tiles instead of two leave room for fewer waves (64 requests 113 us).
#include <climits>
#include <cmath>
#include <type_traits>

#include "hp_packed.hpp"
#include "hp_share.hpp"

#pragma clang fp contract(fast)

namespace {

using namespace hp;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kTile = 64, kHeads = 16;             // states of a wave's tile, heads of a workgroup
constexpr float kMiddle = 8.0f;

struct Params {
    int64_t rows, keys;
    int32_t heads_q, group, groups, dim, head_tiles;
    int32_t units;                                 // of each tile of heads; 0: each row is one
    float scale2;                                  // for exponents of two, of scores in kUnit
    hp_heads_t q, out;
    hp_packed_t k, v;
    const int32_t *ranges;
    float *lse;
    // Rows that lie in several units: the unit that has the beginning writes part 1 of its place, the others part 0.
    // products [heads_k * head_tiles][units][2][part_heads][dim], lse2 the same without dim, rows [rows] first and last unit.
    float *products, *lse2;
    int2 *row_units;
    int32_t part_heads;
};

// The 64 states of a wave in LDS: of each tensor codes [64][GP] of 16 bytes, a row's groups turned so that the same group
// of 8 neighbouring rows lies in different banks, and scales [64][kPairs] (step, low).
template <int GP> struct Layout {
    static constexpr int kPairs = GP == 3 ? 4 : GP;
    static constexpr int kCodes = kTile * GP * kGroupBytes, kTensor = kCodes + kTile * kPairs * 4, kBytes = 2 * kTensor;
    static __device__ __forceinline__ int slot(int row, int g) {
        if constexpr (GP == 8) return g ^ (row & 7);
        else if constexpr (GP == 4) return g ^ (row >> 1 & 3);
        else if constexpr (GP == 2) return g ^ (row >> 2 & 1);
        else return g;
    }
    static __device__ __forceinline__ int at(int row, int g) { return (row * GP + slot(row, g)) * kGroupBytes; }
};

// Brings tiles of one tensor to LDS.  Load n of a lane is so many rows behind load 0, its group turned the same way: one
// offset does for all of them (of three groups, which lie across the loads, three).
template <int GP> struct Loader {
    static constexpr int kPairs = Layout<GP>::kPairs, kLoads = GP + kPairs, kOffsets = GP == 3 ? 3 : 1;
    uint32_t codes[kOffsets], scales;
    __device__ __forceinline__ void plan(const hp_packed_t &t, int groups, int lane) {
#pragma unroll
        for (int n = 0; n < kOffsets; ++n) {
            const int e = n * kWave + lane, row = e / GP, g = Layout<GP>::slot(row, e % GP);     // slot() is its own inverse
            codes[n] = g < groups ? (uint32_t)(row * (int)t.code_row_stride + g * kGroupBytes) : kOutside;
        }
        const int g = lane % kPairs;
        scales = g < groups ? (uint32_t)(lane / kPairs * (int)t.scale_row_stride * 2 + 4 * g) : kOutside;
    }
    // left: states from the tile's first on that are seen
    __device__ __forceinline__ void fetch(char *to, const hp_packed_t &t, int64_t first, int head, int left, int lane) const {
        const char *const codes_at = (const char *)t.codes + first * t.code_row_stride + (int64_t)head * t.code_head_stride;
        const uint16_t *const pairs_at = (const uint16_t *)t.scales + first * t.scale_row_stride + (int64_t)head * t.scale_head_stride;
        constexpr int kRows = kWave / GP, kPairRows = kWave / kPairs;         // of a load
#pragma unroll
        for (int n = 0; n < GP; ++n)
            if constexpr (kOffsets == 1) pieces_to_lds(codes_at, to + n * kWave * 16, lane / GP < left - n * kRows ? codes[0] : kOutside, n * kRows * (int)t.code_row_stride);
            else pieces_to_lds(codes_at, to + n * kWave * 16, (n * kWave + lane) / GP < left ? codes[n % kOffsets] : kOutside, 0);
#pragma unroll
        for (int n = 0; n < kPairs; ++n)
            words_to_lds(pairs_at, to + Layout<GP>::kCodes + n * kWave * 4, lane / kPairs < left - n * kPairRows ? scales : kOutside, n * kPairRows * (int)t.scale_row_stride * 2);
    }
};

__device__ __forceinline__ float2 across_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Of quarters 0 and 1 (and 2 and 3): the first has both its own x and the second's, the second both their y.
__device__ __forceinline__ float2 across_rows(float x, float y) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Over the four lanes of a column.
__device__ __forceinline__ float column_max(float x) {
    const float2 a = across_halves(x), b = across_rows(fmaxf(a.x, a.y), fmaxf(a.x, a.y));
    return fmaxf(b.x, b.y);
}
__device__ __forceinline__ float column_sum(float x) {
    const float2 a = across_halves(x), b = across_rows(a.x + a.y, a.x + a.y);
    return b.x + b.y;
}

// What a row sees, and the tiles of it: one for rows that see nothing, so that somebody writes their zeros.
struct Range {
    int lo, hi;
    __device__ __forceinline__ int tiles() const { return max(1, (hi - lo + kTile - 1) / kTile); }
};
__device__ __forceinline__ Range range_of(const Params &p, int64_t row) {
    Range r{0, (int)p.keys};
    if (p.ranges) {
        r.lo = max(p.ranges[2 * row], 0);
        r.hi = min(p.ranges[2 * row + 1], (int)p.keys);
    }
    if (r.lo >= r.hi) r.lo = r.hi = 0;
    return r;
}

// All rows' tiles lie one behind the other, and the units take equal shares, whatever the rows' lengths: each wave adds up
// the lengths for itself, a few rows a lane.  A row begins with a tile more for each wave, for what it takes to begin and end
// one (30 requests of 1 to 2305 states in heads of 72: 35 us without, 31.7 so, 34 with two).  The tiles of a unit: `left` of
// them, the first of which is the skip-th of `row` and the at-th of all.
constexpr int kRowsALane = 8, kMostShared = kRowsALane * kWave;
template <int WAVES> struct Share {
    int64_t row;
    int skip, left, at, total, units;
    Range held;                                    // of row `lane`, where there are no more rows than lanes
    bool few;
    static __device__ __forceinline__ int cost(const Range &r) { return WAVES + r.tiles(); }
    __device__ __forceinline__ Range now(const Params &p) const {
        if (!few) return range_of(p, row);
        return Range{__builtin_amdgcn_readlane(held.lo, (int)row), __builtin_amdgcn_readlane(held.hi, (int)row)};
    }
};
template <int WAVES> __device__ __forceinline__ Share<WAVES> share_of(const Params &p, int unit, int lane) {
    Share<WAVES> s{unit, 0, 0, 0, 0, 0, Range{}, false};
    if (!p.units) {
        s.left = s.cost(range_of(p, unit));
        return s;
    }
    const int rows = (int)p.rows, each = (rows + kWave - 1) / kWave, mine = lane * each;
    s.few = each == 1;
    int own = 0;
    if (s.few) {
        s.held = range_of(p, min(lane, rows - 1));
        own = lane < rows ? s.cost(s.held) : 0;
    } else {
        for (int i = 0; i < each; ++i)
            if (mine + i < rows) own += s.cost(range_of(p, mine + i));
    }
    int upto = own;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int before = __shfl_up(upto, d);
        if (lane >= d) upto += before;
    }
    s.total = __builtin_amdgcn_readlane(upto, kWave - 1);
    s.units = min(p.units, (s.total + WAVES - 1) / WAVES);         // none with less than a tile for each wave
    s.at = unit < s.units ? first_of(s.total, unit, s.units) : 0;
    s.left = unit < s.units ? first_of(s.total, unit + 1, s.units) - s.at : 0;
    // the lane whose rows have that tile, then the row
    const int at_lane = __builtin_ctzll(__ballot(upto > s.at));
    int before = __builtin_amdgcn_readlane(upto - own, at_lane), row = at_lane * each;
    if (!s.few)
        for (;; ++row) {
            const int n = s.cost(range_of(p, row));
            if (before + n > s.at) break;
            before += n;
        }
    s.row = row, s.skip = s.at - before;
    return s;
}

// x of lane I of this lane's row of 16.
template <int I> __device__ __forceinline__ float of_lane(float x) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x150 + I, 0xf, 0xf, true));
}
// f(0) to f(N - 1), as constants.
template <int N, class F> __device__ __forceinline__ void each(const F &f) {
    if constexpr (N > 0) {
        each<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

constexpr int kSideHeads = 4;                      // of a state head, at most, for the three terms of each to stand side by side
constexpr float kLag = 8.0f;                       // the maximum is raised when a score passes it by 2^8

// Waves of a workgroup, and workgroups of a compute unit: as registers and LDS let run (of 160 KiB, which two workgroups of 80
// or four of 40 do not share: 1024 of these took two turns, 64 requests 88 us instead of 77).
template <int GP> constexpr int kWaves = GP == 8 ? 7 : 4;
template <class T, int GP, bool SIDE = false> constexpr int kResident = SIDE && GP <= 3 ? 3 : sizeof(T) == 2 || SIDE ? (GP <= 3 ? 4 : GP == 4 ? 3 : 1) : (GP <= 2 ? 3 : GP <= 4 ? 2 : 1);
// One row of few tiles: one workgroup for each tile of heads, with more waves.
constexpr int kMostWaves = 8;
template <int GP> constexpr int kFewWaves = GP == 8 ? 7 : kMostWaves;
template <class T, int GP, int WAVES, bool SIDE> constexpr int kWavesASimd = WAVES == kWaves<GP> ? (WAVES * kResident<T, GP, SIDE> + 3) / 4 : (WAVES + 3) / 4;

// Where a state head has four heads at most, the three bfloat16 terms of their binary32 queries and weights stand side by side,
// term t in the columns 4t and on of one product, in the place of three products one behind the other; their sums meet once
// for the scores and once at the end.  64 requests of 576 to 6404 states, 32 heads of 128 on 8: 126 us without, 120 so; heads of
// 256, whose registers hold no three operands of each kind, 44 and 32.
struct Side {
    float first, second;                           // whether this lane's term is behind the first, the second
    __device__ __forceinline__ explicit Side(int term) : first(term >= 1 ? 1.0f : 0.0f), second(term >= 2 ? 1.0f : 0.0f) {}
    __device__ __forceinline__ __bf16 operator()(float x) const {
        x = __builtin_fmaf(-first, upper_half(x), x);
        return half_of(__builtin_fmaf(-second, upper_half(x), x));
    }
};
// Over the four lanes of a row of 16 that have the same head's terms, in all of them alike.
template <int BY> __device__ __forceinline__ float turned(float x) {
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x120 + BY, 0xf, 0xf, true));
}
__device__ __forceinline__ float side_sum(float x) {
    x += turned<8>(x);
    return x + turned<4>(x);
}

template <class T, int GP, int WAVES, bool SIDE> __global__ __launch_bounds__((WAVES * kWave), (kWavesASimd<T, GP, WAVES, SIDE>)) void packed_attend_kernel(Params p) {
    typedef Layout<GP> L;
    constexpr float kLift = Codes<T>::kLift, kUnit = Codes<T>::kUnit;
    constexpr bool kCentred = kLift == -kMiddle;
    constexpr int N = SIDE ? 1 : kTerms<T>, kSets = (GP + 3) / 4, kWaves = WAVES;
    __shared__ __attribute__((aligned(16))) char lds[kWaves * L::kBytes];
    static_assert(sizeof(lds) >= 16 * kWaves * 2 * GP * kWave + 8 * kWaves * kHeads, "room for the join");
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), col = lane % 16, quarter = lane / 16;
    const int unit = (int)blockIdx.x, state_head = (int)blockIdx.y / p.head_tiles, first_head = ((int)blockIdx.y % p.head_tiles) * kHeads;
    const int col_head = SIDE ? col % kSideHeads : col, term = SIDE ? col / kSideHeads : 0;
    const Side side(term);
    const bool spare = SIDE && term == kTerms<T>;  // columns without a term: zeros
    const int heads = min(p.group - first_head, kHeads), head0 = state_head * p.group + first_head;
    char *const k_tile = lds + wave * L::kBytes, *const v_tile = k_tile + L::kTensor;
    const uint32_t *const k_scales = (const uint32_t *)(k_tile + L::kCodes), *const v_scales = (const uint32_t *)(v_tile + L::kCodes);
    Loader<GP> ks, vs;
    ks.plan(p.k, p.groups, lane);
    vs.plan(p.v, p.groups, lane);
    // of a quarter's states 16 a + 4 quarter + i, a and i < 4, lane 4 a + i has the steps and brings the transposed codes
    const int own = 16 * (col / 4) + 4 * quarter + col % 4;
    const auto split = [&](float x, Frag (&f)[N], int i) {
        if constexpr (SIDE) f[0][i] = side(x);
        else terms(x, f, i);
    };
    const Frag centre = all_of(-kLift - kMiddle);
    const Codes<T> codes;

    Share share = share_of<kWaves>(p, unit, lane);
    for (; share.left > 0; ++share.row, share.skip = 0) {
        const int64_t row = share.row;
        const Range see = share.now(p);
        const int lo = see.lo, hi = see.hi, n_tiles = see.tiles();
        const int first = share.at - share.skip, cost = share.cost(see), taken = min(cost - share.skip, share.left);    // first: the row's place among all
        const int begin = max(share.skip - kWaves, 0), end = share.skip + taken - kWaves;
        share.left -= taken, share.at += taken;
        if (end <= begin) break;                   // the next unit has the row's first tile
        const bool whole = begin == 0 && end == n_tiles;
        if (p.units && begin == 0 && blockIdx.y == 0 && tid == 0)
            p.row_units[row] = make_int2(unit, whole ? unit : unit_of(share.total, first + cost - 1, share.units));

        // the queries, and the right operand that puts the lows in: for each pair (step, low) of four groups the values
        // (-lift sum q, sum q), split into three numbers over the quarters
        Frag q[GP][N], sums[kSets] = {};
        const T *q_row = (const T *)p.q.data + row * p.q.row_stride + (int64_t)(head0 + min(col_head, heads - 1)) * p.q.head_stride;
        Vec<T, 8> x[GP];
        int dim = p.dim;
        asm volatile("" : "+s"(dim));                  // or the places of all channels would be kept over the rows
        if (dim % 8 == 0) {                            // pieces are there or not
#pragma unroll
            for (int g = 0; g < GP; ++g) {
                const int d = kGroup * g + 8 * quarter;
                x[g] = *(const typename VecOf<T, 8>::mem *)(q_row + (d < dim ? d : 0));
                if (d >= dim) x[g] = Vec<T, 8>{};
            }
        } else {
#pragma unroll
            for (int g = 0; g < GP; ++g) {
                const int d = kGroup * g + 8 * quarter;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const T one = q_row[min(d + i, dim - 1)];
                    x[g][i] = d + i < dim ? one : (T)0.0f;
                }
                __builtin_amdgcn_sched_barrier(0);     // no more of them at a time than registers hold
            }
        }
        // the first tiles are under way while the queries are made operands
        __builtin_amdgcn_sched_barrier(0);
        if (begin + wave < end) {
            const int key0 = lo + (begin + wave) * kTile;
            ks.fetch(k_tile, p.k, key0, state_head, hi - key0, lane);
            vs.fetch(v_tile, p.v, key0, state_head, hi - key0, lane);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < GP; ++g) {
            if constexpr (SIDE)
#pragma unroll
                for (int i = 0; i < 8; ++i) q[g][0][i] = side(spare ? 0.0f : (float)x[g][i]);
            else terms<T>(x[g], q[g]);
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum += (float)x[g][i];
            sum = column_sum(sum);
            const __bf16 a = (__bf16)sum, b = (__bf16)(sum - (float)a), c = (__bf16)(sum - (float)a - (float)b);
            const float part = quarter == 0 ? (float)a : quarter == 1 ? (float)b : quarter == 2 ? (float)c : 0.0f, of_this = term == 0 ? part : 0.0f;
            sums[g / 4][2 * (g % 4)] = (__bf16)(-kLift * kUnit * of_this);
            sums[g / 4][2 * (g % 4) + 1] = (__bf16)(kUnit * of_this);
        }

        float top = -INFINITY, sum = 0.0f;
        Quad out[2 * GP] = {}, rest = {};
        for (int tile = begin + wave; tile < end; tile += kWaves) {
            const int key0 = lo + tile * kTile, next = key0 + kWaves * kTile;
            const bool more = tile + kWaves < end;
            __builtin_amdgcn_s_waitcnt(but(Loader<GP>::kLoads));   // all but V's
            settle();
            Quad s[4];
            const Vec<uint32_t, L::kPairs> k_pairs = *(const Vec<uint32_t, L::kPairs> *)(k_scales + L::kPairs * own);
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                s[a] = Quad{};
                const Vec<uint32_t, L::kPairs> pairs = *(const Vec<uint32_t, L::kPairs> *)(k_scales + L::kPairs * (16 * a + col));
#pragma unroll
                for (int h = 0; h < kSets; ++h) {
                    Words w = {};
#pragma unroll
                    for (int j = 0; j < 4 && 4 * h + j < L::kPairs; ++j) w[j] = pairs[4 * h + j];
                    s[a] = mma(__builtin_bit_cast(Frag, w), sums[h], s[a]);
                }
            }
            each<GP>([&](auto g) {
                each<4>([&](auto a) {
                    const Frag c = codes(*(const uint32_t *)(k_tile + L::at(16 * a + col, g) + 4 * quarter));
                    Quad d = {};
#pragma unroll
                    for (int n = 0; n < N; ++n) d = mma(c, q[g][n], d);
                    each<4>([&](auto i) { s[a][i.value] += of_lane<4 * a + i>(step_of(k_pairs[g.value])) * d[i.value]; });
                });
            });
            if constexpr (SIDE)
#pragma unroll
                for (int a = 0; a < 4; ++a)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[a][i] = side_sum(s[a][i]);
            // here, not behind the branch, where all these products' results would have to be kept until then
#pragma unroll
            for (int a = 0; a < 4; ++a) asm("" : "+v"(s[a]));
            reads_done();
            if (more) ks.fetch(k_tile, p.k, next, state_head, hi - next, lane);

            if (key0 + kTile > hi)
#pragma unroll
                for (int a = 0; a < 4; ++a)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[a][i] = key0 + 16 * a + 4 * quarter + i < hi ? s[a][i] : -INFINITY;
            float most = s[0][0];
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int i = 0; i < 4; ++i) most = fmaxf(most, s[a][i]);
            most = column_max(most) * p.scale2;
            const bool grows = most > top + kLag;
            if (__any(grows)) {
                const float keep = grows ? __builtin_amdgcn_exp2f(top - most) : 1.0f;
                top = grows ? most : top;
                sum *= keep;
                rest *= keep;
#pragma unroll
                for (int c = 0; c < 2 * GP; ++c) out[c] *= keep;
            }
            const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    s[a][i] = __builtin_amdgcn_exp2f(s[a][i] * p.scale2 - base);
                    sum += s[a][i];
                    if constexpr (SIDE) s[a][i] = spare ? 0.0f : s[a][i];
                }

            if (more) __builtin_amdgcn_s_waitcnt(but(Loader<GP>::kLoads));
            else __builtin_amdgcn_s_waitcnt(but(0));
            settle();
            if constexpr (kCentred) {
                // sum p (8 step + low): row g of the left operand has group g's pairs as they lie there, the right one 8p and p by
                // turns, so that what is large of either meets in the product and does not add up by itself (binary32 would lose
                // three bits of outputs that are small beside the values)
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    Words pairs;
                    Frag weights[N];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        pairs[i] = v_scales[L::kPairs * (16 * a + 4 * quarter + i) + col % L::kPairs];
                        split(kMiddle * s[a][i], weights, 2 * i);
                        split(s[a][i], weights, 2 * i + 1);
                    }
#pragma unroll
                    for (int n = 0; n < N; ++n) rest = mma(__builtin_bit_cast(Frag, pairs), weights[n], rest);
                }
            } else {
                // 8 sum p step + sum p low: row 2g of the left operand has group g's steps, row 2g + 1 its lows
                typedef short Four __attribute__((ext_vector_type(4)));
                typedef __attribute__((address_space(3))) Four *Lds;
                // 16 lanes bring four states' pairs, 8 bytes a lane; beyond a state's pairs rows of the product are not read
                const uint32_t *line = v_scales + L::kPairs * (4 * quarter + col / 4) + 2 * (col % 4 % (L::kPairs / 2));
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const Four even = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(line + L::kPairs * 32 * b)), odd = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(line + L::kPairs * (32 * b + 16)));
                    const Frag pairs = __builtin_bit_cast(Frag, __builtin_shufflevector(even, odd, 0, 1, 2, 3, 4, 5, 6, 7));
                    Frag weights[N];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        split(s[2 * b][i], weights, i);
                        split(s[2 * b + 1][i], weights, 4 + i);
                    }
#pragma unroll
                    for (int n = 0; n < N; ++n) rest = mma(pairs, weights[n], rest);
                }
            }
            const Vec<uint32_t, L::kPairs> v_pairs = *(const Vec<uint32_t, L::kPairs> *)(v_scales + L::kPairs * own);
            each<GP>([&](auto g) {
                Frag weights[2][N];
                each<8>([&](auto e) {
                    constexpr int b = e / 4, i = e % 4;
                    const float step = step_of(v_pairs[g.value]);
                    split(of_lane<8 * b + i>(step) * s[2 * b][i], weights[b], 2 * i);
                    split(of_lane<8 * b + 4 + i>(step) * s[2 * b + 1][i], weights[b], 2 * i + 1);
                });
                typedef int Pair __attribute__((ext_vector_type(2)));
                typedef __attribute__((address_space(3))) Pair *Lds;
                const char *line = v_tile + L::at(own, g);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const Pair w = __builtin_amdgcn_ds_read_tr4_b64_v2i32((Lds)(line + 8 * c));
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const Frag l = codes((uint32_t)w[b]);
#pragma unroll
                        for (int n = 0; n < N; ++n) {
                            if constexpr (!kCentred) out[2 * g + c] = mma(centre, weights[b][n], out[2 * g + c]);
                            out[2 * g + c] = mma(l, weights[b][n], out[2 * g + c]);
                        }
                    }
                }
            });
            reads_done();
            if (more) vs.fetch(v_tile, p.v, next, state_head, hi - next, lane);
        }
        sum = column_sum(sum);

        // join the waves in the tiles' place: statistics, then the products, of which each wave adds up every kWaves-th tile
        Quad *const join = (Quad *)lds;                // [wave][2 GP][lane]
        float *const tops = (float *)(join + kWaves * 2 * GP * kWave), *const totals = tops + kWaves * kHeads;
        __syncthreads();
        if (quarter == 0) {
            tops[wave * kHeads + col] = top;
            totals[wave * kHeads + col] = sum;
        }
        __syncthreads();
        float most = -INFINITY, total = 0.0f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) most = fmaxf(most, tops[w * kHeads + col]);
        // a wave without a maximum has seen nothing, or NaN alone
        const auto weight = [&](float t) { return t == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(t - most); };
#pragma unroll
        for (int w = 0; w < kWaves; ++w) total += totals[w * kHeads + col] * weight(tops[w * kHeads + col]);
        const float part_of_all = total == 0.0f ? 0.0f : weight(top) / total;
        const float lse2 = total == 0.0f ? -INFINITY : most + __builtin_amdgcn_logf(total);
#pragma unroll
        for (int g = 0; g < GP; ++g) {
            const int from = kCentred ? 16 * (g / 4) + col : 16 * (g / 2) + col;
            float more;
            if constexpr (kCentred) more = __shfl(rest[g % 4], from);
            else more = kMiddle * __shfl(rest[2 * (g % 2)], from) + __shfl(rest[2 * (g % 2) + 1], from);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                // rows of the transposed load are a word's bits in order: even channels in one quarter, odd ones in the next
                const Quad v = (out[2 * g + c] * (1.0f / kUnit) + more) * part_of_all;
                const float2 a = across_rows(v[0], v[2]), b = across_rows(v[1], v[3]);
                join[(wave * 2 * GP + 2 * g + c) * kWave + lane] = Quad{a.x, a.y, b.x, b.y};
            }
        }
        __syncthreads();
        const int64_t part = ((int64_t)blockIdx.y * p.units + unit) * 2 + (begin == 0);
        for (int t = wave; t < 2 * GP; t += kWaves) {
            const int d = 16 * t + 4 * quarter;
            Quad v = {};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) v += join[(w * 2 * GP + t) * kWave + lane];
            if constexpr (SIDE)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = side_sum(v[i]);
            if (col >= heads || d >= p.dim) continue;
            if (!whole) {
                store<4>(p.products + (part * p.part_heads + col) * p.dim + d, v, p.dim - d);
            } else {
                Vec<T, 4> o;
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = (T)v[i];
                store<4>((T *)p.out.data + row * p.out.row_stride + (int64_t)(head0 + col) * p.out.head_stride + d, o, p.dim - d);
            }
        }
        if (wave == 0 && quarter == 0 && col < heads) {
            if (!whole) p.lse2[part * p.part_heads + col] = lse2;
            else if (p.lse) p.lse[row * p.heads_q + head0 + col] = lse2 * kLn2;
        }
        __syncthreads();                               // the next row's tiles come where this was
    }
}

// Joins the parts of rows that lie in several units.  A row and head has `waves` waves, which take every waves-th part; a
// workgroup is one row and head of four or sixteen waves, or four heads of one.  4 to 7 us, a launch and three loads one behind
// the other: which units, their sums, their products (asking for the first products ahead changed nothing).
constexpr int kMostJoin = 16;
template <class T> __global__ __launch_bounds__(kMostJoin * kWave) void packed_join_kernel(Params p, int waves) {
    __shared__ __attribute__((aligned(16))) float shared[kMostJoin][HP_ATTEND_MAX_DIM];
    const int lane = (int)threadIdx.x % kWave, index = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), wave = index % waves;
    const int64_t row = blockIdx.x;
    const int2 units = p.row_units[row];
    if (units.x == units.y) return;                // written as it was made
    const int head = (int)(blockIdx.y * (blockDim.x / kWave / waves)) + index / waves, state_head = head / p.group, in_group = head - state_head * p.group;
    if (head >= p.heads_q) return;                 // whole waves, and only where each works by itself
    const int64_t line = (int64_t)(state_head * p.head_tiles + in_group / kHeads) * p.units;
    const auto part = [&](int u) { return ((line + u) * 2 + (u == units.x)) * p.part_heads + in_group % kHeads; };
    // of the first 64 parts each lane keeps one's logarithm
    const int first = units.x + lane;
    const float own = first <= units.y ? p.lse2[part(first)] : -INFINITY;
    float top = own;
    for (int u = first + kWave; u <= units.y; u += kWave) top = fmaxf(top, p.lse2[part(u)]);
#pragma unroll
    for (int d = kWave / 2; d; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
    // nothing seen in a part: no weight; NaN stays, of the products too, which are added up whatever their weight
    const auto weight = [&](float t) { return t == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(t - top); };
    const float mine = weight(own);
    float sum = mine;
    for (int u = first + kWave; u <= units.y; u += kWave) sum += weight(p.lse2[part(u)]);
    sum = wave_sum(sum);
    Quad acc = {};
    const int d = 4 * lane;
    for (int u = units.x + wave; u <= units.y; u += waves) {
        const Quad v = load<4>(p.products + part(u) * p.dim + d, p.dim - d);
        const float w = u - units.x < kWave ? __shfl(mine, u - units.x) : weight(p.lse2[part(u)]);
        acc += w * v;
    }
    if (waves > 1) {
        *(Quad *)&shared[wave][d] = acc;
        __syncthreads();
        if (wave) return;
        for (int w = 1; w < waves; ++w) acc += *(const Quad *)&shared[w][d];
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    Vec<T, 4> o;
#pragma unroll
    for (int t = 0; t < 4; ++t) o[t] = (T)(acc[t] * inv);
    store<4>((T *)p.out.data + row * p.out.row_stride + (int64_t)head * p.out.head_stride + d, o, p.dim - d);
    if (p.lse && lane == 0) p.lse[row * p.heads_q + head] = sum == 0.0f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * kLn2;
}

// ---- host ------------------------------------------------------------------------------------------------------

int64_t align16(int64_t n) { return (n + 15) / 16 * 16; }

int head_tiles_of(const hp_packed_attend_args_t &a) { return (a.heads_q / a.heads_k + kHeads - 1) / kHeads; }

template <class T, bool SIDE = false> int resident_of(int groups) {
    return groups <= 2 ? kResident<T, 2, SIDE> : groups <= 3 ? kResident<T, 3, SIDE> : groups <= 4 ? kResident<T, 4, SIDE> : kResident<T, 8, SIDE>;
}
bool side_by_side(const hp_packed_attend_args_t &a) { return a.dtype == HP_F32 && a.heads_q / a.heads_k <= kSideHeads; }

// Units of each tile of heads, and whether they are workgroups of more waves.
//
// One row of up to two tiles a wave of such a workgroup is left in one, which needs no join: one request of 63, 576 and 1000
// states 7.8, 10.1 and 12.3 us, shared out with the launch that joins its parts 10.3, 12.5 and 12.6 (32 heads of 128 on 8); 2000
// states in two such workgroups took 17 us and took 12.6 with smaller ones.  Several rows are not, however little each sees: the
// workgroup would take them one behind the other, 5 us each (2 requests of 60 states 13 us, shared out 10; 8 of 7 states 44 and
// 10; 16 of 3 states 84 and 10).  All others get as many units as run at once.  Sharing out evenly costs rows of like lengths the
// cuts and the join (256 requests of 500 states 60 us, with a workgroup each 51; of 50 to 2000 states 105 and 96), but nobody
// knows here how long the longest is, and of 20000 states one workgroup would have 80 tiles a wave.  More than kMostShared rows,
// whose lengths no wave adds up by itself, are a workgroup each (513 requests of 50 to 2000 states 180 us, 512 shared out 176).
struct Cut {
    int32_t units;
    bool few;
};
Cut cut_of(const hp_packed_attend_args_t &a) {
    const int64_t columns = (int64_t)a.heads_k * head_tiles_of(a), tiles = a.keys / kTile + 1;
    if (a.rows > kMostShared || a.rows * (tiles + kMostWaves) > INT_MAX) return Cut{0, false};
    const int groups = groups_of(a.dim), waves = groups <= 4 ? kWaves<4> : kWaves<8>;
    if (a.rows == 1 && tiles <= 2 * (groups <= 4 ? kFewWaves<4> : kFewWaves<8>)) return Cut{1, true};
    const int64_t slots = kComputeUnits * (a.dtype == HP_BF16 ? resident_of<__bf16>(groups) : side_by_side(a) ? resident_of<float, true>(groups) : resident_of<float>(groups));
    const int64_t fit = slots / columns, most = (a.rows * (tiles + waves) + waves - 1) / waves, units = fit < most ? fit : most;
    return Cut{(int32_t)(units > 1 ? units : 1), false};
}

int check_sizes(const hp_packed_attend_args_t *a) {
    if (!a) return HP_EINVAL;
    if (a->dtype != HP_BF16 && a->dtype != HP_F32) return HP_EINVAL;
    if (a->dim < 1 || a->dim > HP_ATTEND_MAX_DIM || a->heads_k < 1 || a->heads_q < 1) return HP_EINVAL;
    if (a->heads_q % a->heads_k || a->heads_q > 16384) return HP_ELAYOUT;
    if (a->rows < 0 || a->keys < 0) return HP_EINVAL;
    // up to 448 lanes a row, of launches below 2^32; states are counted in 32 bits, with tiles to spare
    if (a->rows > 1 << 23 || a->rows > ((1 << 30) - 1024) / (a->heads_q / a->heads_k) || a->keys > INT_MAX - 1024) return HP_ELAYOUT;
    return HP_OK;
}

float scale2_of(const hp_packed_attend_args_t &a) { return a.scale * kLog2e / (a.dtype == HP_BF16 ? Codes<__bf16>::kUnit : Codes<float>::kUnit); }

int part_heads_of(const hp_packed_attend_args_t &a) { return a.heads_q / a.heads_k < kHeads ? a.heads_q / a.heads_k : kHeads; }

int64_t workspace_of(const hp_packed_attend_args_t &a) {
    const int64_t units = a.rows > 0 ? cut_of(a).units : 0, parts = 2 * units * a.heads_k * head_tiles_of(a) * part_heads_of(a);
    return units > 0 ? align16(4 * parts * a.dim) + align16(4 * parts) + align16(8 * a.rows) : 0;
}

int check(const hp_packed_attend_args_t *a) {
    if (const int rc = check_sizes(a)) return rc;
    if (!(a->scale > 0) || !std::isfinite(a->scale) || !std::isfinite(scale2_of(*a))) return HP_EINVAL;
    const int size = a->dtype == HP_BF16 ? 2 : 4;
    for (const hp_heads_t *t : {&a->q, &a->out}) {
        if (a->rows > 0 && !t->data) return HP_EINVAL;
        if ((uintptr_t)t->data % size) return HP_EALIGN;
    }
    for (const hp_packed_t *t : {&a->k, &a->v}) {
        if (const int rc = check_packed(*t, a->keys, a->heads_k)) return rc;
        if (!short_strides(*t, a->keys)) return HP_ELAYOUT;
    }
    if ((uintptr_t)a->ranges % 4 || (uintptr_t)a->lse % 4 || (uintptr_t)a->workspace % 16) return HP_EALIGN;
    const int64_t need = a->rows > 0 ? workspace_of(*a) : 0;
    if (need > 0 && (!a->workspace || a->workspace_bytes < need)) return HP_EINVAL;
    return HP_OK;
}

template <class T, int GP, bool SIDE> void launch(bool few, const Params &p, const dim3 &grid, hipStream_t s) {
    if (few) packed_attend_kernel<T, GP, kFewWaves<GP>, SIDE><<<grid, kFewWaves<GP> * kWave, 0, s>>>(p);
    else packed_attend_kernel<T, GP, kWaves<GP>, SIDE><<<grid, kWaves<GP> * kWave, 0, s>>>(p);
}
template <class T, bool SIDE> void launch(bool few, const Params &p, const dim3 &grid, hipStream_t s) {
    if (p.groups <= 2) launch<T, 2, SIDE>(few, p, grid, s);
    else if (p.groups == 3) launch<T, 3, SIDE>(few, p, grid, s);
    else if (p.groups == 4) launch<T, 4, SIDE>(few, p, grid, s);
    else launch<T, 8, SIDE>(few, p, grid, s);
}

template <class T> void join(const Params &p, hipStream_t s) {
    const int64_t items = p.rows * p.heads_q;
    // few rows and heads have many parts each, many few
    const int waves = items <= kComputeUnits ? kMostJoin : items <= 4 * kComputeUnits ? 4 : 1, each = waves == 1 ? 4 : 1;
    packed_join_kernel<T><<<dim3((uint32_t)p.rows, (uint32_t)((p.heads_q + each - 1) / each)), waves * each * kWave, 0, s>>>(p, waves);
}

}  // namespace

extern "C" {

int64_t hp_packed_attend_workspace(const hp_packed_attend_args_t *a) {
    if (const int rc = check_sizes(a)) return rc;
    return workspace_of(*a);
}

int hp_packed_attend_step(const hp_packed_attend_args_t *a, void *stream) {
    if (const int rc = check(a)) return rc;
    if (a->rows == 0) return HP_OK;
    const hipStream_t s = (hipStream_t)stream;
    Params p{};
    p.rows = a->rows, p.keys = a->keys;
    p.heads_q = a->heads_q, p.group = a->heads_q / a->heads_k, p.groups = groups_of(a->dim), p.dim = a->dim;
    const Cut cut = cut_of(*a);
    p.units = cut.units, p.head_tiles = head_tiles_of(*a), p.part_heads = part_heads_of(*a);
    p.scale2 = scale2_of(*a);
    p.q = a->q, p.out = a->out, p.k = without_unused(a->k, a->keys), p.v = without_unused(a->v, a->keys), p.ranges = a->ranges, p.lse = a->lse;
    const int64_t parts = (int64_t)2 * p.units * a->heads_k * p.head_tiles * p.part_heads;
    char *ws = (char *)a->workspace;
    p.products = (float *)ws;
    p.lse2 = (float *)(ws + align16(4 * parts * p.dim));
    p.row_units = (int2 *)(ws + align16(4 * parts * p.dim) + align16(4 * parts));
    const dim3 grid((uint32_t)(p.units ? p.units : p.rows), (uint32_t)(a->heads_k * p.head_tiles));
    if (a->dtype == HP_BF16) launch<__bf16, false>(cut.few, p, grid, s);
    else if (side_by_side(*a)) launch<float, true>(cut.few, p, grid, s);
    else launch<float, false>(cut.few, p, grid, s);
    if (hip_failed(hipGetLastError())) return HP_EHIP;
    if (p.units <= 1) return HP_OK;                // no row has parts
    if (a->dtype == HP_BF16) join<__bf16>(p, s);
    else join<float>(p, s);
    return hip_failed(hipGetLastError()) ? HP_EHIP : HP_OK;
}

}  // extern "C"
