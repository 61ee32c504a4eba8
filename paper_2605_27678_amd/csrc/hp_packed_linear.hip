// A few rows times a matrix held in 4 bits: out[r][n] = sum_k x[r][k] w[n][k], with a group's value = low + step * code
//     = sum_g (step_ng sum_k x_rk code_nk + low_ng sum_k x_rk)            (k in group g)
// The rows of x are the left operand of products of 16 x 16 x 32, a group of 16 rows of w at a time the right one, so that a
// lane has results of one row of w, whose step and low are its own.  The sums of x over a group are products with ones; for
// four groups at a time they are, split into numbers of 8 bits over the quarters (two of bfloat16's, which leave 2^-18 of a
// group's sum out; three of binary32's), the left operand of one more product, whose right one is the pairs (step, low) as
// they lie in memory: it puts sum x low in and takes off what the codes are lifted by.
// The waves of a workgroup share out the inner axis, 64 to 256 of it at a time, and add up at the end in their order.  Each brings its
// own pieces of x and w to LDS, ahead of their use and without barriers: the operands' rows lie in neighbouring lanes, and
// loads straight into registers took the caches 64 cycles each, one a lane, where runs of 64 and 256 bytes take 16
// (12288 x 12288 by 16 rows: 36 us, this way 29).
//
// The weights are 5 bits a value, read once by up to 32 rows: 95 MB of these 12288 x 12288 are 18 us at the rate of a large
// copy.  The call takes 29 with nothing in the caches (26 where the 256 MB cache has a part of them), its loads without the
// computing 27.  With more rows the caches are busier with x: of 8192 x 8192 by 64 rows every compute unit reads half of x,
// 0.5 MB, for its 64 rows of w, 128 MB next to 2 x 44; that takes 25 us, the loads alone 18, where a copy of the 44 MB takes 9.
// Binary32 has three products for each: 60 us.
#include "hp_packed.hpp"

#pragma clang fp contract(fast)

namespace {

using namespace hp;

constexpr int kOuts = 16;                          // rows of w of a tile
constexpr int kWaves = 8, kBlock = kWaves * kWave;

struct Params {
    int64_t rows;
    int32_t n_in, n_out, groups, waves_k;          // waves_k: that share a tile's inner axis, a power of two
    const void *x;
    int64_t x_stride;
    hp_packed_t w;
    void *out;
    int64_t out_stride;
};

// How a launch is cut.  A wave has in LDS, of a chunk of CH groups, R rows of x (4, or tiles of 16) and 16 MT rows of w's
// codes and pairs (step, low), DEPTH chunks in turn.  The 16-byte pieces of a row are turned, so that the same piece of
// neighbouring rows lies in different banks.  EXACT: rows of x are whole aligned pieces, which loads bring to LDS by themselves.
template <class T, int R_, int CH_, int MT_, int DEPTH_, bool EXACT_> struct Cut {
    typedef T type;
    static constexpr int R = R_, CH = CH_, MT = MT_, DEPTH = DEPTH_, N = kTerms<T>, NT = (R + 15) / 16;
    static constexpr bool EXACT = EXACT_;
    static constexpr int kPiece = 16 / (int)sizeof(T), kPieces = CH * kGroup / kPiece, kRowBytes = 16 * kPieces;      // of x
    static constexpr int kXLoads = R * kPieces / kWave, kWLoads = (MT * CH + 3) / 4;                                  // kWLoads: of codes, and of pairs
    static constexpr int kCodes = R * kRowBytes, kPairs = kCodes + kWLoads * kWave * 16, kBytes = kPairs + kWLoads * kWave * 4;
    static constexpr int kLoads = (EXACT ? kXLoads : 0) + 2 * kWLoads, kLds = kWaves * DEPTH * kBytes;
    // binary32 operands are two pieces, which stay neighbours
    static __device__ __forceinline__ int x_slot(int row, int piece) { return sizeof(T) == 2 ? piece ^ (row & (kPieces - 1)) : piece ^ (2 * row & (kPieces - 2)); }
    static __device__ __forceinline__ int code_slot(int row, int piece) { return piece ^ ((CH == 8 ? row : row / (16 / CH)) & (CH - 1)); }
    static_assert(CH <= 8, "a load has as many rows of w as are turned in a period");
    // loads of x whose pieces are turned alike are so many rows and loads apart
    static constexpr int kRowsALoad = kWave / kPieces, kPeriod = sizeof(T) == 2 ? kPieces : kPieces / 2;
    static constexpr int kKinds = kPeriod / kRowsALoad < kXLoads ? kPeriod / kRowsALoad : kXLoads;
    static_assert(kLds <= 160 * 1024 && kLds >= kWaves * MT * NT * kWave * 16, "fits, and has room for the sums");
    static_assert((DEPTH - 1) * kLoads < 64, "what a wave can wait for");
};

template <class C> __global__ __launch_bounds__(kBlock) void packed_linear_kernel(Params p) {
    typedef typename C::type T;
    constexpr int R = C::R, CH = C::CH, MT = C::MT, DEPTH = C::DEPTH, N = C::N, NT = C::NT, kSets = (CH + 3) / 4;
    constexpr float kLift = Codes<T>::kLift, kUnit = Codes<T>::kUnit;
    extern __shared__ __attribute__((aligned(16))) char shared[];
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), col = lane % 16, quarter = lane / 16;
    const int turn = wave & (p.waves_k - 1), tiles = kWaves / p.waves_k;
    const int n0 = ((int)blockIdx.x * tiles + wave / p.waves_k) * kOuts * MT;
    const int64_t r0 = (int64_t)blockIdx.y * R;
    const int rows = (int)min(p.rows - r0, (int64_t)R);
    // whole chunks of this wave, and one that is not whole behind the last
    const int all = n0 < p.n_out ? p.n_in / (CH * kGroup) : 0, chunks = (all - turn + p.waves_k - 1) / p.waves_k;
    char *const mine = shared + wave * (DEPTH * C::kBytes);

    const T *const x0 = (const T *)p.x + r0 * p.x_stride;
    const char *const codes = (const char *)p.w.codes + n0 * p.w.code_row_stride;
    const uint16_t *const pairs = (const uint16_t *)p.w.scales + n0 * p.w.scale_row_stride;
    // what a lane brings
    int x_piece[C::kKinds], x_row[C::kKinds];
    uint32_t x_at[C::kKinds], code_at[C::kWLoads], pair_at[C::kWLoads];
#pragma unroll
    for (int n = 0; n < C::kKinds; ++n) {
        x_row[n] = n * C::kRowsALoad + lane / C::kPieces;
        x_piece[n] = C::x_slot(x_row[n], lane % C::kPieces);
        x_at[n] = (uint32_t)(x_row[n] * (int)p.x_stride * (int)sizeof(T) + 16 * x_piece[n]);
    }
    const int w_row = lane / CH, code_piece = C::code_slot(w_row, lane % CH);
#pragma unroll
    for (int n = 0; n < C::kWLoads; ++n) {
        const int row = n * (kWave / CH) + w_row;
        const bool there = row < kOuts * MT && n0 + row < p.n_out;
        code_at[n] = there ? (uint32_t)(row * (int)p.w.code_row_stride + kGroupBytes * code_piece) : kOutside;
        pair_at[n] = there ? (uint32_t)(row * (int)p.w.scale_row_stride * 2 + 4 * (lane % CH)) : kOutside;
    }
    const auto fetch_w = [&](char *to, int g0, bool whole) {
#pragma unroll
        for (int n = 0; n < C::kWLoads; ++n) {
            pieces_to_lds(codes, to + C::kCodes + n * kWave * 16, whole || g0 + code_piece < p.groups ? code_at[n] : kOutside, g0 * kGroupBytes);
            words_to_lds(pairs, to + C::kPairs + n * kWave * 4, whole || g0 + lane % CH < p.groups ? pair_at[n] : kOutside, g0 * 4);
        }
    };
    const auto fetch_x = [&](char *to, int g0, bool whole) {
#pragma unroll
        for (int n = 0; n < C::kXLoads; ++n) {
            const int kind = n % C::kKinds, behind = n / C::kKinds * C::kPeriod;
            const bool there = x_row[kind] + behind < rows && (whole || g0 * kGroup + x_piece[kind] * C::kPiece < p.n_in);
            pieces_to_lds(x0, to + n * kWave * 16, there ? x_at[kind] : kOutside, (behind * (int)p.x_stride + g0 * kGroup) * (int)sizeof(T));
        }
    };
    // rows that are no whole pieces pass through registers
    typedef Vec<T, C::kPiece> Piece;
    const auto from_row = [&](int n) { return x0 + min(x_row[n % C::kKinds] + n / C::kKinds * C::kPeriod, rows - 1) * p.x_stride + x_piece[n % C::kKinds] * C::kPiece; };

    Quad acc[MT][NT] = {};
    const Frag ones = all_of(1.0f);
    const Codes<T> codes_of;
    // whether this quarter's number of a sum is behind the first, the second
    const float first = quarter >= 1 ? -1.0f : 0.0f, second = quarter >= 2 ? -1.0f : 0.0f;
    const auto add = [&](const char *from) {
        Words low[MT][kSets] = {};                 // for four groups at a time
        Frag sums[NT][kSets] = {};
#pragma unroll
        for (int j = 0; j < CH; ++j) {
            Frag a[NT][N];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int row = 16 * t + (R < 16 ? col % R : col);
                Vec<T, 8> x;
                if constexpr (sizeof(T) == 2) {
                    x = *(const Vec<T, 8> *)(from + row * C::kRowBytes + 16 * C::x_slot(row, 4 * j + quarter));
                } else {
                    const Quad lower = *(const Quad *)(from + row * C::kRowBytes + 16 * C::x_slot(row, 8 * j + 2 * quarter));
                    const Quad upper = *(const Quad *)(from + row * C::kRowBytes + 16 * C::x_slot(row, 8 * j + 2 * quarter + 1));
                    x = __builtin_shufflevector(lower, upper, 0, 1, 2, 3, 4, 5, 6, 7);
                }
                terms<T>(x, a[t]);
                Quad sum = {};                     // of this lane's row of x, in all four numbers
#pragma unroll
                for (int n = 0; n < N; ++n) sum = mma(ones, a[t][n], sum);
                // the quarter's number of it; what stands in quarters without one meets zeros
                float part = __builtin_fmaf(first, (float)(__bf16)sum[0], sum[0]);
                if constexpr (N > 1) part = __builtin_fmaf(second, (float)(__bf16)part, part);
                sums[t][j / 4][2 * (j % 4)] = (__bf16)(-kLift * kUnit * part);
                sums[t][j / 4][2 * (j % 4) + 1] = (__bf16)(kUnit * part);
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const int row = kOuts * m + col;
                const Frag l = codes_of(*(const uint32_t *)(from + C::kCodes + (row * CH + C::code_slot(row, j)) * kGroupBytes + 4 * quarter));
                const uint32_t pair = *(const uint32_t *)(from + C::kPairs + (row * CH + j) * 4);
                const float step = step_of(pair);
                low[m][j / 4][j % 4] = quarter <= (N > 1 ? 2 : 1) ? pair : 0;
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    Quad d = {};
#pragma unroll
                    for (int n = 0; n < N; ++n) d = mma(a[t][n], l, d);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[m][t][i] += step * d[i];
                }
            }
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < kSets; ++h) acc[m][t] = mma(sums[t][h], __builtin_bit_cast(Frag, low[m][h]), acc[m][t]);
    };

    const auto group_of = [&](int i) { return (turn + i * p.waves_k) * CH; };
    const auto stage = [&](int i) { return mine + i % DEPTH * C::kBytes; };
    for (int i = 0; i < DEPTH - 1 && i < chunks; ++i) {
        fetch_w(stage(i), group_of(i), true);
        if constexpr (C::EXACT) fetch_x(stage(i), group_of(i), true);
    }
    Piece held[C::EXACT ? 1 : C::kXLoads];
    if (!C::EXACT && chunks > 0)
#pragma unroll
        for (int n = 0; n < C::kXLoads; ++n) held[C::EXACT ? 0 : n] = *(const typename VecOf<T, C::kPiece>::mem *)(from_row(n) + group_of(0) * kGroup);
    for (int i = 0; i < chunks; ++i) {
        const bool more = i + DEPTH - 1 < chunks;
        if (more) fetch_w(stage(i + DEPTH - 1), group_of(i + DEPTH - 1), true);
        if constexpr (C::EXACT) {
            if (more) {
                fetch_x(stage(i + DEPTH - 1), group_of(i + DEPTH - 1), true);
                __builtin_amdgcn_s_waitcnt(but((DEPTH - 1) * C::kLoads));
            } else {
                __builtin_amdgcn_s_waitcnt(but(0));
            }
        } else {
#pragma unroll
            for (int n = 0; n < C::kXLoads; ++n) *(Piece *)(stage(i) + (n * kWave + lane) * 16) = held[n];
            // w's chunk i came before the pieces; this waits for the chunk asked for last as well, so that what is further
            // ahead than the next one is not of use here
            __builtin_amdgcn_s_waitcnt(but(0));
#pragma unroll
            for (int n = 0; n < C::kXLoads; ++n) held[n] = *(const typename VecOf<T, C::kPiece>::mem *)(from_row(n) + group_of(i + 1 < chunks ? i + 1 : i) * kGroup);
        }
        settle();
        add(stage(i));
        reads_done();
    }
    if (n0 < p.n_out && p.n_in % (CH * kGroup) && all % p.waves_k == turn) {
        const int g0 = all * CH;
        fetch_w(mine, g0, false);
        if constexpr (C::EXACT) {
            fetch_x(mine, g0, false);
        } else {
#pragma unroll
            for (int n = 0; n < C::kXLoads; ++n) *(Piece *)(mine + (n * kWave + lane) * 16) = load<C::kPiece>(from_row(n) + g0 * kGroup, p.n_in - g0 * kGroup - x_piece[n % C::kKinds] * C::kPiece);
        }
        __builtin_amdgcn_s_waitcnt(but(0));
        settle();
        add(mine);
        reads_done();
    }
    if (p.waves_k > 1) {
        __syncthreads();
        Quad *const parts = (Quad *)shared;        // [wave][MT][NT][lane]
        if (turn)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int t = 0; t < NT; ++t) parts[((wave * MT + m) * NT + t) * kWave + lane] = acc[m][t];
        __syncthreads();
        if (turn) return;
        for (int w = 1; w < p.waves_k; ++w)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[m][t] += parts[(((wave + w) * MT + m) * NT + t) * kWave + lane];
    }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int n = n0 + kOuts * m + col;
        if (n >= p.n_out) continue;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 16 * t + 4 * quarter + i;
                if (r < rows) ((T *)p.out)[(r0 + r) * p.out_stride + n] = (T)(acc[m][t][i] * (1.0f / kUnit));
            }
    }
}

int check(const hp_packed_linear_args_t *a) {
    if (!a) return HP_EINVAL;
    if (a->dtype != HP_BF16 && a->dtype != HP_F32) return HP_EINVAL;
    if (a->rows < 0 || a->n_in < 1 || a->n_out < 0) return HP_EINVAL;
    if (a->n_in > HP_PACKED_MAX_DIM || a->n_out > 1 << 24 || a->rows > 1 << 20) return HP_ELAYOUT;
    const int size = a->dtype == HP_BF16 ? 2 : 4;
    const bool any = a->rows > 0 && a->n_out > 0;
    if (any && (!a->x || !a->out)) return HP_EINVAL;
    if ((uintptr_t)a->x % size || (uintptr_t)a->out % size) return HP_EALIGN;
    if (const int rc = check_packed(a->w, any ? a->n_out : 0, 1)) return rc;
    return short_strides(a->w, a->n_out) ? HP_OK : HP_ELAYOUT;
}

// Workgroups of a launch, along w's rows and x's; p.waves_k is set for them.
template <class C> dim3 blocks_of(Params &p) {
    const int64_t tiles = (p.n_out + kOuts * C::MT - 1) / (kOuts * C::MT), chunks = (p.groups + C::CH - 1) / C::CH;
    p.waves_k = 1;
    while (p.waves_k < kWaves && 2 * p.waves_k <= chunks) p.waves_k *= 2;
    const int64_t each = kWaves / p.waves_k;
    return dim3((uint32_t)((tiles + each - 1) / each), (uint32_t)((p.rows + C::R - 1) / C::R));
}

// The first of these cuts, the smallest, of which the compute units take all workgroups at once; otherwise the last.  A
// larger tile reads x and waits for the join less often, a second turn costs as much as the first (us, bfloat16, each cut by itself):
//   4096 x 4096 by 16 rows in tiles of 16 / 32 rows of w   6.0 / 7.1      12288 x 12288: 16 / 32 / 48 / 64   46 / 38 / 29 / 30
//   8192 x 2048 by 64 rows in tiles of 16 x 32 / 32 x 32 / 32 x 64 (rows of x times rows of w)   11.3 / 14.7 / 22
//   8192 x 8192 by 64 rows, the same                                                             45 / 30 / 25
// Up to four rows in bfloat16 are the exception: their workgroups are small enough that several share a compute unit, and
// tiles of 16 were the fastest throughout (12288 x 4096 by one row 8.6, of 48 11.6; 28672 x 4096 17.7 and 23.3).
template <class C, class... More> void launch(Params &p, hipStream_t s) {
    const dim3 blocks = blocks_of<C>(p);
    if constexpr (sizeof...(More) > 0)
        if ((int64_t)blocks.x * blocks.y > kComputeUnits) return launch<More...>(p, s);
    packed_linear_kernel<C><<<blocks, kBlock, C::kLds, s>>>(p);
}

// Chunks are as long as LDS allows, for few and long requests to the caches, or fewer and more in turn, for loads to be ahead: two
// waves a SIMD hide the loads of a single chunk if there is enough to do with it (8192 x 8192 by 64 rows in tiles of 32 x 64: one
// chunk of 128 channels 25 us, two of 64 in turn 28; 4096 x 4096 by 16 rows: three of 64 6.0, one of 128 6.5).  Where workgroups
// are small, two chunks in turn leave room for four of them (28672 x 4096 by one row 17.7 us, four chunks 21.2).
//
// Rows of x that are no whole aligned pieces of 16 bytes pass through registers, and each chunk waits for x's and w's next
// (12288 x 8195 by 16 rows: 40 us, of 8192 21).  Binary32 has three products for one and twice x's bytes.
template <class T> void choose(Params &p, hipStream_t s) {
    constexpr int kPiece = 16 / sizeof(T);
    const bool exact = (uintptr_t)p.x % 16 == 0 && p.n_in % kPiece == 0 && p.x_stride % kPiece == 0 && p.x_stride >= 0 && p.x_stride <= kMostStride / 4;
    if (!exact) {
        if (p.rows <= 4) launch<Cut<T, 4, 4, 1, 4, false>, Cut<T, 4, 4, 2, 4, false>>(p, s);
        else if (p.rows <= 16) launch<Cut<T, 16, 2, 1, 3, false>, Cut<T, 16, 2, 2, 3, false>>(p, s);
        else launch<Cut<T, 32, 2, 2, 2, false>>(p, s);
    } else if constexpr (sizeof(T) == 2) {
        if (p.rows <= 4) launch<Cut<T, 4, 4, 1, 2, true>>(p, s);
        else if (p.rows <= 16) launch<Cut<T, 16, 2, 1, 3, true>, Cut<T, 16, 4, 2, 1, true>, Cut<T, 16, 4, 3, 2, true>, Cut<T, 16, 8, 4, 1, true>>(p, s);
        else launch<Cut<T, 16, 4, 2, 3, true>, Cut<T, 32, 4, 2, 1, true>, Cut<T, 32, 4, 3, 1, true>, Cut<T, 32, 4, 4, 1, true>>(p, s);
    } else {
        if (p.rows <= 4) launch<Cut<T, 4, 4, 1, 2, true>, Cut<T, 4, 4, 2, 2, true>, Cut<T, 4, 4, 3, 2, true>, Cut<T, 4, 4, 4, 1, true>>(p, s);
        else if (p.rows <= 16) launch<Cut<T, 16, 2, 1, 3, true>, Cut<T, 16, 2, 2, 3, true>, Cut<T, 16, 2, 3, 3, true>, Cut<T, 16, 2, 4, 2, true>>(p, s);
        else launch<Cut<T, 16, 2, 2, 3, true>, Cut<T, 32, 2, 2, 2, true>, Cut<T, 32, 2, 2, 1, true>>(p, s);
    }
}

}  // namespace

extern "C" {

int hp_packed_linear(const hp_packed_linear_args_t *a, void *stream) {
    if (const int rc = check(a)) return rc;
    if (a->rows == 0 || a->n_out == 0) return HP_OK;
    Params p{};
    p.rows = a->rows, p.n_in = a->n_in, p.n_out = a->n_out, p.groups = groups_of(a->n_in);
    p.x = a->x, p.x_stride = a->rows > 1 ? a->x_stride : 0, p.w = without_unused(a->w, a->n_out), p.out = a->out, p.out_stride = a->out_stride;
    const hipStream_t s = (hipStream_t)stream;
    if (a->dtype == HP_BF16) choose<__bf16>(p, s);
    else choose<float>(p, s);
    return hip_failed(hipGetLastError()) ? HP_EHIP : HP_OK;
}

}  // extern "C"
