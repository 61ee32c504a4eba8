// A few rows times a matrix held in 4 bits: out[r][n] = sum_k x[r][k] w[n][k], with a group's value = low + step * code
//     = sum_g (step_ng sum_k x_rk code_nk + low_ng sum_k x_rk)            (k in group g)
// The rows of x are the left operand of products of 16 x 16 x 32, a group of 16 rows of w at a time the right one, so that a
// lane has results of one row of w, whose step and low are its own.  The sums of x over a group are products with ones; for
// four groups at a time they are, split into numbers of 8 bits over the quarters, the left operand of one more product, whose
// right one is the pairs (step, low) as they lie in memory: it puts sum x low in and takes off what the codes are lifted by.
// The waves of a workgroup share out the inner axis, 128 of it at a time, and add up at the end in their order.  Each brings its
// own pieces of x and w to LDS, ahead of their use and without barriers: the operands' rows lie in neighbouring lanes, and
// loads straight into registers took the caches 64 cycles each, one a lane, where runs of 64 and 256 bytes take 16
// (12288 x 12288 by 16 rows: 36 us, with AAA).
#include <climits>
#include <cmath>

#include "hp_packed.hpp"

#pragma clang fp contract(fast)

namespace {

using namespace hp;

constexpr int kOuts = 16;                          // rows of w of a tile
constexpr int kChunk = 4, kChannels = kChunk * kGroup;                   // groups and channels at a time
constexpr int kMostWaves = 8;

struct Params {
    int64_t rows;
    int32_t n_in, n_out, groups, waves_k;          // waves_k: that share a tile's inner axis, a power of two
    const void *x;
    int64_t x_stride;
    hp_packed_t w;
    void *out;
    int64_t out_stride;
};

// What a wave has in LDS of a chunk: R rows of x, 16 MT rows of w's codes and as many of its pairs (step, low).  The 16-byte
// pieces of a row are turned, so that the same piece of neighbouring rows lies in different banks.
template <class T, int R, int MT> struct Stage {
    static constexpr int kPieces = kChannels * (int)sizeof(T) / 16, kRowBytes = 16 * kPieces;         // of a row of x
    static constexpr int kX = R * kRowBytes, kCodes = MT * kOuts * kChunk * kGroupBytes, kPairs = MT * kOuts * kChunk * 4, kBytes = kX + kCodes + kPairs;
    static constexpr int kXLoads = R * kPieces / kWave, kLoads = kXLoads + 2 * MT;
    // binary32 operands are two pieces, which stay neighbours
    static __device__ __forceinline__ int x_slot(int row, int piece) { return sizeof(T) == 2 ? piece ^ (row & 15) : piece ^ (2 * row & 30); }
    static __device__ __forceinline__ int code_slot(int row, int piece) { return piece ^ (row >> 1 & 3); }
};

// R: rows of x (4, or tiles of 16), MT: tiles of w of a wave, DEPTH: chunks in LDS, EXACT: rows of x are whole aligned pieces
// that loads bring to LDS by themselves.
template <class T, int R, int MT, int DEPTH, bool EXACT> __global__ __launch_bounds__(kMostWaves * kWave) void packed_linear_kernel(Params p) {
    typedef Stage<T, R, MT> S;
    constexpr int N = kTerms<T>, NT = (R + 15) / 16;
    constexpr float kLift = Codes<T>::kLift;
    extern __shared__ __attribute__((aligned(16))) char shared[];
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), col = lane % 16, quarter = lane / 16;
    const int turn = wave & (p.waves_k - 1), tiles = (int)blockDim.x / kWave / p.waves_k;
    const int n0 = ((int)blockIdx.x * tiles + wave / p.waves_k) * kOuts * MT;
    const int64_t r0 = (int64_t)blockIdx.y * R;
    const int rows = (int)min(p.rows - r0, (int64_t)R), all = n0 < p.n_out ? (p.groups + kChunk - 1) / kChunk : 0;
    const int chunks = (all - turn + p.waves_k - 1) / p.waves_k;
    char *const mine = shared + wave * (DEPTH * S::kBytes);

    const T *const x0 = (const T *)p.x + r0 * p.x_stride;
    const char *const codes = (const char *)p.w.codes + n0 * p.w.code_row_stride;
    const uint16_t *const pairs = (const uint16_t *)p.w.scales + n0 * p.w.scale_row_stride;
    // what a lane brings: of x a piece of every kWave / kPieces rows, of the codes piece and of the pairs pair lane % 4 of row lane / 4
    constexpr int kRowsALoad = kWave / S::kPieces, kKinds = 16 / kRowsALoad < S::kXLoads ? 16 / kRowsALoad : S::kXLoads;
    int x_piece[kKinds];
    uint32_t x_at[kKinds];
#pragma unroll
    for (int n = 0; n < kKinds; ++n) {
        const int row = n * kRowsALoad + lane / S::kPieces;
        x_piece[n] = S::x_slot(row, lane % S::kPieces);
        x_at[n] = (uint32_t)(row * (int)p.x_stride * (int)sizeof(T) + 16 * x_piece[n]);
    }
    const int w_row = lane / 4, code_piece = S::code_slot(w_row, lane % 4);
    const uint32_t code_at = (uint32_t)(w_row * (int)p.w.code_row_stride + kGroupBytes * code_piece), pair_at = (uint32_t)(w_row * (int)p.w.scale_row_stride * 2 + 4 * (lane % 4));

    // Chunk i of this wave; beyond its last one, and of rows and groups that are not there, zeros, which are not read.
    const auto fetch = [&](int i) {
        char *to = mine + i % DEPTH * S::kBytes;
        const int c = i < chunks ? turn + i * p.waves_k : all, g0 = c * kChunk;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            const bool there = i < chunks && n0 + kOuts * m + w_row < p.n_out;
            pieces_to_lds(codes, to + S::kX + m * kWave * 16, there && g0 + code_piece < p.groups ? code_at + g0 * kGroupBytes : kOutside, kOuts * m * (int)p.w.code_row_stride);
            words_to_lds(pairs, to + S::kX + S::kCodes + m * kWave * 4, there && g0 + lane % 4 < p.groups ? pair_at + 4 * g0 : kOutside, 2 * kOuts * m * (int)p.w.scale_row_stride);
        }
#pragma unroll
        for (int n = 0; n < S::kXLoads; ++n) {
            const int row = n * kRowsALoad + lane / S::kPieces, piece = x_piece[n % kKinds], k = c * kChannels + piece * (16 / (int)sizeof(T));
            if constexpr (EXACT) {
                pieces_to_lds(x0, to + n * kWave * 16, i < chunks && row < rows && k < p.n_in ? x_at[n % kKinds] + c * S::kRowBytes : kOutside, n / kKinds * 16 * (int)p.x_stride * (int)sizeof(T));
            } else {
                *(Vec<T, 16 / sizeof(T)> *)(to + (n * kWave + lane) * 16) = load<16 / sizeof(T)>(x0 + row * p.x_stride + k, i < chunks && row < rows ? p.n_in - k : 0);
            }
        }
    };
    Quad acc[MT][NT] = {};
    const Frag ones = all_of(1.0f);
    const Codes<T> codes_of;
    const auto add = [&](const char *from) {
        Words w[MT], pairs[MT];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            w[m] = *(const Words *)(from + S::kX + (m * kOuts + col) * kChunk * kGroupBytes + kGroupBytes * S::code_slot(col, quarter));
            pairs[m] = *(const Words *)(from + S::kX + S::kCodes + (m * kOuts + col) * kChunk * 4);
            across_quarters(w[m]);
        }
        Frag sums[NT];
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            Frag a[NT][N];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const int row = 16 * t + (R < 16 ? col % R : col);
                Vec<T, 8> x;
                if constexpr (sizeof(T) == 2) {
                    x = *(const Vec<T, 8> *)(from + row * S::kRowBytes + 16 * S::x_slot(row, 4 * j + quarter));
                } else {
                    const Quad lower = *(const Quad *)(from + row * S::kRowBytes + 16 * S::x_slot(row, 8 * j + 2 * quarter));
                    const Quad upper = *(const Quad *)(from + row * S::kRowBytes + 16 * S::x_slot(row, 8 * j + 2 * quarter + 1));
                    x = __builtin_shufflevector(lower, upper, 0, 1, 2, 3, 4, 5, 6, 7);
                }
                terms<T>(x, a[t]);
                Quad sum = {};                     // of this lane's row of x, in all four numbers
#pragma unroll
                for (int n = 0; n < N; ++n) sum = mma(ones, a[t][n], sum);
                const float first = (float)(__bf16)sum[0], second = (float)(__bf16)(sum[0] - first);
                const float part = quarter == 0 ? first : quarter == 1 ? second : N > 1 && quarter == 2 ? sum[0] - first - second : 0.0f;
                sums[t][2 * j] = (__bf16)(-kLift * part);
                sums[t][2 * j + 1] = (__bf16)part;
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const Frag l = codes_of(w[m][j]);
                const float step = step_of(pairs[m][j]);
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
            for (int t = 0; t < NT; ++t) acc[m][t] = mma(sums[t], __builtin_bit_cast(Frag, pairs[m]), acc[m][t]);
    };
    for (int i = 0; i < DEPTH - 1; ++i) fetch(i);
    for (int i = 0; i < chunks; ++i) {
        fetch(i + DEPTH - 1);
        if constexpr (EXACT) __builtin_amdgcn_s_waitcnt(but((DEPTH - 1) * S::kLoads));
        else __builtin_amdgcn_s_waitcnt(but(0));
        settle();
        add(mine + i % DEPTH * S::kBytes);
        reads_done();
    }
    if (p.waves_k > 1) {
        __builtin_amdgcn_s_waitcnt(but(0));        // zeros still on their way would come into what follows
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
                if (r < rows) ((T *)p.out)[(r0 + r) * p.out_stride + n] = (T)acc[m][t][i];
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

template <class T, int R, int MT, int DEPTH, int WAVES, bool EXACT> void launch(Params &p, hipStream_t s) {
    constexpr int kLds = WAVES * DEPTH * Stage<T, R, MT>::kBytes;
    static_assert(kLds <= 160 * 1024 && kLds >= WAVES * MT * ((R + 15) / 16) * kWave * 16, "fits, and has room for the sums");
    static_assert((DEPTH - 1) * Stage<T, R, MT>::kLoads < 64, "what a wave can wait for");
    const int64_t tiles = (p.n_out + kOuts * MT - 1) / (kOuts * MT), chunks = (p.groups + kChunk - 1) / kChunk;
    p.waves_k = 1;
    while (p.waves_k < WAVES && 2 * p.waves_k <= chunks) p.waves_k *= 2;
    const int64_t each = WAVES / p.waves_k;
    packed_linear_kernel<T, R, MT, DEPTH, EXACT><<<dim3((uint32_t)((tiles + each - 1) / each), (uint32_t)((p.rows + R - 1) / R)), WAVES * kWave, kLds, s>>>(p);
}

template <class T> void launch(Params &p, hipStream_t s) {
    constexpr int kSize = sizeof(T);
    const bool exact = (uintptr_t)p.x % 16 == 0 && (p.rows <= 1 || (p.x_stride % (16 / kSize) == 0 && p.x_stride >= 0 && p.x_stride <= kMostStride / 2)) && p.n_in % (16 / kSize) == 0;
    const int per = (p.n_out + kOuts * kComputeUnits - 1) / (kOuts * kComputeUnits);       // tiles of a workgroup a compute unit
    if (!exact) {
        if (p.rows <= 4) launch<T, 4, 1, 2, 8, false>(p, s);
        else if (p.rows <= 16 && per < 2) launch<T, 16, 1, 2, 4, false>(p, s);
        else if (p.rows <= 16) launch<T, 16, 2, 2, 4, false>(p, s);
        else launch<T, 32, 2, 2, 4, false>(p, s);
        return;
    }
    if (p.rows <= 4) {
        if (per >= 4) {
            if constexpr (kSize == 2) launch<T, 4, 4, 3, 8, true>(p, s);
            else launch<T, 4, 4, 2, 8, true>(p, s);
        }
        else if (per == 3) launch<T, 4, 3, 3, 8, true>(p, s);
        else if (per == 2) launch<T, 4, 2, 4, 8, true>(p, s);
        else launch<T, 4, 1, 4, 8, true>(p, s);
        return;
    }
    if constexpr (kSize == 2) {
        if (p.rows <= 16) {
            if (per >= 4) launch<T, 16, 4, 2, 8, true>(p, s);
            else if (per == 3) launch<T, 16, 3, 2, 8, true>(p, s);
            else if (per == 2) launch<T, 16, 2, 3, 8, true>(p, s);
            else launch<T, 16, 1, 3, 8, true>(p, s);
        } else if (p.rows <= 32) {
            if (per >= 2) launch<T, 32, 2, 3, 4, true>(p, s);
            else launch<T, 32, 1, 3, 4, true>(p, s);
        } else {
            if (per >= 2) launch<T, 64, 2, 2, 4, true>(p, s);
            else launch<T, 64, 1, 2, 4, true>(p, s);
        }
    } else {
        if (p.rows <= 16) {
            if (per >= 2) launch<T, 16, 2, 3, 4, true>(p, s);
            else launch<T, 16, 1, 3, 4, true>(p, s);
        } else {
            if (per >= 2) launch<T, 32, 2, 2, 4, true>(p, s);
            else launch<T, 32, 1, 2, 4, true>(p, s);
        }
    }
}

}  // namespace

extern "C" {

int hp_packed_linear(const hp_packed_linear_args_t *a, void *stream) {
    if (const int rc = check(a)) return rc;
    if (a->rows == 0 || a->n_out == 0) return HP_OK;
    Params p{};
    p.rows = a->rows, p.n_in = a->n_in, p.n_out = a->n_out, p.groups = groups_of(a->n_in);
    p.x = a->x, p.x_stride = a->x_stride, p.w = a->w, p.out = a->out, p.out_stride = a->out_stride;
    const hipStream_t s = (hipStream_t)stream;
    if (a->dtype == HP_BF16) launch<__bf16>(p, s);
    else launch<float>(p, s);
    return hip_failed(hipGetLastError()) ? HP_EHIP : HP_OK;
}

}  // extern "C"
