// A few rows times a matrix held in 4 bits: out[r][n] = sum_k x[r][k] w[n][k], with a group's value = low + step * code
//     = sum_g (step_ng sum_k x_rk code_nk + low_ng sum_k x_rk)            (k in group g)
// The rows of x are the left operand of products of 16 x 16 x 32, a group of 16 rows of w at a time the right one, so that a
// lane has results of one row of w, whose step and low are its own.  sum x is such a product too, with one number for every
// code: less their lift.  In bfloat16 it takes the lift off and, times -low / lift, puts the lows in; in binary32 codes are
// less 8 and not lifted, and it puts low + 8 step in.
// The waves of a workgroup share out the inner axis, 128 of it at a time, and add up at the end in their order.
#include <climits>
#include <cmath>

#include "hp_packed.hpp"

#pragma clang fp contract(fast)

namespace {

using namespace hp;

constexpr int kWaves = 8, kBlock = kWaves * kWave;
constexpr int kOuts = 16;                          // rows of w of a wave
constexpr int kChunk = 4;                          // groups at a time

struct Params {
    int64_t rows;
    int32_t n_in, n_out, groups, waves_k;          // waves_k: that share a tile's inner axis, a power of two
    const void *x;
    int64_t x_stride;
    hp_packed_t w;
    void *out;
    int64_t out_stride;
};

// What a wave reads of 16 rows of w and 16 NT rows of x for a chunk.
template <class T, int NT> struct Chunk {
    Words codes, pairs;
    Vec<T, 8> x[kChunk][NT];
};

template <class T, int NT> __global__ __launch_bounds__(kBlock) void packed_linear_kernel(Params p) {
    constexpr int N = kTerms<T>;
    __shared__ Quad shared[kWaves][NT][kWave];
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), col = lane % 16, quarter = lane / 16;
    const int turn = wave & (p.waves_k - 1), tiles = kWaves / p.waves_k;
    const int n0 = ((int)blockIdx.x * tiles + wave / p.waves_k) * kOuts;
    const int64_t r0 = (int64_t)blockIdx.y * (16 * NT);
    const int chunks = n0 < p.n_out ? (p.groups + kChunk - 1) / kChunk : 0;
    const auto codes = buffer_at((const char *)p.w.codes + n0 * p.w.code_row_stride);
    const auto pairs = buffer_at((const uint16_t *)p.w.scales + n0 * p.w.scale_row_stride);
    const bool there = n0 + col < p.n_out;
    const uint32_t code_at = (uint32_t)(col * (int)p.w.code_row_stride) + quarter * kGroupBytes, pair_at = (uint32_t)(col * (int)p.w.scale_row_stride * 2);
    const T *x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int64_t r = r0 + 16 * t + col;
        x[t] = (const T *)p.x + (r < p.rows ? r : p.rows - 1) * p.x_stride + 8 * quarter;
    }
    const auto fetch = [&](int c) {
        Chunk<T, NT> f;
        const int g0 = c * kChunk;
        const bool whole = (g0 + kChunk) * kGroup <= p.n_in;
        const uint32_t at = there && g0 + quarter < p.groups ? code_at + g0 * kGroupBytes : kOutside;
        f.codes = __builtin_bit_cast(Words, __builtin_amdgcn_raw_buffer_load_b128(codes, (int)at, 0, 0));
        if (whole) {
            f.pairs = __builtin_bit_cast(Words, __builtin_amdgcn_raw_buffer_load_b128(pairs, (int)(there ? pair_at + 4 * g0 : kOutside), 0, 0));
#pragma unroll
            for (int j = 0; j < kChunk; ++j)
#pragma unroll
                for (int t = 0; t < NT; ++t) f.x[j][t] = load<8>(x[t] + (g0 + j) * kGroup, 8);
        } else {
#pragma unroll
            for (int j = 0; j < kChunk; ++j) {
                f.pairs[j] = __builtin_amdgcn_raw_buffer_load_b32(pairs, (int)(there && g0 + j < p.groups ? pair_at + 4 * (g0 + j) : kOutside), 0, 0);
#pragma unroll
                for (int t = 0; t < NT; ++t) f.x[j][t] = load<8>(x[t] + (g0 + j) * kGroup, p.n_in - (g0 + j) * kGroup - 8 * quarter);
            }
        }
        return f;
    };
    Quad acc[NT] = {};
    constexpr float kLift = Codes<T>::kLift;
    const Frag lift = all_of(-kLift);
    const Codes<T> codes_of;
    Chunk<T, NT> next;
    if (turn < chunks) next = fetch(turn);
    for (int c = turn; c < chunks; c += p.waves_k) {
        const Chunk<T, NT> f = next;
        if (c + p.waves_k < chunks) next = fetch(c + p.waves_k);
        Words w = f.codes;
        across_quarters(w);
#pragma unroll
        for (int j = 0; j < kChunk; ++j) {
            const Frag l = codes_of(w[j]);
            const float step = step_of(f.pairs[j]), low = low_of(f.pairs[j]) * (-1.0f / kLift) + (kLift < 0.0f ? step : 0.0f);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                Frag a[N];
                terms<T>(f.x[j][t], a);
                Quad sum = {};
#pragma unroll
                for (int n = 0; n < N; ++n) sum = mma(a[n], lift, sum);
                Quad d = kLift < 0.0f ? Quad{} : sum;
#pragma unroll
                for (int n = 0; n < N; ++n) d = mma(a[n], l, d);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][i] += step * d[i] + low * sum[i];
            }
        }
    }
    if (p.waves_k > 1) {
        if (turn)
#pragma unroll
            for (int t = 0; t < NT; ++t) shared[wave][t][lane] = acc[t];
        __syncthreads();
        if (turn) return;
        for (int w = 1; w < p.waves_k; ++w)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] += shared[wave + w][t][lane];
    }
    if (!there) return;
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = r0 + 16 * t + 4 * quarter + i;
            if (r < p.rows) ((T *)p.out)[r * p.out_stride + n0 + col] = (T)acc[t][i];
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

template <class T, int NT> void launch(Params &p, hipStream_t s) {
    const int64_t tiles = (p.n_out + kOuts - 1) / kOuts, chunks = (p.groups + kChunk - 1) / kChunk;
    p.waves_k = 1;
    while (p.waves_k < kWaves && 2 * p.waves_k <= chunks) p.waves_k *= 2;
    const int64_t each = kWaves / p.waves_k;
    packed_linear_kernel<T, NT><<<dim3((uint32_t)((tiles + each - 1) / each), (uint32_t)((p.rows + 16 * NT - 1) / (16 * NT))), kBlock, 0, s>>>(p);
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
    if (a->dtype == HP_BF16) {
        if (a->rows <= 16) launch<__bf16, 1>(p, s);
        else if (a->rows <= 32) launch<__bf16, 2>(p, s);
        else launch<__bf16, 4>(p, s);
    } else {
        if (a->rows <= 16) launch<float, 1>(p, s);
        else launch<float, 2>(p, s);
    }
    return hip_failed(hipGetLastError()) ? HP_EHIP : HP_OK;
}

}  // extern "C"
