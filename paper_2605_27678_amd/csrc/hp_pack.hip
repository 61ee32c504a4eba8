// Packing rows into groups of 32 values with codes of 4 bits, and back.
//     low = min, rounded down;  step = (max - low) / 15, rounded up;  code = nearest of low + step * {0 .. 15}, the lower of two
// A lane that packs takes 16 channels, half a group, and one row after the other; one that reads back 8.  (Eight when packing,
// four lanes a group: four times the group's arithmetic for one use.)  Bound by memory, 2 (or 4) bytes and 0.625 a value, and a
// copy of as much takes what this does but for the last twentieth: 40139 rows of 8 heads of 128, k and v, packed and read back,
// 432 MB, 87 us (83 at the rate of a large copy).  Binary32 rows of heads of 72, the last group of 8: 37 us for 124 MB
// (24); 123 MB of whole groups, heads of 128, take 29, so it is the short group that costs (bfloat16 alike: 57 us and 36).
#include <cfloat>
#include <cmath>

#include "hp_packed.hpp"

#pragma clang fp contract(off)

namespace {

using namespace hp;

constexpr int kThreads = 256;
constexpr int64_t kMostBlocks = 1 << 20;           // of rows; more are taken in turns
constexpr int64_t kPackBlocks = 1 << 16;           // of packing: more rows keep their place (40139 rows of 8 heads: 49 us, with 8192 51, with 2048 58)

struct PackParams {
    int64_t rows;
    int32_t dim, words;                            // words of codes a row and head: four a group
    int32_t heads[HP_PACK_MAX_TENSORS], rows_per_block[HP_PACK_MAX_TENSORS];
    hp_heads_t x[HP_PACK_MAX_TENSORS];
    hp_packed_t packed[HP_PACK_MAX_TENSORS];
};

constexpr int kUnit = 16;                           // channels of a lane that packs: two words of codes, half a group
// Where in a word the code of its i-th channel is.
__device__ __forceinline__ constexpr int place_of(int i) { return 4 * (i / 2) + 16 * (i % 2); }

// x of the other lane of a pair.
__device__ __forceinline__ float of_neighbour(float x) { return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0xb1, 0xf, 0xf, true)); }

// The bfloat16 that is next below (or equal), and next above for numbers that are not negative.
__device__ __forceinline__ float down(float x) {
    const uint32_t b = __float_as_uint(x);
    return __uint_as_float((b >> 31 ? b + 0xffffu : b) & 0xffff0000u);
}
__device__ __forceinline__ float up(float x) { return __uint_as_float((__float_as_uint(x) + 0xffffu) & 0xffff0000u); }
__device__ __forceinline__ float up(double x) {
    float f = (float)x;
    if ((double)f < x) f = __uint_as_float(__float_as_uint(f) + 1);
    return up(f);
}

struct Scale {
    float step, low;
    bool plain;                                    // the borders low + (k + 1/2) step are exact in binary32
};

// Where step and low are not too far apart, low + 15 step and the borders between the levels are sums of two numbers of 13
// bits and 8 that binary32 holds exactly, and comparing with them decides as the definition does; elsewhere (a low value
// that is less than 2^-12 of a step but not zero, or more than 2^14 steps) 64 bits do.
__device__ __forceinline__ Scale scale_of(float least, float most) {
    Scale s;
    s.low = down(least);
    const float d = most - s.low, about = d * (1.0f / 15.0f);
    float step = up(about);
    const float lower = __uint_as_float(__float_as_uint(step) - 0x10000u), higher = __uint_as_float(__float_as_uint(step) + 0x10000u);
    s.step = __builtin_fmaf(15.0f, lower, s.low) >= most ? lower : __builtin_fmaf(15.0f, step, s.low) >= most ? step : higher;
    const float size = fabsf(s.low);
    s.plain = d >= 0x1p-100f && d <= 0x1p100f && (size == 0.0f || (size >= 0x1p-12f * s.step && size <= 0x1p14f * s.step));
    if (d == 0.0f) s.step = 0.0f, s.plain = true;
    return s;
}
__device__ __forceinline__ float careful_step(float low, float most) {
    const double each = ((double)most - (double)low) / 15.0;
    return each >= 0x1p-126 ? up(each) : 0.0f;
}

// A code is the level below a value, found roughly, and one more if the value lies beyond the border behind that level.
__device__ __forceinline__ uint32_t code_of(float x, const Scale &s, float inv, float from, float border) {
    const float below = floorf(__builtin_fmaf(x, inv, from));
    return (uint32_t)(int)below + (x > __builtin_fmaf(below, s.step, border) ? 1u : 0u);
}
__device__ __forceinline__ uint32_t careful_code(float x, float low, float step) {
    const double d = (double)x - (double)low, half = 0.5 * (double)step;
    double c = fmin(rint(d / (double)step), 15.0);
    const double v = d - c * (double)step;          // the product is exact
    if (v > half && c < 15.0) c += 1.0;
    else if (v <= -half && c > 0.0) c -= 1.0;
    return (uint32_t)c;
}

// WHOLE: rows are whole groups.
template <class T, bool WHOLE> __global__ __launch_bounds__(kThreads) void pack_kernel(PackParams p) {
    const int t = (int)blockIdx.z, units = p.words / 2, per_row = p.heads[t] * units, rows_per_block = p.rows_per_block[t];
    const int item = (int)(blockIdx.y * kThreads + threadIdx.x);
    const int in_block = rows_per_block > 1 ? item / per_row : 0, at_row = item - in_block * per_row;
    if (in_block >= rows_per_block || at_row >= per_row) return;                 // both lanes of a group alike
    const int head = at_row / units, unit = at_row - head * units, valid = p.dim - kUnit * unit;
    const int64_t first = (int64_t)blockIdx.x * rows_per_block + in_block, step_rows = (int64_t)gridDim.x * rows_per_block;
    const T *from = (const T *)p.x[t].data + (int64_t)head * p.x[t].head_stride + kUnit * unit;
    char *const codes = (char *)p.packed[t].codes + (int64_t)head * p.packed[t].code_head_stride + 8 * unit;
    uint16_t *const scales = (uint16_t *)p.packed[t].scales + (int64_t)head * p.packed[t].scale_head_stride + unit / 2 * 2;
    const auto read = [&](int64_t row, Vec<T, 8> (&v)[2]) {
        const T *src = from + row * p.x[t].row_stride;
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] = WHOLE ? *(const typename VecOf<T, 8>::mem *)(src + 8 * h) : load<8>(src + 8 * h, valid - 8 * h);
    };
    Vec<T, 8> next[2];
    if (first < p.rows) read(first, next);
    for (int64_t row = first; row < p.rows; row += step_rows) {
        float x[kUnit], least = INFINITY, most = -INFINITY, none = 0.0f;
#pragma unroll
        for (int i = 0; i < kUnit; ++i) x[i] = (float)next[i / 8][i % 8];
        if (row + step_rows < p.rows) read(row + step_rows, next);
#pragma unroll
        for (int i = 0; i < kUnit; ++i) {
            none = __builtin_fmaf(x[i], 0.0f, none);                             // NaN if any is infinite or NaN
            least = fminf(least, WHOLE || i < valid ? x[i] : INFINITY);
            most = fmaxf(most, WHOLE || i < valid ? x[i] : -INFINITY);
        }
        if (!(none == 0.0f)) least = -INFINITY;
        least = fminf(least, of_neighbour(least)), most = fmaxf(most, of_neighbour(most));
        Scale s = scale_of(least, most);
        if constexpr (!WHOLE)                                                    // channels that are not there: code 0
#pragma unroll
            for (int i = 0; i < kUnit; ++i) x[i] = i < valid ? x[i] : s.low;
        const bool good = s.low >= -FLT_MAX;
        uint32_t w[2] = {};
        if (__all(s.plain || !good)) {
            const float inv = s.step > 0.0f ? __builtin_amdgcn_rcpf(s.step) : 0.0f, begin = -s.low * inv, border = __builtin_fmaf(0.5f, s.step, s.low);
#pragma unroll
            for (int i = 0; i < kUnit; ++i) w[i / 8] |= code_of(x[i], s, inv, begin, border) << place_of(i % 8);
        } else {
            if (good) s.step = careful_step(s.low, most);
#pragma unroll 1
            for (int i = 0; i < kUnit; ++i) {
                float one = x[0];
#pragma unroll
                for (int j = 1; j < kUnit; ++j) one = i == j ? x[j] : one;
                const uint32_t code = (s.step > 0.0f ? careful_code(one, s.low, s.step) : 0u) << place_of(i % 8);
                w[0] |= i < 8 ? code : 0u, w[1] |= i < 8 ? 0u : code;
            }
        }
        if (!good) s.low = s.step = __uint_as_float(0x7fc00000u), w[0] = w[1] = 0;
        *(Vec<uint32_t, 2> *)(codes + row * p.packed[t].code_row_stride) = Vec<uint32_t, 2>{w[0], w[1]};
        if (unit % 2 == 0) *(uint32_t *)(scales + row * p.packed[t].scale_row_stride) = __float_as_uint(s.step) >> 16 | (__float_as_uint(s.low) & 0xffff0000u);
    }
}

template <class T> __global__ __launch_bounds__(kThreads) void unpack_kernel(PackParams p) {
    const int t = (int)blockIdx.z, per_row = p.heads[t] * p.words, rows_per_block = p.rows_per_block[t];
    const int item = (int)(blockIdx.y * kThreads + threadIdx.x);
    const int in_block = rows_per_block > 1 ? item / per_row : 0, at_row = item - in_block * per_row;
    if (in_block >= rows_per_block || at_row >= per_row) return;
    const int head = at_row / p.words, word = at_row - head * p.words, valid = p.dim - 8 * word;
    const hp_heads_t &to = p.x[t];
    const hp_packed_t &from = p.packed[t];
    for (int64_t row = (int64_t)blockIdx.x * rows_per_block + in_block; row < p.rows; row += (int64_t)gridDim.x * rows_per_block) {
        const uint32_t w = ((const uint32_t *)((const char *)from.codes + row * from.code_row_stride + (int64_t)head * from.code_head_stride))[word];
        const uint32_t pair = ((const uint32_t *)((const uint16_t *)from.scales + row * from.scale_row_stride + (int64_t)head * from.scale_head_stride))[word / 4];
        const float step = step_of(pair), low = low_of(pair);
        Vec<T, 8> v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (T)__builtin_fmaf((float)(w >> place_of(i) & 15u), step, low);
        T *const at = (T *)to.data + row * to.row_stride + (int64_t)head * to.head_stride + 8 * word;
        // past the caches: 40139 rows of 8 heads, packed and read back, 95 -> 87 us
        if (valid >= 8) __builtin_nontemporal_store(v, (typename VecOf<T, 8>::mem *)at);
        else store<8>(at, v, valid);
    }
}

int check(const hp_pack_args_t *a) {
    if (!a) return HP_EINVAL;
    if (a->dtype != HP_BF16 && a->dtype != HP_F32) return HP_EINVAL;
    if (a->n_tensors < 1 || a->n_tensors > HP_PACK_MAX_TENSORS || a->rows < 0) return HP_EINVAL;
    if (a->dim < 1 || a->dim > HP_PACKED_MAX_DIM) return HP_EINVAL;
    const int size = a->dtype == HP_BF16 ? 2 : 4;
    for (int t = 0; t < a->n_tensors; ++t) {
        if (a->heads[t] < 0 || a->heads[t] > 65536) return HP_EINVAL;
        const int64_t rows = a->heads[t] > 0 ? a->rows : 0;
        if (rows > 0 && !a->x[t].data) return HP_EINVAL;
        if ((uintptr_t)a->x[t].data % size) return HP_EALIGN;
        if (const int rc = check_packed(a->packed[t], rows, a->heads[t])) return rc;
    }
    return HP_OK;
}

int run(const hp_pack_args_t *a, bool back, hipStream_t stream) {
    if (const int rc = check(a)) return rc;
    PackParams p{};
    p.rows = a->rows, p.dim = a->dim, p.words = 4 * groups_of(a->dim);
    const int32_t lanes = back ? p.words : p.words / 2;       // of a row and head
    int64_t blocks = 0, lines = 0;
    for (int t = 0; t < a->n_tensors; ++t)
        if ((int64_t)a->heads[t] * p.words > (int64_t)65535 * kThreads) return HP_ELAYOUT;     // blocks of a launch's second axis
    for (int t = 0; t < a->n_tensors; ++t) {
        const int64_t per_row = (int64_t)a->heads[t] * lanes;
        p.heads[t] = a->heads[t], p.x[t] = a->x[t], p.packed[t] = a->packed[t];
        p.rows_per_block[t] = per_row > 0 && per_row < kThreads ? (int32_t)(kThreads / per_row) : 1;
        if (per_row == 0) continue;
        const int64_t b = (a->rows + p.rows_per_block[t] - 1) / p.rows_per_block[t], l = (per_row + kThreads - 1) / kThreads;
        blocks = b > blocks ? b : blocks, lines = l > lines ? l : lines;
    }
    if (blocks == 0) return HP_OK;
    // packing keeps its place over several rows: as many workgroups as run at once, a few times over
    const int64_t all = back ? kMostBlocks : kPackBlocks / (lines * a->n_tensors) + 1;
    const dim3 grid((uint32_t)(blocks < all ? blocks : all), (uint32_t)lines, (uint32_t)a->n_tensors);
    const bool whole = a->dim % kGroup == 0;
    if (a->dtype == HP_BF16) {
        if (back) unpack_kernel<__bf16><<<grid, kThreads, 0, stream>>>(p);
        else if (whole) pack_kernel<__bf16, true><<<grid, kThreads, 0, stream>>>(p);
        else pack_kernel<__bf16, false><<<grid, kThreads, 0, stream>>>(p);
    } else {
        if (back) unpack_kernel<float><<<grid, kThreads, 0, stream>>>(p);
        else if (whole) pack_kernel<float, true><<<grid, kThreads, 0, stream>>>(p);
        else pack_kernel<float, false><<<grid, kThreads, 0, stream>>>(p);
    }
    return hip_failed(hipGetLastError()) ? HP_EHIP : HP_OK;
}

}  // namespace

extern "C" {

int hp_pack(const hp_pack_args_t *a, void *stream) { return run(a, false, (hipStream_t)stream); }
int hp_unpack(const hp_pack_args_t *a, void *stream) { return run(a, true, (hipStream_t)stream); }

}  // extern "C"
