// Rotary positions.  A pair (a, b) of a head's channels is turned by the angle
// that belongs to its row's position:
//     out_a = x_a c - x_b s,   out_b = x_b c + x_a s,
// with (c, s) from a table of binary32 pairs.  The gradient is the same turn
// with -s.  Bound by memory: every value is read and written once, 3 operations
// each; the table's row (8 bytes a pair) is read once a lane and used for
// two heads.  16384 rows of 12 heads of 128 bf16: 19.5 us, 5.6 TB/s; 40139 rows of
// 32 heads of 72 binary32, interleaved, by two axes: 183 us, 4.1 TB/s (a large
// copy: 5.2).
#include <cmath>

#include "hp_device.hpp"
#include "hp_operators.h"

#pragma clang fp contract(fast)

namespace {

using namespace hp;

constexpr int kThreads = 256, kMostThreads = 512;

// Heads that a lane turns with the pairs that it has read from the table.  Four are 2 % faster on large tensors and slower
// on small ones (8 rows of 40 heads: 5.2 us a call, with two 4.0).
constexpr int kHeads = 2;

// Results are written past the caches: 16384 rows of 12 heads of 128 bf16 27.5 -> 19.2 us.
template <int N, class T> __device__ __forceinline__ void leave(T *p, Vec<T, N> v) { __builtin_nontemporal_store(v, (typename VecOf<T, N>::mem *)p); }

struct RotaryParams {
    int64_t rows, table_rows, axis_stride;
    const float *table;
    const int32_t *positions;
    int32_t n_tensors, n_heads;               // of all tensors together
    int32_t dim, half, n_axes, inverse;
    int32_t groups, reserved;                         // of heads that a lane takes one each of
    int32_t units, copies, per_row, rows_per_block;   // lanes of a head, those of them that copy, lanes of a row, and rows of a block
    int32_t axis_end[HP_ROTARY_MAX_AXES];
    int32_t heads[HP_ROTARY_MAX_TENSORS];
    hp_heads_t x[HP_ROTARY_MAX_TENSORS], out[HP_ROTARY_MAX_TENSORS];
};

// One lane: a vector of VEC channels and the one that they turn with, VEC pairs, or VEC interleaved channels, VEC / 2
// pairs, or VEC copied channels; of one row, in kHeads heads.  Consecutive lanes take consecutive vectors, then the next
// heads, so that a wave reads and writes runs of a head or half a head.
template <class T, int VEC, bool INTERLEAVED> __global__ __launch_bounds__(kMostThreads) void rotary_kernel(RotaryParams p) {
    const int item = (int)(blockIdx.y * blockDim.x + threadIdx.x);
    const int in_block = p.rows_per_block > 1 ? item / p.per_row : 0;
    const int at_row = item - in_block * p.per_row;
    if (in_block >= p.rows_per_block || at_row >= p.per_row) return;
    const int group = at_row / p.units, u = at_row - group * p.units;
    constexpr int PAIRS = INTERLEAVED ? VEC / 2 : VEC;
    const int turned = p.units - p.copies;
    const int behind = 2 * p.half + (u - turned) * VEC;                        // a copying lane's first channel
    for (int64_t block = blockIdx.x; block * p.rows_per_block < p.rows; block += gridDim.x) {
        const int64_t row = block * p.rows_per_block + in_block;
        if (row >= p.rows) break;
        // the values first: what the table gives is two loads, one behind the other
        Vec<T, VEC> a[kHeads], b[kHeads];
        T *to[kHeads];
#pragma unroll
        for (int k = 0; k < kHeads; ++k) {
            int h = group + k * p.groups;              // lanes side by side have heads side by side: whole lines
            to[k] = nullptr;
            if (h >= p.n_heads) continue;
            int t = 0;
            while (t < p.n_tensors - 1 && h >= p.heads[t]) h -= p.heads[t++];
            const T *from = (const T *)p.x[t].data + row * p.x[t].row_stride + h * p.x[t].head_stride;
            to[k] = (T *)p.out[t].data + row * p.out[t].row_stride + h * p.out[t].head_stride;
            if (u >= turned) {
                a[k] = load<VEC>(from + behind, p.dim - behind);
            } else {
                a[k] = load<VEC>(from + u * VEC, VEC);
                if constexpr (!INTERLEAVED) b[k] = load<VEC>(from + p.half + u * VEC, VEC);
            }
        }
        float c[PAIRS], s[PAIRS];
        if (u < turned) {
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) c[j] = s[j] = __builtin_nanf("");
            const auto axis_of = [&](int i) {
                int axis = 0;
                for (int a = 0; a < HP_ROTARY_MAX_AXES - 1; ++a) axis += a < p.n_axes - 1 && i >= p.axis_end[a];
                return axis;
            };
            const int axis0 = axis_of(u * PAIRS);
            if (PAIRS == 1 || axis_of(u * PAIRS + PAIRS - 1) == axis0) {       // all but the few lanes at an axis's border
                const int64_t pos = p.positions[axis0 * p.axis_stride + row];
                if (pos >= 0 && pos < p.table_rows) {
                    const Vec<float, 2 * PAIRS> t = load<2 * PAIRS>(p.table + (pos * p.half + u * PAIRS) * 2, 2 * PAIRS);
#pragma unroll
                    for (int j = 0; j < PAIRS; ++j) c[j] = t[2 * j], s[j] = t[2 * j + 1];
                }
            } else {
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) {
                    const int i = u * PAIRS + j;
                    const int64_t pos = p.positions[axis_of(i) * p.axis_stride + row];
                    if (pos >= 0 && pos < p.table_rows) {
                        const Vec<float, 2> t = load<2>(p.table + (pos * p.half + i) * 2, 2);
                        c[j] = t[0], s[j] = t[1];
                    }
                }
            }
            if (p.inverse)
#pragma unroll
                for (int j = 0; j < PAIRS; ++j) s[j] = -s[j];
        }
#pragma unroll
        for (int k = 0; k < kHeads; ++k) {
            if (!to[k]) continue;
            if (u >= turned) {
                store<VEC>(to[k] + behind, a[k], p.dim - behind);
                continue;
            }
            Vec<T, VEC> ra, rb;
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) {
                const float xa = at<VEC, T>(a[k], INTERLEAVED ? 2 * j : j), xb = INTERLEAVED ? at<VEC, T>(a[k], 2 * j + 1) : at<VEC, T>(b[k], j);
                const float ya = xa * c[j] - xb * s[j], yb = xb * c[j] + xa * s[j];
                put<VEC, T>(ra, INTERLEAVED ? 2 * j : j, ya);
                if constexpr (INTERLEAVED) put<VEC, T>(ra, 2 * j + 1, yb);
                else put<VEC, T>(rb, j, yb);
            }
            leave<VEC>(to[k] + u * VEC, ra);
            if constexpr (!INTERLEAVED) leave<VEC>(to[k] + p.half + u * VEC, rb);
        }
    }
}

template <class T, int VEC, bool INTERLEAVED> void launch(RotaryParams &p, bool copies, hipStream_t stream) {
    p.copies = copies ? (p.dim - 2 * p.half + VEC - 1) / VEC : 0;
    p.units = (INTERLEAVED ? 2 * p.half : p.half) / VEC + p.copies;
    p.groups = (p.n_heads + kHeads - 1) / kHeads;
    p.per_row = p.units * p.groups;
    // as many rows as make about 256 lanes, or one row in lanes up to 512, or that in parts
    p.rows_per_block = p.per_row >= kThreads ? 1 : kThreads / p.per_row;
    const int lanes = p.rows_per_block * p.per_row, parts = (lanes + kMostThreads - 1) / kMostThreads;
    const int threads = ((lanes + parts - 1) / parts + kWave - 1) / kWave * kWave;
    const int64_t blocks = (p.rows + p.rows_per_block - 1) / p.rows_per_block;
    const dim3 grid((uint32_t)(blocks < (1 << 22) ? blocks : (1 << 22)), (uint32_t)parts);
    rotary_kernel<T, VEC, INTERLEAVED><<<grid, threads, 0, stream>>>(p);
}

// The widest lanes that divide the channels they turn, 16 bytes at most.
template <class T> void launch(RotaryParams &p, bool interleaved, bool copies, hipStream_t stream) {
    const int run = interleaved ? 2 * p.half : p.half;
    if constexpr (sizeof(T) == 2)
        if (run % 8 == 0) return interleaved ? launch<T, 8, true>(p, copies, stream) : launch<T, 8, false>(p, copies, stream);
    if (run % 4 == 0) return interleaved ? launch<T, 4, true>(p, copies, stream) : launch<T, 4, false>(p, copies, stream);
    if (run % 2 == 0) return interleaved ? launch<T, 2, true>(p, copies, stream) : launch<T, 2, false>(p, copies, stream);
    launch<T, 1, false>(p, copies, stream);            // an odd half: interleaved runs are even
}

struct TableParams {
    float *table;
    int64_t n, first;
    int32_t half, kind;
    double log_base, factor, original, low, high, amplitude;
};

__global__ __launch_bounds__(kThreads) void table_kernel(TableParams t) {
    const int64_t total = t.n * t.half;
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < total; e += (int64_t)gridDim.x * kThreads) {
        const int64_t p = e / t.half;
        const int i = (int)(e - p * t.half);
        double f = exp(-t.log_base * i / t.half);
        if (t.kind == HP_ROTARY_LINEAR) {
            f /= t.factor;
        } else if (t.kind == HP_ROTARY_BY_TURNS) {
            const double turns = t.original * f / 6.283185307179586476925;
            double keep = (turns - t.low) / (t.high - t.low);
            keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
            f = f * keep + f / t.factor * (1 - keep);
        }
        double s, c;
        sincos((double)(t.first + p) * f, &s, &c);
        t.table[2 * e] = (float)(t.amplitude * c);
        t.table[2 * e + 1] = (float)(t.amplitude * s);
    }
}

bool misaligned(const void *p, int to) { return (uintptr_t)p % to != 0; }

}  // namespace

extern "C" {

int hp_rotary_table(float *table, int64_t n, int64_t first, int32_t rot, const hp_rotary_scaling_t *scaling,
                    void *stream) {
    if (!scaling || n < 0 || first < 0 || rot < 2 || rot % 2 || (n > 0 && !table)) return HP_EINVAL;
    if (n > ((int64_t)1 << 40) / rot || first > ((int64_t)1 << 40)) return HP_EINVAL;
    const hp_rotary_scaling_t &s = *scaling;
    if (s.kind < HP_ROTARY_PLAIN || s.kind > HP_ROTARY_BY_TURNS) return HP_EINVAL;
    if (!(s.base > 0) || !std::isfinite(s.base) || !std::isfinite(s.amplitude)) return HP_EINVAL;
    if (s.kind != HP_ROTARY_PLAIN && (!(s.factor > 0) || !std::isfinite(s.factor))) return HP_EINVAL;
    if (s.kind == HP_ROTARY_BASE && rot < 4) return HP_EINVAL;
    if (s.kind == HP_ROTARY_BY_TURNS && (!(s.original_length > 0) || !std::isfinite(s.original_length) || !(s.low_turns < s.high_turns) ||
                                         !std::isfinite(s.high_turns - s.low_turns)))
        return HP_EINVAL;
    if (misaligned(table, 4)) return HP_EALIGN;
    if (n == 0) return HP_OK;
    TableParams t{table, n, first, rot / 2, s.kind, std::log(s.base), s.factor, s.original_length, s.low_turns, s.high_turns, s.amplitude};
    if (s.kind == HP_ROTARY_BASE) t.log_base += std::log(s.factor) * rot / (rot - 2);
    const int64_t blocks = (n * t.half + kThreads - 1) / kThreads;
    table_kernel<<<(uint32_t)(blocks < 65536 ? blocks : 65536), kThreads, 0, (hipStream_t)stream>>>(t);
    return hip_failed(hipGetLastError()) ? HP_EHIP : HP_OK;
}

int hp_rotary(const hp_rotary_args_t *a, void *stream) {
    if (!a) return HP_EINVAL;
    if (a->dtype != HP_BF16 && a->dtype != HP_F32) return HP_EINVAL;
    if (a->n_tensors < 1 || a->n_tensors > HP_ROTARY_MAX_TENSORS || a->rows < 0 || a->table_rows < 1) return HP_EINVAL;
    if (a->dim < 2 || a->dim > 1024 || a->rot < 2 || a->rot % 2 || a->rot > a->dim) return HP_EINVAL;
    if (a->n_axes < 1 || a->n_axes > HP_ROTARY_MAX_AXES) return HP_EINVAL;
    RotaryParams p{};
    p.half = a->rot / 2;
    if (a->n_axes > 1) {
        int64_t sum = 0;
        for (int i = 0; i < a->n_axes; ++i) {
            if (a->sections[i] < 0) return HP_EINVAL;
            sum += a->sections[i];
            if (sum > p.half) return HP_EINVAL;
            p.axis_end[i] = (int32_t)sum;
        }
        if (sum != p.half) return HP_EINVAL;
    }
    const int size = a->dtype == HP_BF16 ? 2 : 4;
    bool in_place = true;
    int64_t n_heads = 0;
    for (int t = 0; t < a->n_tensors; ++t) {
        if (a->heads[t] < 0 || a->heads[t] > 4096) return HP_EINVAL;
        if (a->rows > 0 && a->heads[t] > 0 && (!a->x[t].data || !a->out[t].data)) return HP_EINVAL;
        if (misaligned(a->x[t].data, size) || misaligned(a->out[t].data, size)) return HP_EALIGN;
        // strides that no address goes by do not count: empty tensors, single rows and single heads
        const bool same = a->x[t].data == a->out[t].data, some = a->rows > 0 && a->heads[t] > 0;
        if (same && some && ((a->rows > 1 && a->x[t].row_stride != a->out[t].row_stride) ||
                             (a->heads[t] > 1 && a->x[t].head_stride != a->out[t].head_stride)))
            return HP_EINVAL;
        in_place = in_place && same;
        n_heads += a->heads[t];
        p.heads[t] = a->heads[t];
        p.x[t] = a->x[t];
        p.out[t] = a->out[t];
    }
    if (a->rows > 0 && n_heads > 0 && (!a->table || !a->positions)) return HP_EINVAL;
    if (misaligned(a->table, 4) || misaligned(a->positions, 4)) return HP_EALIGN;
    if (a->rows == 0 || n_heads == 0) return HP_OK;
    p.rows = a->rows;
    p.table_rows = a->table_rows;
    p.axis_stride = a->axis_stride;
    p.table = a->table;
    p.positions = a->positions;
    p.n_tensors = a->n_tensors;
    p.n_heads = (int32_t)n_heads;
    p.dim = a->dim;
    p.n_axes = a->n_axes;
    p.inverse = a->inverse != 0;
    const bool copies = !in_place && a->dim > a->rot;
    if (a->dtype == HP_BF16) launch<__bf16>(p, a->interleaved != 0, copies, (hipStream_t)stream);
    else launch<float>(p, a->interleaved != 0, copies, (hipStream_t)stream);
    return hip_failed(hipGetLastError()) ? HP_EHIP : HP_OK;
}

}  // extern "C"
