// Norms around a block, fused with the block's gate and the residual stream:
//     n = y w1 r1,  r1 = 1 / sqrt(mean y^2 + eps);   h = a x + t n;   z = h w2 r2,  r2 = 1 / sqrt(mean h^2 + eps)
// and, with D the whole gradient of h,
//     D  = dh + r2 dz w2 - h r2^3 mean(h dz w2);        dx = a D
//     dy = r1 e - y r1^3 mean(y e),  e = D t w1
//     A  = sum over rows of D y r1:  dw1 = t A,  dt = w1 A;     dw2 = sum over rows of dz h r2.
// Bound by memory: forward reads x and y and writes h and z, backward reads dh,
// dz, x and y and writes dx and dy, each once.  A row stays in the registers of
// one group of waves between its loads and its stores, weights stay there for
// all rows of a workgroup, and so do the sums over rows (A alone serves w1 and
// the gate), which leave as one line for each group of waves and are added up in
// a fixed order by a second kernel.  16384 rows of 8192 bf16 forward and back:
// 500 us, 5.4 TB/s (a large copy: 5.2); 4099 rows of 2305 binary32: 91 us.
#include <cmath>

#include "hp_device.hpp"
#include "hp_operators.h"

#pragma clang fp contract(fast)

namespace {

using namespace hp;

// Rows go past the caches: 16384 rows of 8192 bf16 forward and back 512 -> 502 us, 4099 of 2305 binary32 96 -> 91.
template <int N, class T> __device__ __forceinline__ void stream_out(T *p, Vec<T, N> v, int valid) {
    if (valid >= N) __builtin_nontemporal_store(v, (typename VecOf<T, N>::mem *)p);
    else store<N>(p, v, valid);
}

struct Norm {
    int64_t rows;
    int32_t hidden, gate_size, gate_tanh, unit_offset;
    float scale, eps;
    const void *x, *y;
    void *h, *z;
    int64_t xs, ys, hs, zs;
    const void *w1, *gate, *w2;
    float *rstd;
    const void *dh, *dz;
    void *dx, *dy;
    int64_t dhs, dzs, dxs, dys;
    float *partial;            // [groups][2][hidden]: A, dw2
};

// Rows that a workgroup holds at a time: WAVES waves hold one, CHUNKS vectors of 16 bytes a lane.
template <int WAVES> constexpr int kGroups = WAVES == 1 ? 4 : 1;

// The sums of N values over the waves that share a row.  Wave sums pass through `slots`, of which a call takes one of
// two sets in turn: a wave may be one call ahead of another, not two, for each call has a barrier in it.
template <int WAVES, int N> struct RowSum {
    float (*slots)[N][16];
    int turn = 0;
    __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
        if constexpr (WAVES > 1) {
            const int wave = (int)threadIdx.x / kWave, lane = (int)threadIdx.x % kWave;
            if (lane == 0)
#pragma unroll
                for (int i = 0; i < N; ++i) slots[turn][i][wave] = v[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float s = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) s += slots[turn][i][w];
                v[i] = s;
            }
            turn ^= 1;
        }
    }
};

// t w1 and w2 of a lane's channels
template <class T, int VEC, int CHUNKS, int STEP>
__device__ __forceinline__ void coefficients(const Norm &p, int lane, float (&tw)[CHUNKS][VEC], float (&w2)[CHUNKS][VEC]) {
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int e = (c * STEP + lane) * VEC, left = p.hidden - e;
        const Vec<T, VEC> one = load<VEC>((const T *)p.w1 + e, p.w1 ? left : 0), two = load<VEC>((const T *)p.w2 + e, p.w2 ? left : 0);
        const Vec<T, VEC> gate = load<VEC>((const T *)p.gate + e, p.gate && p.gate_size > 1 ? left : 0);
        const float g1 = p.gate && p.gate_size == 1 ? (float)*(const T *)p.gate : 1.0f;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            float t = p.gate && p.gate_size > 1 ? at<VEC, T>(gate, j) : g1;
            if (p.gate_tanh && p.gate) t = tanhf(t);
            const float off = p.unit_offset ? 1.0f : 0.0f;
            tw[c][j] = j < left ? t * (p.w1 ? at<VEC, T>(one, j) + off : 1.0f) : 0.0f;
            w2[c][j] = j < left ? at<VEC, T>(two, j) + off : 0.0f;
        }
    }
}

template <class T, int WAVES, int CHUNKS>
__global__ __launch_bounds__(WAVES * kGroups<WAVES> * kWave) void norm_forward_kernel(Norm p) {
    constexpr int VEC = 16 / sizeof(T), STEP = WAVES * kWave;
    __shared__ float slots[2][1][16];
    RowSum<WAVES, 1> sum{slots};
    const int group = (int)threadIdx.x / STEP, lane = (int)threadIdx.x % STEP;
    float tw[CHUNKS][VEC], w2[CHUNKS][VEC];
    coefficients<T, VEC, CHUNKS, STEP>(p, lane, tw, w2);
    const float inv = 1.0f / (float)p.hidden;
    const int64_t stride = (int64_t)gridDim.x * kGroups<WAVES>;
    Vec<T, VEC> x[CHUNKS], y[CHUNKS];
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int e = (c * STEP + lane) * VEC, left = p.hidden - e;
            x[c] = load<VEC>((const T *)p.x + row * p.xs + e, left);
            y[c] = load<VEC>((const T *)p.y + row * p.ys + e, p.y ? left : 0);
        }
    };
    int64_t row = (int64_t)blockIdx.x * kGroups<WAVES> + group;
    if (row < p.rows) fetch(row);
    for (; row < p.rows; row += stride) {      // waves that share rows take the same turns: the barriers meet
        float h[CHUNKS][VEC], v[1] = {0.0f}, yf[CHUNKS][VEC];
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                h[c][j] = p.scale * at<VEC, T>(x[c], j);
                yf[c][j] = at<VEC, T>(y[c], j);
                v[0] += yf[c][j] * yf[c][j];
            }
        if (row + stride < p.rows) fetch(row + stride);
        float r1 = 1.0f, r2 = 1.0f;
        if (p.w1) {
            sum(v);
            r1 = 1.0f / sqrtf(v[0] * inv + p.eps);
        }
        v[0] = 0.0f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                h[c][j] += yf[c][j] * r1 * tw[c][j];
                v[0] += h[c][j] * h[c][j];
            }
        if (p.w2) {
            sum(v);
            r2 = 1.0f / sqrtf(v[0] * inv + p.eps);
        }
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int e = (c * STEP + lane) * VEC, left = p.hidden - e;
            Vec<T, VEC> oh, oz;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                put<VEC, T>(oh, j, h[c][j]);
                put<VEC, T>(oz, j, h[c][j] * r2 * w2[c][j]);
            }
            if (p.h) stream_out<VEC>((T *)p.h + row * p.hs + e, oh, left);
            if (p.z) stream_out<VEC>((T *)p.z + row * p.zs + e, oz, left);
        }
        if (p.rstd && lane == 0) {
            p.rstd[row] = r1;
            p.rstd[p.rows + row] = r2;
        }
    }
}

template <class T, int WAVES, int CHUNKS>
__global__ __launch_bounds__(WAVES * kGroups<WAVES> * kWave) void norm_backward_kernel(Norm p) {
    constexpr int VEC = 16 / sizeof(T), STEP = WAVES * kWave;
    __shared__ float slots[2][3][16];
    RowSum<WAVES, 3> sum{slots};
    const int group = (int)threadIdx.x / STEP, lane = (int)threadIdx.x % STEP;
    float tw[CHUNKS][VEC], w2[CHUNKS][VEC], sum_a[CHUNKS][VEC] = {}, sum_w[CHUNKS][VEC] = {};
    coefficients<T, VEC, CHUNKS, STEP>(p, lane, tw, w2);
    const float inv = 1.0f / (float)p.hidden;
    const int64_t stride = (int64_t)gridDim.x * kGroups<WAVES>;
    Vec<T, VEC> x[CHUNKS], y[CHUNKS], dh[CHUNKS], dz[CHUNKS];
    float next_r1 = 1.0f, next_r2 = 1.0f;
    auto fetch = [&](int64_t row) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int e = (c * STEP + lane) * VEC, left = p.hidden - e;
            x[c] = load<VEC>((const T *)p.x + row * p.xs + e, left);
            y[c] = load<VEC>((const T *)p.y + row * p.ys + e, p.y ? left : 0);
            dh[c] = load<VEC>((const T *)p.dh + row * p.dhs + e, p.dh ? left : 0);
            dz[c] = load<VEC>((const T *)p.dz + row * p.dzs + e, p.dz ? left : 0);
        }
        next_r1 = p.rstd[row];
        next_r2 = p.rstd[p.rows + row];
    };
    const int64_t first = (int64_t)blockIdx.x * kGroups<WAVES> + group;
    if (first < p.rows) fetch(first);
    for (int64_t row = first; row < p.rows; row += stride) {
        const float r1 = next_r1, r2 = next_r2;
        float h[CHUNKS][VEC], d[CHUNKS][VEC], yr[CHUNKS][VEC], v[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float g = at<VEC, T>(dz[c], j) * r2, q = g * w2[c][j];
                yr[c][j] = at<VEC, T>(y[c], j) * r1;
                h[c][j] = p.scale * at<VEC, T>(x[c], j) + yr[c][j] * tw[c][j];
                sum_w[c][j] += g * h[c][j];
                d[c][j] = at<VEC, T>(dh[c], j) + q;
                v[0] += h[c][j] * q;                      // r2 * sum h dz w2
                v[1] += yr[c][j] * tw[c][j] * d[c][j];    // sum of y r1 t w1 D without D's last term ..
                v[2] += yr[c][j] * tw[c][j] * h[c][j];    // .. and what that term multiplies
            }
        if (row + stride < p.rows) fetch(row + stride);
        sum(v);
        const float k2 = p.w2 ? r2 * r2 * v[0] * inv : 0.0f;
        const float k1 = p.w1 ? (v[1] - k2 * v[2]) * inv : 0.0f;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            const int e = (c * STEP + lane) * VEC, left = p.hidden - e;
            Vec<T, VEC> ox, oy;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float whole = d[c][j] - h[c][j] * k2;
                sum_a[c][j] += whole * yr[c][j];
                put<VEC, T>(ox, j, p.scale * whole);
                put<VEC, T>(oy, j, r1 * (tw[c][j] * whole - yr[c][j] * k1));
            }
            if (p.dx) stream_out<VEC>((T *)p.dx + row * p.dxs + e, ox, left);
            if (p.dy) stream_out<VEC>((T *)p.dy + row * p.dys + e, oy, left);
        }
    }
    if (!p.partial) return;
    float *line = p.partial + first * 2 * p.hidden;        // every group leaves a line, of zeros where it had no row
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int e = (c * STEP + lane) * VEC, left = p.hidden - e;
        Vec<float, VEC> a, w;
#pragma unroll
        for (int j = 0; j < VEC; ++j) a[j] = sum_a[c][j], w[j] = sum_w[c][j];
        store<VEC>(line + e, a, left);
        store<VEC>(line + p.hidden + e, w, left);
    }
}

struct Finish {
    const float *partial;
    int32_t lines, hidden, gate_size, gate_tanh, unit_offset;
    const void *w1, *gate;
    void *dw1, *dgate, *dw2;
    float *sums;                // hidden values of A for the one gate of all channels, or NULL
};

constexpr int kColumns = 32, kLines = 32;                  // of a finishing workgroup

// Adds the lines up: a workgroup takes 32 columns, each of its 32 rows of lanes every 32nd line, in ascending order.
template <class T> __global__ __launch_bounds__(kColumns * kLines) void norm_finish_kernel(Finish f) {
    __shared__ float part[2][kLines][kColumns];
    const int c = (int)threadIdx.x % kColumns, l = (int)threadIdx.x / kColumns, col = (int)blockIdx.x * kColumns + c;
    float a = 0.0f, w = 0.0f;
    if (col < f.hidden)
        for (int i = l; i < f.lines; i += kLines) {
            a += f.partial[(int64_t)i * 2 * f.hidden + col];
            w += f.partial[((int64_t)i * 2 + 1) * f.hidden + col];
        }
    part[0][l][c] = a;
    part[1][l][c] = w;
    __syncthreads();
    if (l || col >= f.hidden) return;
    for (int i = 1; i < kLines; ++i) {
        a += part[0][i][c];
        w += part[1][i][c];
    }
    float t = 1.0f, slope = 1.0f;
    if (f.gate) {
        t = (float)((const T *)f.gate)[f.gate_size > 1 ? col : 0];
        if (f.gate_tanh) {
            // 1 - tanh^2 without the difference, which has no bits left from gates of 9 on: 4 e / (1 + e)^2, e = exp(-2 |gate|)
            const float e = expf(-2.0f * fabsf(t));
            slope = 4.0f * e / ((1.0f + e) * (1.0f + e));
            t = tanhf(t);
        }
    }
    const float w1 = f.w1 ? (float)((const T *)f.w1)[col] + (f.unit_offset ? 1.0f : 0.0f) : 1.0f;
    if (f.dw1) ((T *)f.dw1)[col] = (T)(t * a);
    if (f.dw2) ((T *)f.dw2)[col] = (T)w;
    if (f.sums) f.sums[col] = w1 * a * slope;
    else if (f.dgate) ((T *)f.dgate)[col] = (T)(w1 * a * slope);
}

// The one gate's gradient: the sum over the channels.
template <class T> __global__ __launch_bounds__(1024) void norm_gate_kernel(const float *sums, int32_t hidden, void *dgate) {
    __shared__ float part[16];
    float s = 0.0f;
    for (int i = (int)threadIdx.x; i < hidden; i += 1024) s += sums[i];
    s = wave_sum(s);
    if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = s;
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 1; i < 16; ++i) s += part[i];
    *(T *)dgate = (T)s;
}

// How many waves hold a row: as few as keep it within two or three vectors a lane, so that weights, sums and the next row's
// values stay in registers too.  That holds for rows of up to 1024 vectors backward in bf16 (8192 channels) and 1536 in binary32
// (6144); wider ones go through scratch memory for every row: 8192 rows of 12288 bf16 forward and back 800 us (a copy of as
// many bytes: 390; forward alone 151), of 16384 bf16 1440 (519), of 8192 binary32 640 (519).  Forward does so from 2049 vectors
// on in bf16 and 4097 in binary32 (both 16385 channels).
struct Shape {
    int waves, chunks;
};
Shape shape_of(int hidden, int vec) {
    const int lanes = (hidden + vec - 1) / vec;            // that one vector each would take
    for (const Shape s : {Shape{1, 1}, Shape{1, 2}, Shape{4, 1}, Shape{4, 2}, Shape{4, 3}, Shape{8, 2}, Shape{8, 3}, Shape{16, 2}, Shape{16, 4}})
        if (lanes <= s.waves * kWave * s.chunks) return s;
    return {16, 8};
}

// Workgroups of a launch: about what the compute units hold at a time, each with rows of its own.
int64_t blocks_of(int64_t rows, const Shape &s, bool backward) {
    const int64_t per_block = s.waves == 1 ? 4 : 1;
    const int64_t blocks = (rows + per_block - 1) / per_block;
    const int64_t most = kComputeUnits * (s.waves == 16 ? 1 : s.waves == 8 ? (backward ? 1 : 2) : (backward ? 2 : 4));
    return blocks < most ? blocks : most;
}

template <class T, int W, int C> void launch(const Norm &p, bool backward, int64_t blocks, hipStream_t stream) {
    const dim3 block(W * kGroups<W> * kWave);
    if (backward) norm_backward_kernel<T, W, C><<<(uint32_t)blocks, block, 0, stream>>>(p);
    else norm_forward_kernel<T, W, C><<<(uint32_t)blocks, block, 0, stream>>>(p);
}

template <class T> void launch(const Norm &p, const Shape &s, bool backward, int64_t blocks, hipStream_t stream) {
    if (s.waves == 1) {
        if (s.chunks == 1) launch<T, 1, 1>(p, backward, blocks, stream);
        else launch<T, 1, 2>(p, backward, blocks, stream);
    } else if (s.waves == 4) {
        if (s.chunks == 1) launch<T, 4, 1>(p, backward, blocks, stream);
        else if (s.chunks == 2) launch<T, 4, 2>(p, backward, blocks, stream);
        else launch<T, 4, 3>(p, backward, blocks, stream);
    } else if (s.waves == 8) {
        if (s.chunks == 2) launch<T, 8, 2>(p, backward, blocks, stream);
        else launch<T, 8, 3>(p, backward, blocks, stream);
    } else {
        if (s.chunks == 2) launch<T, 16, 2>(p, backward, blocks, stream);
        else if (s.chunks == 4) launch<T, 16, 4>(p, backward, blocks, stream);
        else if constexpr (sizeof(T) == 4) launch<T, 16, 8>(p, backward, blocks, stream);   // 32768 values of 4 bytes
    }
}

bool misaligned(const void *p, int to) { return (uintptr_t)p % to != 0; }

// Whether rows written in the place of others that are read lie elsewhere than these: a row would be overwritten before
// another group of waves has read it.
bool crosses(const Norm &p, const void *from, int64_t from_stride, const void *to, int64_t to_stride) {
    return to && from == to && from_stride != to_stride && p.rows > 1;
}

// Checks what both calls read and fills in the kernels' struct.
int take(const hp_norm_args_t *a, Norm *p) {
    if (!a) return HP_EINVAL;
    if (a->dtype != HP_BF16 && a->dtype != HP_F32) return HP_EINVAL;
    if (a->rows < 0 || a->hidden < 1 || a->hidden > HP_NORM_MAX_HIDDEN) return HP_EINVAL;
    if (!std::isfinite(a->residual_scale) || !(a->eps >= 0) || !std::isfinite(a->eps)) return HP_EINVAL;
    if (a->gate && a->gate_size != 1 && a->gate_size != a->hidden) return HP_EINVAL;
    if (!a->y && (a->w_post || a->gate)) return HP_EINVAL;
    if (a->rows > 0 && !a->x) return HP_EINVAL;
    const int size = a->dtype == HP_BF16 ? 2 : 4;
    for (const void *q : {a->x, a->y, a->w_post, a->gate, a->w_pre})
        if (misaligned(q, size)) return HP_EALIGN;
    if (misaligned(a->rstd, 4)) return HP_EALIGN;
    *p = Norm{};
    p->rows = a->rows;
    p->hidden = a->hidden;
    p->gate_size = a->hidden == 1 ? 1 : a->gate_size;
    p->gate_tanh = a->gate_tanh != 0;
    p->unit_offset = a->unit_offset != 0;
    p->scale = a->residual_scale;
    p->eps = a->eps;
    p->x = a->x, p->y = a->y, p->xs = a->x_stride, p->ys = a->y_stride;
    p->w1 = a->w_post, p->gate = a->gate, p->w2 = a->w_pre;
    p->rstd = a->rstd;
    return HP_OK;
}

int64_t workspace_of(int64_t rows, int32_t hidden) {
    // for either type: that of fewer values to a vector takes more waves, the other more groups
    int64_t lines = 0;
    for (const int vec : {4, 8}) {
        const Shape s = shape_of(hidden, vec);
        const int64_t n = blocks_of(rows, s, true) * (s.waves == 1 ? 4 : 1);
        lines = n > lines ? n : lines;
    }
    return (lines * 2 + 1) * hidden * (int64_t)sizeof(float);
}

}  // namespace

extern "C" {

int hp_gated_norm(const hp_norm_args_t *a, void *stream) {
    Norm p;
    if (const int rc = take(a, &p)) return rc;
    const int size = a->dtype == HP_BF16 ? 2 : 4;
    if (misaligned(a->h, size) || misaligned(a->z, size)) return HP_EALIGN;
    if (a->z && !a->w_pre) return HP_EINVAL;
    if (a->rows == 0) return HP_OK;
    if (!a->h && !a->z) return HP_EINVAL;
    p.h = a->h, p.z = a->z, p.hs = a->h_stride, p.zs = a->z_stride;
    if (crosses(p, p.x, p.xs, p.h, p.hs) || crosses(p, p.y, p.ys, p.h, p.hs)) return HP_EINVAL;
    if (crosses(p, p.x, p.xs, p.z, p.zs) || crosses(p, p.y, p.ys, p.z, p.zs)) return HP_EINVAL;
    const Shape s = shape_of(p.hidden, 16 / size);
    const int64_t blocks = blocks_of(p.rows, s, false);
    if (a->dtype == HP_BF16) launch<__bf16>(p, s, false, blocks, (hipStream_t)stream);
    else launch<float>(p, s, false, blocks, (hipStream_t)stream);
    return hip_failed(hipGetLastError()) ? HP_EHIP : HP_OK;
}

int64_t hp_gated_norm_workspace(int64_t rows, int32_t hidden) {
    if (rows < 0 || hidden < 1 || hidden > HP_NORM_MAX_HIDDEN) return HP_EINVAL;
    return workspace_of(rows, hidden);
}

int hp_gated_norm_backward(const hp_norm_args_t *a, const hp_norm_grads_t *g, void *stream) {
    Norm p;
    if (const int rc = take(a, &p)) return rc;
    if (!g) return HP_EINVAL;
    const int size = a->dtype == HP_BF16 ? 2 : 4;
    const bool sums = g->dw_post || g->dgate || g->dw_pre;
    for (const void *q : {g->dh, g->dz, (const void *)g->dx, (const void *)g->dy, (const void *)g->dw_post, (const void *)g->dgate, (const void *)g->dw_pre})
        if (misaligned(q, size)) return HP_EALIGN;
    if ((g->dz && !a->w_pre) || (g->dy && !a->y)) return HP_EINVAL;
    if ((g->dw_post && !a->w_post) || (g->dgate && !a->gate) || (g->dw_pre && !a->w_pre)) return HP_EINVAL;
    if (sums && (!g->workspace || g->workspace_bytes < workspace_of(a->rows, a->hidden))) return HP_EINVAL;
    if (misaligned(g->workspace, 16)) return HP_EALIGN;
    if (a->rows > 0 && (!a->rstd || (!g->dh && !g->dz))) return HP_EINVAL;
    p.dh = g->dh, p.dz = g->dz, p.dx = g->dx, p.dy = g->dy;
    p.dhs = g->dh_stride, p.dzs = g->dz_stride, p.dxs = g->dx_stride, p.dys = g->dy_stride;
    if (crosses(p, p.dh, p.dhs, p.dx, p.dxs) || crosses(p, p.dz, p.dzs, p.dx, p.dxs)) return HP_EINVAL;
    if (crosses(p, p.dh, p.dhs, p.dy, p.dys) || crosses(p, p.dz, p.dzs, p.dy, p.dys)) return HP_EINVAL;
    p.partial = sums ? (float *)g->workspace : nullptr;
    const hipStream_t st = (hipStream_t)stream;
    const Shape s = shape_of(p.hidden, 16 / size);
    const int64_t blocks = blocks_of(p.rows, s, true);
    if (p.rows > 0 && (g->dx || g->dy || sums)) {
        if (a->dtype == HP_BF16) launch<__bf16>(p, s, true, blocks, st);
        else launch<float>(p, s, true, blocks, st);
        if (hip_failed(hipGetLastError())) return HP_EHIP;
    }
    if (!sums) return HP_OK;
    Finish f{p.partial, (int32_t)(p.rows > 0 ? blocks * (s.waves == 1 ? 4 : 1) : 0), p.hidden, p.gate_size, p.gate_tanh, p.unit_offset,
             p.w1, p.gate, g->dw_post, g->dgate, g->dw_pre, nullptr};
    if (g->dgate && p.gate_size == 1) f.sums = p.partial + (int64_t)f.lines * 2 * p.hidden;
    const uint32_t grid = (uint32_t)((p.hidden + kColumns - 1) / kColumns);
    if (a->dtype == HP_BF16) norm_finish_kernel<__bf16><<<grid, kColumns * kLines, 0, st>>>(f);
    else norm_finish_kernel<float><<<grid, kColumns * kLines, 0, st>>>(f);
    if (f.sums) {
        if (hip_failed(hipGetLastError())) return HP_EHIP;
        if (a->dtype == HP_BF16) norm_gate_kernel<__bf16><<<1, 1024, 0, st>>>(f.sums, p.hidden, g->dgate);
        else norm_gate_kernel<float><<<1, 1024, 0, st>>>(f.sums, p.hidden, g->dgate);
    }
    return hip_failed(hipGetLastError()) ? HP_EHIP : HP_OK;
}

}  // extern "C"
