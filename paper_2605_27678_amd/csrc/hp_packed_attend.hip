// Attention of single tokens to states held in 4 bits: row r sees the states lo(r) .. hi(r) - 1, and with a group's
// value = low + step * code,
//     s_j = scale sum_g (step_jg sum_c q_c code_jc + low_jg sum_c q_c),  p_j = exp(s_j - m) / sum,
//     out_c = sum_j (p_j step_jg) code_jc + sum_j p_j low_jg              (g the group of channel c)
// in one pass with a running maximum m and sum.  The codes go into the matrix units as they are (hp_packed.hpp).
//
// A wave takes 64 states at a time by itself.  S^T = K Q^T, so that a lane has scores of one head, four states of each 16.
// Its four words of a 16-byte group change places with those of three other lanes, and it has 8 channels of one state for
// each product.  The steps go over a group's 16 x 16 results before they add up.  out^T = V^T P^T has the states as inner
// values: the transposing LDS load brings a lane 16 states of one channel, in the order in which it has their weights, so
// that no weight leaves its lane; the weights, times the group's steps, are rounded to bfloat16 (three such numbers in
// binary32).  What the codes' lift puts into a product, and 8 more so that codes lie around zero and cancel little, is taken
// off by a product with -24 throughout, from the very same rounded weights (in binary32 they lie there as they are);
// 8 * sum p step + sum p low come from one more product, whose left rows are the groups' steps and lows.
#include <climits>
#include <cmath>

#include "hp_join.hpp"
#include "hp_packed.hpp"

#pragma clang fp contract(fast)

namespace {

using namespace hp;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kWaves = 4, kBlock = kWaves * kWave;
constexpr int kTile = 64, kHeads = 16;             // states of a wave's tile, heads of a workgroup
constexpr float kMiddle = 8.0f;

struct Params {
    int64_t rows, keys;
    int32_t heads_q, group, groups, dim, splits, head_tiles;
    float scale2;                                  // for exponents of two
    hp_heads_t q, out;
    hp_packed_t k, v;
    const int32_t *ranges;
    float *lse;
    float *part, *part_lse;                        // [splits][rows * heads_q][dim], [splits][rows * heads_q]
};

// The 64 states of a wave in LDS: of each tensor codes [64][GP] of 16 bytes, a row's groups turned so that the same group
// of 8 neighbouring rows lies in different banks, and scales [GP][64] pairs.
template <int GP> struct Layout {
    static constexpr int kCodes = kTile * GP * kGroupBytes, kTensor = kCodes + kTile * GP * 4, kBytes = 2 * kTensor;
    static __device__ __forceinline__ int slot(int row, int g) {
        if constexpr (GP == 8) return g ^ (row & 7);
        else if constexpr (GP == 4) return g ^ (row >> 1 & 3);
        else if constexpr (GP == 2) return g ^ (row >> 2 & 1);
        else return g;
    }
    static __device__ __forceinline__ int at(int row, int g) { return (row * GP + slot(row, g)) * kGroupBytes; }
};

// Brings tiles of one tensor to LDS, 2 GP loads each.
template <int GP> struct Loader {
    uint32_t codes[GP], scales;
    __device__ __forceinline__ void plan(const hp_packed_t &t, int groups, int lane) {
#pragma unroll
        for (int n = 0; n < GP; ++n) {
            const int e = n * kWave + lane, row = e / GP, g = Layout<GP>::slot(row, e % GP);     // slot() is its own inverse
            codes[n] = g < groups ? (uint32_t)(row * (int)t.code_row_stride + g * kGroupBytes) : kOutside;
        }
        scales = (uint32_t)(lane * (int)t.scale_row_stride * 2);
    }
    // left: states from the tile's first on that are seen
    __device__ __forceinline__ void fetch(char *to, const hp_packed_t &t, int64_t first, int head, int left, int groups, int lane) const {
        typedef __attribute__((address_space(3))) void *Lds;
        const auto from = buffer_at((const char *)t.codes + first * t.code_row_stride + (int64_t)head * t.code_head_stride);
#pragma unroll
        for (int n = 0; n < GP; ++n)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (Lds)(to + n * kWave * 16), 16, (int)((n * kWave + lane) / GP < left ? codes[n] : kOutside), 0, 0, 0);
        const auto pairs = buffer_at((const uint16_t *)t.scales + first * t.scale_row_stride + (int64_t)head * t.scale_head_stride);
#pragma unroll
        for (int g = 0; g < GP; ++g)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(pairs, (Lds)(to + Layout<GP>::kCodes + g * kWave * 4), 4, (int)(lane < left && g < groups ? scales + 4 * g : kOutside), 0, 0, 0);
    }
};

__device__ __forceinline__ float2 across_halves(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float2 across_rows(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Over the four lanes of a column.
__device__ __forceinline__ float column_max(float x) {
    const float2 a = across_halves(x), b = across_rows(fmaxf(a.x, a.y));
    return fmaxf(b.x, b.y);
}
__device__ __forceinline__ float column_sum(float x) {
    const float2 a = across_halves(x), b = across_rows(a.x + a.y);
    return b.x + b.y;
}

constexpr float kLag = 8.0f;                       // the maximum is raised when a score passes it by 2^8

// Waves of a SIMD: as many as registers (128, 168 and 256 of them) and LDS (10 KiB a wave for heads of 128) let run.
template <class T, int GP> constexpr int kResident = sizeof(T) == 2 ? (GP <= 4 ? 4 : 2) : (GP <= 3 ? 3 : 2);

template <class T, int GP> __global__ __launch_bounds__(kBlock, (kResident<T, GP>)) void packed_attend_kernel(Params p) {
    typedef Layout<GP> L;
    constexpr float kLift = Codes<T>::kLift;
    constexpr bool kCentred = kLift == -kMiddle;
    constexpr int N = kTerms<T>, kSets = (GP + 3) / 4, kRow = kGroup * GP + 4;
    __shared__ __attribute__((aligned(16))) char lds[kWaves * L::kBytes];
    static_assert(sizeof(lds) >= sizeof(float) * kWaves * kHeads * (kRow + 2), "room for the join");
    const int tid = (int)threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), col = lane % 16, quarter = lane / 16;
    const int64_t row = blockIdx.x;
    const int state_head = (int)blockIdx.y / p.head_tiles, first_head = ((int)blockIdx.y % p.head_tiles) * kHeads, split = (int)blockIdx.z;
    const int heads = min(p.group - first_head, kHeads), head0 = state_head * p.group + first_head;
    int lo = 0, hi = (int)p.keys;
    if (p.ranges) {
        lo = max(p.ranges[2 * row], 0);
        hi = min(p.ranges[2 * row + 1], (int)p.keys);
    }
    if (lo >= hi) lo = hi = 0;

    // the queries, and the right operand that puts the lows in: for each pair (step, low) of four groups the values
    // (-lift sum q, sum q), split into three numbers over the quarters
    Frag q[GP][N], sums[kSets] = {};
    const T *q_row = (const T *)p.q.data + row * p.q.row_stride + (int64_t)(head0 + min(col, heads - 1)) * p.q.head_stride;
#pragma unroll
    for (int g = 0; g < GP; ++g) {
        const int d = kGroup * g + 8 * quarter;
        const Vec<T, 8> x = load<8>(q_row + d, p.dim - d);
        terms<T>(x, q[g]);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += (float)x[i];
        sum = column_sum(sum);
        const __bf16 a = (__bf16)sum, b = (__bf16)(sum - (float)a), c = (__bf16)(sum - (float)a - (float)b);
        const float part = quarter == 0 ? (float)a : quarter == 1 ? (float)b : quarter == 2 ? (float)c : 0.0f;
        sums[g / 4][2 * (g % 4)] = (__bf16)(-kLift * part);
        sums[g / 4][2 * (g % 4) + 1] = (__bf16)part;
    }

    char *const k_tile = lds + wave * L::kBytes, *const v_tile = k_tile + L::kTensor;
    const uint32_t *const k_scales = (const uint32_t *)(k_tile + L::kCodes), *const v_scales = (const uint32_t *)(v_tile + L::kCodes);
    Loader<GP> ks, vs;
    ks.plan(p.k, p.groups, lane);
    vs.plan(p.v, p.groups, lane);
    // a wave's tiles are its own: no barriers, only its own loads to wait for and its own reads to finish
    const auto settle = [] {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    const auto read = [&] {
        __builtin_amdgcn_s_waitcnt(0xc07f);        // lgkmcnt(0)
        settle();
    };

    float top = -INFINITY, sum = 0.0f;
    Quad out[2 * GP] = {}, rest = {};
    const Frag centre = all_of(-kLift - kMiddle);
    const Codes<T> codes;
    const int n_tiles = (hi - lo + kTile - 1) / kTile;
    const int begin = (int)((int64_t)n_tiles * split / p.splits), end = (int)((int64_t)n_tiles * (split + 1) / p.splits);
    if (begin + wave < end) {
        const int key0 = lo + (begin + wave) * kTile;
        ks.fetch(k_tile, p.k, key0, state_head, hi - key0, p.groups, lane);
        vs.fetch(v_tile, p.v, key0, state_head, hi - key0, p.groups, lane);
    }
    for (int tile = begin + wave; tile < end; tile += kWaves) {
        const int key0 = lo + tile * kTile, next = key0 + kWaves * kTile;
        const bool more = tile + kWaves < end;
        __builtin_amdgcn_s_waitcnt(but(2 * GP));   // all but V's
        settle();
        Quad s[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            s[a] = Quad{};
#pragma unroll
            for (int h = 0; h < kSets; ++h) {
                union {
                    Words w;
                    Frag f;
                } u;
#pragma unroll
                for (int j = 0; j < 4; ++j) u.w[j] = 4 * h + j < GP ? k_scales[(4 * h + j) * kTile + 16 * a + col] : 0u;
                s[a] = mma(u.f, sums[h], s[a]);
            }
        }
#pragma unroll
        for (int j = 0; j < GP; ++j) {
            // pieces 4j .. 4j + 3 of this column's four states of GP groups, one a quarter
            const int mine = 4 * j + quarter;
            Words w = *(const Words *)(k_tile + L::at(16 * (mine / GP) + col, mine % GP));
            across_quarters(w);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int a = (4 * j + t) / GP, g = (4 * j + t) % GP;
                const Frag c = codes(w[t]);
                Quad d = {};
#pragma unroll
                for (int n = 0; n < N; ++n) d = mma(c, q[g][n], d);
                const Words pairs = *(const Words *)(k_scales + g * kTile + 16 * a + 4 * quarter);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[a][i] += step_of(pairs[i]) * d[i];
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // here, not behind the branch, where all these products' results would have to be kept until then
#pragma unroll
        for (int a = 0; a < 4; ++a) asm("" : "+v"(s[a]));
        read();
        if (more) ks.fetch(k_tile, p.k, next, state_head, hi - next, p.groups, lane);

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
            }

        if (more) __builtin_amdgcn_s_waitcnt(but(2 * GP));
        else __builtin_amdgcn_s_waitcnt(but(0));
        settle();
        // 8 sum p step + sum p low: row 2g of the left operand has group g's steps, row 2g + 1 its lows
        {
            const uint32_t *line = v_scales + min(col / 2, GP - 1) * kTile + 4 * quarter;
            const uint32_t half = col % 2 ? 0x07060302u : 0x05040100u;
            Frag weights[2][N];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const Words even = *(const Words *)(line + 32 * b), odd = *(const Words *)(line + 32 * b + 16);
                union {
                    Words w;
                    Frag f;
                } u;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    u.w[i] = __builtin_amdgcn_perm(odd[i], even[i], half);
                    terms(s[2 * b][i], weights[b], 2 * i);
                    terms(s[2 * b + 1][i], weights[b], 2 * i + 1);
                }
#pragma unroll
                for (int n = 0; n < N; ++n) rest = mma(u.f, weights[b][n], rest);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int g = 0; g < GP; ++g) {
            Frag weights[2][N];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const Words even = *(const Words *)(v_scales + g * kTile + 32 * b + 4 * quarter), odd = *(const Words *)(v_scales + g * kTile + 32 * b + 16 + 4 * quarter);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    terms(s[2 * b][i] * step_of(even[i]), weights[b], 2 * i);
                    terms(s[2 * b + 1][i] * step_of(odd[i]), weights[b], 2 * i + 1);
                }
            }
            typedef int Pair __attribute__((ext_vector_type(2)));
            typedef __attribute__((address_space(3))) Pair *Lds;
            const char *line = v_tile + L::at(16 * (col / 4) + 4 * quarter + col % 4, g);      // the 16 lanes of a quarter: its states
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
            __builtin_amdgcn_sched_barrier(0);
        }
        read();
        if (more) vs.fetch(v_tile, p.v, next, state_head, hi - next, p.groups, lane);
    }
    sum = column_sum(sum);

    // join the waves in the tiles' place: statistics, then the products of each
    float *const join = (float *)lds, *const tops = join + kWaves * kHeads * kRow, *const totals = tops + kWaves * kHeads;
    __syncthreads();
    if (quarter == 0) {
        tops[wave * kHeads + col] = top;
        totals[wave * kHeads + col] = sum;
    }
    __syncthreads();
    float most = -INFINITY, total = 0.0f;
    for (int w = 0; w < kWaves; ++w) most = fmaxf(most, tops[w * kHeads + col]);
    // a wave without a maximum has seen nothing, or NaN alone
    const auto weight = [&](float t) { return t == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(t - most); };
    for (int w = 0; w < kWaves; ++w) total += totals[w * kHeads + col] * weight(tops[w * kHeads + col]);
    const float share = total == 0.0f ? 0.0f : weight(top) / total;
    const float lse2 = total == 0.0f ? -INFINITY : most + __builtin_amdgcn_logf(total);
#pragma unroll
    for (int g = 0; g < GP; ++g) {
        const int from = 16 * (g / 2) + col;
        const float more = kMiddle * __shfl(rest[2 * (g % 2)], from) + __shfl(rest[2 * (g % 2) + 1], from);
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)            // rows of the transposed load are a word's bits in order
                join[(wave * kHeads + col) * kRow + kGroup * g + 16 * c + 8 * (quarter / 2) + 2 * i + quarter % 2] = (out[2 * g + c][i] + more) * share;
    }
    __syncthreads();
    const int64_t n = p.rows * p.heads_q, out_row = row * p.heads_q + head0;
    for (int e = tid; e < heads * 8 * GP; e += kBlock) {
        const int m = e / (8 * GP), d = 4 * (e % (8 * GP));
        if (d >= p.dim) continue;
        Quad v = {};
        for (int w = 0; w < kWaves; ++w) v += *(const Quad *)(join + (w * kHeads + m) * kRow + d);
        if (p.splits > 1) {
            store<4>(p.part + (split * n + out_row + m) * p.dim + d, v, p.dim - d);
        } else {
            Vec<T, 4> o;
#pragma unroll
            for (int t = 0; t < 4; ++t) o[t] = (T)v[t];
            store<4>((T *)p.out.data + row * p.out.row_stride + (int64_t)(head0 + m) * p.out.head_stride + d, o, p.dim - d);
        }
    }
    if (wave == 0 && quarter == 0 && col < heads) {
        if (p.splits > 1) p.part_lse[split * n + out_row + col] = lse2;
        else if (p.lse) p.lse[out_row + col] = lse2 * kLn2;
    }
}

// ---- host ------------------------------------------------------------------------------------------------------

int64_t align16(int64_t n) { return (n + 15) / 16 * 16; }

int head_tiles_of(const hp_packed_attend_args_t &a) { return (a.heads_q / a.heads_k + kHeads - 1) / kHeads; }

// Parts of each row's range.
int32_t splits_of(const hp_packed_attend_args_t &a) {
    const int64_t each = a.rows * a.heads_k * head_tiles_of(a);
    if (each == 0) return 1;
    const int64_t want = (each <= kComputeUnits / 2 ? 2 * kComputeUnits : 8 * kComputeUnits) / each;
    const int64_t most = a.keys / (kWaves * kTile) < kMostParts ? a.keys / (kWaves * kTile) : kMostParts;
    const int64_t n = want < most ? want : most;
    return (int32_t)(n < 1 ? 1 : n);
}

int check_sizes(const hp_packed_attend_args_t *a) {
    if (!a) return HP_EINVAL;
    if (a->dtype != HP_BF16 && a->dtype != HP_F32) return HP_EINVAL;
    if (a->dim < 1 || a->dim > HP_ATTEND_MAX_DIM || a->heads_k < 1 || a->heads_q < 1) return HP_EINVAL;
    if (a->heads_q % a->heads_k || a->heads_q > 16384) return HP_ELAYOUT;
    if (a->rows < 0 || a->keys < 0) return HP_EINVAL;
    // 256 lanes a row, and in the join one wave or workgroup a row and head, of launches below 2^32
    if (a->rows > 1 << 23 || a->rows * a->heads_q > (1 << 24) - 1 || a->keys > INT_MAX - 1024) return HP_ELAYOUT;
    return HP_OK;
}

int64_t workspace_of(const hp_packed_attend_args_t &a) {
    const int64_t splits = splits_of(a), outs = a.rows * a.heads_q;
    return splits > 1 ? align16(4 * splits * outs) + 4 * splits * outs * a.dim : 0;
}

int check(const hp_packed_attend_args_t *a) {
    if (const int rc = check_sizes(a)) return rc;
    if (!(a->scale > 0) || !std::isfinite(a->scale) || !std::isfinite(a->scale * kLog2e)) return HP_EINVAL;
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

template <class T> void launch(const Params &p, const dim3 &grid, hipStream_t s) {
    if (p.groups <= 2) packed_attend_kernel<T, 2><<<grid, kBlock, 0, s>>>(p);
    else if (p.groups == 3) packed_attend_kernel<T, 3><<<grid, kBlock, 0, s>>>(p);
    else if (p.groups == 4) packed_attend_kernel<T, 4><<<grid, kBlock, 0, s>>>(p);
    else packed_attend_kernel<T, 8><<<grid, kBlock, 0, s>>>(p);
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
    p.splits = splits_of(*a), p.head_tiles = head_tiles_of(*a);
    p.scale2 = a->scale * kLog2e;
    p.q = a->q, p.out = a->out, p.k = a->k, p.v = a->v, p.ranges = a->ranges, p.lse = a->lse;
    if (p.splits > 1) {
        p.part_lse = (float *)a->workspace;
        p.part = (float *)((char *)a->workspace + align16(4 * p.splits * p.rows * p.heads_q));
    }
    const dim3 grid((uint32_t)p.rows, (uint32_t)(a->heads_k * p.head_tiles), (uint32_t)p.splits);
    if (a->dtype == HP_BF16) launch<__bf16>(p, grid, s);
    else launch<float>(p, grid, s);
    if (hip_failed(hipGetLastError())) return HP_EHIP;
    if (p.splits == 1) return HP_OK;
    return join_parts(Parts{p.part, p.part_lse, p.splits}, a->dtype, p.rows, p.heads_q, p.dim, p.out, p.lse, s);
}

}  // extern "C"
