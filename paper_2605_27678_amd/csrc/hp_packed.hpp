// What the kernels over packed values share: codes of 4 bits as operands of matrix products.
//
// A group's value is low + step * code, so that a sum over its channels is
//     sum x value = step * sum x code + low * sum x:
// the matrix units take the codes as they are, which bfloat16 holds exactly, and the step goes over the 4 results that a
// lane has of 32 channels instead of over the 8 codes that it has unpacked.
#pragma once

#include "hp_device.hpp"
#include "hp_packed.h"

namespace hp {

typedef Vec<__bf16, 8> Frag;
typedef Vec<float, 4> Quad;
typedef Vec<uint32_t, 4> Words;

constexpr int kGroup = HP_PACKED_GROUP, kGroupBytes = 16;

inline __host__ __device__ int groups_of(int dim) { return (dim + kGroup - 1) / kGroup; }

// The products of 16 x 16 x 32: lane l has, of the left operand, row l % 16, of the right one column l % 16, of both the
// inner values 8(l / 16) and on, and of the result column l % 16 and rows 4(l / 16) and on.
__device__ __forceinline__ Quad mma(const Frag &a, const Frag &b, const Quad &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// A word's eight codes as an operand of products, (code + kLift) * kUnit, in the order of their channels.
//
// For bfloat16 results a code's four bits go below the leading one of 16: 0x4180 | code << 3 is 16 + code, two at a time with
// a shift and an and-or, one instruction a code.  (128 + code would save one shift in eight and cost the sums three more bits
// to cancel.)  What the 16 adds is taken off again with sum x, which the matrix units make too.
//
// Binary32 results would feel that the lift cancels (1.8e-6 of their size off instead of 8e-7): there a code less 8 goes
// through binary32, by the conversion of 4-bit whole numbers, which gives sixteenths.
template <class T> struct Codes;
template <> struct Codes<__bf16> {
    static constexpr float kLift = 16.0f, kUnit = 1.0f;
    uint32_t sixteen = 0x41804180u;
    // in a vector register: an and-or takes one constant from a scalar one
    __device__ __forceinline__ Codes() { asm("" : "+v"(sixteen)); }
    __device__ __forceinline__ Frag operator()(uint32_t w) const {
        constexpr uint32_t kBits = 0x00780078u;
        return __builtin_bit_cast(Frag, Words{(w << 3 & kBits) | sixteen, (w >> 1 & kBits) | sixteen, (w >> 5 & kBits) | sixteen, (w >> 9 & kBits) | sixteen});
    }
};
template <> struct Codes<float> {
    static constexpr float kLift = -8.0f, kUnit = 0.0625f;
    __device__ __forceinline__ Frag operator()(uint32_t w) const {
        // bytes' lower halves, and one shift for the upper ones; the conversion picks bytes by itself
        const uint32_t even = w ^ 0x88888888u;
        uint32_t odd = even >> 4;
        asm("" : "+v"(odd));
        Frag f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (__bf16)__builtin_amdgcn_cvt_off_f32_i4((int)((i / 2 % 2 ? odd : even) >> (8 * (i / 4) + 16 * (i % 2)) & 0xffu));
        return f;
    }
};

__device__ __forceinline__ Frag all_of(float x) {
    Frag f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (__bf16)x;
    return f;
}

// The two halves of a pair (step, low) as it lies in memory.
__device__ __forceinline__ float step_of(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float low_of(uint32_t pair) { return __uint_as_float(pair & 0xffff0000u); }

// The bfloat16 numbers that stand for a value of type T as an operand: itself (rounded, if it is a result), or three that add
// up to its 24 bits, 8 bits each.
template <class T> constexpr int kTerms = sizeof(T) == 2 ? 1 : 3;
__device__ __forceinline__ float upper_half(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ __bf16 half_of(float x) { return __builtin_bit_cast(__bf16, (uint16_t)(__float_as_uint(x) >> 16)); }
template <int N> __device__ __forceinline__ void terms(float x, Frag (&f)[N], int i) {
    if constexpr (N == 1) {
        f[0][i] = (__bf16)x;
    } else {
#pragma unroll
        for (int t = 0; t < N; ++t) {
            f[t][i] = half_of(x);
            x -= upper_half(x);
        }
    }
}
template <class T> __device__ __forceinline__ void terms(const Vec<T, 8> &x, Frag (&f)[kTerms<T>]) {
    if constexpr (sizeof(T) == 2) {
        f[0] = x;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) terms(x[i], f, i);
    }
}

// What a wave brings to LDS is its own: no barriers, only its own loads to wait for, and its own reads to finish before the
// next loads write there.
__device__ __forceinline__ void settle() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ void reads_done() {
    __builtin_amdgcn_s_waitcnt(0xc07f);            // lgkmcnt(0)
    settle();
}

constexpr int64_t kMostStride = 1 << 24;           // bytes or elements, of rows: 63 of them stay below kOutside
// Loads of a wave that write LDS: 16 or 4 bytes a lane from `offset` (the lane's) and `more` (the wave's) bytes behind
// `base`, one lane's behind the other from `to`; zeros for lanes with kOutside.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const void *base) {
    return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, 0x7fffffff, 0x00020000);
}
__device__ __forceinline__ void pieces_to_lds(const void *base, char *to, uint32_t offset, int more) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer_at(base), (__attribute__((address_space(3))) void *)to, 16, (int)offset, more, 0, 0);
}
__device__ __forceinline__ void words_to_lds(const void *base, char *to, uint32_t offset, int more) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(buffer_at(base), (__attribute__((address_space(3))) void *)to, 4, (int)offset, more, 0, 0);
}

// What hp_packed_t has to be, for so many rows and heads; strides that no address goes by do not count.
inline int check_packed(const hp_packed_t &t, int64_t rows, int64_t heads) {
    if (rows > 0 && heads > 0 && (!t.codes || !t.scales)) return HP_EINVAL;
    if ((uintptr_t)t.codes % 16 || (uintptr_t)t.scales % 4) return HP_EALIGN;
    if (rows > 1 && (t.code_row_stride % 16 || t.scale_row_stride % 2)) return HP_EALIGN;
    if (heads > 1 && (t.code_head_stride % 16 || t.scale_head_stride % 2)) return HP_EALIGN;
    return HP_OK;
}
// Row strides that offsets of 32 bits hold for a tile's rows; a single row has none.
inline bool short_strides(const hp_packed_t &t, int64_t rows) {
    return rows <= 1 || (t.code_row_stride >= 0 && t.code_row_stride <= kMostStride && t.scale_row_stride >= 0 && t.scale_row_stride <= kMostStride);
}

inline hp_packed_t without_unused(hp_packed_t t, int64_t rows) {
    if (rows <= 1) t.code_row_stride = t.scale_row_stride = 0;
    return t;
}

}  // namespace hp
