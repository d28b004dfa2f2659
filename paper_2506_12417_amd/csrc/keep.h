// Values kept in 8 bits, 64 neighbouring columns of a row with a scale: what keep.hip and ffn_train.hip share.
//
//   m = max |v| of the block     scale = m / 127     q = v 127 / m to the nearest integer, ties to even     read back: q scale
//
// (ffn_train.hip multiplies by a reciprocal, which is off by 2^-15 of a step at most: ties go either way.)
// The error is at most half a scale, m / 254.  POSITIVE (ReLU): negative values are kept as 0 and what is above zero as at least 1, so that the
// activation's slope is not lost.  A block that holds an infinity or a NaN has a scale of NaN; one whose m is below
// MOE_KEEP_LEAST is kept as zeros (127 / m would leave fp32's range).
#pragma once
#include "common.h"
#include "gemm_util.h"

namespace {

constexpr int KEEP_BLOCK = 64;
constexpr float MOE_KEEP_LEAST = 0x1p-100f;

// The largest magnitude as a bit pattern: NaN > infinity > numbers, so that neither gets lost.
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ unsigned max_u32(unsigned a, unsigned b) { return a > b ? a : b; }

struct KeepScale {
    float scale, to_q;       // q = v to_q
};
__device__ __forceinline__ KeepScale keep_scale(unsigned most) {
    const float m = __uint_as_float(most);
    KeepScale k;
    k.scale = most >= 0x7f800000u ? __builtin_nanf("") : m < MOE_KEEP_LEAST ? 0.f : m * (1.f / 127.f);
    // (v_rcp_f32 gives zero for a reciprocal below the normal numbers: m is brought down before, exactly)
    k.to_q = most >= 0x7f800000u || m < MOE_KEEP_LEAST ? 0.f : (127.f * 0x1p-16f) * __builtin_amdgcn_rcpf(m * 0x1p-16f);
    return k;
}
// v to_q, rounded, in the low 8 bits (adding 1.5 * 2^23 leaves the rounded integer there, two's complement)
template <bool POSITIVE> __device__ __forceinline__ unsigned keep_value(float v, float to_q) {
    float q = v * to_q;
    if (POSITIVE) q = v > 0.f && to_q > 0.f ? __builtin_fmaxf(q, 1.f) : 0.f;
    return __float_as_uint(q + 12582912.f);
}
// The same to the nearest for certain: 127 v - q m tells on which side of the tie the quotient lies (m and v are brought down, exactly, so
// that it has room).  m: the block's largest magnitude.
__device__ __forceinline__ unsigned keep_nearest(float v, float m, float to_q) {
    const float q = __builtin_rintf(v * to_q), down = to_q > 0.f ? m * 0x1p-16f : __builtin_inff();
    const float p = q * down, rest = fmaf(q, down, -p), twice = 2.f * (fmaf(v * 0x1p-16f, 127.f, -p) - rest);
    const bool odd = ((int)q & 1) != 0;
    const float up = twice > down || (twice == down && odd) ? 1.f : 0.f, less = twice < -down || (twice == -down && odd) ? 1.f : 0.f;
    return __float_as_uint(q + (up - less) + 12582912.f);
}
// the low bytes of four words
__device__ __forceinline__ unsigned pack_bytes(unsigned a, unsigned b, unsigned c, unsigned d) {
    const unsigned ab = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), cd = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
    return ab | cd;
}
template <bool POSITIVE> __device__ __forceinline__ unsigned keep_four(float a, float b, float c, float d, float to_q) {
    return pack_bytes(keep_value<POSITIVE>(a, to_q), keep_value<POSITIVE>(b, to_q), keep_value<POSITIVE>(c, to_q), keep_value<POSITIVE>(d, to_q));
}
template <int I> __device__ __forceinline__ float byte_value(unsigned w) { return (float)((int)(w << (24 - 8 * I)) >> 24); }

}  // namespace
