// Exchanges between lanes and what the routers build on them: comparisons, sums and the best of a wavefront in 64 bits; the gates' exponential.
#pragma once
#include "common.h"

namespace {

__device__ __forceinline__ bool beats(float av, int ae, float bv, int be) { return av > bv || (av == bv && ae < be); }
__device__ __forceinline__ bool beats(double av, int ae, double bv, int be) { return av > bv || (av == bv && ae < be); }

// exchange inside groups of 4 (steps 0, 1), 8 (step 2) and 16 (step 3) neighbouring lanes
template <int STEP> __device__ __forceinline__ int dpp_xchg(int v) {
    if (STEP == 0) return __builtin_amdgcn_update_dpp(v, v, 0xB1, 0xf, 0xf, false);    // quad_perm [1,0,3,2]
    if (STEP == 1) return __builtin_amdgcn_update_dpp(v, v, 0x4E, 0xf, 0xf, false);    // quad_perm [2,3,0,1]
    if (STEP == 2) return __builtin_amdgcn_update_dpp(v, v, 0x141, 0xf, 0xf, false);   // row_half_mirror
    return __builtin_amdgcn_update_dpp(v, v, 0x140, 0xf, 0xf, false);                  // row_mirror
}
template <int STEP> __device__ __forceinline__ float dpp_xchg(float v) {
    return __int_as_float(dpp_xchg<STEP>(__float_as_int(v)));
}
// the same for doubles: exchanges inside a row of 16 lanes stay in the vector unit (a __shfl goes through
// LDS and takes ten times as long)
template <int STEP> __device__ __forceinline__ double dpp_xchg(double v) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = (unsigned)dpp_xchg<STEP>((int)(unsigned)u), hi = (unsigned)dpp_xchg<STEP>((int)(unsigned)(u >> 32));
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
__device__ __forceinline__ double lane_f64(double v, int lane) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)u, lane), hi = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)(u >> 32), lane);
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
__device__ __forceinline__ double row_sum_f64(double v) {
    v += dpp_xchg<0>(v);
    v += dpp_xchg<1>(v);
    v += dpp_xchg<2>(v);
    v += dpp_xchg<3>(v);
    return v;
}
__device__ __forceinline__ double wave_sum_f64(double v) {
    v = row_sum_f64(v);
    return (lane_f64(v, 0) + lane_f64(v, 16)) + (lane_f64(v, 32) + lane_f64(v, 48));
}
// the best of each row of 16 lanes, or (all) of the wavefront
__device__ __forceinline__ void row_best_f64(double& v, int& e, bool all) {
    double ov; int oe;
    ov = dpp_xchg<0>(v); oe = dpp_xchg<0>(e); if (beats(ov, oe, v, e)) { v = ov; e = oe; }
    ov = dpp_xchg<1>(v); oe = dpp_xchg<1>(e); if (beats(ov, oe, v, e)) { v = ov; e = oe; }
    ov = dpp_xchg<2>(v); oe = dpp_xchg<2>(e); if (beats(ov, oe, v, e)) { v = ov; e = oe; }
    ov = dpp_xchg<3>(v); oe = dpp_xchg<3>(e); if (beats(ov, oe, v, e)) { v = ov; e = oe; }
    if (all) {
#pragma unroll
        for (int off = 16; off <= 32; off <<= 1) {
            ov = __shfl_xor(v, off);
            oe = __shfl_xor(e, off);
            if (beats(ov, oe, v, e)) { v = ov; e = oe; }
        }
    }
}

// exp(v) = 2^t for t = v log2(e), with what the rounding of t took away put back (v is up to tens, so t alone costs several
// units in the last place of the result).
__device__ __forceinline__ float gate_exp(float v) {
    constexpr float L = 1.44269504088896340736f, L_REST = (float)(1.44269504088896340736 - (double)L), LN2 = 0.69314718055994530942f;
    const float t = v * L, rest = fmaf(v, L_REST, fmaf(v, L, -t)), e = __builtin_amdgcn_exp2f(t);
    return e > 0.f ? fmaf(e, rest * LN2, e) : e;     // (rest is no number for an infinite v)
}

}  // namespace
