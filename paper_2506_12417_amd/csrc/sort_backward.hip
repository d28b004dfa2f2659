// The gradients of the token sort and of the weighted combine (moe_permute, moe_unpermute_combine):
//
//   moe_unpermute_combine_backward   dy_perm[r] = gate_w[a] dy[t]     dgate_w[a] = sum_c dy[t,c] y_perm[r,c]      r = inv_perm[a], a = t k + j
//   moe_permute_backward             dx[t] = dx_add[t] + sum_j dx_perm[inv_perm[t k + j]]
//
// HBM bound: every row is read once and written once, past the caches, whole lines an instruction.  An assignment without a row (inv_perm negative)
// has dgate_w 0 and adds nothing.  8192 tokens, k = 4, d = 2048, rows in fp32, the rest in bf16: 92 us for 436 MB and 65 us for 370 MB.
// (With eight neighbouring columns a lane, so that fp32 rows were moved in halves of 32 bytes, a pass of both took 8 us more.)
#include "common.h"
#include "gemm_util.h"
#include "lanes.h"

namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(8))) float f32x8;
constexpr int NTH = 256;
constexpr int GROUP = 4;                                   // rows of a token whose loads are under way together

// a lane's values of a piece of 512 columns: four neighbours of either half (VEC: an instruction moves whole lines), else every 64th
template <bool VEC> __device__ __forceinline__ int col_of(int piece, int lane, int i) { return piece * 512 + (VEC ? (i & 4) * 64 + lane * 4 + (i & 3) : i * 64 + lane); }

template <bool VEC> __device__ __forceinline__ void fetch(const float* row, int d, int piece, int lane, bool on, float (&v)[8]) {
    if constexpr (VEC) {
        const int c = col_of<true>(piece, lane, 0);
        f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
        if (on && c < d) a = __builtin_nontemporal_load((const f32x4*)(row + c));
        if (on && c + 256 < d) b = __builtin_nontemporal_load((const f32x4*)(row + c + 256));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < 4 ? a[i & 3] : b[i & 3];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = col_of<false>(piece, lane, i);
            v[i] = on && c < d ? row[c] : 0.f;
        }
    }
}
template <bool VEC> __device__ __forceinline__ void put(float* row, int d, int piece, int lane, const float (&v)[8]) {
    if constexpr (VEC) {
        const int c = col_of<true>(piece, lane, 0);
        if (c < d) __builtin_nontemporal_store(f32x4{v[0], v[1], v[2], v[3]}, (f32x4*)(row + c));
        if (c + 256 < d) __builtin_nontemporal_store(f32x4{v[4], v[5], v[6], v[7]}, (f32x4*)(row + c + 256));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col_of<false>(piece, lane, i) < d) row[col_of<false>(piece, lane, i)] = v[i];
    }
}
template <bool VEC> __device__ __forceinline__ void put(uint16_t* row, int d, int piece, int lane, const float (&v)[8]) {
    if constexpr (VEC) {
        const int c = col_of<true>(piece, lane, 0);
        const f32x8 f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
        const u32x4 w = __builtin_bit_cast(u32x4, __builtin_convertvector(f, bf16x8));
        if (c < d) __builtin_nontemporal_store(u32x2{w[0], w[1]}, (u32x2*)(row + c));
        if (c + 256 < d) __builtin_nontemporal_store(u32x2{w[2], w[3]}, (u32x2*)(row + c + 256));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col_of<false>(piece, lane, i) < d) row[col_of<false>(piece, lane, i)] = __builtin_bit_cast(uint16_t, (__bf16)v[i]);
    }
}

__device__ __forceinline__ float wave_sum(float v) {
    v += dpp_xchg<0>(v);
    v += dpp_xchg<1>(v);
    v += dpp_xchg<2>(v);
    v += dpp_xchg<3>(v);
    const int b = __float_as_int(v);
    return (__int_as_float(__builtin_amdgcn_readlane(b, 0)) + __int_as_float(__builtin_amdgcn_readlane(b, 16))) +
           (__int_as_float(__builtin_amdgcn_readlane(b, 32)) + __int_as_float(__builtin_amdgcn_readlane(b, 48)));
}

// The same through a buffer descriptor of the row, without branches (behind these the compiler waits for all loads that are under way): what lies behind the
// row's end, or in a row that is none, reads as zero.
[[maybe_unused]] constexpr int NONTEMPORAL = 2;
template <bool VEC> __device__ __forceinline__ void fetch(const float*, __amdgpu_buffer_rsrc_t row, int piece, int lane, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += VEC ? 4 : 1) {
        const unsigned at = (unsigned)col_of<VEC>(piece, lane, i) * 4u;
        if constexpr (VEC) {
            const f32x4 a = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(row, at, 0, NONTEMPORAL));
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i + j] = a[j];
        } else {
            v[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(row, at, 0, NONTEMPORAL));
        }
    }
}
template <bool VEC> __device__ __forceinline__ void fetch(const uint16_t*, __amdgpu_buffer_rsrc_t row, int piece, int lane, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; i += VEC ? 4 : 1) {
        const unsigned at = (unsigned)col_of<VEC>(piece, lane, i) * 2u;
        if constexpr (VEC) {
            const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(row, at, 0, NONTEMPORAL));
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i + j] = __uint_as_float(j & 1 ? a[j >> 1] & 0xffff0000u : a[j >> 1] << 16);
        } else {
            v[i] = bf16_to_f32((uint16_t)__builtin_amdgcn_raw_buffer_load_b16(row, at, 0, NONTEMPORAL));
        }
    }
}

// A wavefront has a token; its rows go GROUP at a time, so that dy is fetched once for up to four of them.  A piece's loads are issued before the stores of
// the piece before it: loads and stores are counted together, a load behind stores waits for their way to memory.
template <typename D, typename P, bool VEC>
__global__ __launch_bounds__(NTH) void combine_backward_kernel(const D* __restrict__ dy, const float* __restrict__ y_perm, const int32_t* __restrict__ inv_perm,
                                                               const float* __restrict__ gate_w, int T, int d, int k, P* __restrict__ dy_perm,
                                                               float* __restrict__ dgate_w) {
#ifdef __HIP_DEVICE_COMPILE__                              // (the host's pass has no buffer descriptors)
    const int t = sgpr((int)(blockIdx.x * (NTH / 64) + (threadIdx.x >> 6))), lane = threadIdx.x & 63;
    if (t >= T) return;
    const __amdgpu_buffer_rsrc_t from = make_rsrc(dy + (size_t)t * d, (unsigned)d * (unsigned)sizeof(D));
    const int pieces = (d + 511) / 512;
    for (int j0 = 0; j0 < k; j0 += GROUP) {
        int row[GROUP];
        float w[GROUP], sum[GROUP];
        __amdgpu_buffer_rsrc_t ys[GROUP];
#pragma unroll
        for (int j = 0; j < GROUP; ++j) {
            const size_t a = (size_t)t * k + j0 + j;
            const bool on = j0 + j < k;
            row[j] = sgpr(on ? inv_perm[a] : -1);
            w[j] = on && gate_w ? gate_w[a] : 1.f;
            sum[j] = 0.f;
            ys[j] = make_rsrc(y_perm + (size_t)(row[j] < 0 ? 0 : row[j]) * d, dgate_w && row[j] >= 0 ? (unsigned)d * 4u : 0u);
        }
        struct Piece { float g[8], y[GROUP][8]; };
        auto load = [&](int piece, Piece& p) {
            fetch<VEC>(dy, from, piece, lane, p.g);
#pragma unroll
            for (int j = 0; j < GROUP; ++j) fetch<VEC>(y_perm, ys[j], piece, lane, p.y[j]);
        };
        auto step = [&](int piece, const Piece& here, Piece& next) {
            load(piece + 1, next);                         // (behind the last: zeros)
#pragma unroll
            for (int j = 0; j < GROUP; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[j] = fmaf(here.g[i], here.y[j][i], sum[j]);
            if (dy_perm) {
#pragma unroll
                for (int j = 0; j < GROUP; ++j) {
                    if (row[j] < 0) continue;
                    float v[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] = w[j] * here.g[i];
                    put<VEC>(dy_perm + (size_t)row[j] * d, d, piece, lane, v);
                }
            }
        };
        Piece a, b;
        load(0, a);
        for (int piece = 0; piece < pieces; piece += 2) {
            step(piece, a, b);
            if (piece + 1 < pieces) step(piece + 1, b, a);
        }
        if (dgate_w) {
#pragma unroll
            for (int j = 0; j < GROUP; ++j) {
                const float s = wave_sum(sum[j]);
                if (j0 + j < k && lane == 0) dgate_w[(size_t)t * k + j0 + j] = row[j] < 0 ? 0.f : s;
            }
        }
    }
#endif
}

template <typename P, bool VEC>
__global__ __launch_bounds__(NTH) void permute_backward_kernel(const float* __restrict__ dx_perm, const int32_t* __restrict__ inv_perm, int T, int d, int k,
                                                               const float* dx_add, P* dx, int pieces) {      // (dx may be dx_add)
    const size_t id = (size_t)blockIdx.x * (NTH / 64) + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int t = sgpr((int)(id / (unsigned)pieces)), piece = sgpr((int)(id % (unsigned)pieces));
    if (t >= T) return;
    float acc[8];
    fetch<VEC>(dx_add + (size_t)t * d, d, piece, lane, dx_add != nullptr, acc);
    for (int j0 = 0; j0 < k; j0 += GROUP) {
        float y[GROUP][8];
#pragma unroll
        for (int j = 0; j < GROUP; ++j) {
            const int r = j0 + j < k ? inv_perm[(size_t)t * k + j0 + j] : -1;
            fetch<VEC>(dx_perm + (size_t)(r < 0 ? 0 : r) * d, d, piece, lane, r >= 0, y[j]);
        }
#pragma unroll
        for (int j = 0; j < GROUP; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] += y[j][i];
    }
    put<VEC>(dx + (size_t)t * d, d, piece, lane, acc);
}

bool whole_pieces(int d, std::initializer_list<const void*> ps) {
    uintptr_t all = 0;
    for (const void* p : ps) all |= (uintptr_t)p;
    return d % 8 == 0 && (all & 15) == 0;
}

// A launch has less than 2^32 threads: work-groups of NTH, the last one whole.
bool wavefronts_fit(long long n) { return (n + NTH / 64 - 1) / (NTH / 64) < (1ll << 32) / NTH; }

}  // namespace

extern "C" int moe_unpermute_combine_backward(const void* dy, moe_dtype dy_dt, const float* y_perm, const int32_t* inv_perm, const float* gate_w, int T, int d,
                                              int k, void* dy_perm, moe_dtype perm_dt, float* dgate_w, void* stream) {
    MOE_REQUIRE(T >= 0 && d >= 1 && k >= 1, MOE_ERR_ARG, "moe_unpermute_combine_backward: T=%d d=%d k=%d", T, d, k);
    MOE_REQUIRE(moe_dtype_ok(dy_dt) && moe_dtype_ok(perm_dt), MOE_ERR_UNSUPPORTED, "moe_unpermute_combine_backward: dtypes %d, %d", (int)dy_dt, (int)perm_dt);
    MOE_REQUIRE((long long)T * k < (1ll << 31) && wavefronts_fit(T) && d < (1 << 29), MOE_ERR_UNSUPPORTED, "moe_unpermute_combine_backward: T=%d d=%d k=%d", T, d, k);
    if (T == 0) return MOE_OK;
    MOE_REQUIRE(dy && inv_perm && (dy_perm || dgate_w) && (y_perm || !dgate_w), MOE_ERR_ARG, "moe_unpermute_combine_backward: null pointer");
    const bool vec = whole_pieces(d, {dy, y_perm, dy_perm});
    auto go = [&](auto kern, auto* from, auto* to) {
        hipLaunchKernelGGL(kern, dim3((T + NTH / 64 - 1) / (NTH / 64)), dim3(NTH), 0, (hipStream_t)stream, from, y_perm, inv_perm, gate_w, T, d, k, to, dgate_w);
    };
    auto types = [&](auto* from, auto* to) {
        using D = std::remove_const_t<std::remove_pointer_t<decltype(from)>>;
        using P = std::remove_pointer_t<decltype(to)>;
        vec ? go(combine_backward_kernel<D, P, true>, from, to) : go(combine_backward_kernel<D, P, false>, from, to);
    };
    if (dy_dt == MOE_F32) perm_dt == MOE_F32 ? types((const float*)dy, (float*)dy_perm) : types((const float*)dy, (uint16_t*)dy_perm);
    else perm_dt == MOE_F32 ? types((const uint16_t*)dy, (float*)dy_perm) : types((const uint16_t*)dy, (uint16_t*)dy_perm);
    MOE_CHECK_LAUNCH("moe_unpermute_combine_backward");
    return MOE_OK;
}

extern "C" int moe_permute_backward(const float* dx_perm, const int32_t* inv_perm, int T, int d, int k, const float* dx_add, void* dx, moe_dtype dx_dt,
                                    void* stream) {
    MOE_REQUIRE(T >= 0 && d >= 1 && k >= 1, MOE_ERR_ARG, "moe_permute_backward: T=%d d=%d k=%d", T, d, k);
    MOE_REQUIRE(moe_dtype_ok(dx_dt), MOE_ERR_UNSUPPORTED, "moe_permute_backward: dtype %d", (int)dx_dt);
    const int pieces = (int)(((long long)d + 511) / 512);  // (of a wavefront each)
    MOE_REQUIRE((long long)T * k < (1ll << 31) && wavefronts_fit((long long)T * pieces), MOE_ERR_UNSUPPORTED, "moe_permute_backward: T=%d d=%d k=%d", T, d, k);
    if (T == 0) return MOE_OK;
    MOE_REQUIRE(dx_perm && inv_perm && dx, MOE_ERR_ARG, "moe_permute_backward: null pointer");
    const bool vec = whole_pieces(d, {dx_perm, dx_add, dx});
    const unsigned grid = (unsigned)(((long long)T * pieces + NTH / 64 - 1) / (NTH / 64));
    auto go = [&](auto kern, auto* to) {
        hipLaunchKernelGGL(kern, dim3(grid), dim3(NTH), 0, (hipStream_t)stream, dx_perm, inv_perm, T, d, k, dx_add, to, pieces);
    };
    if (dx_dt == MOE_F32) vec ? go(permute_backward_kernel<float, true>, (float*)dx) : go(permute_backward_kernel<float, false>, (float*)dx);
    else vec ? go(permute_backward_kernel<uint16_t, true>, (uint16_t*)dx) : go(permute_backward_kernel<uint16_t, false>, (uint16_t*)dx);
    MOE_CHECK_LAUNCH("moe_permute_backward");
    return MOE_OK;
}
