// moe_keep_rows and moe_keep_restore: rows of activations kept in 8 bits with a scale for every 64 columns (keep.h), and read back.
// Eight lanes hold a block, eight values each, so that its largest value takes three exchanges inside a row of lanes.  HBM bound: 8192 x 2048
// in fp32 there and back in 27 us (136 MB, 5.0 TB/s), rows of 777 values, one by one, 1501 of them in 9.5 us, of which most is the two launches.
#include "common.h"
#include "keep.h"
#include "lanes.h"

namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(8))) float f32x8;
constexpr int NTH = 256;

// VEC: rows are whole pieces of eight values, aligned; a lane's values are neighbours.  Else every eighth of its block's.
template <bool VEC> __device__ __forceinline__ int col_of(int block, int l8, int i) { return block * KEEP_BLOCK + (VEC ? l8 * 8 + i : i * 8 + l8); }

template <typename E, bool VEC> __device__ __forceinline__ void fetch(const E* row, int n, int block, int l8, float (&v)[8]) {
    if constexpr (VEC) {
        const int c = col_of<true>(block, l8, 0);
        const bool on = c < n;
        if constexpr (sizeof(E) == 4) {
            f32x4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
            if (on) { a = ((const f32x4*)(row + c))[0]; b = ((const f32x4*)(row + c))[1]; }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < 4 ? a[i & 3] : b[i & 3];
        } else {
            u32x4 a = {0u, 0u, 0u, 0u};
            if (on) a = *(const u32x4*)(row + c);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(i & 1 ? a[i >> 1] & 0xffff0000u : a[i >> 1] << 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = col_of<false>(block, l8, i);
            v[i] = c < n ? load_as_f32(row + c) : 0.f;
        }
    }
}

template <typename E, bool VEC>
__global__ __launch_bounds__(NTH) void keep_rows_kernel(const E* __restrict__ x, size_t blocks, int n, int nb, int8_t* __restrict__ q, float* __restrict__ scale) {
    const size_t at = ((size_t)blockIdx.x * NTH + threadIdx.x) >> 3;
    const int l8 = threadIdx.x & 7;
    const bool on = at < blocks;                           // (all lanes take part in the exchanges)
    const size_t row = on ? at / (unsigned)nb : 0;
    const int block = on ? (int)(at - row * nb) : 0;
    float v[8];
    fetch<E, VEC>(x + row * n, n, block, l8, v);
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max_u32(most, magnitude(v[i]));
    most = max_u32(most, (unsigned)dpp_xchg<0>((int)most));
    most = max_u32(most, (unsigned)dpp_xchg<1>((int)most));
    most = max_u32(most, (unsigned)dpp_xchg<2>((int)most));
    if (!on) return;
    const KeepScale k = keep_scale(most);
    auto nearest = [&](float a) { return keep_nearest(a, __uint_as_float(most), k.to_q); };
    if (l8 == 0) scale[at] = k.scale;
    int8_t* to = q + row * n;
    if constexpr (VEC) {
        const int c = col_of<true>(block, l8, 0);
        const u32x2 w = {pack_bytes(nearest(v[0]), nearest(v[1]), nearest(v[2]), nearest(v[3])), pack_bytes(nearest(v[4]), nearest(v[5]), nearest(v[6]), nearest(v[7]))};
        if (c < n) *(u32x2*)(to + c) = w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = col_of<false>(block, l8, i);
            if (c < n) to[c] = (int8_t)nearest(v[i]);
        }
    }
}

template <typename E, bool VEC>
__global__ __launch_bounds__(NTH) void keep_restore_kernel(const int8_t* __restrict__ q, const float* __restrict__ scale, size_t blocks, int n, int nb, E* __restrict__ out) {
    const size_t at = ((size_t)blockIdx.x * NTH + threadIdx.x) >> 3;
    const int l8 = threadIdx.x & 7;
    if (at >= blocks) return;
    const size_t row = at / (unsigned)nb;
    const int block = (int)(at - row * nb);
    const float s = scale[at];
    const int8_t* from = q + row * n;
    E* to = out + row * n;
    if constexpr (VEC) {
        const int c = col_of<true>(block, l8, 0);
        if (c >= n) return;
        const u32x2 w = *(const u32x2*)(from + c);
        const f32x8 f = {byte_value<0>(w[0]) * s, byte_value<1>(w[0]) * s, byte_value<2>(w[0]) * s, byte_value<3>(w[0]) * s,
                         byte_value<0>(w[1]) * s, byte_value<1>(w[1]) * s, byte_value<2>(w[1]) * s, byte_value<3>(w[1]) * s};
        if constexpr (sizeof(E) == 4) {
            ((f32x4*)(to + c))[0] = f32x4{f[0], f[1], f[2], f[3]};
            ((f32x4*)(to + c))[1] = f32x4{f[4], f[5], f[6], f[7]};
        } else {
            *(u32x4*)(to + c) = __builtin_bit_cast(u32x4, __builtin_convertvector(f, bf16x8));      // to nearest, ties to even
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = col_of<false>(block, l8, i);
            if (c >= n) break;
            const float f = (float)from[c] * s;
            if constexpr (sizeof(E) == 4) to[c] = f;
            else to[c] = __builtin_bit_cast(uint16_t, (__bf16)f);
        }
    }
}

int keep_grid(const char* what, long long rows, int n, size_t* blocks, unsigned* grid) {
    *blocks = (size_t)rows * (size_t)((n + KEEP_BLOCK - 1) / KEEP_BLOCK);
    const size_t g = (*blocks * 8 + NTH - 1) / NTH;        // (a launch has less than 2^32 threads)
    MOE_REQUIRE(g < (1ull << 24), MOE_ERR_UNSUPPORTED, "%s: %lld rows of %d values", what, rows, n);
    *grid = (unsigned)g;
    return MOE_OK;
}

}  // namespace

extern "C" int moe_keep_rows(const void* x, moe_dtype dt, long long rows, int n, int8_t* q, float* scale, void* stream) {
    MOE_REQUIRE(rows >= 0 && n >= 1, MOE_ERR_ARG, "moe_keep_rows: rows=%lld n=%d", rows, n);
    MOE_REQUIRE(moe_dtype_ok(dt), MOE_ERR_UNSUPPORTED, "moe_keep_rows: dtype %d", (int)dt);
    MOE_REQUIRE(rows < (1ll << 40), MOE_ERR_UNSUPPORTED, "moe_keep_rows: rows=%lld", rows);
    size_t blocks;
    unsigned grid;
    const int ok = keep_grid("moe_keep_rows", rows, n, &blocks, &grid);
    if (ok != MOE_OK) return ok;
    if (rows == 0) return MOE_OK;
    MOE_REQUIRE(x && q && scale, MOE_ERR_ARG, "moe_keep_rows: null pointer");
    MOE_REQUIRE(((uintptr_t)x & (moe_elem_size(dt) - 1)) == 0 && ((uintptr_t)scale & 3) == 0, MOE_ERR_UNSUPPORTED, "moe_keep_rows: pointers not aligned to their type");
    const bool vec = n % 8 == 0 && ((uintptr_t)x & 15) == 0 && ((uintptr_t)q & 7) == 0;
    const int nb = (n + KEEP_BLOCK - 1) / KEEP_BLOCK;
    auto go = [&](auto kern, auto* p) { hipLaunchKernelGGL(kern, dim3(grid), dim3(NTH), 0, (hipStream_t)stream, p, blocks, n, nb, q, scale); };
    if (dt == MOE_F32) vec ? go(keep_rows_kernel<float, true>, (const float*)x) : go(keep_rows_kernel<float, false>, (const float*)x);
    else vec ? go(keep_rows_kernel<uint16_t, true>, (const uint16_t*)x) : go(keep_rows_kernel<uint16_t, false>, (const uint16_t*)x);
    MOE_CHECK_LAUNCH("moe_keep_rows");
    return MOE_OK;
}

extern "C" int moe_keep_restore(const int8_t* q, const float* scale, long long rows, int n, void* x, moe_dtype dt, void* stream) {
    MOE_REQUIRE(rows >= 0 && n >= 1, MOE_ERR_ARG, "moe_keep_restore: rows=%lld n=%d", rows, n);
    MOE_REQUIRE(moe_dtype_ok(dt), MOE_ERR_UNSUPPORTED, "moe_keep_restore: dtype %d", (int)dt);
    MOE_REQUIRE(rows < (1ll << 40), MOE_ERR_UNSUPPORTED, "moe_keep_restore: rows=%lld", rows);
    size_t blocks;
    unsigned grid;
    const int ok = keep_grid("moe_keep_restore", rows, n, &blocks, &grid);
    if (ok != MOE_OK) return ok;
    if (rows == 0) return MOE_OK;
    MOE_REQUIRE(x && q && scale, MOE_ERR_ARG, "moe_keep_restore: null pointer");
    MOE_REQUIRE(((uintptr_t)x & (moe_elem_size(dt) - 1)) == 0 && ((uintptr_t)scale & 3) == 0, MOE_ERR_UNSUPPORTED, "moe_keep_restore: pointers not aligned to their type");
    const bool vec = n % 8 == 0 && ((uintptr_t)x & 15) == 0 && ((uintptr_t)q & 7) == 0;
    const int nb = (n + KEEP_BLOCK - 1) / KEEP_BLOCK;
    auto go = [&](auto kern, auto* p) { hipLaunchKernelGGL(kern, dim3(grid), dim3(NTH), 0, (hipStream_t)stream, q, scale, blocks, n, nb, p); };
    if (dt == MOE_F32) vec ? go(keep_restore_kernel<float, true>, (float*)x) : go(keep_restore_kernel<float, false>, (float*)x);
    else vec ? go(keep_restore_kernel<uint16_t, true>, (uint16_t*)x) : go(keep_restore_kernel<uint16_t, false>, (uint16_t*)x);
    MOE_CHECK_LAUNCH("moe_keep_restore");
    return MOE_OK;
}
