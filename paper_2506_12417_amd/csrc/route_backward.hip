// moe_route_topk_backward: from the gradients of the gate values to those of the logits, of x, of the router's matrix and of its bias.
//
//   g_j = gate_w[t,j] of expert i_j;   D = sum_j g_j dgate_w[t,j]
//   softmax over all E logits:  dl[t,e] = p_e (sum_{j: i_j = e} dgate_w[t,j] - D)      p = softmax(logits[t])
//   over the k chosen (renorm): dl[t,i_j] = g_j (dgate_w[t,j] - D), 0 elsewhere
//   dl += dlogits_add     dx = dx_add + dl W_g^T     dW_g = x^T dl     db = sum_t dl
//
// Both products are fp32 throughout (v_mfma_f32_16x16x4_f32): dl is never rounded.  dW_g and db are summed over ranges of tokens, whose
// parts a second launch adds up in their order: no atomics.
#include "common.h"
#include "gemm_util.h"

namespace {

constexpr int NTH = 256;

__device__ __forceinline__ float shfl_sum(float v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ float shfl_max(float v) {
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

// ---- dl: a wavefront has a token, a lane up to four experts
__global__ __launch_bounds__(NTH) void dlogits_kernel(const float* __restrict__ dgate_w, const float* __restrict__ gate_w, const int32_t* __restrict__ idx,
                                                      const float* __restrict__ logits, const float* __restrict__ add, int T, int E, int k, int renorm,
                                                      float* __restrict__ dl) {
    const int t = (int)(blockIdx.x * (NTH / 64) + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
    if (t >= T) return;
    float g = 0.f, dg = 0.f;
    int e_of = -1;
    if (lane < k) {
        g = gate_w[(size_t)t * k + lane];
        dg = dgate_w[(size_t)t * k + lane];
        e_of = idx[(size_t)t * k + lane];
    }
    const bool lost = __ballot(lane < k && (e_of < 0 || e_of >= E)) != 0;      // (a token whose logits are NaN)
    const float D = shfl_sum(g * dg);
    float p[4], v[4];
    if (!renorm) {
        float most = -__builtin_inff(), sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = i * 64 + lane;
            p[i] = e < E ? logits[(size_t)t * E + e] : -__builtin_inff();
            most = fmaxf(most, p[i]);
        }
        most = shfl_max(most);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = i * 64 + lane < E ? expf(p[i] - most) : 0.f;
            sum += p[i];
        }
        sum = shfl_sum(sum);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] /= sum;
            v[i] = -D;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = p[i] = 0.f;
    }
    for (int j = 0; j < k; ++j) {
        const int e = __shfl(e_of, j);
        const float a = renorm ? __shfl(g, j) * (__shfl(dg, j) - D) : __shfl(dg, j);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (e == i * 64 + lane) v[i] += a;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = i * 64 + lane;
        if (e >= E) continue;
        const size_t at = (size_t)t * E + e;
        float r = renorm ? v[i] : p[i] * v[i];
        if (add) r += add[at];
        dl[at] = lost ? __builtin_nanf("") : r;
    }
}

// ---- dx: 64 tokens x 64 columns a work-group, a wavefront 16 tokens; terms (experts) 32 at a time through LDS
constexpr int KC = 32, PAD = KC + 4;
template <typename W>
__global__ __launch_bounds__(NTH) void dx_kernel(const float* __restrict__ dl, const W* __restrict__ w, const float* __restrict__ add, int T, int d, int E,
                                                 float* __restrict__ dx) {
    __shared__ __attribute__((aligned(16))) float sl[64 * PAD], sw[64 * PAD];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, lq = lane >> 4;
    const int t0 = blockIdx.y * 64, c0 = blockIdx.x * 64;
    f32x4 acc[4] = {};
    for (int e0 = 0; e0 < E; e0 += KC) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 64 * KC / NTH; ++i) {
            const int r = (i * NTH + tid) / KC, c = tid % KC;
            sl[r * PAD + c] = t0 + r < T && e0 + c < E ? dl[(size_t)(t0 + r) * E + e0 + c] : 0.f;
            sw[r * PAD + c] = c0 + r < d && e0 + c < E ? load_as_f32(w + (size_t)(c0 + r) * E + e0 + c) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < KC; s += 16) {
            const f32x4 b = *(const f32x4*)(sl + (wave * 16 + l16) * PAD + s + lq * 4);
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                const f32x4 a = *(const f32x4*)(sw + (n * 16 + l16) * PAD + s + lq * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], acc[n], 0, 0, 0);
            }
        }
    }
    const int t = t0 + wave * 16 + l16;
    if (t >= T) return;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const int c = c0 + n * 16 + lq * 4;
        if (c >= d) continue;                              // (d is a multiple of 8)
        const size_t at = (size_t)t * d + c;
        f32x4 v = acc[n];
        if (add) v += *(const f32x4*)(add + at);
        *(f32x4*)(dx + at) = v;
    }
}

// ---- dW_g over a range of tokens: 64 rows (of x's columns) x 64 experts a work-group, a wavefront 16 rows; 32 tokens at a time through LDS
constexpr int TC = 32, ROW = 64 + 16;
template <typename X>
__global__ __launch_bounds__(NTH) void dw_kernel(const X* __restrict__ x, const float* __restrict__ dl, int T, int d, int E, int range, float* __restrict__ part) {
    __shared__ __attribute__((aligned(16))) float sx[TC * ROW], sl[TC * ROW];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, lq = lane >> 4;
    const int c0 = blockIdx.x * 64, e0 = blockIdx.y * 64, first = blockIdx.z * range, last = first + range < T ? first + range : T;
    f32x4 acc[4] = {};
    float db = 0.f;
    for (int t0 = first; t0 < last; t0 += TC) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TC * 64 / NTH; ++i) {
            const int r = i * (NTH / 64) + wave, t = t0 + r;
            sx[r * ROW + lane] = x && t < last && c0 + lane < d ? load_as_f32(x + (size_t)t * d + c0 + lane) : 0.f;
            sl[r * ROW + lane] = t < last && e0 + lane < E ? dl[(size_t)t * E + e0 + lane] : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < TC; s += 4) {
            const float b = sx[(s + lq) * ROW + wave * 16 + l16];
#pragma unroll
            for (int n = 0; n < 4; ++n)
                acc[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(sl[(s + lq) * ROW + n * 16 + l16], b, acc[n], 0, 0, 0);
        }
        if (wave == 0 && blockIdx.x == 0)
            for (int r = 0; r < TC; ++r) db += sl[r * ROW + lane];
    }
    // part: [range][d + 1][E], the last row for db
    float* to = part + (size_t)blockIdx.z * (d + 1) * E;
    const int c = c0 + wave * 16 + l16;
    if (c < d) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (e0 + n * 16 + lq * 4 + i < E) to[(size_t)c * E + e0 + n * 16 + lq * 4 + i] = acc[n][i];
    }
    if (wave == 0 && blockIdx.x == 0 && e0 + lane < E) to[(size_t)d * E + e0 + lane] = db;
}
__global__ __launch_bounds__(NTH) void dw_sum_kernel(const float* __restrict__ part, int ranges, int d, int E, float* __restrict__ dw, float* __restrict__ db) {
    const size_t i = (size_t)blockIdx.x * NTH + threadIdx.x, n = (size_t)d * E, step = n + E;
    if (i >= step) return;
    float s = 0.f;
    for (int r = 0; r < ranges; ++r) s += part[r * step + i];
    if (i < n) {
        if (dw) dw[i] = s;
    } else if (db) {
        db[i - n] = s;
    }
}

// Ranges of tokens that dW_g is summed over: enough work-groups for the chip, 64 tokens at least.
int ranges_of(int T, int d, int E) {
    const int tiles = ((d + 63) / 64) * ((E + 63) / 64);
    int n = (1024 + tiles - 1) / tiles;
    const int most = (T + 63) / 64;
    if (n > most) n = most;
    if (n < 1) n = 1;
    const int range = ((T + n - 1) / n + TC - 1) / TC * TC;
    return range > 0 ? (T + range - 1) / range : 1;
}

}  // namespace

size_t moe_route_back_bytes(int T, int d, int E) {
    if (T < 1 || d < 1 || E < 1) return 0;
    return (size_t)ranges_of(T, d, E) * (d + 1) * E * sizeof(float);
}

extern "C" int moe_route_topk_backward(const float* dgate_w, const float* gate_w, const int32_t* expert_idx, const float* logits, const float* dlogits_add,
                                       const void* x, const void* w_gate, int T, int d, int E, int k, int renorm, moe_dtype dt, float* dlogits,
                                       const float* dx_add, float* dx, float* dw_gate, float* dbias, void* ws, size_t ws_bytes, void* stream) {
    const char* me = "moe_route_topk_backward";
    MOE_REQUIRE(T >= 0 && d >= 1 && E >= 1 && k >= 1 && k <= E, MOE_ERR_ARG, "%s: T=%d d=%d E=%d k=%d", me, T, d, E, k);
    MOE_REQUIRE(moe_dtype_ok(dt), MOE_ERR_UNSUPPORTED, "%s: dtype %d", me, (int)dt);
    MOE_REQUIRE(E <= MOE_MAX_EXPERTS && k <= MOE_MAX_TOPK && d % 8 == 0, MOE_ERR_UNSUPPORTED, "%s: d=%d E=%d k=%d", me, d, E, k);
    MOE_REQUIRE(T <= 64 * 65535, MOE_ERR_UNSUPPORTED, "%s: T=%d", me, T);
    const bool sums = dw_gate || dbias;
    const size_t need = sums ? moe_route_back_bytes(T, d, E) : 0;
    if (T > 0) {
        MOE_REQUIRE(dgate_w && gate_w && expert_idx && (logits || renorm) && dlogits && (w_gate || !dx) && (x || !dw_gate), MOE_ERR_ARG, "%s: null pointer", me);
        MOE_REQUIRE(!sums || (ws && ws_bytes >= need), MOE_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", me, ws_bytes, need);
        MOE_REQUIRE((((uintptr_t)dx | (uintptr_t)dx_add) & 15) == 0 && (((uintptr_t)ws | (uintptr_t)dlogits) & 3) == 0, MOE_ERR_UNSUPPORTED, "%s: dx and dx_add have to be aligned to 16 bytes", me);
    }
    if (T == 0 && !sums) return MOE_OK;
    const hipStream_t st = (hipStream_t)stream;
    int ranges = 0;
    if (T > 0) {
        hipLaunchKernelGGL(dlogits_kernel, dim3((T + 3) / 4), dim3(NTH), 0, st, dgate_w, gate_w, expert_idx, logits, dlogits_add, T, E, k, renorm, dlogits);
        if (dx) {
            const dim3 grid((d + 63) / 64, (T + 63) / 64);
            if (dt == MOE_F32) hipLaunchKernelGGL(dx_kernel<float>, grid, dim3(NTH), 0, st, dlogits, (const float*)w_gate, dx_add, T, d, E, dx);
            else hipLaunchKernelGGL(dx_kernel<uint16_t>, grid, dim3(NTH), 0, st, dlogits, (const uint16_t*)w_gate, dx_add, T, d, E, dx);
        }
        if (sums) {
            ranges = ranges_of(T, d, E);
            const int range = ((T + ranges - 1) / ranges + TC - 1) / TC * TC;
            const dim3 grid(dw_gate ? (d + 63) / 64 : 1, (E + 63) / 64, ranges);
            if (dt == MOE_F32) hipLaunchKernelGGL(dw_kernel<float>, grid, dim3(NTH), 0, st, (const float*)(dw_gate ? x : nullptr), dlogits, T, d, E, range, (float*)ws);
            else hipLaunchKernelGGL(dw_kernel<uint16_t>, grid, dim3(NTH), 0, st, (const uint16_t*)(dw_gate ? x : nullptr), dlogits, T, d, E, range, (float*)ws);
        }
    }
    if (sums) {
        const size_t n = (size_t)(d + 1) * E;
        hipLaunchKernelGGL(dw_sum_kernel, dim3((unsigned)((n + NTH - 1) / NTH)), dim3(NTH), 0, st, (const float*)ws, ranges, d, E, dw_gate, dbias);
    }
    MOE_CHECK_LAUNCH("moe_route_topk_backward");
    return MOE_OK;
}
