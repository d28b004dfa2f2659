// moe_route_topk_backward: from the gradients of the gate values to those of the logits, of x, of the router's matrix and of its bias.
//
//   g_j = gate_w[t,j] of expert i_j;   D = sum_j g_j dgate_w[t,j]
//   softmax over all E logits:  dl[t,e] = p_e (sum_{j: i_j = e} dgate_w[t,j] - D)      p = softmax(logits[t])
//   over the k chosen (renorm): dl[t,i_j] = g_j (dgate_w[t,j] - D), 0 elsewhere
//   dl += dlogits_add     dx = dx_add + dl W_g^T     dW_g = x^T dl     db = sum_t dl
//
// Both products are made by the 16-bit matrix instruction of fp32 values taken apart: v = hi + mid + lo, each bf16 (24 bits in all), whose products are exact
// and whose sums are fp32.  dl has three parts, x and W_g one where they are bf16 and three where they are fp32 (then without the products
// below 2^-24).  dW_g and db are summed over ranges of tokens, whose parts a second launch adds up in their order: no atomics.
//
// The least there is to move: x, dx_add and dx once, the logits and dl.  Measured, us (dl, dx, dW_g, its sum): 16384 tokens of 768 in bf16, 128 experts
// 8.4, 27, 22.5, 4.8 (a pass 66, at 5.5 TB/s 26 would do); 1501 of 1032 in fp32, 60 experts 3.0, 6.3, 8.8, 3.0 (a pass 19).  dx moves 100 MB, at 3.9
// TB/s; dW_g is bound by latencies: a work-group has thirteen steps of 32 tokens, whose dl every column tile fetches and takes apart
// again, and more work-groups store more parts (twice as many 27 + 6 us, half 26 + 4).
#include <type_traits>
#include "common.h"
#include "gemm_util.h"
#include "lanes.h"

namespace {

constexpr int NTH = 256;

// Sum and largest over the lanes: in rows of sixteen by exchanges, the rows' through scalar registers.
__device__ __forceinline__ float lane_f32(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
__device__ __forceinline__ float wave_sum(float v) {
    v += dpp_xchg<0>(v);
    v += dpp_xchg<1>(v);
    v += dpp_xchg<2>(v);
    v += dpp_xchg<3>(v);
    return (lane_f32(v, 0) + lane_f32(v, 16)) + (lane_f32(v, 32) + lane_f32(v, 48));
}
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp_xchg<0>(v));
    v = fmaxf(v, dpp_xchg<1>(v));
    v = fmaxf(v, dpp_xchg<2>(v));
    v = fmaxf(v, dpp_xchg<3>(v));
    return fmaxf(fmaxf(lane_f32(v, 0), lane_f32(v, 16)), fmaxf(lane_f32(v, 32), lane_f32(v, 48)));
}

// ---- dl: a wavefront has a token, a lane N experts
template <int N>
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
    const float D = wave_sum(g * dg);
    float p[N], v[N];
    if (!renorm) {
        float most = -__builtin_inff(), sum = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int e = i * 64 + lane;
            p[i] = e < E ? logits[(size_t)t * E + e] : -__builtin_inff();
            most = fmaxf(most, p[i]);
        }
        most = wave_max(most);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            p[i] = i * 64 + lane < E ? expf(p[i] - most) : 0.f;
            sum += p[i];
        }
        sum = wave_sum(sum);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            p[i] /= sum;
            v[i] = -D;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = p[i] = 0.f;
    }
    for (int j = 0; j < k; ++j) {
        const int e = __builtin_amdgcn_readlane(e_of, j);
        const float a = renorm ? lane_f32(g, j) * (lane_f32(dg, j) - D) : lane_f32(dg, j);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (e == i * 64 + lane) v[i] += a;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int e = i * 64 + lane;
        if (e >= E) continue;
        const size_t at = (size_t)t * E + e;
        float r = renorm ? v[i] : p[i] * v[i];
        if (add) r += add[at];
        dl[at] = lost ? __builtin_nanf("") : r;
    }
}

// ---- fp32 values in parts
template <int N> struct Parts { bf16x8 p[N]; };
__device__ __forceinline__ Parts<3> take_apart(__attribute__((ext_vector_type(8))) float v) {
    Parts<3> r;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const __bf16 hi = (__bf16)v[i];
        const float rest = v[i] - (float)hi;
        const __bf16 mid = (__bf16)rest;
        r.p[0][i] = hi;
        r.p[1][i] = mid;
        r.p[2][i] = (__bf16)(rest - (float)mid);
    }
    return r;
}
// acc += a b: the products of the parts, the small ones first
template <int NA, int NB> __device__ __forceinline__ void multiply(const Parts<NA>& a, const Parts<NB>& b, f32x4& acc) {
#pragma unroll
    for (int s = 2; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.p[i], b.p[s - i], acc, 0, 0, 0);
}
// Rows that a work-group reads, through a buffer descriptor: what is not `on`, or lies behind a row's n values, reads as zero without a branch (behind
// branches with loads in them the compiler waits for all that is under way).  Eight neighbours of row r from column c on.  VEC: n is a multiple of
// this (8, 4 or 1) and the rows are aligned to as many values.
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(4))) unsigned short u16x4;
typedef __attribute__((ext_vector_type(8))) unsigned short u16x8;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
constexpr unsigned NOWHERE = 0xFFFFFF00u;
[[maybe_unused]] constexpr int NONTEMPORAL = 2;
template <int VEC> __device__ __forceinline__ f32x8 fetch8(const float*, __amdgpu_buffer_rsrc_t rows, int n, unsigned r, int c, bool on) {
    const unsigned at = (r * (unsigned)n + (unsigned)c) * 4u;
    f32x8 v;
    if constexpr (VEC >= 4) {
        const f32x4 a = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, on && c < n ? at : NOWHERE, 0, 0));
        const f32x4 b = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, on && c + 4 < n ? at + 16u : NOWHERE, 0, 0));
        v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rows, on && c + i < n ? at + 4u * i : NOWHERE, 0, 0));
    }
    return v;
}
template <int VEC> __device__ __forceinline__ u16x8 fetch8(const uint16_t*, __amdgpu_buffer_rsrc_t rows, int n, unsigned r, int c, bool on) {
    const unsigned at = (r * (unsigned)n + (unsigned)c) * 2u;
    u16x8 v;
    if constexpr (VEC == 8) {
        v = __builtin_bit_cast(u16x8, __builtin_amdgcn_raw_buffer_load_b128(rows, on && c < n ? at : NOWHERE, 0, 0));
    } else if constexpr (VEC == 4) {
        const u16x4 a = __builtin_bit_cast(u16x4, __builtin_amdgcn_raw_buffer_load_b64(rows, on && c < n ? at : NOWHERE, 0, 0));
        const u16x4 b = __builtin_bit_cast(u16x4, __builtin_amdgcn_raw_buffer_load_b64(rows, on && c + 4 < n ? at + 8u : NOWHERE, 0, 0));
        v = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_amdgcn_raw_buffer_load_b16(rows, on && c + i < n ? at + 2u * i : NOWHERE, 0, 0);
    }
    return v;
}
template <typename E> struct Eight { typedef f32x8 type; };
template <> struct Eight<uint16_t> { typedef u16x8 type; };
__device__ __forceinline__ Parts<1> take_apart(u16x8 v) { return Parts<1>{__builtin_bit_cast(bf16x8, v)}; }
template <typename E> constexpr int PARTS = sizeof(E) == 4 ? 3 : 1;

// ---- dx: a work-group has dl of TT tokens in LDS, in parts, and goes over columns: a wavefront 32 of every 128, whose rows of W_g and added values are fetched
// while the 32 before are multiplied.  (With dl in registers and every wavefront fetching W_g for itself those fetches took 30 us: 16384 x 768, E = 128.)
// LDS: [part][token][32 KS experts], 16-byte pieces turned by the token, so that the reads of sixteen tokens touch all banks.
template <typename W, int KS, int VEC>
__global__ __launch_bounds__(NTH) void dx_kernel(const float* __restrict__ dl, const W* __restrict__ w, const float* add, int T, int d, int E, int columns,
                                                 float* dx) {       // (dx may be add)
#ifdef __HIP_DEVICE_COMPILE__                              // (the host's pass has no buffer descriptors)
    constexpr int TT = KS <= 4 ? 64 : 32, N = TT / 16, P = KS * 4, ROW = P * 16, TURN = P < 16 ? 16 / P : 1;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[3 * TT * ROW];
    auto place = [](int t, int piece) { return t * ROW + ((piece ^ (t / TURN & (P < 16 ? P - 1 : 15))) << 4); };
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, lq = lane >> 4;
    const int t0 = (int)blockIdx.x * TT;
    const unsigned rows = (unsigned)(T - t0 < TT ? T - t0 : TT);
    const __amdgpu_buffer_rsrc_t rl = make_rsrc(dl + (size_t)t0 * E, rows * (unsigned)E * 4u), rm = make_rsrc(w, (unsigned)d * (unsigned)E * (unsigned)sizeof(W));
    const __amdgpu_buffer_rsrc_t ra = make_rsrc(add + (size_t)t0 * d, add ? rows * (unsigned)d * 4u : 0u), ro = make_rsrc(dx + (size_t)t0 * d, rows * (unsigned)d * 4u);
    const int first = (int)blockIdx.y * columns, last = first + columns < d ? first + columns : d;
    typename Eight<W>::type next[KS][2];
    f32x4 old[2][N][2];
    auto fetch = [&](int c0, f32x4 (&o)[N][2]) {
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) next[s][h] = fetch8<VEC>(w, rm, E, (unsigned)(c0 + 16 * h + l16), s * 32 + lq * 8, c0 + 16 * h + l16 < last);
        const int c = c0 + lq * 4;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                o[n][h] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                        ra, c + 16 * h < last ? ((unsigned)(n * 16 + l16) * (unsigned)d + (unsigned)(c + 16 * h)) * 4u : NOWHERE, 0, 0));
    };
    f32x8 raw[TT * P / NTH];
#pragma unroll
    for (int i = 0; i < TT * P / NTH; ++i) raw[i] = fetch8<VEC>(dl, rl, E, (unsigned)((i * NTH + tid) / P), (i * NTH + tid) % P * 8, true);
    fetch(first + wave * 32, old[0]);
#pragma unroll
    for (int i = 0; i < TT * P / NTH; ++i) {
        const Parts<3> v = take_apart(raw[i]);
#pragma unroll
        for (int q = 0; q < 3; ++q) *(bf16x8*)(lds + q * TT * ROW + place((i * NTH + tid) / P, (i * NTH + tid) % P)) = v.p[q];
    }
    __syncthreads();
    auto step = [&](int c0, f32x4 (&here)[N][2], f32x4 (&later)[N][2]) {
        Parts<PARTS<W>> m[KS][2];
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int h = 0; h < 2; ++h) m[s][h] = take_apart(next[s][h]);
        fetch(c0 + 128, later);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            f32x4 acc[2] = {};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                Parts<3> g;
#pragma unroll
                for (int q = 0; q < 3; ++q) g.p[q] = *(const bf16x8*)(lds + q * TT * ROW + place(n * 16 + l16, s * 4 + lq));
#pragma unroll
                for (int h = 0; h < 2; ++h) multiply(m[s][h], g, acc[h]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {                  // (d is a multiple of 8)
                const int c = c0 + lq * 4 + 16 * h;
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[h] + here[n][h]), ro,
                                                       c < last ? ((unsigned)(n * 16 + l16) * (unsigned)d + (unsigned)c) * 4u : NOWHERE, 0, NONTEMPORAL);
            }
        }
    };
    for (int c0 = first + wave * 32; c0 < last; c0 += 256) {
        step(c0, old[0], old[1]);
        if (c0 + 128 < last) step(c0 + 128, old[1], old[0]);
    }
#endif
}

// ---- dW_g over a range of tokens: 64 of x's columns x 128 experts a work-group, 32 tokens at a time through LDS (fetched while the 32 before are multiplied);
// a wavefront has 64 columns x 32 experts.  The contraction lies outermost in both operands: the reads that transpose bring a column's terms together.
// LDS: panels of 32 tokens x 64 columns, 128 bytes a row, whose 32-byte pieces are turned by the row, so that the reads touch all banks.
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
constexpr int TC = 32;
[[maybe_unused]] constexpr int PANEL = TC * 128;
__device__ __forceinline__ int panel_at(int row, int c) { return row * 128 + (((c >> 4) ^ (row >> 1 & 3)) * 32) + (c & 15) * 2; }      // of column c < 64
__device__ __forceinline__ bf16x8 read_transposed(const unsigned char* panel, int block, int l16, int lq) {
    typedef __attribute__((ext_vector_type(8))) short s16x8;
    s16x4 v[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(panel + panel_at(i * 16 + lq * 4 + (l16 >> 2), block * 16 + (l16 & 3) * 4)));
    const s16x8 r = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, r);
}
template <int N> __device__ __forceinline__ void put8(unsigned char* at, int step, const Parts<N>& v) {
#pragma unroll
    for (int i = 0; i < N; ++i) *(bf16x8*)(at + i * step) = v.p[i];
}

template <typename X, int VEC>
__global__ __launch_bounds__(NTH) void dw_kernel(const X* __restrict__ x, const float* __restrict__ dl, int T, int d, int E, int range, float* __restrict__ part) {
#ifdef __HIP_DEVICE_COMPILE__
    constexpr int NX = PARTS<X>, BUF = (NX + 6) * PANEL;   // x's parts, then dl's: [part][two panels]
    __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * BUF];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, lq = lane >> 4;
    const int c0 = blockIdx.x * 64, e0 = blockIdx.y * 128, first = blockIdx.z * range, last = first + range < T ? first + range : T;
    // a thread has eight columns of x and, twice, eight experts of dl
    const int xr = tid >> 3, xc = (tid & 7) * 8, er = tid >> 4, ec = (tid & 15) * 8;
    // (two sets: what the step after the next needs is on its way)
    typename Eight<X>::type gx[2];
    f32x8 ge[2][2];
    float db[8] = {};
    auto fetch = [&](int t0, int set) {
        const unsigned rows = (unsigned)(last - t0 < 0 ? 0 : last - t0 < TC ? last - t0 : TC);
        const __amdgpu_buffer_rsrc_t rx = make_rsrc(x + (size_t)t0 * d, x ? rows * (unsigned)d * (unsigned)sizeof(X) : 0u), rl = make_rsrc(dl + (size_t)t0 * E, rows * (unsigned)E * 4u);
        gx[set] = fetch8<8>(x, rx, d, (unsigned)xr, c0 + xc, true);
#pragma unroll
        for (int i = 0; i < 2; ++i) ge[set][i] = fetch8<VEC>(dl, rl, E, (unsigned)(er + i * 16), e0 + ec, true);
    };
    f32x4 acc[4][2] = {};
    auto step = [&](int t0, int buf) {
        unsigned char* to = lds + buf * BUF;
        put8(to + panel_at(xr, xc), PANEL, take_apart(gx[buf]));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            put8(to + NX * PANEL + (ec >> 6) * PANEL + panel_at(er + i * 16, ec & 63), 2 * PANEL, take_apart(ge[buf][i]));
#pragma unroll
            for (int c = 0; c < 8; ++c) db[c] += ge[buf][i][c];
        }
        fetch(t0 + 2 * TC, buf);                           // (behind the range: zeros)
        __syncthreads();                                   // (one is enough: whoever writes this buffer again has passed the next)
        const unsigned char* from = lds + buf * BUF;
        Parts<3> e[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 3; ++i) e[b].p[i] = read_transposed(from + (NX + 2 * i + (wave >> 1)) * PANEL, (wave & 1) * 2 + b, l16, lq);
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            Parts<NX> v;
#pragma unroll
            for (int i = 0; i < NX; ++i) v.p[i] = read_transposed(from + i * PANEL, m, l16, lq);
#pragma unroll
            for (int b = 0; b < 2; ++b) multiply(e[b], v, acc[m][b]);
        }
    };
    fetch(first, 0);
    fetch(first + TC, 1);
    for (int t0 = first; t0 < last; t0 += 2 * TC) {
        step(t0, 0);
        if (t0 + TC < last) step(t0 + TC, 1);
    }
    // part: [range][d + 1][E], the last row for db
    float* to = part + (size_t)blockIdx.z * (d + 1) * E;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const int c = c0 + m * 16 + l16;
        if (c >= d || !x) continue;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int e = e0 + wave * 32 + b * 16 + lq * 4;
            if constexpr (VEC >= 4) {
                if (e < E) *(f32x4*)(to + (size_t)c * E + e) = acc[m][b];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (e + i < E) to[(size_t)c * E + e + i] = acc[m][b][i];
            }
        }
    }
    if (blockIdx.x == 0) {                                 // sixteen threads have each column
        float* sums = (float*)lds;
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 8; ++c) sums[er * 128 + ec + c] = db[c];
        __syncthreads();
        if (tid < 128 && e0 + tid < E) {
            float s = 0.f;
            for (int r = 0; r < 16; ++r) s += sums[r * 128 + tid];
            to[(size_t)d * E + e0 + tid] = s;
        }
    }
#endif
}
__global__ __launch_bounds__(NTH) void dw_sum_kernel(const float* __restrict__ part, int ranges, int d, int E, float* __restrict__ dw, float* __restrict__ db) {
    const size_t i = (size_t)blockIdx.x * NTH + threadIdx.x, n = (size_t)d * E, step = n + E;
    if (i >= step) return;
    float s = 0.f;
#pragma unroll 8
    for (int r = 0; r < ranges; ++r) s += part[r * step + i];
    if (i < n) {
        if (dw) dw[i] = s;
    } else if (db) {
        db[i - n] = s;
    }
}

// Ranges of tokens that dW_g is summed over: enough work-groups for the chip, 64 tokens at least.
int ranges_of(int T, int d, int E) {
    const int tiles = ((d + 63) / 64) * ((E + 127) / 128);
    int n = 512 / tiles;                                   // (two work-groups a CU, and not one more than that)
    const int most = (T + 63) / 64;
    if (n > most) n = most;
    if (n < 1) n = 1;
    const int range = ((T + n - 1) / n + TC - 1) / TC * TC;
    return range > 0 ? (T + range - 1) / range : 1;
}

template <typename F> void by_vec(int vec, F&& f) {
    if (vec == 8) f(std::integral_constant<int, 8>{});
    else if (vec == 4) f(std::integral_constant<int, 4>{});
    else f(std::integral_constant<int, 1>{});
}
template <typename W> void launch_dx(const W* w, int vec, const float* dl, const float* add, int T, int d, int E, float* dx, hipStream_t st) {
    // columns a work-group: as many as leave three of them a CU, 128 at least
    const int tt = E <= 128 ? 64 : 32, groups = (T + tt - 1) / tt;
    int splits = (768 + groups - 1) / groups;
    const int columns = ((d + splits - 1) / splits + 127) / 128 * 128;
    splits = (d + columns - 1) / columns;
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(groups, splits), dim3(NTH), 0, st, dl, w, add, T, d, E, columns, dx); };
    auto by_size = [&](auto v) {
        constexpr int V = decltype(v)::value;
        if (E <= 32) go(dx_kernel<W, 1, V>);
        else if (E <= 64) go(dx_kernel<W, 2, V>);
        else if (E <= 128) go(dx_kernel<W, 4, V>);
        else go(dx_kernel<W, 8, V>);
    };
    by_vec(vec, by_size);
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
    MOE_REQUIRE(T <= 64 * 65535 && d <= (1 << 20), MOE_ERR_UNSUPPORTED, "%s: T=%d d=%d", me, T, d);
    const bool sums = dw_gate || dbias;
    const size_t need = sums ? moe_route_back_bytes(T, d, E) : 0;
    if (T > 0) {
        MOE_REQUIRE(dgate_w && gate_w && expert_idx && (logits || renorm) && dlogits && (w_gate || !dx) && (x || !dw_gate), MOE_ERR_ARG, "%s: null pointer", me);
        MOE_REQUIRE(!sums || (ws && ws_bytes >= need), MOE_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", me, ws_bytes, need);
        MOE_REQUIRE((((uintptr_t)dx | (uintptr_t)dx_add | (uintptr_t)x) & 15) == 0 && (((uintptr_t)ws | (uintptr_t)dlogits) & 3) == 0, MOE_ERR_UNSUPPORTED,
                    "%s: x, dx and dx_add have to be aligned to 16 bytes", me);
    }
    if (T == 0 && !sums) return MOE_OK;
    const hipStream_t st = (hipStream_t)stream;
    int ranges = 0;
    if (T > 0) {
        auto first = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((T + 3) / 4), dim3(NTH), 0, st, dgate_w, gate_w, expert_idx, logits, dlogits_add, T, E, k, renorm, dlogits); };
        E <= 64 ? first(dlogits_kernel<1>) : E <= 128 ? first(dlogits_kernel<2>) : first(dlogits_kernel<4>);
        const int vec = (((uintptr_t)dlogits | (uintptr_t)w_gate | (uintptr_t)ws) & 15) != 0 ? 1 : E % 8 == 0 ? 8 : E % 4 == 0 ? 4 : 1;
        if (dx) dt == MOE_F32 ? launch_dx((const float*)w_gate, vec, dlogits, dx_add, T, d, E, dx, st) : launch_dx((const uint16_t*)w_gate, vec, dlogits, dx_add, T, d, E, dx, st);
        if (sums) {
            ranges = ranges_of(T, d, E);
            const int range = ((T + ranges - 1) / ranges + TC - 1) / TC * TC;
            const dim3 grid(dw_gate ? (d + 63) / 64 : 1, (E + 127) / 128, ranges);
            auto go = [&](auto kern, auto* from) { hipLaunchKernelGGL(kern, grid, dim3(NTH), 0, st, dw_gate ? from : nullptr, dlogits, T, d, E, range, (float*)ws); };
            by_vec(vec < 4 ? 1 : 4, [&](auto v) {          // (dl and the sums are fp32)
                constexpr int V = decltype(v)::value == 8 ? 4 : decltype(v)::value;
                dt == MOE_F32 ? go(dw_kernel<float, V>, (const float*)x) : go(dw_kernel<uint16_t, V>, (const uint16_t*)x);
            });
        }
    }
    if (sums) {
        const size_t n = (size_t)(d + 1) * E;
        hipLaunchKernelGGL(dw_sum_kernel, dim3((unsigned)((n + NTH - 1) / NTH)), dim3(NTH), 0, st, (const float*)ws, ranges, d, E, dw_gate, dbias);
    }
    MOE_CHECK_LAUNCH("moe_route_topk_backward");
    return MOE_OK;
}
