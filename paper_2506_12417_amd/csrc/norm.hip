// The norms before and after a block with its gate and residual scale (moe_norm, moe_block_end,
// moe_block_end_rows) and their gradients.  One row:
//
//   p = n_post(v) w_p + b_p   (or v)      y = alpha h + gate p      u = n_next(y) w_n + b_n
//   n(x) = (x - m) r,   r = 1 / sqrt(mean((x - m)^2) + eps),   m = mean(x) (LAYER) or 0 (RMS)
//
// moe_norm is the last of the three with y = h.  Gradients, from gy' = dy and du, with yn = n_next(y), vn = n_post(v):
//
//   gn = du w_n    gy = dy + r_n (gn - [LAYER] mean(gn) - yn mean(gn yn))     dh = alpha gy     dgate = sum gy p
//   dp = gate gy   gv = dp w_p     dv = r_p (gv - [LAYER] mean(gv) - vn mean(gv vn))
//   dw_n = sum du yn     db_n = sum du     dw_p = sum dp vn     db_p = sum dp        (sums over the rows)
//
// What bounds it: HBM; in calls of few rows the launch and one chain of load, sums over the row, store.  A row is
// held in registers, eight values a thread, so that every tensor is read once and the statistics take two passes over registers
// (mean first, then squares of the differences).  A work-group keeps its columns of the parameters in registers and goes over
// rows, the next row's loads under way while the present one is summed up (at a block's end, backward, rows of more than 4096
// values leave a thread no registers for either: they fetch the parameters again for every row, 4096 x 8192 in 200 us).  All
// arithmetic is fp32; the outputs are rounded once, and u is made of the unrounded y.  The parameters' gradients are summed over a work-group's rows in registers, written
// to the workspace and added up by a second launch in a fixed order: no atomics.
//
// Measured (medians of 50 launches, each by itself; the least are up to a fifth shorter): 16384 x 2048, 16-bit, LAYER, 29 us forward (134 MB, 4.6 TB/s; a copy
// of 1 GiB reaches 5.2) and 51 + 7 backward with the residual stream's gradient (268 MB, 5.3); 8192 x 4096, both norms, 58 forward (268 MB, 4.7) and
// 78 + 7 backward (402 MB, 5.2); the rows form with four experts' rows and a shared one each, 8192 x 2048 88 (438 MB, 5.0), 2048 x 8192 the
// same, 33 x 2048 4.2; 1501 x 777 fp32 4.2, 5.8 + 4.4; 33 x 2048 3 - 3.5.  Beyond 4096 columns, 8192 x 5120, 7168 and 8192 forward 47, 64, 61 and
// backward 67, 133, 102 (+ 8); both norms, 4096 rows of these, 50, 52, 56 and 104, 170, 200 (+ 6).
#include "common.h"
#include "gemm_util.h"
#include <climits>
#include <type_traits>

namespace {

typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;

constexpr int V = 8;                     // values of a row per thread
constexpr int MAXT = 512, MAXT_LONG = 1024;      // threads per row, and in rows of more than 4096 values (LONG)
constexpr int MAXW = MAXT_LONG / 64;
static_assert(MAXT_LONG * V == MOE_NORM_MAX_D && MAXT * V == MOE_NORM_ANY_D, "");

enum { SRC_NONE = 0, SRC_TENSOR = 1, SRC_ROWS = 2 };

// ---- a thread's values of a row: neighbours (VEC, one or two 16-byte pieces) where rows are whole 16-byte pieces, else
// every 64th of its wavefront's
template <bool VEC> __device__ __forceinline__ int column(int i) {
    return VEC ? (int)threadIdx.x * V + i : ((int)threadIdx.x & ~63) * V + i * 64 + ((int)threadIdx.x & 63);
}

// All goes through buffer loads and stores: what lies past the row's d values, or in a row that is not there (`on` false), reads as zero or
// is not written, without a branch; behind branches with loads in them the compiler waits for all that is under way, the next row's
// loads included (8192 x 4096, both norms, the least of 50: 61 forward + 91 us backward, against 50 + 76).
template <typename E, bool VEC> struct Held;
template <> struct Held<float, true> {
    f32x4 a, b;
    __device__ __forceinline__ void fetch(const float* row, int d, bool on) {
        const __amdgpu_buffer_rsrc_t r = make_rsrc(row, on ? (unsigned)d * 4u : 0u);
        a = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, column<true>(0) * 4, 0, 0));
        b = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, column<true>(4) * 4, 0, 0));
    }
    __device__ __forceinline__ float at(int i) const { return i < 4 ? a[i & 3] : b[i & 3]; }
};
template <> struct Held<uint16_t, true> {
    u32x4 a;
    __device__ __forceinline__ void fetch(const uint16_t* row, int d, bool on) {
        a = __builtin_amdgcn_raw_buffer_load_b128(make_rsrc(row, on ? (unsigned)d * 2u : 0u), column<true>(0) * 2, 0, 0);
    }
    __device__ __forceinline__ float at(int i) const {
        const unsigned w = a[i >> 1];
        return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
    }
};
template <typename E> struct Held<E, false> {
    E a[V];
    __device__ __forceinline__ void fetch(const E* row, int d, bool on) {
        const __amdgpu_buffer_rsrc_t r = make_rsrc(row, on ? (unsigned)d * (unsigned)sizeof(E) : 0u);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if constexpr (sizeof(E) == 4) a[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(r, column<false>(i) * 4, 0, 0));
            else a[i] = __builtin_amdgcn_raw_buffer_load_b16(r, column<false>(i) * 2, 0, 0);
        }
    }
    __device__ __forceinline__ float at(int i) const { return load_as_f32(&a[i]); }
};

template <bool VEC> __device__ __forceinline__ void store(float* row, int d, const float (&x)[V], bool on) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(row, on ? (unsigned)d * 4u : 0u);
    if constexpr (VEC) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{x[0], x[1], x[2], x[3]}), r, column<true>(0) * 4, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{x[4], x[5], x[6], x[7]}), r, column<true>(4) * 4, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x[i]), r, column<false>(i) * 4, 0, 0);
    }
}
template <bool VEC> __device__ __forceinline__ void store(uint16_t* row, int d, const float (&x)[V], bool on) {
    const __amdgpu_buffer_rsrc_t r = make_rsrc(row, on ? (unsigned)d * 2u : 0u);
    if constexpr (VEC) {
        const f32x8 f = {x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]};
        const bf16x8 to = __builtin_convertvector(f, bf16x8);    // to nearest, ties to even
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, to), r, column<true>(0) * 2, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, (__bf16)x[i]), r, column<false>(i) * 2, 0, 0);
    }
}
// a parameter's columns; `none` where there is no such parameter
template <bool VEC> __device__ __forceinline__ void params(const float* p, int d, float none, float (&to)[V]) {
    Held<float, VEC> t;
    t.fetch(p, d, p != nullptr);
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = p ? t.at(i) : none;
}

// ---- sums over a row: lanes by exchanges, wavefronts through LDS.  Every thread gets the same bits.  Two buffers in
// turn: whoever writes one again has passed the barrier behind which all have read it.
__device__ __forceinline__ float lanes16_sum(float v) {
    v += __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), 0xB1, 0xf, 0xf, false));     // quad_perm [1,0,3,2]
    v += __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), 0x4E, 0xf, 0xf, false));     // quad_perm [2,3,0,1]
    v += __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), 0x141, 0xf, 0xf, false));    // row_half_mirror
    v += __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), 0x140, 0xf, 0xf, false));    // row_mirror
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
    v = lanes16_sum(v);
    const int i = __float_as_int(v);
    return (__int_as_float(__builtin_amdgcn_readlane(i, 0)) + __int_as_float(__builtin_amdgcn_readlane(i, 16))) +
           (__int_as_float(__builtin_amdgcn_readlane(i, 32)) + __int_as_float(__builtin_amdgcn_readlane(i, 48)));
}
struct RowSum {
    float (*red)[2][MAXW];               // [buffer][value][wavefront]
    int waves, turn;
    __device__ __forceinline__ void operator()(float& a, float& b, bool both) {
        a = wave_sum(a);
        if (both) b = wave_sum(b);
        if (waves > 1) {
            const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
            if (lane == 0) { red[turn][0][wave] = a; red[turn][1][wave] = b; }
            __syncthreads();
            const int at = lane & 15;
            a = red[turn][0][at];        // (past the wavefronts: whatever is there)
            a = lanes16_sum(at < waves ? a : 0.f);
            if (both) {
                b = red[turn][1][at];
                b = lanes16_sum(at < waves ? b : 0.f);
            }
            turn ^= 1;
        }
    }
    __device__ __forceinline__ void operator()(float& a) { float b = 0.f; (*this)(a, b, false); }
};

// x -> n(x); m and r are returned
template <bool VEC>
__device__ __forceinline__ void normalise(float (&x)[V], int kind, float eps, int d, float inv_d, RowSum& sum, float& m, float& r) {
    m = 0.f;
    if (kind == MOE_NORM_LAYER) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) s += x[i];                   // (columns past d hold zeros)
        sum(s);
        m = s * inv_d;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = column<VEC>(i) < d ? x[i] - m : 0.f;
    }
    float q = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) q = fmaf(x[i], x[i], q);
    sum(q);
    r = 1.f / sqrtf(fmaf(q, inv_d, eps));
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] *= r;
}

struct Args {
    const void* v;                       // [T,d], or the experts' rows [T k, d] fp32
    const void* h;                       // [T,d]
    const float *post_w, *post_b, *gate, *next_w, *next_b;
    int T, d, post_kind, next_kind, gate_rows, k;
    int waves, step;                     // of a row; rows in work at a time
    float post_eps, next_eps, alpha, inv_d;
    const int32_t* inv_perm;             // experts' rows only, as gate_w and shared
    const float *gate_w, *shared;
    void *y, *u;                         // (y is null for moe_norm)
    float* stats;                        // [T,4] or, for moe_norm, [T,2]
};

// the experts' rows of a token, weighted and summed as moe_unpermute_combine does it, G of them asked for together
template <int G, bool VEC>
__device__ __forceinline__ void combine_row(const Args& p, int t, float (&x)[V]) {
    const float* rows = (const float*)p.v;
    const size_t a0 = (size_t)t * p.k;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = 0.f;
    Held<float, VEC> s;
    s.fetch(p.shared + (size_t)t * p.d, p.d, p.shared != nullptr);
    for (int j0 = 0; j0 < p.k; j0 += G) {
        Held<float, VEC> r[G];
        float w[G];
        int at[G];
#pragma unroll
        for (int j = 0; j < G; ++j) {
            const int jj = j0 + j < p.k ? j0 + j : p.k - 1;
            w[j] = p.gate_w ? p.gate_w[a0 + jj] : 1.f;
            at[j] = p.inv_perm[a0 + jj];
            r[j].fetch(rows + (size_t)(at[j] < 0 ? 0 : at[j]) * p.d, p.d, true);
        }
#pragma unroll
        for (int j = 0; j < G; ++j)
            if (j0 + j < p.k) {
                const float none = w[j] == 0.f ? 0.f : __builtin_nanf("");
#pragma unroll
                for (int i = 0; i < V; ++i) x[i] = fmaf(w[j], at[j] < 0 ? none : r[j].at(i), x[i]);
            }
    }
    if (p.shared) {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] += s.at(i);
    }
    // (a missing row makes NaN of the columns past d too)
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = column<VEC>(i) < p.d ? x[i] : 0.f;
}

template <typename VT, typename HT, typename UT, bool VEC, int SRC, int G, bool LONG>
__global__ __launch_bounds__(LONG ? MAXT_LONG : MAXT) void norm_kernel(Args p) {
    __shared__ float red[2][2][MAXW];
    RowSum sum = {red, p.waves, 0};
    const int d = p.d, step = p.step;
    float pw[V], pb[V], gate[V], nw[V], nb[V];
    const bool own = SRC != SRC_NONE && p.gate_rows > 1;
    Held<VT, VEC> v_next;
    Held<HT, VEC> h_next;
    Held<float, VEC> gate_next;
    auto fetch = [&](int t) __attribute__((always_inline)) {
        const bool on = t < p.T;
        const size_t at = (size_t)t * d;
        if constexpr (SRC == SRC_TENSOR) v_next.fetch((const VT*)p.v + at, d, on);
        h_next.fetch((const HT*)p.h + at, d, on);
        if constexpr (SRC != SRC_NONE) gate_next.fetch(p.gate + at, d, on && own);
    };
    // a row's mean and factor, by one thread
    auto keep = [&](int t, int which, float m, float r) __attribute__((always_inline)) {
        constexpr int S = SRC == SRC_NONE ? 2 : 4;
        const __amdgpu_buffer_rsrc_t to = make_rsrc(p.stats + (size_t)t * S, p.stats ? S * 4u : 0u);
        __builtin_amdgcn_raw_buffer_store_b64(u32x2{__float_as_uint(m), __float_as_uint(r)}, to, threadIdx.x == 0 ? which * 8 : S * 4, 0, 0);
    };
    int t = sgpr((int)(blockIdx.x * blockDim.y + threadIdx.y));  // (a wavefront for itself, or one row for all)
    fetch(t);
    params<VEC>(SRC == SRC_NONE ? nullptr : p.post_w, d, 1.f, pw);
    params<VEC>(SRC == SRC_NONE ? nullptr : p.post_b, d, 0.f, pb);
    params<VEC>(SRC == SRC_NONE || p.gate_rows != 1 ? nullptr : p.gate, d, 1.f, gate);
    params<VEC>(p.next_w, d, 1.f, nw);
    params<VEC>(p.next_b, d, 0.f, nb);
    for (; t < p.T; t += step) {
        const Held<VT, VEC> v = v_next;
        const Held<HT, VEC> h = h_next;
        const size_t at = (size_t)t * d;
        float y[V];
        float m = 0.f, r = 0.f;
        const Held<float, VEC> own_gate = gate_next;
        if constexpr (SRC == SRC_ROWS) combine_row<G, VEC>(p, t, y);
        fetch(t + step);
        if constexpr (SRC == SRC_NONE) {
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = h.at(i);
        } else {
            if constexpr (SRC == SRC_TENSOR) {
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = v.at(i);
            }
            if (p.post_kind != MOE_NORM_NONE) {
                normalise<VEC>(y, p.post_kind, p.post_eps, d, p.inv_d, sum, m, r);
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = fmaf(y[i], pw[i], pb[i]);
            }
            if constexpr (SRC == SRC_TENSOR) keep(t, 0, m, r);
            if (own) {
#pragma unroll
                for (int i = 0; i < V; ++i) gate[i] = own_gate.at(i);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = fmaf(p.alpha, h.at(i), gate[i] * y[i]);       // (past d: v, h and post_b are zero)
            store<VEC>((HT*)p.y + at, d, y, true);
        }
        if (p.next_kind != MOE_NORM_NONE) {
            normalise<VEC>(y, p.next_kind, p.next_eps, d, p.inv_d, sum, m, r);
            if constexpr (SRC != SRC_ROWS) keep(t, SRC == SRC_NONE ? 0 : 1, m, r);
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = fmaf(y[i], nw[i], nb[i]);
            store<VEC>((UT*)p.u + at, d, y, true);
        }
    }
}

// ---- gradients
enum { D_NEXT_W = 0, D_NEXT_B = 1, D_GATE = 2, D_POST_W = 3, D_POST_B = 4, N_GRADS = 5 };
struct Grads {
    const void *dy, *du;                 // either may be null
    void *dv, *dh;
    float* dgate;                        // the gate of every token's own: [T,d]; else null
    float* part;                         // partial sums [work-group or wavefront][slots][d]
    int slot[N_GRADS];                   // where in them a parameter's gradient stands, -1: not wanted
    int slots;
};

// A thread's sums of the parameters' gradients over its rows: registers, and in long rows, where these do not suffice,
// LDS of its own for all but one.
template <bool LONG> struct Sums {
    float reg[N_GRADS][V];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int g = 0; g < N_GRADS; ++g)
#pragma unroll
            for (int i = 0; i < V; ++i) reg[g][i] = 0.f;
    }
    template <int W, typename F> __device__ __forceinline__ void add(F f) {
#pragma unroll
        for (int i = 0; i < V; ++i) reg[W][i] = f(i, reg[W][i]);
    }
};
__shared__ f32x4 long_sums[(N_GRADS - 1) * (V / 4)][MAXT_LONG];
template <> struct Sums<true> {
    float reg[V];
    static constexpr int slot(int w) { return (w > D_GATE ? w - 1 : w) * (V / 4); }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < (N_GRADS - 1) * (V / 4); ++i) long_sums[i][threadIdx.x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < V; ++i) reg[i] = 0.f;
    }
    template <int W, typename F> __device__ __forceinline__ void add(F f) {
        if constexpr (W == D_GATE) {
#pragma unroll
            for (int i = 0; i < V; ++i) reg[i] = f(i, reg[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V; i += 4) {
                f32x4 s = long_sums[slot(W) + i / 4][threadIdx.x];
#pragma unroll
                for (int j = 0; j < 4; ++j) s[j] = f(i + j, s[j]);
                long_sums[slot(W) + i / 4][threadIdx.x] = s;
            }
        }
    }
};

template <typename VT, typename HT, typename UT, bool VEC, bool HAS_V, bool LONG>
__global__ __launch_bounds__(LONG ? MAXT_LONG : MAXT) void norm_back_kernel(Args p, Grads q) {
    constexpr bool TIGHT = LONG && HAS_V;        // too few registers for parameters, sums and the next row
    __shared__ float red[2][2][MAXW];
    RowSum sum = {red, p.waves, 0};
    const int d = p.d, step = p.step, first = sgpr((int)(blockIdx.x * blockDim.y + threadIdx.y));
    constexpr int S = HAS_V ? 4 : 2;
    const bool own = HAS_V && p.gate_rows > 1;
    float pw[V], pb[V], gate[V], nw[V];
    auto post_params = [&]() __attribute__((always_inline)) {
        params<VEC>(HAS_V ? p.post_w : nullptr, d, 1.f, pw);
        params<VEC>(HAS_V ? p.post_b : nullptr, d, 0.f, pb);
    };
    auto gate_params = [&]() __attribute__((always_inline)) { params<VEC>(!HAS_V || p.gate_rows != 1 ? nullptr : p.gate, d, 1.f, gate); };
    auto next_params = [&]() __attribute__((always_inline)) { params<VEC>(p.next_w, d, 1.f, nw); };
    Sums<TIGHT> acc;
    acc.clear();
    Held<VT, VEC> v_next;
    Held<HT, VEC> h_next, dy_next;
    Held<UT, VEC> du_next;
    Held<float, VEC> gate_next;
    u32x4 st_next = {};
    auto fetch = [&](int t) __attribute__((always_inline)) {
        const bool on = t < p.T;
        const size_t at = (size_t)t * d;
        const __amdgpu_buffer_rsrc_t stats = make_rsrc(p.stats + (size_t)t * S, on ? S * 4u : 0u);
        if constexpr (HAS_V) {
            st_next = __builtin_amdgcn_raw_buffer_load_b128(stats, 0, 0, 0);
        } else {
            const u32x2 two = __builtin_amdgcn_raw_buffer_load_b64(stats, 0, 0, 0);
            st_next = u32x4{two[0], two[1], 0u, 0u};
        }
        if constexpr (HAS_V) v_next.fetch((const VT*)p.v + at, d, on);
        h_next.fetch((const HT*)p.h + at, d, on);
        dy_next.fetch((const HT*)q.dy + at, d, on && q.dy);
        du_next.fetch((const UT*)q.du + at, d, on && q.du);
        if constexpr (HAS_V) gate_next.fetch(p.gate + at, d, on && own);
    };
    if (!TIGHT) { fetch(first); post_params(); gate_params(); next_params(); }
    for (int t = first; t < p.T; t += step) {
        if (TIGHT) { fetch(t); post_params(); gate_params(); }
        const Held<VT, VEC> v = v_next;
        const Held<HT, VEC> h = h_next, dy = dy_next;
        const Held<UT, VEC> du = du_next;
        const size_t at = (size_t)t * d;
        const Held<float, VEC> own_gate = gate_next;
        float st[S];
#pragma unroll
        for (int i = 0; i < S; ++i) st[i] = __uint_as_float(st_next[i]);
        if (!TIGHT) fetch(t + step);
        float vn[V], y[V], gy[V];
        const bool next_layer = p.next_kind == MOE_NORM_LAYER, post_layer = p.post_kind == MOE_NORM_LAYER;
        // (Past d everything is zero, but for what LAYER subtracts the mean from.)
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = h.at(i);
        if constexpr (HAS_V) {
            if (own) {
#pragma unroll
                for (int i = 0; i < V; ++i) gate[i] = own_gate.at(i);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) vn[i] = v.at(i);
            if (post_layer) {
#pragma unroll
                for (int i = 0; i < V; ++i) vn[i] = column<VEC>(i) < d ? vn[i] - st[0] : 0.f;
            }
            if (p.post_kind != MOE_NORM_NONE) {
#pragma unroll
                for (int i = 0; i < V; ++i) vn[i] *= st[1];
            }
#pragma unroll
            for (int i = 0; i < V; ++i) y[i] = fmaf(p.alpha, y[i], gate[i] * fmaf(vn[i], pw[i], pb[i]));     // (without a norm pw is 1 and pb 0)
        }
#pragma unroll
        for (int i = 0; i < V; ++i) gy[i] = 0.f;
        if (q.dy) {
#pragma unroll
            for (int i = 0; i < V; ++i) gy[i] = dy.at(i);
        }
        if (q.du) {
            float a = 0.f, b = 0.f, gn[V];
            if (TIGHT) next_params();
            if (next_layer) {
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = column<VEC>(i) < d ? y[i] - st[S - 2] : 0.f;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                y[i] *= st[S - 1];
                gn[i] = du.at(i) * nw[i];
                a = fmaf(gn[i], y[i], a);
            }
            if (next_layer) {
#pragma unroll
                for (int i = 0; i < V; ++i) b += gn[i];
            }
            if (q.slot[D_NEXT_W] >= 0) acc.template add<D_NEXT_W>([&](int i, float s) __attribute__((always_inline)) { return fmaf(du.at(i), y[i], s); });
            if (q.slot[D_NEXT_B] >= 0) acc.template add<D_NEXT_B>([&](int i, float s) __attribute__((always_inline)) { return s + du.at(i); });
            sum(a, b, next_layer);
            a *= p.inv_d;
            if (next_layer) {
                b *= p.inv_d;
#pragma unroll
                for (int i = 0; i < V; ++i) gn[i] -= b;
            }
#pragma unroll
            for (int i = 0; i < V; ++i) gy[i] = fmaf(st[S - 1], fmaf(-y[i], a, gn[i]), gy[i]);
        }
        float out[V];
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = HAS_V ? p.alpha * gy[i] : gy[i];
        store<VEC>((HT*)q.dh + at, d, out, q.dh != nullptr);
        if constexpr (HAS_V) {
            float a = 0.f, b = 0.f;
            if (TIGHT) { post_params(); gate_params(); }
            if (TIGHT && own) {
                Held<float, VEC> again;
                again.fetch(p.gate + at, d, true);
#pragma unroll
                for (int i = 0; i < V; ++i) gate[i] = again.at(i);
            }
            if (q.slot[D_GATE] >= 0)
                acc.template add<D_GATE>([&](int i, float s) __attribute__((always_inline)) { return fmaf(gy[i], fmaf(vn[i], pw[i], pb[i]), s); });
            if (q.dgate) {
#pragma unroll
                for (int i = 0; i < V; ++i) out[i] = gy[i] * fmaf(vn[i], pw[i], pb[i]);
                store<VEC>(q.dgate + at, d, out, true);
            }
#pragma unroll
            for (int i = 0; i < V; ++i) gy[i] *= gate[i];        // dp
            if (q.slot[D_POST_W] >= 0) acc.template add<D_POST_W>([&](int i, float s) __attribute__((always_inline)) { return fmaf(gy[i], vn[i], s); });
            if (q.slot[D_POST_B] >= 0) acc.template add<D_POST_B>([&](int i, float s) __attribute__((always_inline)) { return s + gy[i]; });
            if (p.post_kind != MOE_NORM_NONE) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    gy[i] *= pw[i];
                    a = fmaf(gy[i], vn[i], a);
                }
                if (post_layer) {
#pragma unroll
                    for (int i = 0; i < V; ++i) b += column<VEC>(i) < d ? gy[i] : 0.f;
                }
                sum(a, b, post_layer);
                a *= p.inv_d;
                if (post_layer) {
                    b *= p.inv_d;
#pragma unroll
                    for (int i = 0; i < V; ++i) gy[i] -= b;
                }
#pragma unroll
                for (int i = 0; i < V; ++i) gy[i] = st[1] * fmaf(-vn[i], a, gy[i]);
            }
            store<VEC>((VT*)q.dv + at, d, gy, q.dv != nullptr);
        }
    }
    auto put = [&](auto which) __attribute__((always_inline)) {
        constexpr int W = decltype(which)::value;
        if (q.slot[W] < 0) return;
        float s[V];
        acc.template add<W>([&](int i, float v) __attribute__((always_inline)) { return s[i] = v; });
        store<VEC>(q.part + ((size_t)first * q.slots + q.slot[W]) * d, d, s, true);
    };
    put(std::integral_constant<int, D_NEXT_W>{});
    put(std::integral_constant<int, D_NEXT_B>{});
    if constexpr (HAS_V) {
        put(std::integral_constant<int, D_GATE>{});
        put(std::integral_constant<int, D_POST_W>{});
        put(std::integral_constant<int, D_POST_B>{});
    }
}

// The partial sums of 16 columns of one parameter, in a fixed order: 64 threads a column, 16 parts each at most, asked for together, then
// four lanes, then the sixteen wavefronts.  (64 columns a work-group are 26 work-groups for two gradients of 777 columns, and took 7.7 us
// for 1024 parts there.)
struct Outs { float* out[N_GRADS]; };
__global__ __launch_bounds__(1024) void sum_parts_kernel(const float* __restrict__ part, int n, int slots, int d, Outs o) {
    __shared__ float s[16][16];
    const int lane = threadIdx.x & 15, row = threadIdx.x >> 4, c = (int)blockIdx.x * 16 + lane, slot = (int)blockIdx.y;
    const float* from = part + (size_t)slot * d + (c < d ? c : 0);
    const size_t pitch = (size_t)slots * d;
    float a[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) a[j] = row + 64 * j < n ? from[(row + 64 * j) * pitch] : 0.f;
#pragma unroll
    for (int w = 8; w; w >>= 1)
#pragma unroll
        for (int j = 0; j < w; ++j) a[j] += a[j + w];
    float v = a[0];
    v += __shfl_xor(v, 16);
    v += __shfl_xor(v, 32);
    if ((threadIdx.x & 63) < 16) s[threadIdx.x >> 6][lane] = v;
    __syncthreads();
    if (threadIdx.x < 16 && c < d) {
        v = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w) v += s[w][lane];
        o.out[slot][c] = v;
    }
}

// ---- launches
bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }

struct Shape { dim3 grid, block; };
// Threads for a row: whole wavefronts, as few as its values need.  Up to 512 columns a wavefront has a row for itself,
// four of them in a work-group.  waves: wavefronts per CU that the kernel's registers leave room for; parts: rows in work at most.
Shape shape(int T, int d, int waves, int parts) {
    const int g = (d + 64 * V - 1) / (64 * V) * 64;
    const int rows = g == 64 ? 4 : 1;
    int blocks = (T + rows - 1) / rows, most = 256 * waves * 64 / (g * rows);
    if (most > parts / rows) most = parts / rows;
    if (blocks > most) blocks = (blocks + (blocks + most - 1) / most - 1) / ((blocks + most - 1) / most);     // (as many rows each)
    return {dim3((unsigned)(blocks < 1 ? 1 : blocks)), dim3((unsigned)g, (unsigned)rows)};
}
Shape forward_shape(int T, int d) { return shape(T, d, 32, 1 << 30); }
// (a row in work is a row of partial sums)
Shape backward_shape(int T, int d, bool has_v) { return shape(T, d, has_v ? 8 : 16, 1024); }

template <typename F> void by_type(int dt, F f) {
    if (dt == MOE_BF16) f(uint16_t{});
    else f(float{});
}

template <int SRC, int G>
int launch_forward(const char* who, Args a, int v_dt, int h_dt, int u_dt, bool vec, hipStream_t st) {
    MOE_REQUIRE(vec || a.d <= MOE_NORM_ANY_D, MOE_ERR_UNSUPPORTED, "%s: d=%d beyond %d needs multiples of 8 and pointers aligned to 16 bytes", who,
                a.d, MOE_NORM_ANY_D);
    const Shape s = forward_shape(a.T, a.d);
    a.waves = (int)s.block.x / 64;
    a.step = (int)(s.grid.x * s.block.y);
    by_type(SRC == SRC_TENSOR ? v_dt : MOE_F32, [&](auto vt) {
        by_type(h_dt, [&](auto ht) {
            by_type(u_dt, [&](auto ut) {
                typedef decltype(vt) VT;
                typedef decltype(ht) HT;
                typedef decltype(ut) UT;
                if constexpr (SRC == SRC_TENSOR || std::is_same<VT, float>::value) {
                    if (a.d > MOE_NORM_ANY_D) hipLaunchKernelGGL((norm_kernel<VT, HT, UT, true, SRC, G < 2 ? G : 2, true>), s.grid, s.block, 0, st, a);
                    else if (vec) hipLaunchKernelGGL((norm_kernel<VT, HT, UT, true, SRC, G, false>), s.grid, s.block, 0, st, a);
                    else hipLaunchKernelGGL((norm_kernel<VT, HT, UT, false, SRC, G, false>), s.grid, s.block, 0, st, a);
                }
            });
        });
    });
    MOE_CHECK_LAUNCH(who);
    return MOE_OK;
}

template <bool HAS_V>
int launch_backward(const char* who, Args a, Grads q, float* const (&want)[N_GRADS], int v_dt, int h_dt, int u_dt, bool vec, hipStream_t st) {
    MOE_REQUIRE(vec || a.d <= MOE_NORM_ANY_D, MOE_ERR_UNSUPPORTED, "%s: d=%d beyond %d needs multiples of 8 and pointers aligned to 16 bytes", who,
                a.d, MOE_NORM_ANY_D);
    Outs o = {};
    q.slots = 0;
    for (int g = 0; g < N_GRADS; ++g) {
        q.slot[g] = want[g] ? q.slots : -1;
        if (want[g]) o.out[q.slots++] = want[g];
    }
    const Shape s = backward_shape(a.T, a.d, HAS_V);
    a.waves = (int)s.block.x / 64;
    a.step = (int)(s.grid.x * s.block.y);
    if (a.T) {
        by_type(HAS_V ? v_dt : MOE_F32, [&](auto vt) {
            by_type(h_dt, [&](auto ht) {
                by_type(u_dt, [&](auto ut) {
                    typedef decltype(vt) VT;
                    typedef decltype(ht) HT;
                    typedef decltype(ut) UT;
                    if constexpr (HAS_V || std::is_same<VT, float>::value) {
                        if (a.d > MOE_NORM_ANY_D) hipLaunchKernelGGL((norm_back_kernel<VT, HT, UT, true, HAS_V, true>), s.grid, s.block, 0, st, a, q);
                        else if (vec) hipLaunchKernelGGL((norm_back_kernel<VT, HT, UT, true, HAS_V, false>), s.grid, s.block, 0, st, a, q);
                        else hipLaunchKernelGGL((norm_back_kernel<VT, HT, UT, false, HAS_V, false>), s.grid, s.block, 0, st, a, q);
                    }
                });
            });
        });
        MOE_CHECK_LAUNCH(who);
    }
    if (q.slots) {
        hipLaunchKernelGGL(sum_parts_kernel, dim3((unsigned)((a.d + 15) / 16), (unsigned)q.slots), dim3(1024), 0, st, q.part,
                           a.T ? (int)(s.grid.x * s.block.y) : 0, q.slots, a.d, o);
        MOE_CHECK_LAUNCH(who);
    }
    return MOE_OK;
}

// ---- checks
bool kind_ok(int kind, bool none) { return kind == MOE_NORM_RMS || kind == MOE_NORM_LAYER || (none && kind == MOE_NORM_NONE); }

int check_shape(const char* who, int T, int d) {
    MOE_REQUIRE(T >= 0 && d >= 1, MOE_ERR_ARG, "%s: T=%d d=%d", who, T, d);
    MOE_REQUIRE(d <= MOE_NORM_MAX_D, MOE_ERR_UNSUPPORTED, "%s: d=%d is beyond %d", who, d, MOE_NORM_MAX_D);
    // (a row's number and the rows in work at a time add up to an int)
    MOE_REQUIRE(T <= INT_MAX - (1 << 20), MOE_ERR_UNSUPPORTED, "%s: T=%d is beyond %d", who, T, INT_MAX - (1 << 20));
    return MOE_OK;
}
int check_norms(const char* who, int T, int post_kind, float post_eps, const float* post_w, const float* post_b, const float* gate, int gate_rows,
                int next_kind, float next_eps, const float* next_w, const float* next_b) {
    MOE_REQUIRE(kind_ok(post_kind, true) && kind_ok(next_kind, true), MOE_ERR_ARG, "%s: norm kinds %d, %d", who, post_kind, next_kind);
    MOE_REQUIRE(post_eps >= 0.f && next_eps >= 0.f, MOE_ERR_ARG, "%s: eps %g, %g", who, (double)post_eps, (double)next_eps);
    MOE_REQUIRE(post_kind != MOE_NORM_NONE || (!post_w && !post_b), MOE_ERR_ARG, "%s: parameters of a norm that is none (post)", who);
    MOE_REQUIRE(next_kind != MOE_NORM_NONE || (!next_w && !next_b), MOE_ERR_ARG, "%s: parameters of a norm that is none (next)", who);
    MOE_REQUIRE(gate ? gate_rows == 1 || gate_rows == T : gate_rows == 0, MOE_ERR_ARG, "%s: gate_rows=%d with T=%d and %s gate", who, gate_rows, T,
                gate ? "a" : "no");
    return MOE_OK;
}
#define MOE_PASS(call) do { const int rc_ = (call); if (rc_ != MOE_OK) return rc_; } while (0)

int group_of(int k) { return k <= 1 ? 1 : k <= 2 ? 2 : k <= 4 ? 4 : 8; }

}  // namespace

size_t moe_norm_back_bytes(int T, int d, bool block_end, int grads) {
    if (T < 0 || d < 1 || d > MOE_NORM_MAX_D) return 0;
    const Shape s = backward_shape(T, d, block_end);
    return (size_t)s.grid.x * s.block.y * grads * d * sizeof(float);
}

extern "C" int moe_norm(const void* x, moe_dtype x_dt, const float* w, const float* b, int T, int d, moe_norm_kind kind, float eps, void* u,
                        moe_dtype u_dt, float* stats, void* stream) {
    MOE_PASS(check_shape("moe_norm", T, d));
    MOE_REQUIRE(moe_dtype_ok(x_dt) && moe_dtype_ok(u_dt), MOE_ERR_UNSUPPORTED, "moe_norm: dtypes %d, %d", (int)x_dt, (int)u_dt);
    MOE_REQUIRE(kind_ok(kind, false), MOE_ERR_ARG, "moe_norm: norm kind %d", (int)kind);
    MOE_REQUIRE(eps >= 0.f, MOE_ERR_ARG, "moe_norm: eps %g", (double)eps);
    if (T == 0) return MOE_OK;
    MOE_REQUIRE(x && u, MOE_ERR_ARG, "moe_norm: null pointer");
    Args a = {};
    a.h = x; a.next_w = w; a.next_b = b; a.T = T; a.d = d; a.next_kind = kind; a.next_eps = eps; a.inv_d = 1.f / (float)d; a.u = u; a.stats = stats;
    const bool vec = d % V == 0 && aligned(x) && aligned(u) && aligned(w) && aligned(b);
    return launch_forward<SRC_NONE, 1>("moe_norm", a, 0, x_dt, u_dt, vec, (hipStream_t)stream);
}

extern "C" int moe_norm_backward(const void* du, moe_dtype u_dt, const void* x, moe_dtype x_dt, const float* w, const float* stats, int T, int d,
                                 moe_norm_kind kind, const void* dx_add, void* dx, float* dw, float* db, void* ws, size_t ws_bytes, void* stream) {
    MOE_PASS(check_shape("moe_norm_backward", T, d));
    MOE_REQUIRE(moe_dtype_ok(x_dt) && moe_dtype_ok(u_dt), MOE_ERR_UNSUPPORTED, "moe_norm_backward: dtypes %d, %d", (int)x_dt, (int)u_dt);
    MOE_REQUIRE(kind_ok(kind, false), MOE_ERR_ARG, "moe_norm_backward: norm kind %d", (int)kind);
    MOE_REQUIRE(T == 0 || (du && x && stats), MOE_ERR_ARG, "moe_norm_backward: null pointer");
    if (dw || db) {
        const size_t need = T ? moe_norm_back_bytes(T, d, false, (dw != nullptr) + (db != nullptr)) : 0;
        MOE_REQUIRE(need == 0 || (ws && ws_bytes >= need), MOE_ERR_WORKSPACE, "moe_norm_backward: workspace of %zu bytes, %zu needed", ws_bytes, need);
    }
    Args a = {};
    a.h = x; a.next_w = w; a.T = T; a.d = d; a.next_kind = kind; a.inv_d = 1.f / (float)d; a.stats = const_cast<float*>(stats);
    Grads q = {};
    q.dy = dx_add; q.du = du; q.dh = dx; q.part = (float*)ws;
    float* const want[N_GRADS] = {dw, db, nullptr, nullptr, nullptr};
    const bool vec = d % V == 0 && aligned(x) && aligned(du) && aligned(w) && aligned(dx_add) && aligned(dx) && aligned(ws);
    return launch_backward<false>("moe_norm_backward", a, q, want, 0, x_dt, u_dt, vec, (hipStream_t)stream);
}

extern "C" int moe_block_end(const void* v, moe_dtype v_dt, const void* h, moe_dtype h_dt, int T, int d, moe_norm_kind post_kind, float post_eps,
                             const float* post_w, const float* post_b, const float* gate, int gate_rows, float alpha, moe_norm_kind next_kind,
                             float next_eps, const float* next_w, const float* next_b, void* y, void* u, moe_dtype u_dt, float* stats, void* stream) {
    MOE_PASS(check_shape("moe_block_end", T, d));
    MOE_REQUIRE(moe_dtype_ok(v_dt) && moe_dtype_ok(h_dt) && moe_dtype_ok(u_dt), MOE_ERR_UNSUPPORTED, "moe_block_end: dtypes %d, %d, %d", (int)v_dt,
                (int)h_dt, (int)u_dt);
    MOE_PASS(check_norms("moe_block_end", T, post_kind, post_eps, post_w, post_b, gate, gate_rows, next_kind, next_eps, next_w, next_b));
    if (T == 0) return MOE_OK;
    MOE_REQUIRE(v && h && y && (u || next_kind == MOE_NORM_NONE), MOE_ERR_ARG, "moe_block_end: null pointer");
    Args a = {};
    a.v = v; a.h = h; a.post_w = post_w; a.post_b = post_b; a.gate = gate; a.next_w = next_w; a.next_b = next_b; a.T = T; a.d = d;
    a.post_kind = post_kind; a.next_kind = next_kind; a.gate_rows = gate_rows; a.post_eps = post_eps; a.next_eps = next_eps; a.alpha = alpha;
    a.inv_d = 1.f / (float)d; a.y = y; a.u = u; a.stats = stats;
    const bool vec = d % V == 0 && aligned(v) && aligned(h) && aligned(post_w) && aligned(post_b) && aligned(gate) && aligned(next_w) &&
                     aligned(next_b) && aligned(y) && aligned(u);
    return launch_forward<SRC_TENSOR, 1>("moe_block_end", a, v_dt, h_dt, u_dt, vec, (hipStream_t)stream);
}

extern "C" int moe_block_end_rows(const float* y_perm, const int32_t* inv_perm, const float* gate_w, const float* shared, int k, const void* h,
                                  moe_dtype h_dt, int T, int d, moe_norm_kind post_kind, float post_eps, const float* post_w, const float* post_b,
                                  const float* gate, int gate_rows, float alpha, moe_norm_kind next_kind, float next_eps, const float* next_w,
                                  const float* next_b, void* y, void* u, moe_dtype u_dt, void* stream) {
    MOE_PASS(check_shape("moe_block_end_rows", T, d));
    MOE_REQUIRE(k >= 1, MOE_ERR_ARG, "moe_block_end_rows: k=%d", k);
    MOE_REQUIRE(moe_dtype_ok(h_dt) && moe_dtype_ok(u_dt), MOE_ERR_UNSUPPORTED, "moe_block_end_rows: dtypes %d, %d", (int)h_dt, (int)u_dt);
    MOE_PASS(check_norms("moe_block_end_rows", T, post_kind, post_eps, post_w, post_b, gate, gate_rows, next_kind, next_eps, next_w, next_b));
    if (T == 0) return MOE_OK;
    MOE_REQUIRE(y_perm && inv_perm && h && y && (u || next_kind == MOE_NORM_NONE), MOE_ERR_ARG, "moe_block_end_rows: null pointer");
    Args a = {};
    a.v = y_perm; a.inv_perm = inv_perm; a.gate_w = gate_w; a.shared = shared; a.k = k; a.h = h; a.post_w = post_w; a.post_b = post_b; a.gate = gate;
    a.next_w = next_w; a.next_b = next_b; a.T = T; a.d = d; a.post_kind = post_kind; a.next_kind = next_kind; a.gate_rows = gate_rows;
    a.post_eps = post_eps; a.next_eps = next_eps; a.alpha = alpha; a.inv_d = 1.f / (float)d; a.y = y; a.u = u;
    const bool vec = d % V == 0 && aligned(y_perm) && aligned(shared) && aligned(h) && aligned(post_w) && aligned(post_b) && aligned(gate) &&
                     aligned(next_w) && aligned(next_b) && aligned(y) && aligned(u);
    const char* who = "moe_block_end_rows";
    switch (group_of(k)) {
        case 1: return launch_forward<SRC_ROWS, 1>(who, a, 0, h_dt, u_dt, vec, (hipStream_t)stream);
        case 2: return launch_forward<SRC_ROWS, 2>(who, a, 0, h_dt, u_dt, vec, (hipStream_t)stream);
        case 4: return launch_forward<SRC_ROWS, 4>(who, a, 0, h_dt, u_dt, vec, (hipStream_t)stream);
        default: return launch_forward<SRC_ROWS, 8>(who, a, 0, h_dt, u_dt, vec, (hipStream_t)stream);
    }
}

extern "C" int moe_block_end_backward(const void* dy, const void* du, moe_dtype u_dt, const void* v, moe_dtype v_dt, const void* h, moe_dtype h_dt,
                                      int T, int d, moe_norm_kind post_kind, const float* post_w, const float* post_b, const float* gate,
                                      int gate_rows, float alpha, moe_norm_kind next_kind, const float* next_w, const float* stats, void* dv,
                                      void* dh, float* dpost_w, float* dpost_b, float* dgate, float* dnext_w, float* dnext_b, void* ws,
                                      size_t ws_bytes, void* stream) {
    const char* who = "moe_block_end_backward";
    MOE_PASS(check_shape(who, T, d));
    MOE_REQUIRE(moe_dtype_ok(v_dt) && moe_dtype_ok(h_dt) && moe_dtype_ok(u_dt), MOE_ERR_UNSUPPORTED, "%s: dtypes %d, %d, %d", who, (int)v_dt,
                (int)h_dt, (int)u_dt);
    MOE_PASS(check_norms(who, T, post_kind, 0.f, post_w, post_b, gate, gate_rows, next_kind, 0.f, next_w, nullptr));
    MOE_REQUIRE(post_kind != MOE_NORM_NONE || (!dpost_w && !dpost_b), MOE_ERR_ARG, "%s: gradients of a norm that is none (post)", who);
    MOE_REQUIRE(next_kind != MOE_NORM_NONE || (!dnext_w && !dnext_b && !du), MOE_ERR_ARG, "%s: gradients of a norm that is none (next)", who);
    MOE_REQUIRE(gate || !dgate, MOE_ERR_ARG, "%s: gradient of a gate that is none", who);
    MOE_REQUIRE(du || (!dnext_w && !dnext_b), MOE_ERR_ARG, "%s: parameters' gradients without du", who);
    MOE_REQUIRE(T == 0 || (v && h && stats && (dy || du)), MOE_ERR_ARG, "%s: null pointer", who);
    const bool own = gate_rows != 1;     // (a row for every token; no tokens: dgate has no rows)
    float* const want[N_GRADS] = {dnext_w, dnext_b, own ? nullptr : dgate, dpost_w, dpost_b};
    int n = 0;
    for (float* w : want) n += w != nullptr;
    if (n) {
        const size_t need = T ? moe_norm_back_bytes(T, d, true, n) : 0;
        MOE_REQUIRE(need == 0 || (ws && ws_bytes >= need), MOE_ERR_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need);
    }
    Args a = {};
    a.v = v; a.h = h; a.post_w = post_w; a.post_b = post_b; a.gate = gate; a.next_w = next_w; a.T = T; a.d = d; a.post_kind = post_kind;
    a.next_kind = next_kind; a.gate_rows = gate_rows; a.alpha = alpha; a.inv_d = 1.f / (float)d; a.stats = const_cast<float*>(stats);
    Grads q = {};
    q.dy = dy; q.du = du; q.dv = dv; q.dh = dh; q.dgate = own ? dgate : nullptr; q.part = (float*)ws;
    const bool vec = d % V == 0 && aligned(dy) && aligned(du) && aligned(v) && aligned(h) && aligned(post_w) && aligned(post_b) && aligned(gate) &&
                     aligned(next_w) && aligned(dv) && aligned(dh) && aligned(q.dgate) && aligned(ws);
    return launch_backward<true>(who, a, q, want, v_dt, h_dt, u_dt, vec, (hipStream_t)stream);
}
