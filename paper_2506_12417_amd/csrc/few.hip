// moe_layer_few: a whole MoE layer for a few tokens (T <= 64) in two launches.
//
//   launch 1   routing, then   H[r,:] = act(x[token of r] . W_in^T)            for every row r = (expert, token)
//   launch 2   y[t,:] = sum_j gate[t,j] H[row of (t,j)] . W_out^T  (+ shared expert)
//
// What bounds it: the fetch of the active experts' weights, each once; then launches and chains of latencies.  The general path's
// five launches (routing, sort, plan, two products, combine) read the same weights, and its sort and plan are there to
// balance rows, of which there are none to balance here.  So the sort is a table of bits in LDS (one bit per expert and token),
// made by every work-group for itself, and there is no plan: an active expert is a list of items.
//
// Launch 1, one work-group of sixteen wavefronts per CU.  Every work-group routes all tokens for itself (what it reads for
// that, W_g and x, comes from the L2s; waiting for another work-group's answer, or another launch, costs more): logits on the matrix
// cores in fp32 over 32 terms at a time, added up in fp64, with a rigorous error bound; logits closer than the bound are
// computed again in fp64, so that the choice is that of exact arithmetic.  Then its wavefronts take items of 16 weight rows, each
// alone over the whole contraction: no barrier, no partial sums.
// Launch 2: a work-group owns 8 or 16 output columns for all tokens and all experts.  The (expert, 128-byte line) pairs of its
// contraction are dealt out to its sixteen wavefronts in equal runs; a wavefront adds each expert's products, times the gates, to
// sums per token of its own in LDS, and the sixteen are added in a fixed order.  So the combine costs no pass over memory, no atomics and no
// second launch, and all CUs read equal shares of the weights whatever the routing.
//
// Weights and rows come in whole 128-byte lines, eight rows a load, several lines in flight per wavefront, and
// are turned into the matrix instruction's fragments in a piece of LDS of the wavefront's own (fragments straight from global memory touch 16
// lines per quarter wavefront instead of 2, and the vector cache is then what a CU waits for).
#include <climits>
#include "common.h"
#include "ffn_kernels.h"
#include "gemm_util.h"
#include "lanes.h"

namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef const __attribute__((address_space(1))) unsigned char* gptr;
typedef const __attribute__((address_space(1))) u32x4* gpiece;

constexpr int NW = 16, NTH = NW * 64;            // wavefronts and threads of a work-group
constexpr int MAXT = MOE_FEW_MAX_T, MAXE = MOE_MAX_EXPERTS, MAXA = MAXT * MOE_MAX_TOPK;
static_assert(MAXT == 64, "a token is a bit of two words");

enum { BF = 0, HF = 1, FP = 2 };                 // what the operands are: bf16, half, fp32

// D[i][j] += sum of a 16-byte piece's terms of A row i and B row j (every lane gives the pieces of its row lane % 16; which
// terms a lane's piece holds matters only in so far as both operands agree)
template <int TY> __device__ __forceinline__ f32x4 mma(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (TY == BF) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else if constexpr (TY == HF) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
        return c;
    }
}

// ---- the rows of the active experts
struct Lists {
    unsigned bits[MAXE][2];              // the tokens of an expert
    int first[MAXE + 1];                 // its first row
    int active[MAXE];                    // the experts with tokens, rising
    int n_active;
    unsigned short a[MAXA];              // a row's assignment t k + j
    int id[MAXA];
    float gate[MAXA];                    // by assignment
};
constexpr int TURN_PIECES = 2 * 16 * 8;  // 16 weight rows and 16 rows of 128 bytes, in 16-byte pieces

// ids (in l.id) -> lists.  An id outside [0,E) has no row.  All threads; a barrier before and behind.
__device__ __forceinline__ void make_lists(Lists& l, int T, int E, int k) {
    const int tid = threadIdx.x, A = T * k;
    for (int i = tid; i < 2 * MAXE; i += NTH) (&l.bits[0][0])[i] = 0u;
    __syncthreads();
    int e = -1, t = 0;
    if (tid < A) {
        e = l.id[tid];
        t = tid / k;
        if ((unsigned)e < (unsigned)E) atomicOr(&l.bits[e][t >> 5], 1u << (t & 31));
    }
    __syncthreads();
    if (tid < 64) {
        unsigned rows = 0, act = 0;      // of the experts before
#pragma unroll
        for (int j = 0; j < MAXE / 64; ++j) {
            const int x = j * 64 + tid;
            const unsigned n = __popc(l.bits[x][0]) + __popc(l.bits[x][1]), up = moe_wave_scan_u32(n);
            const unsigned long long on = __ballot(n != 0);
            l.first[x] = (int)(rows + up - n);
            if (n) l.active[act + __popcll(on & ((1ull << tid) - 1ull))] = x;
            rows += (unsigned)__builtin_amdgcn_readlane((int)up, 63);
            act += (unsigned)__popcll(on);
        }
        if (tid == 0) { l.first[MAXE] = (int)rows; l.n_active = (int)act; }
    }
    __syncthreads();
    if ((unsigned)e < (unsigned)E) {
        const unsigned lo = l.bits[e][0], hi = l.bits[e][1], below = (1u << (t & 31)) - 1u;
        l.a[l.first[e] + (t < 32 ? __popc(lo & below) : __popc(lo) + __popc(hi & below))] = (unsigned short)tid;
    }
    __syncthreads();
}

// ---- acc[g] += 16 weight rows (A) x the 16 activation rows of group g (B) over the 128-byte lines [l0, l1)
// WL: weight loads of eight rows (1: rows 8 - 15 of the product mean nothing), XL: loads of a group's activation rows, U: lines in
// flight.  w0, w1: the two eights of weight rows; x_at: byte offsets of the lane's rows, beyond the buffer for rows that are not there.
template <int TY, int G, int XL, int WL, int U>
__device__ __forceinline__ void lines_product(const unsigned char* w0, const unsigned char* w1, unsigned w_off, __amdgpu_buffer_rsrc_t x,
                                              const unsigned (&x_at)[4][2], int l0, int l1, f32x4 (&acc)[4], u32x4* turn) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4;
    // (rows of eight pieces, piece p of row r at place p ^ (r & 7): no bank conflicts either way)
    const int st_at = (lane >> 3) * 8 + ((lane & 7) ^ (lane >> 3)), rd_at = l16 * 8 + (lq ^ (l16 & 7));
    u32x4* const xturn = turn + 16 * 8;
    for (int l = l0; l < l1; l += U) {
        u32x4 w[U][WL], b[U][G][XL];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = (l + u < l1 ? l + u : l1 - 1) * 128;          // (past the end: the last line again, not multiplied)
            w[u][0] = *(gpiece)((gptr)(uintptr_t)(w0 + at) + w_off);
            if constexpr (WL == 2) w[u][1] = *(gpiece)((gptr)(uintptr_t)(w1 + at) + w_off);
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int i = 0; i < XL; ++i) b[u][g][i] = __builtin_amdgcn_raw_buffer_load_b128(x, (int)x_at[g][i], at, 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (l + u < l1) {
#pragma unroll
                for (int i = 0; i < WL; ++i) turn[i * 64 + st_at] = w[u][i];
                u32x4 wf[2] = {turn[rd_at], turn[rd_at ^ 4]};
#pragma unroll
                for (int g = 0; g < G; ++g) {
#pragma unroll
                    for (int i = 0; i < XL; ++i) xturn[i * 64 + st_at] = b[u][g][i];
#pragma unroll
                    for (int v = 0; v < 2; ++v) acc[g] = mma<TY>(wf[v], xturn[rd_at ^ (4 * v)], acc[g]);
                }
            }
        }
    }
}
// the same for m rows (m <= 64), as many groups as they need
template <int TY, int WL>
__device__ __forceinline__ int lines_product_rows(int m, const unsigned char* w0, const unsigned char* w1, unsigned w_off, __amdgpu_buffer_rsrc_t x,
                                                  const unsigned (&x_at)[4][2], int l0, int l1, f32x4 (&acc)[4], u32x4* turn) {
#pragma unroll
    for (int g = 0; g < 4; ++g) acc[g] = f32x4{0.f, 0.f, 0.f, 0.f};
    if (m <= 8) lines_product<TY, 1, 1, WL, WL == 2 ? 6 : 8>(w0, w1, w_off, x, x_at, l0, l1, acc, turn);
    else if (m <= 16) lines_product<TY, 1, 2, WL, WL == 2 ? 4 : 6>(w0, w1, w_off, x, x_at, l0, l1, acc, turn);
    else if (m <= 32) lines_product<TY, 2, 2, WL, WL == 2 ? 3 : 4>(w0, w1, w_off, x, x_at, l0, l1, acc, turn);
    else if (m <= 48) lines_product<TY, 3, 2, WL, 2>(w0, w1, w_off, x, x_at, l0, l1, acc, turn);
    else lines_product<TY, 4, 2, WL, 2>(w0, w1, w_off, x, x_at, l0, l1, acc, turn);
    // (the last matrix instructions stand before a branch, across which the compiler does not keep the distance to the use of
    // their results: sixteen cycles and more here)
    asm volatile("s_nop 15\n\ts_nop 3" : "+v"(acc[0]), "+v"(acc[1]), "+v"(acc[2]), "+v"(acc[3]));
    return (m + 15) >> 4;
}

constexpr unsigned NOWHERE = 0x80000000u;        // beyond every buffer here (they are smaller than 2 GiB)

// ---- routing
struct Route {
    const uint16_t *x, *w;               // x [T,d], W_g prepared [E,d]
    const float *norm2, *bias;
    int32_t* idx;                        // [T,k], out
    float* gate;
    int T, d, E, k, renorm;
};
template <int TT> struct RouteLds {      // TT: groups of 16 tokens
    double part[NW * 16][TT * 16 + 1];   // [contraction part, expert][token]
    float xsq[NW][TT * 16];
    float most[NW];
};

constexpr int TERMS = 32;                // terms summed up in fp32, by one matrix instruction

// fp64 product of token row and expert row by a wavefront
__device__ __forceinline__ double exact_dot(const uint16_t* xr, const uint16_t* wr, int d) {
    const int lane = threadIdx.x & 63;
    double s0 = 0.0, s1 = 0.0;
    for (int i = lane * 8; i < d; i += 1024) {
        u32x4 xv[2], wv[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            xv[u] = wv[u] = u32x4{0u, 0u, 0u, 0u};
            if (i + u * 512 < d) { xv[u] = *(const u32x4*)(xr + i + u * 512); wv[u] = *(const u32x4*)(wr + i + u * 512); }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s0 = fma((double)__uint_as_float(xv[u][j] << 16), (double)__uint_as_float(wv[u][j] << 16), s0);
                s1 = fma((double)__uint_as_float(xv[u][j] & 0xffff0000u), (double)__uint_as_float(wv[u][j] & 0xffff0000u), s1);
            }
    }
    return wave_sum_f64(s0 + s1);
}

// exp(v) for v <= 0 in 64 bits: what the rounding of v to fp32 took away is put back
__device__ __forceinline__ float exp_of(double v) {
    const float hi = (float)v, e = expf(hi);
    return e > 0.f ? fmaf(e, (float)(v - (double)hi), e) : e;
}

template <int TT>
__device__ __forceinline__ void route_all(const Route& p, RouteLds<TT>& s, Lists& l, bool write) {
    const int tid = threadIdx.x, lane = tid & 63, wave = sgpr(tid >> 6), l16 = lane & 15, lq = lane >> 4;
    const int T = p.T, d = p.d, E = p.E, k = p.k;
    // NB blocks of 16 experts, the contraction in KS parts; wavefront = block + NB part
    const int blocks = (E + 15) >> 4, NB = blocks <= 1 ? 1 : blocks <= 2 ? 2 : blocks <= 4 ? 4 : blocks <= 8 ? 8 : 16, KS = NW / NB;
    const int block = wave % NB, part = wave / NB;
    const float my_norm = tid < E ? p.norm2[tid] : 0.f;
    double acc[TT][4];
#pragma unroll
    for (int g = 0; g < TT; ++g)
#pragma unroll
        for (int r = 0; r < 4; ++r) acc[g][r] = 0.0;
    float xsq[TT] = {};
    if (block < blocks) {
        const int e = block * 16 + l16 < E ? block * 16 + l16 : E - 1;
        const uint16_t* wr = p.w + (size_t)e * d + lq * 8;
        const uint16_t* xr[TT];
#pragma unroll
        for (int g = 0; g < TT; ++g) xr[g] = p.x + (size_t)(g * 16 + l16 < T ? g * 16 + l16 : T - 1) * d + lq * 8;
        constexpr int U = TT == 1 ? 6 : TT == 2 ? 4 : TT == 3 ? 3 : 2;   // 32-term steps in flight
        const int steps = d / TERMS;
        for (int c = part; c < steps; c += KS * U) {
            u32x4 w[U], x[U][TT];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = (c + u * KS < steps ? c + u * KS : c) * TERMS;
                w[u] = *(const u32x4*)(wr + at);
#pragma unroll
                for (int g = 0; g < TT; ++g) x[u][g] = *(const u32x4*)(xr[g] + at);
            }
            if (block == 0) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (c + u * KS < steps) {
#pragma unroll
                        for (int g = 0; g < TT; ++g)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float a = __uint_as_float(x[u][g][j] << 16), b = __uint_as_float(x[u][g][j] & 0xffff0000u);
                                xsq[g] = fmaf(a, a, fmaf(b, b, xsq[g]));
                            }
                    }
            }
            // (no branch between a matrix instruction and the use of its result: the compiler does not keep
            // their distance across one.  Steps past the end give zeros.)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool in = c + u * KS < steps;
                f32x4 v[TT];
#pragma unroll
                for (int g = 0; g < TT; ++g) v[g] = mma<BF>(w[u], x[u][g], f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                for (int g = 0; g < TT; ++g)
#pragma unroll
                    for (int r = 0; r < 4; ++r) acc[g][r] += (double)(in ? v[g][r] : 0.f);
            }
        }
    }
    // D[i][j]: lane holds token j = l16, experts i = 4 lq + r
#pragma unroll
    for (int g = 0; g < TT; ++g) {
#pragma unroll
        for (int r = 0; r < 4; ++r) s.part[wave * 16 + 4 * lq + r][g * 16 + l16] = acc[g][r];
        float q = xsq[g];
        q += __shfl_xor(q, 16);
        q += __shfl_xor(q, 32);
        if (block == 0 && lq == 0) s.xsq[part][g * 16 + l16] = q;
    }
    const float most = moe_wave_max_nonneg(my_norm);
    if (lane == 0) s.most[wave] = most;
    __syncthreads();
    float wn = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) wn = fmaxf(wn, s.most[w]);

    // a wavefront chooses for a token; lane holds experts lane, lane + 64, ...
    constexpr int NJ = MAXE / 64;
    constexpr double NONE = -__builtin_huge_val();
    for (int t = wave; t < T; t += NW) {
        double v[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const int e = lane + 64 * j;
            v[j] = NONE;
            if (e < E) {
                v[j] = p.bias ? (double)p.bias[e] : 0.0;
                for (int q = 0; q < KS; ++q) v[j] += s.part[(q * NB + (e >> 4)) * 16 + (e & 15)][t];
            }
        }
        float xs = 0.f;
        for (int q = 0; q < KS; ++q) xs += s.xsq[q][t];
        // |error| of a logit: two roundings per term of a matrix instruction (the order inside it is not known), the
        // sums of norms rounded up; twice that is what two logits may be wrong by against one another
        const float tau = 2.1f * 5.9604645e-8f * (2 * TERMS + 6) * (sqrtf(xs) * 1.0001f) * (sqrtf(wn) * 1.0001f);
        const int rounds = k + 1 < E ? k + 1 : E;
        double sv = NONE;                // lane r: the r-th choice
        int se = INT_MAX;
        auto choose = [&]() __attribute__((always_inline)) {
            unsigned taken = 0;          // of this lane's experts
            for (int r = 0; r < rounds; ++r) {
                double bv = NONE;
                int be = INT_MAX;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
                    if (j * 64 < E && !(taken >> j & 1) && lane + 64 * j < E && beats(v[j], lane + 64 * j, bv, be)) { bv = v[j]; be = lane + 64 * j; }
                row_best_f64(bv, be, true);
                if (be != INT_MAX && (be & 63) == lane) taken |= 1u << (be >> 6);
                if (lane == r) { sv = bv; se = be; }
            }
        };
        choose();
        const double next = __shfl(sv, lane + 1 < 64 ? lane + 1 : lane);
        // (written so that a bound or a difference that is no number counts as near)
        if (__ballot(lane + 1 < rounds && !(sv - next >= (double)tau))) {
            // near one another: these logits again, in fp64
            const double last = lane_f64(sv, k - 1) - (double)tau;
            unsigned again = 0;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int e = lane + 64 * j;
                bool near = false;
                if (j * 64 < E)
                    for (int r = 0; r < rounds; ++r) {
                        const double o = lane_f64(sv, r);
                        const int oe = __builtin_amdgcn_readlane(se, r);
                        near = near || (oe != e && !(fabs(v[j] - o) >= (double)tau));
                    }
                if (e < E && near && !(v[j] < last)) again |= 1u << j;
            }
#pragma unroll
            for (int j = 0; j < NJ; ++j)
                for (unsigned long long m = __ballot(again >> j & 1); m; m &= m - 1) {
                    const int src = __builtin_ctzll(m), e = src + 64 * j;
                    const double dot = exact_dot(p.x + (size_t)t * d, p.w + (size_t)e * d, d) + (p.bias ? (double)p.bias[e] : 0.0);
                    if (lane == src) v[j] = dot;
                }
            choose();
        }
        const double top = lane_f64(sv, 0);
        float e = 0.f;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            if (lane + 64 * j < E) e += exp_of(v[j] - top);
        e += dpp_xchg<0>(e);
        e += dpp_xchg<1>(e);
        e += dpp_xchg<2>(e);
        e += dpp_xchg<3>(e);
        const float all = (__int_as_float(__builtin_amdgcn_readlane(__float_as_int(e), 0)) + __int_as_float(__builtin_amdgcn_readlane(__float_as_int(e), 16))) +
                          (__int_as_float(__builtin_amdgcn_readlane(__float_as_int(e), 32)) + __int_as_float(__builtin_amdgcn_readlane(__float_as_int(e), 48)));
        const float mine = se == INT_MAX ? __builtin_nanf("") : exp_of(sv - top);
        float chosen = 0.f;
        for (int r = 0; r < k; ++r) chosen += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), r));
        if (lane < k) {
            const float over = p.renorm && all == all ? chosen : all;    // (a logit that is no number: nor is any gate)
            l.id[t * k + lane] = se;
            if (write) {
                p.idx[t * k + lane] = se;
                p.gate[t * k + lane] = mine / over;
            }
        }
    }
    __syncthreads();
}

// ---- launch 1
struct Hidden {
    Route route;
    const void* x;
    const void* const *w_in, *const *s_w_in;
    unsigned char *h, *s_h;              // hidden activations of the rows [A,F] and of the shared expert [T,shared_F]
    int F, shared_F, glu;
};
__device__ __forceinline__ uint16_t half_of(float v) {           // saturating, nearest-even
    return __builtin_bit_cast(uint16_t, (_Float16)__builtin_amdgcn_fmed3f(v, -65504.f, 65504.f));
}

// TT: groups of 16 tokens that every work-group routes itself; 0: idx is there already
template <bool F32, int TT>
__global__ __launch_bounds__(NTH) void few_hidden_kernel(Hidden p) {
    constexpr int ES = F32 ? 4 : 2, TY = F32 ? FP : BF;
    constexpr size_t TURNS = sizeof(u32x4) * TURN_PIECES * NW, ROUTE = TT ? sizeof(RouteLds<TT ? TT : 1>) : 0;
    __shared__ __attribute__((aligned(16))) unsigned char smem[TURNS > ROUTE ? TURNS : ROUTE];
    __shared__ Lists l;
    const int tid = threadIdx.x, lane = tid & 63, wave = sgpr(tid >> 6), l16 = lane & 15, lq = lane >> 4;
    const int T = p.route.T, d = p.route.d, E = p.route.E, k = p.route.k;
    if constexpr (TT > 0) {
        route_all<TT>(p.route, *(RouteLds<TT>*)smem, l, blockIdx.x == 0);
    } else {
        if (tid < T * k) l.id[tid] = p.route.idx[tid];
        __syncthreads();
    }
    make_lists(l, T, E, k);
    u32x4* const turn = (u32x4*)smem + wave * TURN_PIECES;
    const __amdgpu_buffer_rsrc_t x = make_rsrc(p.x, (unsigned)(T * d) * ES);
    const unsigned w_off = (unsigned)(lane >> 3) * (unsigned)d * ES + (unsigned)(lane & 7) * 16u, piece = (unsigned)(lane & 7) * 16u;
    const size_t row_bytes = (size_t)d * ES;
    // items of 16 weight rows: the shared expert's first (they have the most rows), then the active experts'
    const int s_items = p.shared_F / 8, per = p.F / (p.glu ? 8 : 16), items = s_items + sgpr(l.n_active) * per;
    for (int item = wave * (int)gridDim.x + (int)blockIdx.x; item < items; item += NW * (int)gridDim.x) {
        const bool shared = item < s_items, glu = shared || p.glu;
        const int rest = item - s_items, ai = shared ? 0 : rest / per, q = shared ? item : rest - ai * per;
        const int e = shared ? 0 : sgpr(l.active[ai]), r0 = shared ? 0 : sgpr(l.first[e]);
        const int m = shared ? T : sgpr(l.first[e + 1]) - r0;
        const unsigned char* w = (const unsigned char*)sgpr_ptr(shared ? p.s_w_in[0] : p.w_in[e]);
        // Packed rows (moe_pack_weights): 16-bit rows 16 h + j of a block of 32 are outputs 2 j + h, fp32 rows are in order; with SwiGLU
        // blocks of 32 gate and 32 up rows alternate.  An item is 16 rows of a block, or 8 gate rows and their 8 up rows.
        const int p0 = glu ? (q >> 2) * 64 + (q & 3) * 8 : q * 16;
        const int out0 = F32 ? (glu ? (q >> 2) * 32 + (q & 3) * 8 : q * 16)
                             : (glu ? (q >> 2) * 32 + (q & 1) * 16 + ((q >> 1) & 1) : (q >> 1) * 32 + (q & 1));
        constexpr int out_step = F32 ? 1 : 2;
        unsigned x_at[4][2];
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = g * 16 + i * 8 + (lane >> 3);
                x_at[g][i] = NOWHERE;
                if (r < m) x_at[g][i] = (unsigned)(shared ? r : (int)l.a[r0 + r] / k) * (unsigned)row_bytes + piece;
            }
        f32x4 acc[4];
        const unsigned char* w0 = w + p0 * row_bytes;
        const int groups = lines_product_rows<TY, 2>(m, w0, w0 + (glu ? 32 : 8) * row_bytes, w_off, x, x_at, 0, d * ES / 128, acc, turn);
        const int width = shared ? p.shared_F : p.F;
        unsigned char* h = shared ? p.s_h : p.h;
        for (int g = 0; g < groups; ++g) {
            f32x4 a = g == 0 ? acc[0] : g == 1 ? acc[1] : g == 2 ? acc[2] : acc[3];
            const int r = g * 16 + l16;
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float up = __shfl_xor(a[i], 32);
                v[i] = glu ? silu_f(a[i]) * up : fmaxf(a[i], 0.f);
            }
            if (r < m && (!glu || lq < 2)) {
                unsigned char* to = h + ((size_t)(r0 + r) * width + out0 + 4 * lq * out_step) * ES;
                if constexpr (F32) {
                    *(f32x4*)to = f32x4{v[0], v[1], v[2], v[3]};
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) ((uint16_t*)to)[2 * i] = half_of(v[i]);
                }
            }
        }
    }
}

// ---- launch 2
struct Out {
    const int32_t* idx;
    const float* gate;
    const void* const *w_out, *const *s_w_out;
    const unsigned char *h, *s_h;
    void* y;
    int T, d, E, k, F, shared_F, y_f32;
};

// WL: 1 for 8 columns of a work-group, 2 for 16
template <bool F32, int WL>
__global__ __launch_bounds__(NTH) void few_out_kernel(Out p) {
    constexpr int ES = F32 ? 4 : 2, TY = F32 ? FP : HF, COLS = WL * 8;
    __shared__ __attribute__((aligned(16))) unsigned char smem[sizeof(u32x4) * TURN_PIECES * NW];
    __shared__ __attribute__((aligned(16))) float sums[NW][MAXT][COLS];
    __shared__ Lists l;
    __shared__ int lost[MAXT];           // tokens with an assignment to no expert
    const int tid = threadIdx.x, lane = tid & 63, wave = sgpr(tid >> 6), l16 = lane & 15, lq = lane >> 4;
    const int T = p.T, d = p.d, E = p.E, k = p.k, F = p.F;
    if (tid < T) lost[tid] = 0;
    if (tid < T * k) {
        l.id[tid] = p.idx[tid];
        l.gate[tid] = p.gate[tid];
    }
    for (int i = lane; i < T * COLS; i += 64) (&sums[wave][0][0])[i] = 0.f;
    __syncthreads();
    if (tid < T * k && (unsigned)l.id[tid] >= (unsigned)E) lost[tid / k] = 1;
    make_lists(l, T, E, k);
    u32x4* const turn = (u32x4*)smem + wave * TURN_PIECES;
    const int n_active = sgpr(l.n_active), rows = sgpr(l.first[MAXE]);
    const __amdgpu_buffer_rsrc_t h = make_rsrc(p.h, (unsigned)(rows * F) * ES), s_h = make_rsrc(p.s_h, (unsigned)(T * p.shared_F) * ES);
    const int p0 = (int)blockIdx.x * COLS;
    // (expert, line) pairs, the shared expert's behind the others'
    const int L = F * ES / 128, s_L = p.shared_F * ES / 128, units = n_active * L + s_L;
    const int u1 = (int)((long long)units * (wave + 1) / NW);
    for (int u = (int)((long long)units * wave / NW); u < u1;) {
        const int ai = u / L;
        const bool shared = ai >= n_active;
        const int base = shared ? n_active * L : ai * L, l0 = u - base, have = shared ? s_L : L;
        const int l1 = u1 - base < have ? u1 - base : have;
        u = base + l1;
        const int e = shared ? 0 : sgpr(l.active[ai]), r0 = shared ? 0 : sgpr(l.first[e]), m = shared ? T : sgpr(l.first[e + 1]) - r0;
        const size_t row_bytes = (size_t)(shared ? p.shared_F : F) * ES;
        const unsigned char* w = (const unsigned char*)sgpr_ptr(shared ? p.s_w_out[0] : p.w_out[e]) + p0 * row_bytes;
        const unsigned piece = (unsigned)(lane & 7) * 16u, w_off = (unsigned)(lane >> 3) * (unsigned)row_bytes + piece;
        unsigned x_at[4][2];
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = g * 16 + i * 8 + (lane >> 3);
                x_at[g][i] = r < m ? (unsigned)(r0 + r) * (unsigned)row_bytes + piece : NOWHERE;
            }
        f32x4 acc[4];
        const int groups = lines_product_rows<TY, WL>(m, w, w + 8 * row_bytes, w_off, shared ? s_h : h, x_at, l0, l1, acc, turn);
        for (int g = 0; g < groups; ++g) {
            const f32x4 a = g == 0 ? acc[0] : g == 1 ? acc[1] : g == 2 ? acc[2] : acc[3];
            const int r = g * 16 + l16;
            if (r < m && (WL == 2 || lq < 2)) {
                const int as = shared ? 0 : l.a[r0 + r], t = shared ? r : as / k;
                const float gate = shared ? 1.f : l.gate[as];
                f32x4* to = (f32x4*)&sums[wave][t][4 * lq];      // (an expert's rows are different tokens)
                f32x4 s = *to;
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] = fmaf(gate, a[i], s[i]);
                *to = s;
            }
        }
    }
    __syncthreads();
    if (tid < T * COLS) {
        const int t = tid / COLS, c = tid - t * COLS, row = p0 + c;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) v += sums[w][t][c];
        if (lost[t]) v = __builtin_nanf("");                      // (its gates are NaN)
        const int col = F32 ? row : (row & ~31) + 2 * (row & 15) + ((row >> 4) & 1);
        if (p.y_f32) ((float*)p.y)[(size_t)t * d + col] = v;
        else ((uint16_t*)p.y)[(size_t)t * d + col] = f32_to_bf16(v);
    }
}
static_assert(MAXT * 16 <= NTH, "a thread per output of a work-group");

template <bool F32, int TT> void launch_hidden(const Hidden& a, hipStream_t st) {
    hipLaunchKernelGGL((few_hidden_kernel<F32, TT>), dim3(MOE_GEMM_GRID), dim3(NTH), 0, st, a);
}

bool aligned(const void* p) { return ((uintptr_t)p & 15) == 0; }

}  // namespace

extern "C" size_t moe_layer_few_workspace(int T, int F, int k, int shared_F, moe_dtype dt) {
    if (T < 0 || F < 1 || k < 1 || shared_F < 0 || !moe_dtype_ok(dt)) return 0;
    return (size_t)T * ((size_t)k * F + shared_F) * moe_elem_size(dt);
}

extern "C" int moe_layer_few(const void* x, int T, int d, int F, int E, int k, moe_act act, moe_dtype dt, int renorm, const void* w_gate,
                             const float* w_norm2, const float* bias, const void* const* w_in, const void* const* w_out, int shared_F,
                             const void* const* s_w_in, const void* const* s_w_out, int32_t* expert_idx, float* gate_w, void* ws,
                             size_t ws_bytes, void* y, moe_dtype y_dt, void* stream) {
    MOE_REQUIRE(T >= 0 && d >= 1 && F >= 1 && E >= 1 && k >= 1 && k <= E && shared_F >= 0, MOE_ERR_ARG,
                "moe_layer_few: T=%d d=%d F=%d E=%d k=%d shared_F=%d", T, d, F, E, k, shared_F);
    MOE_REQUIRE(act == MOE_RELU || act == MOE_SWIGLU, MOE_ERR_UNSUPPORTED, "moe_layer_few: activation %d", (int)act);
    MOE_REQUIRE(moe_dtype_ok(dt) && moe_dtype_ok(y_dt), MOE_ERR_UNSUPPORTED, "moe_layer_few: dtypes %d, %d", (int)dt, (int)y_dt);
    MOE_REQUIRE(T <= MAXT, MOE_ERR_UNSUPPORTED, "moe_layer_few: T=%d is beyond %d", T, MAXT);
    MOE_REQUIRE(E <= MAXE && k <= MOE_MAX_TOPK, MOE_ERR_UNSUPPORTED, "moe_layer_few: E=%d k=%d", E, k);
    MOE_REQUIRE(d % 64 == 0 && F % 64 == 0 && shared_F % 64 == 0, MOE_ERR_UNSUPPORTED, "moe_layer_few: d=%d F=%d shared_F=%d are not all multiples of 64",
                d, F, shared_F);
    const size_t es = moe_elem_size(dt), two_gib = (size_t)1 << 31;
    MOE_REQUIRE((size_t)8 * d * es < two_gib && (size_t)8 * F * es < two_gib && (size_t)8 * shared_F * es < two_gib && (size_t)T * d * es < two_gib && (size_t)T * k * F * es < two_gib && (size_t)T * shared_F * es < two_gib, MOE_ERR_UNSUPPORTED,
                "moe_layer_few: rows of %d, %d and %d values are too long", d, F, shared_F);
    if (T == 0) return MOE_OK;
    MOE_REQUIRE(x && w_gate && w_in && w_out && expert_idx && gate_w && y && (dt == MOE_F32 || w_norm2) && (!shared_F || (s_w_in && s_w_out)),
                MOE_ERR_ARG, "moe_layer_few: null pointer");
    const size_t need = moe_layer_few_workspace(T, F, k, shared_F, dt);
    MOE_REQUIRE(ws && ws_bytes >= need, MOE_ERR_WORKSPACE, "moe_layer_few: workspace of %zu bytes, %zu needed", ws_bytes, need);
    MOE_REQUIRE(aligned(x) && aligned(w_gate) && aligned(ws), MOE_ERR_UNSUPPORTED, "moe_layer_few: x, w_gate and ws must be aligned to 16 bytes");
    const int dev_ok = moe_check_gemm_device();
    if (dev_ok != MOE_OK) return dev_ok;
    const hipStream_t st = (hipStream_t)stream;
    Hidden a = {};
    a.route = {(const uint16_t*)x, (const uint16_t*)w_gate, w_norm2, bias, expert_idx, gate_w, T, d, E, k, renorm};
    a.x = x; a.w_in = w_in; a.s_w_in = s_w_in; a.F = F; a.shared_F = shared_F; a.glu = act == MOE_SWIGLU;
    a.h = (unsigned char*)ws;
    a.s_h = a.h + (size_t)T * k * F * es;
    if (dt == MOE_F32) {
        const int rc = moe_route_topk(x, w_gate, bias, T, d, E, k, renorm, dt, expert_idx, gate_w, nullptr, stream);
        if (rc != MOE_OK) return rc;
        launch_hidden<true, 0>(a, st);
    } else if (T <= 16) {
        launch_hidden<false, 1>(a, st);
    } else if (T <= 32) {
        launch_hidden<false, 2>(a, st);
    } else if (T <= 48) {
        launch_hidden<false, 3>(a, st);
    } else {
        launch_hidden<false, 4>(a, st);
    }
    MOE_CHECK_LAUNCH("moe_layer_few (routing and first product)");
    Out o = {expert_idx, gate_w, w_out, s_w_out, a.h, a.s_h, y, T, d, E, k, F, shared_F, y_dt == MOE_F32};
    // Sixteen columns where they make a work-group per CU, else eight (a matrix instruction half empty, twice the work-groups)
    const bool wide = d / 16 >= MOE_GEMM_GRID;
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)(d / (wide ? 16 : 8))), dim3(NTH), 0, st, o); };
    if (dt == MOE_F32) wide ? go(few_out_kernel<true, 2>) : go(few_out_kernel<true, 1>);
    else wide ? go(few_out_kernel<false, 2>) : go(few_out_kernel<false, 1>);
    MOE_CHECK_LAUNCH("moe_layer_few (second product and combine)");
    return MOE_OK;
}
