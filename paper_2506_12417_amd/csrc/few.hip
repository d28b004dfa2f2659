// moe_layer_few: a whole MoE layer for a few tokens (T <= 64) in two launches (three: fp32, more than 32 tokens, and a large shared expert).
//
//   launch 1   routing, then   H[r,:] = act(x[token of r] . W_in^T)            for every row r = (expert, token)
//   launch 2   y[t,:] = sum_j gate[t,j] H[row of (t,j)] . W_out^T  (+ shared expert)
//
// What bounds it: the fetch of the active experts' weights, each once; then launches and chains of latencies.  The general path's
// five launches (routing, sort, plan, two products, combine) read the same weights, and its sort and plan are there to
// balance rows, of which there are none to balance here.  So the sort is a table of bits in LDS (one bit per expert and token),
// made by every work-group for itself, and there is no plan: an active expert is a list of items.
//
// Launch 1, one work-group of eight wavefronts per CU.  Every work-group routes all tokens for itself (what it reads for
// that, W_g and x, comes from the L2s; waiting for another work-group's answer, or another launch, costs more): logits on the matrix
// cores in fp32 over 64 terms at a time, added up in fp64, with a rigorous error bound; a token whose logits are closer than the bound
// has those computed again in fp64, so that the choice is that of exact arithmetic.  Then its items of 16 weight rows are shared
// out to its wavefronts in runs of equal cost; an item that several of them have part of is added up in LDS.
// Launch 2: a work-group owns 8 or 16 output columns, for all tokens and experts or, in narrow layers, some of them.  The (expert,
// 128-byte line) pairs of its contraction are shared out in the same way; a wavefront adds each expert's products, times the gates, to
// sums per token of its own in LDS, and these are added in a fixed order.  So the combine costs no pass over memory, no atomics and no
// launch of its own, and all CUs read equal shares of the weights whatever the routing.
//
// The hidden activations are the second product's operands, and so IEEE half in 16 bits (11 significant bits; bf16 would be eight times coarser): that
// rounding is 2.0e-4 of y's norm, and changes the last bit of one bf16 output in thirty (whose own rounding is 1.65e-3 of the norm).
//
// Weights and rows come in whole 128-byte lines, eight rows a load, several lines in flight per wavefront, and
// are turned into the matrix instruction's fragments in a piece of LDS of the wavefront's own (fragments straight from global memory touch 16
// lines per quarter wavefront instead of 2, and the vector cache is then what a CU waits for).
//
// Measured, us for launches 1 and 2 (medians of 50; weights of the chosen experts, TB/s): d=768 F=3072 E=128 k=1 one token 14.4 + 6.6 (9.4 MB), 8 tokens
// 19.5 + 11.6 (69 MB, 2.2); d=4096 F=14336 E=8 k=2, 3 tokens 153 + 70 (1.4 GB, 6.3; 5.6 where they lie elsewhere); d=2048 F=1408 E=60 k=4 with a
// shared expert of 5632, 33 tokens 12 + 92 + 56 with the routing (825 MB, 5.2); fp32 d=320 F=1984 E=16 k=2, 5 tokens 4.7 + 13.6 + 7.8.
// One token, launch 1: logits 4.9, their sums and the choice 3.5, lists 0.7, product 3.
#include <climits>
#include <type_traits>
#include "common.h"
#include "ffn_kernels.h"
#include "gemm_util.h"
#include "lanes.h"

namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int NW = 8, NTH = NW * 64;            // wavefronts and threads of a work-group
constexpr int MAXT = MOE_FEW_MAX_T, MAXE = MOE_MAX_EXPERTS, MAXA = MAXT * MOE_MAX_TOPK;
static_assert(MAXT == 64 && MAXA <= NTH && 2 * MAXE <= NTH, "a token is a bit of two words; a thread per assignment and per word");

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
    int cost[MAXE + 1];                  // what a line of each of the active ones before costs, in all
    int n_active;
    const void* w[MAXE];                 // the experts' matrices
    int id[MAXA];                        // the choice, by assignment
    float gate[MAXA];                    // by row
    unsigned short pair[MAXA];           // a row's assignment: token * k + choice
    unsigned char t[MAXA];               // and its token
};

__device__ __forceinline__ int line_cost(int m);

__device__ __forceinline__ int rows_in(const Lists& l, int x, unsigned long long range) {
    return __popc(l.bits[x][0] & (unsigned)range) + __popc(l.bits[x][1] & (unsigned)(range >> 32));
}
// Every thread's assignment (expert e of token t with weight gate; e outside [0,E): none) -> lists; active and cost of the experts and rows of
// the tokens in `range` only.  The bits are clear.  A barrier before and behind.
__device__ __forceinline__ void make_lists(Lists& l, int E, int e, int t, float gate, unsigned long long range) {
    const int tid = threadIdx.x;
    const bool is = (unsigned)e < (unsigned)E;
    if (is) atomicOr(&l.bits[e][t >> 5], 1u << (t & 31));
    __syncthreads();
    if (tid < 64) {
        unsigned rows = 0, act = 0, cost = 0;    // of the experts before
        for (int x = tid; x - tid < E; x += 64) {
            const unsigned n = (unsigned)rows_in(l, x, ~0ull), in = (unsigned)rows_in(l, x, range), c = in ? (unsigned)line_cost((int)in) : 0u;
            // (both sums in one scan: at most 512 rows, and 256 experts' costs of at most 10)
            const unsigned up = moe_wave_scan_u32(n | c << 16);
            const unsigned long long on = __ballot(in != 0);
            l.first[x] = (int)(rows + (up & 0xffffu) - n);
            if (in) {
                const int at = (int)act + __popcll(on & ((1ull << tid) - 1ull));
                l.active[at] = x;
                l.cost[at] = (int)(cost + (up >> 16) - c);
            }
            const unsigned all = (unsigned)__builtin_amdgcn_readlane((int)up, 63);
            rows += all & 0xffffu;
            cost += all >> 16;
            act += (unsigned)__popcll(on);
        }
        if (tid == 0) {
            l.first[(E + 63) & ~63] = (int)rows;
            l.cost[act] = (int)cost;
            l.n_active = (int)act;
        }
    }
    __syncthreads();
    if (is) {
        const unsigned lo = l.bits[e][0], hi = l.bits[e][1], below = (1u << (t & 31)) - 1u;
        const int r = l.first[e] + (t < 32 ? __popc(lo & below) : __popc(lo) + __popc(hi & below));
        l.pair[r] = (unsigned short)tid;
        l.t[r] = (unsigned char)t;
        l.gate[r] = gate;
    }
    __syncthreads();
}

constexpr unsigned NOWHERE = 0x80000000u;        // beyond every buffer here (they are smaller than 2 GiB)

// Where a product's activations come from: LDS, where they all lie in it (rows in order, 16-byte piece p of row r of every 128 bytes at
// place p ^ (r & 7)); or memory, as fragments, or in whole lines that are turned into fragments in LDS.  (Rows in lines cost
// the vector cache 16 look-ups a load, as fragments 4 for every row: lines are the choice for more than 4 rows that lie in order.)
enum { IN_LDS = 0, FRAGMENTS = 1, LINES = 2 };

// ---- products.  A segment: 16 weight rows times an expert's m <= 64 rows over the 128-byte lines [l0, l1) of the contraction.
struct Segment {
    __amdgpu_buffer_rsrc_t w, x;
    unsigned w_at[2];                    // byte offsets of the lane's two weight rows (eight rows a load)
    // and of its activations: its 16 bytes of group g in the first 64 bytes of a row; beyond the buffer for rows that are not there (in
    // LDS: of any row)
    unsigned x_at[4];
    unsigned row_at[8];                  // LINES: its 16 bytes of the first 128 of row 8 i + lane / 8; IN_LDS, fp32: of row i, for dots()
    int x_step;                          // from one 64 bytes to the next (FRAGMENTS)
    int l0, l1, m;
};

// Eight weight rows a load, a lane's 16 bytes of them times the same 16 bytes of every activation row, in fp32: for a few rows, where the
// matrix instruction's 16 columns would be nearly empty (fp32: eight of 32 cycles a line).  acc[i][r]: row 8 i + lane / 8, activation row r.
template <int WL, int M>
__device__ __forceinline__ void dots(const u32x4 (&w)[WL], const unsigned char* xl, const unsigned (&x_at)[8], int line, float (&acc)[WL][M]) {
#pragma unroll
    for (int r = 0; r < M; ++r) {
        const u32x4 x = *(const u32x4*)(xl + x_at[r] + line * 128);
#pragma unroll
        for (int i = 0; i < WL; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][r] = fmaf(__uint_as_float(w[i][j]), __uint_as_float(x[j]), acc[i][r]);
    }
}
// their sums over the eight lanes of a row, in the matrix instruction's places: lane holds activation row lane % 16, weight rows 4 (lane / 16) + r
template <int WL, int M> __device__ __forceinline__ f32x4 dots_total(float (&acc)[WL][M]) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4;
    float mine[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < WL; ++i)
#pragma unroll
        for (int r = 0; r < M; ++r) {
            float v = acc[i][r];
            v += dpp_xchg<0>(v);
            v += dpp_xchg<1>(v);
            v += dpp_xchg<2>(v);
            mine[i] = (lane & 7) == r ? v : mine[i];
        }
    f32x4 out;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int from = (4 * (lq & 1) + r) * 8 + (l16 & 7);
        const float lo = __shfl(mine[0], from), hi = WL == 2 ? __shfl(mine[1], from) : 0.f;
        out[r] = lq & 2 ? hi : lo;
    }
    return out;
}

// A wavefront's run of segments with G groups of 16 rows: acc[g] = weight rows (A) x rows of group g (B), D lines in flight.
//   WL     weight loads of eight rows (1: rows 8 - 15 of the product mean nothing)
//   M      > 0: at most M rows, by dots() (IN_LDS, fp32)
//   CACHE  CACHE_NT for weights that are fetched once: streamed past what the caches hold they come 5 - 12 % faster (d=4096 F=14336 E=8
//          k=2, 3 tokens 272 - 278 us against 244 - 256, d=2048 F=1408 E=60 k=4, 8 tokens 105 against 99); fetched for several ranges of
//          tokens they are better off in the L2 (fp32 d=320 F=1984, 33 tokens 50 us against 53)
//   next(Segment&)  the segment behind the present one, false if there is none of this kind;   done(Segment const&, acc)
// The loads run on from one segment into the next: in the last D lines of one the next one's first are fetched; a segment takes its lines'
// number rounded up to D.  The weights of a line go through one half of the turning place while the line before is multiplied.
template <int TY, int WL, int G, int M, int D, int X, int CACHE, typename Next, typename Done>
__device__ __forceinline__ void stream(Segment seg, u32x4* turn, const unsigned char* xl, Next next, Done done) {
    static_assert(D % 2 == 0, "the turning place's halves alternate");
    static_assert(M == 0 || (X == IN_LDS && TY == FP && G == 1), "");
    const int lane = threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4;
    // (rows of eight pieces, piece p of row r at place p ^ (r & 7): no bank conflicts either way)
    const int st_at = (lane >> 3) * 8 + ((lane & 7) ^ (lane >> 3)), rd_at = l16 * 8 + (lq ^ (l16 & 7));
    u32x4 a[D][WL], b[X == IN_LDS ? 1 : D][G][2];
    auto fetch = [&](const Segment& from, int u, int l) __attribute__((always_inline)) {
        const bool in = l < from.l1;
        const int at = in ? l : 0;
#pragma unroll
        for (int i = 0; i < WL; ++i) a[u][i] = __builtin_amdgcn_raw_buffer_load_b128(from.w, (int)(in ? from.w_at[i] : NOWHERE), at * 128, CACHE);
        if constexpr (X != IN_LDS) {
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int v = 0; v < 2; ++v)
                    b[u][g][v] = __builtin_amdgcn_raw_buffer_load_b128(from.x, (int)(in ? (X == LINES ? from.row_at[2 * g + v] : from.x_at[g]) : NOWHERE),
                                                                       X == LINES ? at * 128 : (2 * at + v) * from.x_step, 0);
        }
    };
    u32x4 wf[2][2], xf[2][G][2];
    // line l of segment s, fetched at u, becomes fragments
    auto turned = [&](const Segment& s, int u, int l) __attribute__((always_inline)) {
        if constexpr (M == 0) {
            u32x4* const half = turn + (u & 1) * 128;
#pragma unroll
            for (int i = 0; i < WL; ++i) half[i * 64 + st_at] = a[u % D][i];
            wf[u & 1][0] = half[rd_at];
            wf[u & 1][1] = half[rd_at ^ 4];
            if constexpr (X == IN_LDS) {
                const int at = l < s.l1 ? l * 128 : 0;
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int v = 0; v < 2; ++v) xf[u & 1][g][v] = *(const u32x4*)(xl + (s.x_at[g] ^ (64u * v)) + at);
            }
        }
    };
    f32x4 acc[G];
    float dot[WL][M ? M : 1];
    auto multiply = [&](const Segment& s, int u, int l) __attribute__((always_inline)) {
        if constexpr (M > 0) {
            dots<WL, M>(a[u], xl, s.row_at, l, dot);
        } else {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                if constexpr (X == LINES) {
                    u32x4* const third = turn + 256;
#pragma unroll
                    for (int v = 0; v < 2; ++v) third[v * 64 + st_at] = b[u][g][v];
#pragma unroll
                    for (int v = 0; v < 2; ++v) acc[g] = mma<TY>(wf[u & 1][v], third[rd_at ^ (4 * v)], acc[g]);
                } else {
#pragma unroll
                    for (int v = 0; v < 2; ++v) acc[g] = mma<TY>(wf[u & 1][v], X == IN_LDS ? xf[u & 1][g][v] : b[X == IN_LDS ? 0 : u][g][v], acc[g]);
                }
            }
        }
    };
#pragma unroll
    for (int u = 0; u < D; ++u) fetch(seg, u, seg.l0 + u);
    turned(seg, 0, seg.l0);
    for (;;) {
        Segment nxt = seg;
        const bool more = next(nxt);
        if (!more) nxt.l1 = nxt.l0;
#pragma unroll
        for (int g = 0; g < G; ++g) acc[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < WL; ++i)
#pragma unroll
            for (int r = 0; r < (M ? M : 1); ++r) dot[i][r] = 0.f;
        int l = seg.l0;
        for (; l + D < seg.l1 || (more && l < seg.l1); l += D) {
            const bool last = l + D >= seg.l1;
            Segment from = seg;
            int at = l + D;
            if (last) {
                from = nxt;
                at = nxt.l0;
            }
#pragma unroll
            for (int u = 0; u < D; ++u) {
                if (u + 1 < D) turned(seg, u + 1, l + u + 1);
                else turned(from, D, at);                // (the next D's first, fetched at u = 0)
                if (l + u < seg.l1) multiply(seg, u, l + u);
                fetch(from, u, at + u);
                __builtin_amdgcn_sched_barrier(0);       // (lines stay apart: mixed, they need more registers than there are)
            }
        }
        if (!more) {                     // the run's last lines: nothing to fetch
#pragma unroll
            for (int u = 0; u < D; ++u) {
                if (l + u < seg.l1) {
                    if (u + 1 < D) turned(seg, u + 1, l + u + 1);
                    multiply(seg, u, l + u);
                }
            }
        }
        if constexpr (M > 0) acc[0] = dots_total<WL, M>(dot);
        // (the last matrix instructions stand before a branch, across which the compiler does not keep the distance to the use of
        // their results: sixteen cycles and more here)
#pragma unroll
        for (int g = 0; g < G; ++g) asm volatile("s_nop 15\n\ts_nop 3" : "+v"(acc[g]));
        done(seg, acc);
        if (!more) return;
        seg = nxt;
    }
}
// what decides which instance of stream() multiplies m rows
template <int TY, int X, int X_TALL> __device__ __forceinline__ int kind_of(int m) {
    if (TY == FP && X == IN_LDS && m <= 8) return m <= 2 ? -2 : -8;
    if (X_TALL == LINES && m <= 4) return 0;
    return (m + 15) >> 4;
}
// Runs of segments one behind the other, whatever their rows.  current: false if there is none; few: there are few lines in all.
template <int TY, int WL, int X, int X_TALL, int CACHE, typename Current, typename Next, typename Done>
__device__ __forceinline__ void stream_all(u32x4* turn, const unsigned char* xl, bool few, Current current, Next next, Done done) {
    Segment seg;
    constexpr int DEEP = X == IN_LDS ? (WL == 2 ? 10 : 16) : (WL == 2 ? 8 : 12);
    while (current(seg)) {
        const int kind = kind_of<TY, X, X_TALL>(seg.m);
        auto same = [&](Segment& s) __attribute__((always_inline)) { return next(s) && kind_of<TY, X, X_TALL>(s.m) == kind; };
        if constexpr (TY == FP && X == IN_LDS) {
            if (kind == -2) {
                stream<TY, WL, 1, 2, DEEP, X, CACHE>(seg, turn, xl, same, done);
                continue;
            }
            if (kind == -8) {
                stream<TY, WL, 1, 8, 8, X, CACHE>(seg, turn, xl, same, done);
                continue;
            }
        }
        if (kind <= 1 && few) stream<TY, WL, 1, 0, 4, X, CACHE>(seg, turn, xl, same, done);
        else if (kind == 0) stream<TY, WL, 1, 0, DEEP, X, CACHE>(seg, turn, xl, same, done);
        else if (kind == 1) stream<TY, WL, 1, 0, DEEP, X_TALL, CACHE>(seg, turn, xl, same, done);
        else if (kind == 2) stream<TY, WL, 2, 0, 6, X_TALL, CACHE>(seg, turn, xl, same, done);
        else if (kind == 3) stream<TY, WL, 3, 0, 4, X_TALL, CACHE>(seg, turn, xl, same, done);
        else stream<TY, WL, 4, 0, X == IN_LDS ? 4 : 2, X_TALL, CACHE>(seg, turn, xl, same, done);
    }
}
// what a line of an expert with m rows costs a wavefront, in loads
__device__ __forceinline__ int line_cost(int m) { return 2 + (m + 15) / 16 * 2; }

// The lane's place in rows that lie in LDS: its 16 bytes of row r for a fragment, and of row r for dots().
__device__ __forceinline__ unsigned fragment_at(int r, unsigned row_bytes) {
    const int lq = (threadIdx.x & 63) >> 4;
    return (unsigned)r * row_bytes + (unsigned)(lq ^ (r & 7)) * 16u;
}
__device__ __forceinline__ unsigned piece_at(int r, unsigned row_bytes) { return (unsigned)r * row_bytes + (unsigned)((threadIdx.x & 7) ^ (r & 7)) * 16u; }
// `rows` rows of row_bytes (a multiple of 128) from memory into LDS in that order: all wavefronts, a row each; to be waited for (vmcnt) and
// shown to the others by a barrier
__device__ __forceinline__ void rows_to_lds(const void* from, int rows, unsigned row_bytes, unsigned char* to) {
    const int lane = threadIdx.x & 63, wave = sgpr(threadIdx.x >> 6);
    const __amdgpu_buffer_rsrc_t src = make_rsrc(from, (unsigned)rows * row_bytes);
    for (int r = wave; r < rows; r += NW)
        for (unsigned at = 0; at < row_bytes; at += 1024) {
            const unsigned mine = at + (unsigned)((lane & ~7) | ((lane & 7) ^ (r & 7))) * 16u;
            if (mine < row_bytes)        // (the row's end is a multiple of 128 bytes: the place is inside where the source is)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(src, (lds_void_t*)(to + (unsigned)r * row_bytes + at), 16, (unsigned)r * row_bytes + mine, 0, 0, 0);
        }
}

// ---- routing
struct Route {
    const uint16_t *x, *w;               // x [T,d], W_g prepared [E,d]
    const float *norm2, *bias;
    int32_t* idx;                        // [T,k], out
    float* gate;
    int T, d, E, k, renorm;
};
// How T tokens are routed: TT groups of 16, x in LDS or not; a wavefront takes EB blocks of 16 experts, D lines in flight.
// (More experts a wavefront fetch x less often, but their sums take LDS: 128 KB for four blocks and 32 tokens.)
template <int TT_, bool LDS_> struct How {
    static constexpr int TT = TT_, EB = TT_ <= 1 || (TT_ == 2 && !LDS_) ? 4 : 2, D = TT_ == 1 ? 3 : 2;
    static constexpr bool LDS = LDS_;
};
// Beyond that many tokens MOE_BF16 routes in a launch of its own: what every work-group does for itself takes longer than that then (64
// tokens: d=320 F=512 E=24 k=4 38.2 us against 34.9, d=2048 F=1408 E=60 k=4 227 against 220; 17 to 32 tokens: up to 3 us less than with
// a launch).
constexpr int ROUTE_MAXT = 32;
static_assert(ROUTE_MAXT <= NW * 4, "choose: four tokens a wavefront");
template <bool LDS> using Routed = How<0, LDS>;          // the choice is there already
template <typename H> struct RouteLds {
    double part[NW * H::EB * 16][H::TT * 16 + 1];        // [contraction part, expert][token]; the lines' turning places before
    float xsq[NW][H::TT * 16];
    float bias[MAXE];
    float most[NW];
};
template <bool LDS> struct RouteLds<How<0, LDS>> {};

constexpr int TERMS = 64;                // terms summed up in fp32: a line, by two matrix instructions

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

// unsigned numbers in the floats' order; 0 for what is no number
__device__ __forceinline__ unsigned order_of(float v) {
    const unsigned u = __float_as_uint(v);
    return v == v ? u ^ (u >> 31 ? 0xffffffffu : 0x80000000u) : 0u;
}

// A token whose choice (the wavefront's lanes `from` on, expert ids by falling logit) is not certain: the logits that are close to a chosen
// one's are computed again in fp64, and the choice is made again among exact and well separated ones.  A wavefront; returns the choice
// of number lane % 16.
template <typename L>
__device__ __forceinline__ int choose_again(const Route& p, L& s, int t, int se, double tau, int from, int rounds) {
    const int lane = threadIdx.x & 63, E = p.E, k = p.k, d = p.d;
    constexpr int NJ = MAXE / 64;
    constexpr double NONE = -__builtin_huge_val();
    auto close = [&](double a, double b) __attribute__((always_inline)) { return !(fabs(a - b) >= tau + 3e-7 * fabs(a)); };
    const int last_e = __builtin_amdgcn_readlane(se, from + k - 1);
    const double last = last_e == INT_MAX ? NONE : s.part[last_e][t], least = last - (tau + 3e-7 * fabs(last));
    double v[NJ];
    unsigned again = 0;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
        const int e = lane + 64 * j;
        v[j] = e < E ? s.part[e][t] : NONE;
        bool near = false;
        for (int r = 0; r < rounds; ++r) {
            const int oe = __builtin_amdgcn_readlane(se, from + r);
            if (oe != INT_MAX) near = near || (oe != e && close(s.part[oe][t], v[j]));
        }
        if (e < E && near && !(v[j] < least)) again |= 1u << j;
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
        for (unsigned long long m = __ballot(again >> j & 1); m; m &= m - 1) {
            const int src = __builtin_ctzll(m), e = src + 64 * j;
            const double dot = exact_dot(p.x + (size_t)t * d, p.w + (size_t)e * d, d) + (p.bias ? (double)p.bias[e] : 0.0);
            if (lane == src) {
                v[j] = dot;
                s.part[e][t] = dot;
            }
        }
    unsigned taken = 0;                  // of this lane's experts
    int chosen = INT_MAX;
    for (int r = 0; r < rounds; ++r) {
        double bv = NONE;
        int be = INT_MAX;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            if (!(taken >> j & 1) && lane + 64 * j < E && beats(v[j], lane + 64 * j, bv, be)) { bv = v[j]; be = lane + 64 * j; }
        row_best_f64(bv, be, true);
        if (be != INT_MAX && (be & 63) == lane) taken |= 1u << (be >> 6);
        if ((lane & 15) == r) chosen = be;
    }
    return chosen;
}

// Sixteen lanes choose for a token, four tokens a wavefront from t0 on; lane `sub` of them holds experts sub, sub + 16, ... (NI of them) as
// numbers in the order of the logits rounded to fp32.
template <int NI, typename L>
__device__ __forceinline__ void choose(const Route& p, L& s, Lists& l, int t0, float wn, int KS, bool write) {
    const int lane = threadIdx.x & 63, sub = lane & 15, T = p.T, E = p.E, k = p.k, rounds = k + 1 < E ? k + 1 : E;
    const int t = t0 + (lane >> 4), tt = t < T ? t : T - 1;
    double v[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) v[i] = s.part[sub + 16 * i < E ? sub + 16 * i : E - 1][tt];
    unsigned key[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) key[i] = sub + 16 * i < E ? order_of((float)v[i]) : 0u;
    float xs = 0.f;
#pragma unroll
    for (int q = 0; q < NW; ++q) xs += q < KS ? s.xsq[q][tt] : 0.f;
    // A logit is off by two roundings per term of a matrix instruction at most (the order inside it is not known); twice that is
    // what two logits may be wrong by against one another.  The choice compares them rounded to fp32.
    const double tau = 2.1f * 5.9604645e-8f * (2 * TERMS + 6) * (sqrtf(xs) * 1.0001f) * (sqrtf(wn) * 1.0001f);
    int se = INT_MAX;                    // lane `sub`: the choice of that number
    for (int r = 0; r < rounds; ++r) {
        unsigned best = key[0];
#pragma unroll
        for (int i = 1; i < NI; ++i) best = max(best, key[i]);
        unsigned top = best;
        top = max(top, (unsigned)dpp_xchg<0>((int)top));
        top = max(top, (unsigned)dpp_xchg<1>((int)top));
        top = max(top, (unsigned)dpp_xchg<2>((int)top));
        top = max(top, (unsigned)dpp_xchg<3>((int)top));
        // (equal ones: any of them, the exact choice sees to it)
        const int winner = __builtin_ctz((unsigned)(__ballot(best == top) >> (lane & 48)) & 0xffffu);
        int e = 0;
#pragma unroll
        for (int i = NI - 1; i >= 0; --i) e = key[i] == top ? sub + 16 * i : e;
        e = __shfl(e, (lane & 48) + winner);
        se = sub == r && top ? e : se;
#pragma unroll
        for (int i = 0; i < NI; ++i) key[i] = e == sub + 16 * i ? 0u : key[i];
    }
    double sv = se != INT_MAX ? s.part[se][tt] : -__builtin_huge_val();
    const double next = __shfl(sv, lane + 1 < 64 ? lane + 1 : lane);
    // (written so that a bound or a difference that is no number counts as close; a token with a NaN has nothing to be looked at again)
    const unsigned long long look = __ballot(t < T && sub + 1 < rounds && !(fabs(sv - next) >= tau + 3e-7 * fabs(sv)) && xs == xs);
    if (look) {
#pragma nounroll
        for (int q = 0; q < 4; ++q)
            if (look >> (16 * q) & 0xffffu) {
                const int again = choose_again(p, s, t0 + q, se, lane_f64(tau, 16 * q), 16 * q, rounds);
                if ((lane >> 4) == q) se = again;
            }
        sv = se != INT_MAX ? s.part[se][tt] : -__builtin_huge_val();
#pragma unroll
        for (int i = 0; i < NI; ++i) v[i] = s.part[sub + 16 * i < E ? sub + 16 * i : E - 1][tt];
    }
    const double top = __shfl(sv, lane & 48);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NI; ++i) sum += sub + 16 * i < E ? gate_exp((float)(v[i] - top)) : 0.f;
    sum += dpp_xchg<0>(sum);
    sum += dpp_xchg<1>(sum);
    sum += dpp_xchg<2>(sum);
    sum += dpp_xchg<3>(sum);
    const float mine = se == INT_MAX ? __builtin_nanf("") : gate_exp((float)(sv - top));
    float chosen = sub < k ? mine : 0.f;
    chosen += dpp_xchg<0>(chosen);
    chosen += dpp_xchg<1>(chosen);
    chosen += dpp_xchg<2>(chosen);
    chosen += dpp_xchg<3>(chosen);
    if (t < T && sub < k) {
        const float over = p.renorm && sum == sum ? chosen : sum;        // (a logit that is no number: nor is any gate)
        l.id[t * k + sub] = se;
        if (write) {
            p.idx[t * k + sub] = se;
            p.gate[t * k + sub] = mine / over;
        }
    }
}

template <typename H>
__device__ __forceinline__ void route_all(const Route& p, unsigned char* smem, const unsigned char* xl, Lists& l, bool write) {
    constexpr int TT = H::TT, XL = 2, EB = H::EB, D = H::D, PLACE = (EB + (H::LDS ? 0 : TT)) * 128;
    RouteLds<H>& s = *(RouteLds<H>*)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = sgpr(tid >> 6), l16 = lane & 15, lq = lane >> 4;
    const int T = p.T, d = p.d, E = p.E;
    // NB groups of EB blocks of 16 experts, the contraction in KS parts; wavefront = group + NB part
    const int groups = (E + 16 * EB - 1) / (16 * EB), NB = groups <= 1 ? 1 : groups <= 2 ? 2 : groups <= 4 ? 4 : 8, KS = NW / NB;
    const int group = wave % NB, part = wave / NB;
    // (fetched before the product, so that their latency passes under it)
    const float my_norm = tid < E ? p.norm2[tid] : 0.f, my_bias = tid < E && p.bias ? p.bias[tid] : 0.f;
    double acc[EB][TT][4];
#pragma unroll
    for (int b = 0; b < EB; ++b)
#pragma unroll
        for (int g = 0; g < TT; ++g)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[b][g][r] = 0.0;
    float xsq[TT][XL] = {};
    if (group < groups) {
        // whole lines, eight rows a load, turned into fragments in LDS, as in stream()
        const __amdgpu_buffer_rsrc_t w = make_rsrc(p.w, (unsigned)(E * d) * 2u), x = make_rsrc(p.x, (unsigned)(T * d) * 2u);
        u32x4* const turn = (u32x4*)smem + wave * PLACE;
        const int st_at = (lane >> 3) * 8 + ((lane & 7) ^ (lane >> 3)), rd_at = l16 * 8 + (lq ^ (l16 & 7));
        const unsigned piece = (unsigned)(lane & 7) * 16u;
        unsigned w_at[EB][2], x_at[TT][XL];
#pragma unroll
        for (int b = 0; b < EB; ++b)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int e = (group * EB + b) * 16 + i * 8 + (lane >> 3);
                w_at[b][i] = e < E ? (unsigned)e * (unsigned)d * 2u + piece : NOWHERE;
            }
#pragma unroll
        for (int g = 0; g < TT; ++g)
#pragma unroll
            for (int i = 0; i < XL; ++i) {
                const int t = g * 16 + i * 8 + (lane >> 3);
                x_at[g][i] = t < T ? (unsigned)t * (unsigned)d * 2u + piece : NOWHERE;
            }
        unsigned x_in[TT];
#pragma unroll
        for (int g = 0; g < TT; ++g) x_in[g] = fragment_at(g * 16 + l16 < T ? g * 16 + l16 : T - 1, (unsigned)d * 2u);
        const int lines = d / 64;
        u32x4 a[D][EB][2], c[H::LDS ? 1 : D][TT][XL];
        auto fetch = [&](int u, int line) __attribute__((always_inline)) {
            const bool in = line < lines;
            const int at = in ? line * 128 : 0;
            if constexpr (!H::LDS) {
#pragma unroll
                for (int g = 0; g < TT; ++g)
#pragma unroll
                    for (int i = 0; i < XL; ++i) c[u][g][i] = __builtin_amdgcn_raw_buffer_load_b128(x, (int)(in ? x_at[g][i] : NOWHERE), at, 0);
            }
#pragma unroll
            for (int b = 0; b < EB; ++b)
#pragma unroll
                for (int i = 0; i < 2; ++i) a[u][b][i] = __builtin_amdgcn_raw_buffer_load_b128(w, (int)(in ? w_at[b][i] : NOWHERE), at, 0);
        };
#pragma unroll
        for (int u = 0; u < D; ++u) fetch(u, part + u * KS);
        if constexpr (H::LDS) {
            MOE_WAIT_VMCNT(0);           // (x, and the first lines of W_g, which are next anyway)
            __syncthreads();
        }
        for (int line = part; line < lines; line += D * KS) {
#pragma unroll
            for (int u = 0; u < D; ++u) {
                if constexpr (!H::LDS) {
#pragma unroll
                    for (int g = 0; g < TT; ++g)
#pragma unroll
                        for (int i = 0; i < XL; ++i) turn[(EB + g) * 128 + i * 64 + st_at] = c[u][g][i];
                }
#pragma unroll
                for (int b = 0; b < EB; ++b)
#pragma unroll
                    for (int i = 0; i < 2; ++i) turn[b * 128 + i * 64 + st_at] = a[u][b][i];
                if (!H::LDS && group == 0) {
#pragma unroll
                    for (int g = 0; g < TT; ++g)
#pragma unroll
                        for (int i = 0; i < XL; ++i)
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const unsigned v = c[H::LDS ? 0 : u][g][i][j];
                                const float lo = __uint_as_float(v << 16), hi = __uint_as_float(v & 0xffff0000u);
                                xsq[g][i] = fmaf(lo, lo, fmaf(hi, hi, xsq[g][i]));
                            }
                }
                u32x4 xf[TT][2];
#pragma unroll
                for (int g = 0; g < TT; ++g)
#pragma unroll
                    for (int v = 0; v < 2; ++v)
                        xf[g][v] = H::LDS ? *(const u32x4*)(xl + (x_in[g] ^ (64u * v)) + (line + u * KS < lines ? line + u * KS : 0) * 128)
                                          : turn[(EB + g) * 128 + (rd_at ^ (4 * v))];
                // (no branch between a matrix instruction and the use of its result: the compiler does not keep their
                // distance across one)
#pragma unroll
                for (int b = 0; b < EB; ++b) {
                    const u32x4 wf[2] = {turn[b * 128 + rd_at], turn[b * 128 + (rd_at ^ 4)]};
                    f32x4 q[TT];
#pragma unroll
                    for (int g = 0; g < TT; ++g) q[g] = mma<BF>(wf[1], xf[g][1], mma<BF>(wf[0], xf[g][0], f32x4{0.f, 0.f, 0.f, 0.f}));
#pragma unroll
                    for (int g = 0; g < TT; ++g)
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[b][g][r] += H::LDS && line + u * KS >= lines ? 0.0 : (double)q[g][r];
                }
                fetch(u, line + (u + D) * KS);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    } else if constexpr (H::LDS) {
        MOE_WAIT_VMCNT(0);               // (a wavefront without experts has copied rows of x as well)
        __syncthreads();
    }
    __syncthreads();                     // (the sums take the turning places' memory)
    // D[i][j]: lane holds token j = l16, experts i = 4 lq + r
#pragma unroll
    for (int g = 0; g < TT; ++g)
        if (g * 16 + l16 < T) {
#pragma unroll
            for (int b = 0; b < EB; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r) s.part[(wave * EB + b) * 16 + 4 * lq + r][g * 16 + l16] = acc[b][g][r];
        }
    if constexpr (H::LDS) {
        for (int t = wave; t < T; t += NW) {
            float q = 0.f;
            for (int at = lane * 16; at < d * 2; at += 1024) {
                const u32x4 v = *(const u32x4*)(xl + t * d * 2 + at);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float lo = __uint_as_float(v[j] << 16), hi = __uint_as_float(v[j] & 0xffff0000u);
                    q = fmaf(lo, lo, fmaf(hi, hi, q));
                }
            }
            q = (float)wave_sum_f64((double)q);
            if (lane < KS) s.xsq[lane][t] = lane == 0 ? q : 0.f;
        }
    } else if (group == 0) {
#pragma unroll
        for (int g = 0; g < TT; ++g)
#pragma unroll
            for (int i = 0; i < XL; ++i) {
                float q = xsq[g][i];     // the eight lanes of a row
                q += dpp_xchg<0>(q);
                q += dpp_xchg<1>(q);
                q += dpp_xchg<2>(q);
                if ((lane & 7) == 0) s.xsq[part][g * 16 + i * 8 + (lane >> 3)] = q;
            }
    }
    if (tid < E) s.bias[tid] = my_bias;
    const float most = moe_wave_max_nonneg(my_norm);
    if (lane == 0) s.most[wave] = most;
    __syncthreads();
    // the logits, in the first part's place
    const int bits = T <= 1 ? 0 : 32 - __builtin_clz((unsigned)(T - 1));
    for (int i = tid; i < E << bits; i += NTH) {
        const int t = i & ((1 << bits) - 1), e = i >> bits;
        if (t < T) {
            double v[NW];
#pragma unroll
            for (int q = 0; q < NW; ++q) v[q] = s.part[((q < KS ? q : 0) * NB * EB + (e >> 4)) * 16 + (e & 15)][t];
            double sum = (double)s.bias[e];
#pragma unroll
            for (int q = 0; q < NW; ++q) sum += q < KS ? v[q] : 0.0;
            s.part[e][t] = sum;
        }
    }
    float wn = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) wn = fmaxf(wn, s.most[w]);
    __syncthreads();
    if (wave * 4 < T) {                  // (four tokens a wavefront, ROUTE_MAXT in all)
        if (E <= 64) choose<4>(p, s, l, wave * 4, wn, KS, write);
        else if (E <= 128) choose<8>(p, s, l, wave * 4, wn, KS, write);
        else choose<16>(p, s, l, wave * 4, wn, KS, write);
    }
    __syncthreads();
}

constexpr unsigned X_BYTES = 64 << 10;           // of LDS for x

// ---- launch 1
constexpr int ROUTE_EACH = 8;
constexpr unsigned h_bytes(int WL) { return WL == 2 ? 80u << 10 : 93u << 10; }     // and for the hidden activations in launch 2
struct Hidden {
    Route route;
    const void* x;
    const void* const *w_in, *const *s_w_in;
    unsigned char *h, *s_h;              // hidden activations of the rows (A of F) and of the shared expert (T of shared_F)
    int F, shared_F, glu, h_rows;        // h_rows: H in rows, else an expert's rows piece by piece (see finish)
    int route_blocks;                    // R: so many work-groups route
};

// H: how the tokens are routed first, by every work-group; or not at all (Routed).  R (a How; with Routed): a launch of its own for the
// routing, ROUTE_EACH tokens a work-group, and beside it the shared expert's first product, by the other work-groups.
template <bool F32, typename H, typename R>
__global__ __launch_bounds__(NTH) void few_hidden_kernel(Hidden p) {
    constexpr bool FIRST = !std::is_void<R>::value;
    typedef typename std::conditional<FIRST, R, H>::type Router;
    constexpr int ES = F32 ? 4 : 2, TY = F32 ? FP : BF;
    constexpr size_t PLACE = H::LDS ? 256 : 384, PLACES = sizeof(u32x4) * (PLACE + 256) * NW, ROUTE = sizeof(RouteLds<Router>);
    constexpr size_t TURN = sizeof(u32x4) * NW * (Router::EB + (Router::LDS ? 0 : Router::TT)) * 128, SMEM = PLACES > ROUTE ? PLACES : ROUTE;
    __shared__ __attribute__((aligned(16))) unsigned char smem[SMEM > TURN ? SMEM : TURN];
    __shared__ __attribute__((aligned(16))) unsigned char xl[H::LDS || Router::LDS ? X_BYTES : 16];
    __shared__ Lists l;
    __shared__ int head_lines[NW];
    const int tid = threadIdx.x, lane = tid & 63, wave = sgpr(tid >> 6), l16 = lane & 15, lq = lane >> 4;
    const int T = p.route.T, d = p.route.d, E = p.route.E, k = p.route.k;
    const unsigned row_bytes = (unsigned)d * ES;
    int grid = (int)gridDim.x, block = (int)blockIdx.x;
    if constexpr (FIRST) {
        if (block < p.route_blocks) {
            Route r = p.route;
            const int t0 = block * ROUTE_EACH;
            r.x += (size_t)t0 * d;
            r.idx += t0 * k;
            r.gate += t0 * k;
            r.T = T - t0 < ROUTE_EACH ? T - t0 : ROUTE_EACH;
            if constexpr (R::LDS) rows_to_lds(r.x, r.T, row_bytes, xl);
            route_all<R>(r, smem, xl, l, true);
            return;
        }
        grid -= p.route_blocks;
        block -= p.route_blocks;
    }
    if constexpr (H::LDS) rows_to_lds(p.x, T, row_bytes, xl);
    const void* const mine_w = tid < E ? p.w_in[tid] : nullptr;
    if (tid < 2 * MAXE) (&l.bits[0][0])[tid] = 0u;
    int e = -1;
    if constexpr (H::TT > 0) {
        route_all<H>(p.route, smem, xl, l, blockIdx.x == 0);
        if (tid < T * k) e = l.id[tid];
    } else {
        if (!FIRST && tid < T * k) e = p.route.idx[tid];
        if constexpr (H::LDS) MOE_WAIT_VMCNT(0);
        __syncthreads();
    }
    if (tid < E) l.w[tid] = mine_w;
    make_lists(l, E, e, tid / k, 0.f, ~0ull);
    u32x4* const turn = (u32x4*)smem + wave * PLACE;
    f32x4* const heads = (f32x4*)((u32x4*)smem + NW * PLACE);            // [wavefront][group][lane]
    const __amdgpu_buffer_rsrc_t x = make_rsrc(p.x, (unsigned)T * row_bytes);
    const int lines = d * ES / 128;
    // Items of 16 weight rows: the shared expert's first, then the active experts'.  The work-group has every grid-th of them, and its
    // wavefronts equal shares of their lines by what these cost: whole items, and an item's head or tail at either end.
    const int s_items = p.shared_F / 8, per = p.F / (p.glu ? 8 : 16), n_active = sgpr(l.n_active), items = s_items + n_active * per;
    const int mine = items > block ? (items - block + grid - 1) / grid : 0;
    auto cost_of = [&](int n) __attribute__((always_inline)) {           // of a line of the work-group's item n
        const int item = n * grid + block - s_items, e = l.active[item < 0 || n >= mine ? 0 : item / per];
        return n >= mine ? 0u : (unsigned)line_cost(item < 0 ? T : l.first[e + 1] - l.first[e]);
    };
    const unsigned c0 = cost_of(lane), up0 = moe_wave_scan_u32(c0);
    unsigned all = (unsigned)__builtin_amdgcn_readlane((int)up0, 63);
    for (int n0 = 64; n0 < mine; n0 += 64) all += moe_wave_sum_u32(cost_of(n0 + lane));
    const int total = (int)(all * (unsigned)lines), lo = sgpr((int)((unsigned long long)total * (unsigned)wave / NW)),
              hi = sgpr((int)((unsigned long long)total * (unsigned)(wave + 1) / NW));
    // the first item of the share, and where it begins
    int n = 0, base = 0;
    for (int n0 = 0; n0 < mine; n0 += 64) {
        const unsigned up = n0 ? moe_wave_scan_u32(cost_of(n0 + lane)) : up0;
        const int count = (int)__popcll(__ballot(n0 + lane < mine && (base + (int)up) * lines <= lo));
        if (count) base += __builtin_amdgcn_readlane((int)up, count - 1);
        n += count;
        if (count < 64) break;
    }
    base = sgpr(base) * lines;
    // Where the item is: number `ai` of the active experts (-1: the shared one), item q of its.
    auto step = [&](int& ai, int& q) __attribute__((always_inline)) {    // the work-group's next
        q += grid;
        while (q >= (ai < 0 ? s_items : per) && ai < n_active) {
            q -= ai < 0 ? s_items : per;
            ++ai;
        }
    };
    struct Item {
        int r0, m, width, out0;
        bool shared, glu;
        unsigned char* h;
    };
    auto item_of = [&](int ai, int q) __attribute__((always_inline)) {
        Item it;
        const bool shared = ai < 0;
        const int e = shared ? 0 : sgpr(l.active[ai]);
        it.shared = shared;
        it.glu = shared || p.glu;
        it.r0 = shared ? 0 : sgpr(l.first[e]);
        it.m = shared ? T : sgpr(l.first[e + 1]) - it.r0;
        it.width = shared ? p.shared_F : p.F;
        it.h = shared ? p.s_h : p.h;
        it.out0 = F32 ? (it.glu ? (q >> 2) * 32 + (q & 3) * 8 : q * 16)
                      : (it.glu ? (q >> 2) * 32 + (q & 1) * 16 + ((q >> 1) & 1) : (q >> 1) * 32 + (q & 1));
        return it;
    };
    auto finish = [&](const Item& it, f32x4 a, int g) __attribute__((always_inline)) {
        const int r = g * 16 + l16;
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float up = __shfl_xor(a[i], 32);
            v[i] = it.glu ? silu_f(a[i]) * up : relu_f(a[i]);
        }
        if (r < it.m && (!it.glu || lq < 2)) {
            // H in rows by token and choice; or an expert's rows piece by piece, 16 bytes of every row behind one another, so that a fragment
            // of any rows is one run of bytes.  The lane's four outputs are in one piece (16 bits: every other one of its eight).
            const int col = it.out0 + 4 * lq * (F32 ? 1 : 2), piece = col * ES / 16;
            const size_t row = it.width * ES;
            unsigned char* to = it.h + (p.h_rows ? (it.shared ? r : (int)l.pair[it.r0 + r]) * row + piece * 16 : it.r0 * row + ((size_t)piece * it.m + r) * 16);
            if constexpr (F32) {
                *(f32x4*)to = f32x4{v[0], v[1], v[2], v[3]};
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) ((uint16_t*)to)[(col & 1) + 2 * i] = half_bits(v[i]);
            }
        }
    };
    // the segment of an item that lies in the share; false behind its end
    auto segment = [&](Segment& s, int ai, int q, int base) __attribute__((always_inline)) {
        if (base >= hi) return false;    // (the items' costs end where the last share does)
        const bool shared = ai < 0, glu = shared || p.glu;
        const int e = shared ? 0 : sgpr(l.active[ai]), r0 = shared ? 0 : sgpr(l.first[e]);
        s.m = shared ? T : sgpr(l.first[e + 1]) - r0;
        const int cost = line_cost(s.m);
        s.l0 = 0;
        s.l1 = lines;
        if (lo > base) s.l0 = (lo - base + cost - 1) / cost;
        if (hi < base + lines * cost) s.l1 = (hi - base + cost - 1) / cost;
        // Packed rows (moe_pack_weights): 16-bit rows 16 h + j of a block of 32 are outputs 2 j + h, fp32 rows are in order; with SwiGLU
        // blocks of 32 gate and 32 up rows alternate.  An item is 16 rows of a block, or 8 gate rows and their 8 up rows.
        const int p0 = glu ? (q >> 2) * 64 + (q & 3) * 8 : q * 16;
        const unsigned char* w = (const unsigned char*)sgpr_ptr(shared ? p.s_w_in[0] : l.w[e]) + (size_t)p0 * row_bytes;
        const unsigned up = (glu ? 32u : 8u) * row_bytes, at = (unsigned)(lane >> 3) * row_bytes + (unsigned)(lane & 7) * 16u;
        s.w = make_rsrc(w, up + 8u * row_bytes);
        s.w_at[0] = at;
        s.w_at[1] = up + at;
        s.x = x;
        s.x_step = 64;
        auto token = [&](int r) __attribute__((always_inline)) { return shared ? r : (int)l.t[r0 + r]; };
        if constexpr (H::LDS) {
#pragma unroll
            for (int g = 0; g < 4; ++g) s.x_at[g] = fragment_at(token(g * 16 + l16 < s.m ? g * 16 + l16 : s.m - 1), row_bytes);
            if constexpr (F32) {
#pragma unroll
                for (int r = 0; r < 8; ++r) s.row_at[r] = piece_at(token(r < s.m ? r : s.m - 1), row_bytes);
            }
        } else {
            s.x_at[1] = s.x_at[2] = s.x_at[3] = NOWHERE;         // (members without a value end up in scratch memory when copied)
            s.x_at[0] = l16 < s.m ? (unsigned)token(l16 < s.m ? l16 : 0) * row_bytes + (unsigned)lq * 16u : NOWHERE;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = i * 8 + (lane >> 3);
                s.row_at[i] = r < s.m ? (unsigned)token(r < s.m ? r : 0) * row_bytes + (unsigned)(lane & 7) * 16u : NOWHERE;
            }
        }
        return true;
    };
    int ai = -1, q = n * grid + block;
    if (q >= s_items) {
        ai = (q - s_items) / per;
        q = q - s_items - ai * per;
    }
    int tail_ai = 0, tail_q = 0, tail_lines = 0;         // tail_lines > 0: of an item whose rest is with the wavefronts behind
    if (lane == 0) head_lines[wave] = 0;
    stream_all<TY, 2, H::LDS ? IN_LDS : FRAGMENTS, H::LDS ? IN_LDS : LINES, CACHE_NT>(
        turn, xl, hi - lo <= 16,
        [&](Segment& s) __attribute__((always_inline)) {
            while (segment(s, ai, q, base)) {
                if (s.l0 < s.l1) return true;
                base += line_cost(s.m) * lines;
                step(ai, q);
            }
            return false;
        },
        [&](Segment& s) __attribute__((always_inline)) {
            int next_ai = ai, next_q = q;
            step(next_ai, next_q);
            return segment(s, next_ai, next_q, base + line_cost(s.m) * lines) && s.l0 < s.l1;
        },
        [&](const Segment& s, auto& acc) __attribute__((always_inline)) {
            constexpr int G = sizeof(acc) / sizeof(acc[0]);
            if (s.l0 == 0 && s.l1 == lines) {
                const Item it = item_of(ai, q);
#pragma unroll
                for (int g = 0; g < G; ++g) finish(it, acc[g], g);
            } else {
                // (the turning place is free only behind the last segment, which a tail is)
                f32x4* const to = s.l0 ? heads + wave * 256 : (f32x4*)turn;
#pragma unroll
                for (int g = 0; g < G; ++g) to[g * 64 + lane] = acc[g];
                if (s.l0) {
                    if (lane == 0) head_lines[wave] = s.l1 - s.l0;
                } else {
                    tail_ai = ai;
                    tail_q = q;
                    tail_lines = s.l1;
                }
            }
            base += line_cost(s.m) * lines;
            step(ai, q);
        });
    __syncthreads();
    if (tail_lines) {
        const Item it = item_of(tail_ai, tail_q);
        for (int g = 0; g < (it.m + 15) >> 4; ++g) {
            f32x4 a = ((const f32x4*)turn)[g * 64 + lane];
            int have = tail_lines;
            for (int w = wave + 1; have < lines; ++w) {
                const int more = sgpr(head_lines[w]);
                if (more) a += heads[w * 256 + g * 64 + lane];
                have += more;
            }
            finish(it, a, g);
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
    int T, d, E, k, F, shared_F, y_f32, splits, pairs;
};

// WL: 1 for 8 columns of a work-group, 2 for 16.  LDS: the hidden activations (of its tokens) go there first.  splits > 1: that many
// work-groups share a column block: a range of the tokens each (RANGES), or, with one choice per token and no shared expert, the experts.
// pairs (RANGES, LDS): every assignment of the range for itself, so that a token's sums do not depend on what other tokens chose.
template <bool F32, int WL, bool LDS, bool RANGES>
__global__ __launch_bounds__(NTH) void few_out_kernel(Out p) {
    constexpr int ES = F32 ? 4 : 2, TY = F32 ? FP : HF, COLS = WL * 8;
    __shared__ __attribute__((aligned(16))) unsigned char smem[sizeof(u32x4) * 256 * NW];
    __shared__ __attribute__((aligned(16))) unsigned char hl[LDS ? h_bytes(WL) : 16];
    __shared__ __attribute__((aligned(16))) float sums[NW][MAXT][COLS];
    __shared__ Lists l;
    __shared__ int state[MAXT];          // of a token: 0 not this work-group's, 1 to be written, 2 with an assignment to no expert
    const int tid = threadIdx.x, lane = tid & 63, wave = sgpr(tid >> 6), l16 = lane & 15, lq = lane >> 4;
    const int T = p.T, d = p.d, E = p.E, k = p.k, F = p.F, splits = p.splits;
    // (the work-groups of a column block on one XCD where the number of blocks is a multiple of eight)
    const int blocks = d / COLS, split = (int)blockIdx.x / blocks, p0 = ((int)blockIdx.x - split * blocks) * COLS;
    const int t0 = RANGES ? T * split / splits : 0, t1 = RANGES ? T * (split + 1) / splits : T;
    const unsigned long long range = (t1 < 64 ? (1ull << t1) : 0ull) - (1ull << t0);
    const unsigned f_bytes = (unsigned)F * ES, s_bytes = (unsigned)p.shared_F * ES, s_base = (unsigned)((t1 - t0) * k) * f_bytes;
    int e = -1;
    float gate = 0.f;
    if (tid < T * k) {
        e = p.idx[tid];
        gate = p.gate[tid];
    }
    const void* const mine_w = tid < E ? p.w_out[tid] : nullptr;
    if constexpr (LDS) {
        rows_to_lds(p.h + (size_t)(t0 * k) * f_bytes, (t1 - t0) * k, f_bytes, hl);
        if (p.shared_F) rows_to_lds(p.s_h + (size_t)t0 * s_bytes, t1 - t0, s_bytes, hl + s_base);
    }
    if (tid < 2 * MAXE) (&l.bits[0][0])[tid] = 0u;
    if (tid < T) state[tid] = RANGES ? tid >= t0 && tid < t1 : splits == 1;
    for (int i = lane; i < T * COLS; i += 64) (&sums[wave][0][0])[i] = 0.f;
    __syncthreads();
    if (tid < E) l.w[tid] = mine_w;
    if (tid < T * k && (unsigned)e >= (unsigned)E && (RANGES ? state[tid / k] : split == 0)) state[tid / k] = 2;
    if constexpr (LDS) MOE_WAIT_VMCNT(0);
    const bool pairs = RANGES && LDS && p.pairs;
    if (pairs) {
        const int i = tid - t0 * k, n = (t1 - t0) * k;
        if (i >= 0 && i < n) {
            l.active[i] = (unsigned)e < (unsigned)E ? e : -1;
            l.pair[i] = (unsigned short)tid;
            l.t[i] = (unsigned char)(tid / k);
            l.gate[i] = gate;
        }
        if (tid <= n) l.cost[tid] = tid * line_cost(1);
        if (tid == 0) l.n_active = n;
        __syncthreads();
    } else {
        make_lists(l, E, e, tid / k, gate, range);
    }
    u32x4* const turn = (u32x4*)smem + wave * 256;
    const int n_active = sgpr(l.n_active), all_rows = LDS ? 0 : sgpr(l.first[(E + 63) & ~63]);
    const __amdgpu_buffer_rsrc_t h = make_rsrc(p.h, (unsigned)all_rows * f_bytes), s_h = make_rsrc(p.s_h, (unsigned)T * s_bytes);
    // The lines of the active experts' contractions, the shared expert's behind, by what they cost: a wavefront's share of that.
    const int L = F * ES / 128, s_L = p.shared_F * ES / 128, s_cost = line_cost(t1 - t0);
    int ai0 = 0, ai1 = n_active;         // the work-group's experts
    if (!RANGES && splits > 1) {
        const int all = l.cost[n_active];
        int below = 0, upto = 0;
        for (int x = lane; x - lane < n_active; x += 64) {
            const int owner = x < n_active ? l.cost[x] * splits / all : splits;
            below += __popcll(__ballot(owner < split));
            upto += __popcll(__ballot(owner <= split));
        }
        ai0 = below;
        ai1 = upto;
    }
    const int base = sgpr(L * l.cost[ai0]), all = sgpr(L * l.cost[ai1]) - base + s_L * s_cost;
    const int lo = (int)((unsigned long long)all * (unsigned)wave / NW), hi = (int)((unsigned long long)all * (unsigned)(wave + 1) / NW);
    int ai = ai0;
    for (int x = ai0 + lane; x - lane < ai1; x += 64) ai += __popcll(__ballot(x < ai1 && L * l.cost[x + 1] - base <= lo));
    ai = sgpr(ai);
    auto segment = [&](Segment& s, int ai) __attribute__((always_inline)) {
        const bool shared = ai == ai1;
        if (ai > ai1 || (shared && !s_L)) return false;
        const int at = sgpr(L * l.cost[ai]) - base;
        if (at >= hi) return false;
        // the expert's rows (all tokens') begin at `begin` and are `rows`; the work-group's are s.m, `off` behind
        const int chosen = shared ? 0 : sgpr(l.active[ai]), e = pairs && chosen < 0 ? 0 : chosen, have = shared ? s_L : chosen < 0 ? 0 : L;
        const int begin = shared ? 0 : pairs ? ai : sgpr(l.first[e]), rows = shared ? T : pairs ? 1 : sgpr(l.first[e + 1]) - begin;
        const int off = shared ? t0 : pairs ? 0 : sgpr(rows_in(l, e, (1ull << t0) - 1ull)), r0 = begin + off;
        s.m = shared ? t1 - t0 : pairs ? 1 : sgpr(rows_in(l, e, range));
        const int c = line_cost(s.m);
        s.l0 = 0;
        s.l1 = have;
        if (lo > at) s.l0 = (lo - at + c - 1) / c;
        if (hi < at + have * c) s.l1 = (hi - at + c - 1) / c;
        const unsigned row_bytes = shared ? s_bytes : f_bytes, at8 = (unsigned)(lane >> 3) * row_bytes + (unsigned)(lane & 7) * 16u;
        s.w = make_rsrc((const unsigned char*)sgpr_ptr(shared ? p.s_w_out[0] : l.w[e]) + (size_t)p0 * row_bytes, COLS * row_bytes);
        s.w_at[0] = at8;
        s.w_at[1] = at8 + 8u * row_bytes;
        s.x = shared ? s_h : h;
        s.x_step = 64 * rows;
        if constexpr (LDS) {
            const unsigned start = shared ? s_base : 0u;
            auto place = [&](int r) __attribute__((always_inline)) {     // of row r (of the last one, beyond)
                const int at = r < s.m ? r : s.m - 1;
                return shared ? at : (int)l.pair[r0 + at] - t0 * k;
            };
#pragma unroll
            for (int g = 0; g < 4; ++g) s.x_at[g] = start + fragment_at(place(g * 16 + l16), row_bytes);
            if constexpr (F32) {
#pragma unroll
                for (int r = 0; r < 8; ++r) s.row_at[r] = start + piece_at(place(r), row_bytes);
            }
        } else {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int r = g * 16 + l16;
                s.x_at[g] = r < s.m ? (unsigned)begin * row_bytes + (unsigned)(lq * rows + off + r) * 16u : NOWHERE;
            }
        }
        return true;
    };
    stream_all<TY, WL, LDS ? IN_LDS : FRAGMENTS, LDS ? IN_LDS : FRAGMENTS, RANGES ? 0 : CACHE_NT>(
        turn, hl, hi - lo <= 16,
        [&](Segment& s) __attribute__((always_inline)) {
            while (segment(s, ai)) {
                if (s.l0 < s.l1) return true;
                ++ai;
            }
            return false;
        },
        [&](Segment& s) __attribute__((always_inline)) { return segment(s, ai + 1) && s.l0 < s.l1; },
        [&](const Segment& s, auto& acc) __attribute__((always_inline)) {
            constexpr int G = sizeof(acc) / sizeof(acc[0]);
            const bool shared = ai == ai1;
            const int e = shared ? 0 : sgpr(l.active[ai]), r0 = shared ? t0 : pairs ? ai : sgpr(l.first[e] + rows_in(l, e, (1ull << t0) - 1ull));
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const int r = g * 16 + l16;
                if (r < s.m && (WL == 2 || lq < 2)) {
                    const int t = shared ? r0 + r : l.t[r0 + r];
                    const float gate = shared ? 1.f : l.gate[r0 + r];
                    f32x4* to = (f32x4*)&sums[wave][t][4 * lq];          // (an expert's rows are different tokens)
                    f32x4 sum = *to;
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[i] = fmaf(gate, acc[g][i], sum[i]);
                    *to = sum;
                    if (!RANGES && splits > 1) state[t] = 1;
                }
            }
            ++ai;
        });
    __syncthreads();
    for (int i = tid; i < T * COLS; i += NTH) {
        const int t = i / COLS, c = i - t * COLS, row = p0 + c, st = state[t];
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) v += sums[w][t][c];
        if (st == 2) v = __builtin_nanf("");                      // (its gates are NaN)
        const int col = F32 ? row : (row & ~31) + 2 * (row & 15) + ((row >> 4) & 1);
        if (st) {
            if (p.y_f32) ((float*)p.y)[(size_t)t * d + col] = v;
            else ((uint16_t*)p.y)[(size_t)t * d + col] = f32_to_bf16(v);
        }
    }
}
template <bool F32, typename H, typename R = void> void launch_hidden(const Hidden& a, hipStream_t st, int grid = MOE_GEMM_GRID) {
    hipLaunchKernelGGL((few_hidden_kernel<F32, H, R>), dim3((unsigned)grid), dim3(NTH), 0, st, a);
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
    // (offsets inside a buffer are 31 bits: a segment of the first matrix spans 16 rows, with SwiGLU the 8 up rows end 40 rows on; one of the second 16)
    const size_t in_rows = act == MOE_SWIGLU || shared_F ? 40 : 16;
    MOE_REQUIRE(in_rows * d * es < two_gib && (size_t)16 * F * es < two_gib && (size_t)16 * shared_F * es < two_gib && (size_t)T * d * es < two_gib &&
                    (size_t)E * d * es < two_gib && (size_t)T * k * F * es < two_gib && (size_t)T * shared_F * es < two_gib, MOE_ERR_UNSUPPORTED,
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
    // The second launch's work-groups: sixteen columns where they make one per CU, else eight (a matrix instruction half empty, twice the
    // work-groups); where these are few, several share a column block.  With one choice per token they share the experts, and nothing is
    // fetched twice.  Else they share the tokens, and an expert is fetched for every range of tokens that chose it, from the L2 then, while
    // most CUs would have no work.  Ranges of at most eight tokens take every assignment for itself, as few experts are met twice there.
    // (us, unshared / ranges / of assignments: 8 tokens, fp32 d=320 F=1984 E=16 k=2: 51.9 / - / 32.1; 12 tokens, 16-bit d=320 F=512
    // E=24 k=4: 28.7 / 24.8 / 22.1, d=640 F=768 E=24 k=2: - / 28.7 / 26.3; 32 tokens, d=512 F=512 E=24 k=4: - / 31.5 / 32.9)
    const bool apart = k == 1 && !shared_F;
    const bool wide = (long long)(d / 16) * (apart ? T : 1) >= MOE_GEMM_GRID;
    const int blocks = d / (wide ? 16 : 8);
    Out o = {expert_idx, gate_w, w_out, s_w_out, a.h, a.s_h, y, T, d, E, k, F, shared_F, y_dt == MOE_F32, 1, 0};
    while (o.splits < T && blocks * (o.splits + 1) <= MOE_GEMM_GRID) ++o.splits;
    const int range = apart ? T : (T + o.splits - 1) / o.splits;
    // x and the work-group's hidden activations go to LDS first where they fit
    const bool x_lds = (size_t)T * d * es <= X_BYTES, h_lds = (size_t)range * (need / T) <= h_bytes(wide ? 2 : 1);
    a.h_rows = h_lds;
    const bool ranges = !apart && o.splits > 1;      // (then d <= 1024, and eight columns)
    o.pairs = ranges && h_lds && range <= 8;
    // A shared expert whose first matrices take as long to fetch as a launch (16 MB, three microseconds) is worked on while a few work-groups
    // route: d=2048 F=1408 E=60 k=4 shared 5632 (46 MB), us without / with: 1 token 42.9 / 39.7, 9 tokens 106 / 101, 16 tokens 134 / 133, 24
    // tokens 149 / 153 (the routing's loads wait behind the others); d=1152 shared 1600 (7 MB), 4 tokens 29.9 / 31.0.  Eight layers of 17 to 168 MB and
    // d=1024 to 7168, 1 to 16 tokens: with / without 0.96 on the average, 0.80 to 1.06 (d=1024 1.03, d=7168 0.90).
    const bool beside = T <= 16 && (size_t)shared_F * 2 * d * es >= (16u << 20);
    if (dt == MOE_F32) {
        const int rc = moe_route_topk(x, w_gate, bias, T, d, E, k, renorm, dt, expert_idx, gate_w, nullptr, stream);
        if (rc != MOE_OK) return rc;
        x_lds ? launch_hidden<true, Routed<true>>(a, st) : launch_hidden<true, Routed<false>>(a, st);
    } else if (T > ROUTE_MAXT || beside) {
        a.route_blocks = (T + ROUTE_EACH - 1) / ROUTE_EACH;
        const int grid = beside ? MOE_GEMM_GRID : a.route_blocks;
        if (x_lds) launch_hidden<false, Routed<true>, How<1, true>>(a, st, grid);
        else if ((size_t)(T < ROUTE_EACH ? T : ROUTE_EACH) * d * es <= X_BYTES) launch_hidden<false, Routed<false>, How<1, true>>(a, st, grid);
        else launch_hidden<false, Routed<false>, How<1, false>>(a, st, grid);
        MOE_CHECK_LAUNCH("moe_layer_few (routing)");
        if (beside) a.shared_F = 0;      // (its first product is done)
        x_lds ? launch_hidden<false, Routed<true>>(a, st) : launch_hidden<false, Routed<false>>(a, st);
    } else if (T <= 16) {
        x_lds ? launch_hidden<false, How<1, true>>(a, st) : launch_hidden<false, How<1, false>>(a, st);
    } else {
        x_lds ? launch_hidden<false, How<2, true>>(a, st) : launch_hidden<false, How<2, false>>(a, st);
    }
    MOE_CHECK_LAUNCH("moe_layer_few (routing and first product)");
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3((unsigned)(blocks * o.splits)), dim3(NTH), 0, st, o); };
    auto typed = [&](auto f32, auto lds) {
        if (ranges) go(few_out_kernel<f32(), 1, lds(), true>);
        else if (wide) go(few_out_kernel<f32(), 2, lds(), false>);
        else go(few_out_kernel<f32(), 1, lds(), false>);
    };
    if (dt == MOE_F32) h_lds ? typed(std::true_type{}, std::true_type{}) : typed(std::true_type{}, std::false_type{});
    else h_lds ? typed(std::false_type{}, std::true_type{}) : typed(std::false_type{}, std::false_type{});
    MOE_CHECK_LAUNCH("moe_layer_few (second product and combine)");
    return MOE_OK;
}
