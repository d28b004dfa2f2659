// The experts' part of a training step (moe_grouped_ffn_keep, moe_grouped_ffn_backward).  Row r of expert e (offsets[e] <= r < offsets[e+1]) is
// assignment a = perm[r] of token t = a / k with weight w = gate_w[a]:
//
//   keep       z = x[t] W_in     h = relu(z), or silu(g) u of z = (g, u)     z kept in 8 bits (keep.h), h in half
//   backward   s = dy[t] W_out^T     dgate_w[a] = sum_f h s     dh = w s     dz = dh [z > 0], or (dh u sig(g) (1 + g (1 - sig(g))), dh silu(g))
//              dx_perm[r] = dz W_in^T     dW_in = sum_r x[t]^T dz     dW_out = sum_r (w h)^T dy[t]
//
// Three products over an expert's rows (z, s, dx_perm: gemm_nt_kernel, which differ in their operands and in what is done with the result) and two over
// the rows themselves (dW_in, dW_out: gemm_tn_kernel).  What bounds them: arithmetic where experts hold many rows, the fetch of the matrices and the
// stores of their gradients where they hold few.
//
// Both kernels: work-groups of four wavefronts, one a CU (two where gemm_tn_kernel's tiles are of 128), persistent, take items one after another:
// 256 features of 256, 128 or 64 rows (gemm_nt_kernel), 256 x 256 or 128 x 128 values of a gradient (gemm_tn_kernel).  The contraction goes through
// two or three buffers of 64 terms in LDS, or four of 32 rows, filled by loads that go there directly and run on into the next items, so
// that these start without a pause.  The fragments of the next 32 terms are read while those before are multiplied.
//
// Measured (us, medians: z with its 8 bits, s with dz and w h, dx, dW; parts of the whole calls):
//   8192 tokens, top-4 of 60 experts of 2048 x 1408, SwiGLU     502   306   453   886     0.75, 0.62, 0.83, 0.64 PFLOP/s
//   16384 tokens, top-1 of 128 experts of d = 768, F = 4 d      209   224   194   518     z: 3.7 TB/s
//   8192 tokens, top-2 of 8 experts of 4096 x 14336, SwiGLU    3601  2145  3722  5421     1.07, 0.90, 1.03, 1.07 PFLOP/s
// What bounds them now.  The loops: the way from the L2s to LDS and the matrix instructions together (dW: 64 KB a stage of 64 rows, 1.4 us for the
// fetch alone, 2.0 with its multiplications; the L2s deliver 8.5 TB/s, the matrix units are busy 60% of the time).  An item's end: nothing covers the
// epilogue (13 us of the backward pass's first product, mostly vector instructions), and loads behind an item's stores are counted behind
// them, which dW feels where experts hold few rows: 16384 tokens 545 us, 320 without its stores
// (1.2 GB), when both were measured; 518 now.
//
// Rounded on the way: dz and w h, once, to bf16 (the matrix instruction's type), and what is kept in 8 bits.  Sums are fp32.
#include <type_traits>
#include "common.h"
#include "ffn_kernels.h"
#include "gemm_util.h"
#include "keep.h"

namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(8))) float f32x8;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int NTH = 256;
[[maybe_unused]] constexpr int XCD = 8;
constexpr int GROUP_ROWS = 8;              // row tiles of an expert that are taken together, column block after column block

// (nothing may move across: neither memory operations nor matrix-core work)
__device__ __forceinline__ void wg_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
}

// A buffer descriptor as four registers, for loads written as assembly: the compiler counts a global -> LDS load that it knows of as a store
// that any LDS read may depend on, and waits for all of them before reads that it cannot tell apart from their targets (the transposing
// ones, row tables): the loads here have no register that is written, and the kernels wait for them by themselves.
__device__ __forceinline__ u32x4 descriptor(const void* p, unsigned bytes) {
    const uint64_t u = (uint64_t)p;
    return u32x4{(unsigned)sgpr((int)(unsigned)u), (unsigned)sgpr((int)(unsigned)(u >> 32)) & 0xffffu, (unsigned)sgpr((int)bytes), 0x00020000u};
}
// What a load below may read: the words in scalar registers, which a vector instruction (the lane read that brings them there, where the compiler holds
// them in vector registers over a loop) has not written for five wait states.  The hardware does not check this, and the compiler sees to it for
// its own loads only; the build counts the states in the assembly.  settled: with the wait.  pinned: at this place, for a load with matrix instructions
// before it, once for a half's loads (in front of each load they would be two states ahead of it; with the wait a backward pass over 8192 tokens, 8 experts of
// 4096 x 14336, takes 11.5 ms instead of 11.2).
__device__ __forceinline__ u32x4 scalars(const u32x4& r) {
    return u32x4{(unsigned)sgpr((int)r[0]), (unsigned)sgpr((int)r[1]), (unsigned)sgpr((int)r[2]), (unsigned)sgpr((int)r[3])};
}
__device__ __forceinline__ u32x4 pinned(const u32x4& r) {
    u32x4 d = scalars(r);
    asm volatile("" : "+s"(d));
    __builtin_amdgcn_sched_barrier(0);
    return d;
}
__device__ __forceinline__ u32x4 settled(const u32x4& r) {
    u32x4 d = scalars(r);
    asm volatile("s_nop 4" : "+s"(d));
    return d;
}
// 16 bytes a lane to LDS at base + at (bytes, wave-uniform) + 16 lane, from voff + add (the sum saturates: an offset beyond everything stays that);
// only this one is range-checked, soff is not.  (M0 may not be used in the instruction behind the one that sets it: the sum stands between.)
__device__ __forceinline__ void load_to_lds(const u32x4& r, unsigned base, unsigned at, unsigned voff, unsigned add, unsigned soff) {
    unsigned sum;
    asm volatile("s_add_u32 m0, %1, %2\n\tv_add_u32_e64 %0, %3, %4 clamp\n\tbuffer_load_dwordx4 %0, %5, %6 offen lds"
                 : "=&v"(sum) : "s"(base), "i"(at), "v"(voff), "s"(add), "s"(r), "s"(soff) : "memory", "scc");
}
// 4 bytes a lane
__device__ __forceinline__ void load_to_lds4(const u32x4& r, unsigned to, unsigned voff) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(to), "v"(voff), "s"(r) : "memory");
}

// A store of 16 bytes.  Its data registers may not be written in the instruction behind it: with an offset in a scalar register the compiler takes
// that for safe, and with two wavefronts a SIMD the last lanes' first values came out as what was written there next.
// STREAM: past the caches, for results that are larger than these.  Only where an instruction writes whole lines of 128 bytes (halves of lines are
// put together in the caches: a gradient stored so in halves took 15% longer, in whole lines 5% less), and to leave in them what is read again: a
// backward pass of 100 tokens over 128 experts of d = 768, F = 4 d, took 338 us instead of 400, of 16384 tokens 970 instead of 1025.
constexpr int STREAM = 2;
template <int AUX = 0> __device__ __forceinline__ void store_b128(u32x4 v, __amdgpu_buffer_rsrc_t r, unsigned voff, unsigned soff) {
    __builtin_amdgcn_raw_buffer_store_b128(v, r, voff, soff, AUX);
    asm volatile("s_nop 1" : : "v"(v) : "memory");         // (they live until behind it)
}

// Two pieces of 16 bytes of a row l16 of sixteen, 64 bytes apart, to whole lines for a store: rows l16 % 8 (a) and 8 + l16 % 8 (b), the second 64 bytes in
// lanes 8 to 15.
__device__ __forceinline__ void to_lines(u32x4& a, u32x4& b) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int lo = (int)a[i], hi = (int)b[i];
        a[i] = (unsigned)__builtin_amdgcn_update_dpp(lo, hi, 0x128, 0xf, 0xc, false);      // (turned by eight lanes of sixteen)
        b[i] = (unsigned)__builtin_amdgcn_update_dpp(hi, lo, 0x128, 0xf, 0x3, false);
    }
}

// The lane's number, formed where it is used: held in a register over the loops it ends up in scratch memory, and the wait for its way back is one
// for all loads under way.
__device__ __forceinline__ int lane_now() {
    int v;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(v));
    return v;
}

// What was issued before `LOADS` loads and an item's stores is there once only those (at least `stores` of the latter) are under way.
template <int LOADS> __device__ __forceinline__ void wait_landed(int stores) {
    static_assert(LOADS <= 30, "vmcnt range");
    if (stores >= 63 - LOADS) MOE_WAIT_VMCNT(63);
    else if (stores >= 32) MOE_WAIT_VMCNT(LOADS + 32);
    else if (stores >= 16) MOE_WAIT_VMCNT(LOADS + 16);
    else MOE_WAIT_VMCNT(LOADS);
}

// a / k for a < 2^30, m = (2^32 - 1) / k: the product is one too small at most (k = 1 too)
__device__ __forceinline__ unsigned divided(unsigned a, unsigned k, unsigned m) {
    const unsigned q = __umulhi(a, m);
    return a - q * k >= k ? q + 1 : q;
}

// Sum and largest over the four lanes l16, l16 + 16, l16 + 32, l16 + 48; all four get it.
__device__ __forceinline__ float quarter_sum(float v) {
    const unsigned b = __float_as_uint(v);
    const u32x2 p = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    const unsigned c = __float_as_uint(__uint_as_float(p[0]) + __uint_as_float(p[1]));
    const u32x2 q = __builtin_amdgcn_permlane32_swap(c, c, false, false);
    return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}
__device__ __forceinline__ unsigned quarter_max(unsigned v) {
    const u32x2 p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    const unsigned c = max_u32(p[0], p[1]);
    const u32x2 q = __builtin_amdgcn_permlane32_swap(c, c, false, false);
    return max_u32(q[0], q[1]);
}
__device__ __forceinline__ u32x4 to_bf16(const float (&v)[8]) {
    const f32x8 f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
    return __builtin_bit_cast(u32x4, __builtin_convertvector(f, bf16x8));      // to nearest, ties to even
}

// Running sums over the experts, four of them a lane (E <= 256): lane l holds the sums up to and with experts 4 l .. 4 l + 3.
struct Sums {
    int s[4];
    __device__ __forceinline__ int total() const { return __builtin_amdgcn_readlane(s[3], 63); }
    // up to, and without, expert e
    __device__ __forceinline__ int before(int e) const {
        if (e == 0) return 0;
        const int l = (e - 1) >> 2, j = (e - 1) & 3;
        const int a = __builtin_amdgcn_readlane(s[0], l), b = __builtin_amdgcn_readlane(s[1], l);
        const int c = __builtin_amdgcn_readlane(s[2], l), d = __builtin_amdgcn_readlane(s[3], l);
        return j == 0 ? a : j == 1 ? b : j == 2 ? c : d;
    }
    // the expert in whose share `at` lies
    __device__ __forceinline__ int find(int at) const {
        return __popcll(__ballot(s[0] <= at)) + __popcll(__ballot(s[1] <= at)) + __popcll(__ballot(s[2] <= at)) + __popcll(__ballot(s[3] <= at));
    }
};
template <typename F> __device__ __forceinline__ Sums sums_over_experts(const int32_t* offsets, int E, int lane, F share) {
    Sums r;
    int at[5];
#pragma unroll
    for (int j = 0; j < 5; ++j) at[j] = offsets[4 * lane + j < E ? 4 * lane + j : E];
    int sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        sum += 4 * lane + j < E ? share(at[j + 1] - at[j]) : 0;
        r.s[j] = sum;
    }
    const int before = (int)moe_wave_scan_u32((unsigned)sum) - sum;
#pragma unroll
    for (int j = 0; j < 4; ++j) r.s[j] += before;
    return r;
}

// ------------------------------------------------------------------------------------------ products over an expert's rows
// D[feature][row] = sum over terms of W[feature][term] R[row][term]: the features are the matrix instruction's rows, so that a lane has eight
// neighbouring features of one row and can load and store them in whole pieces.
enum { KEEP_RELU = 0, KEEP_SWIGLU = 1, HID_RELU = 2, HID_SWIGLU = 3, DX = 4 };

struct NtArgs {
    const uint16_t* rows;          // x, dy [T,K] (gathered) or dz [A, ld_rows]
    const int32_t *offsets, *perm;
    const void* const* w_ptrs;     // KEEP: packed [N,K] matrices
    const uint16_t *w0, *w1;       // else: [E] matrices of N rows of ld_w values; w1 continues w0's contraction (DX, SwiGLU)
    size_t w_stride;
    int T, k, E, N, KT, KT0;       // stages, of them with w0
    int ld_rows, ld_w, F, Z, parts;
    const int8_t* q_in;
    const float *scale_in, *gate_w;
    int8_t* q_out;
    float *scale_out, *dx_perm, *dgate_part;
    uint16_t *h, *dz, *wh;
};

template <int TR> struct Nt {
    static constexpr int NI = TR / 64;                     // 32-row blocks of a wavefront (two wavefronts share the rows, block by block)
    static constexpr int F_BYTES = 256 * 128, R_BYTES = TR * 128, STAGE = F_BYTES + R_BYTES;
    static constexpr int NFL = 8, NRL = TR / 32, LPS = NFL + NRL;      // loads per thread and stage
    // Stages in LDS: two of 256 rows (all that there is room for), three of fewer, whose time is the way of the matrices from HBM.
    static constexpr int RING = TR == 256 ? 2 : 3, ROWS_AT = RING * STAGE;
    static constexpr size_t SMEM = ROWS_AT + 8 * TR * 4;
};
template <int TR> using NtAcc = f32x4[Nt<TR>::NI][2][4][2];            // [32-row block][its half][32-feature block][its half]
template <int TR> struct NtFrags { bf16x8 f[4][2], r[Nt<TR>::NI][2]; };

struct NtItem { int e, row0, rc, n0; };

template <int TR> __device__ __forceinline__ NtItem nt_locate(const NtArgs& a, const Sums& tiles, int ncb, int item) {
    NtItem it;
    const int tile_at = item / ncb;
    it.e = sgpr(tiles.find(tile_at));
    const int first = tiles.before(it.e);
    const int begin = a.offsets[it.e], n = a.offsets[it.e + 1] - begin;
    const int R = (n + TR - 1) / TR;
    const int local = item - first * ncb;
    const int grp = local / (GROUP_ROWS * ncb), rem = local - grp * GROUP_ROWS * ncb;
    const int gs = R - grp * GROUP_ROWS < GROUP_ROWS ? R - grp * GROUP_ROWS : GROUP_ROWS;
    const int cb = rem / gs, tile = grp * GROUP_ROWS + rem - cb * gs;
    it.row0 = sgpr(begin + tile * TR);
    it.rc = sgpr(n - tile * TR < TR ? n - tile * TR : TR);
    it.n0 = sgpr(cb * 256);
    return it;
}

// The loader's place in the stream of stages: it runs RING of them ahead of the multiplications, across the items' borders.
template <int TR> struct NtLoader {
    u32x4 rr, rf;
    unsigned vr[Nt<TR>::NRL], vf;  // byte offsets: of this thread's rows, of its first feature
    int item, kt, buf, seq;
};
struct NtWork {
    int ncb, end, stride;
    unsigned ring, rinfo, div;     // LDS addresses; for the division by k
    int wave, lane, ld_row;
    unsigned piece;
};

// (gather) the assignments of an item's rows: eight items' tables in turn
template <int TR> __device__ __forceinline__ void nt_fetch_rows(const NtArgs& a, const NtWork& w, const NtItem& it, int seq) {
    if (w.wave * 64 < TR)
        load_to_lds4(settled(descriptor(a.perm + it.row0, (unsigned)it.rc * 4u)), w.rinfo + (unsigned)((seq & 7) * TR + w.wave * 64) * 4u, (unsigned)(w.wave * 64 + w.lane) * 4u);
}

template <int KIND, int TR> __device__ __forceinline__ void nt_turn(const NtArgs& a, const NtWork& w, const Sums& tiles, const int* rinfo, NtLoader<TR>& L) {
    if (L.item >= w.end) {                                 // past the last item: nothing is fetched, the schedule stays
        L.rr = L.rf = descriptor(a.rows, 0u);
        return;
    }
    const NtItem it = nt_locate<TR>(a, tiles, w.ncb, L.item);
    const int nr = a.N - it.n0 < 256 ? a.N - it.n0 : 256;
    const unsigned bytes = (unsigned)nr * (unsigned)a.ld_w * 2u;
    if constexpr (KIND <= KEEP_SWIGLU) {
        L.rf = descriptor((const uint16_t*)a.w_ptrs[it.e] + (size_t)it.n0 * a.ld_w, bytes);
    } else {
        const size_t at = (size_t)it.e * a.w_stride + (size_t)it.n0 * a.ld_w;
        L.rf = descriptor(a.w0 + at, bytes);
    }
    if constexpr (KIND == DX) {
        L.rr = descriptor(a.rows + (size_t)it.row0 * a.ld_rows, (unsigned)it.rc * (unsigned)a.ld_rows * 2u);
    } else {
        L.rr = descriptor(a.rows, (unsigned)a.T * (unsigned)a.ld_rows * 2u);
#pragma unroll
        for (int q = 0; q < Nt<TR>::NRL; ++q) {
            const int row = q * 32 + w.ld_row;
            unsigned src = (unsigned)rinfo[(L.seq & 7) * TR + row];
            src = divided(src, (unsigned)a.k, w.div);
            // (a row past the tile's end gets an offset beyond the matrix: the range check reads zeros)
            L.vr[q] = row < it.rc ? src * (unsigned)a.ld_rows * 2u + w.piece : 0xFFFFFFF0u;
        }
        if (L.item + w.stride < w.end) nt_fetch_rows<TR>(a, w, nt_locate<TR>(a, tiles, w.ncb, L.item + w.stride), L.seq + 1);
        ++L.seq;
    }
}

// load Q of the loader's stage (the features first)
struct NtFrom { u32x4 rr, rf; };
template <int KIND, int TR, int Q> __device__ __forceinline__ void nt_load(const NtArgs& a, const NtWork& w, const NtLoader<TR>& L, const NtFrom& from) {
    const unsigned to = w.ring + (unsigned)(L.buf * Nt<TR>::STAGE + w.wave * 1024);
    if constexpr (Q < Nt<TR>::NFL)
        load_to_lds(from.rf, to, Q * 4096, L.vf, (unsigned)(Q * 32) * (unsigned)a.ld_w * 2u, (unsigned)(KIND == DX && L.kt >= a.KT0 ? L.kt - a.KT0 : L.kt) * 128u);
    else
        load_to_lds(from.rr, to, Nt<TR>::F_BYTES + (Q - Nt<TR>::NFL) * 4096, L.vr[Q - Nt<TR>::NFL], 0u, (unsigned)L.kt * 128u);
}
template <int KIND, int TR, int FROM, int TO> __device__ __forceinline__ void nt_loads(const NtArgs& a, const NtWork& w, const NtLoader<TR>& L, const NtFrom& from) {
    if constexpr (FROM < TO) {
        nt_load<KIND, TR, FROM>(a, w, L, from);
        nt_loads<KIND, TR, FROM + 1, TO>(a, w, L, from);
    }
}
// after the last load of a stage
template <int KIND, int TR> __device__ __forceinline__ void nt_advance(const NtArgs& a, const NtWork& w, const Sums& tiles, const int* rinfo, NtLoader<TR>& L) {
    L.buf = L.buf + 1 == Nt<TR>::RING ? 0 : L.buf + 1;
    ++L.kt;
    if (KIND == DX && L.kt == a.KT0 && L.kt < a.KT)        // the second matrix: its place in the first one's stead
        L.rf = descriptor((const void*)(((uint64_t)L.rf[1] << 32 | L.rf[0]) + ((uint64_t)a.w1 - (uint64_t)a.w0)), L.rf[2]);
    if (L.kt == a.KT) {
        L.kt = 0;
        if (L.item < w.end) L.item += w.stride;
        nt_turn<KIND, TR>(a, w, tiles, rinfo, L);
    }
}

struct NtLane { int f_rd, r_rd; };              // first half's fragment of the first block

// fragment read j of a half (32 terms): features first
template <int TR> __device__ __forceinline__ void nt_read(NtFrags<TR>& fr, const unsigned char* ring, int j, int at_f, int at_r) {
    if (j < 8) fr.f[j >> 1][j & 1] = *(const bf16x8*)(ring + at_f + (j >> 1) * 4096 + (j & 1) * 2048);
    else fr.r[(j - 8) >> 1][j & 1] = *(const bf16x8*)(ring + at_r + ((j - 8) >> 1) * 8192 + (j & 1) * 2048);
}

// Half S of the stage in buffer `buf`: multiplies set S, reads the other.  Half 1 issues the loads of the stage after the next into the buffer that
// this one has left.  FIRST: of an item's first RING - 1 stages,
// behind whose loads the stores of the item before (at least `stores`) may be under way.
template <int KIND, int TR, int S, bool FULL, int t>
__device__ __forceinline__ void nt_groups(const NtArgs& a, const NtWork& w, const NtLoader<TR>& L, const NtFrom& from, const unsigned char* ring, int at_f, int at_r,
                                          NtAcc<TR>& acc, NtFrags<TR> (&fr)[2], int ni_on) {
    constexpr int G = Nt<TR>::NI * 4, READS = 8 + 2 * Nt<TR>::NI, SPREAD = G >= 16 ? 12 : G, LPS = Nt<TR>::LPS;
    if constexpr (t < G) {
        constexpr int ni = t >> 2, n16 = (t >> 1) & 1, b0 = (t & 1) * 2;
        if (FULL || ni < ni_on) {
#pragma unroll
            for (int b = b0; b < b0 + 2; ++b)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    acc[ni][n16][b][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fr[S].f[b][h], fr[S].r[ni][n16], acc[ni][n16][b][h], 0, 0, 0);
        }
        if (t < SPREAD) {
#pragma unroll
            for (int j = t * READS / SPREAD; j < (t + 1) * READS / SPREAD; ++j) nt_read<TR>(fr[S ^ 1], ring, j, at_f, at_r);
        }
        if constexpr (S == 1) nt_loads<KIND, TR, t * LPS / G, (t + 1) * LPS / G>(a, w, L, from);
        __builtin_amdgcn_sched_barrier(0);
        nt_groups<KIND, TR, S, FULL, t + 1>(a, w, L, from, ring, at_f, at_r, acc, fr, ni_on);
    }
}
template <int KIND, int TR, int S, bool FIRST, bool FULL>
__device__ __forceinline__ void nt_half(const NtArgs& a, const NtWork& w, const Sums& tiles, const int* rinfo, NtLoader<TR>& L, const NtLane& ln, const unsigned char* ring, int& buf,
                                        NtAcc<TR>& acc, NtFrags<TR> (&fr)[2], int stores, int ni_on) {
    if (S == 1) buf = buf + 1 == Nt<TR>::RING ? 0 : buf + 1;
    const int at_f = buf * Nt<TR>::STAGE + (ln.f_rd ^ (S == 0 ? 64 : 0)), at_r = buf * Nt<TR>::STAGE + (ln.r_rd ^ (S == 0 ? 64 : 0));
    NtFrom from = {};
    if (S == 1) from = NtFrom{KIND == DX ? pinned(L.rr) : scalars(L.rr), scalars(L.rf)};      // (the others the compiler holds in scalar registers)
    nt_groups<KIND, TR, S, FULL, 0>(a, w, L, from, ring, at_f, at_r, acc, fr, ni_on);
    if (S == 0) {
        // everybody has read all of this stage, and the next one is there
        MOE_WAIT_LGKMCNT(0);
        if (FIRST) wait_landed<(Nt<TR>::RING - 2) * Nt<TR>::LPS>(stores);
        else MOE_WAIT_VMCNT((Nt<TR>::RING - 2) * Nt<TR>::LPS);
        wg_barrier();
        nt_advance<KIND, TR>(a, w, tiles, rinfo, L);
    }
}

template <int KIND, int TR, bool FULL>
__device__ __forceinline__ void nt_contract(const NtArgs& a, const NtWork& w, const Sums& tiles, const int* rinfo, NtLoader<TR>& L, const NtLane& ln, const unsigned char* ring,
                                            int& buf, NtAcc<TR>& acc, NtFrags<TR> (&fr)[2], int stores, int ni_on) {
    nt_half<KIND, TR, 0, true, FULL>(a, w, tiles, rinfo, L, ln, ring, buf, acc, fr, stores, ni_on);
    nt_half<KIND, TR, 1, false, FULL>(a, w, tiles, rinfo, L, ln, ring, buf, acc, fr, 0, ni_on);
    int kt = 1;
    if (Nt<TR>::RING > 2 && kt < a.KT) {
        nt_half<KIND, TR, 0, true, FULL>(a, w, tiles, rinfo, L, ln, ring, buf, acc, fr, stores, ni_on);
        nt_half<KIND, TR, 1, false, FULL>(a, w, tiles, rinfo, L, ln, ring, buf, acc, fr, 0, ni_on);
        ++kt;
    }
#pragma clang loop unroll(disable)
    for (; kt < a.KT; ++kt) {
        nt_half<KIND, TR, 0, false, FULL>(a, w, tiles, rinfo, L, ln, ring, buf, acc, fr, 0, ni_on);
        nt_half<KIND, TR, 1, false, FULL>(a, w, tiles, rinfo, L, ln, ring, buf, acc, fr, 0, ni_on);
    }
}

// (v_rcp_f32 is off by one unit in the last place at most)
__device__ __forceinline__ float sigmoid(float v) { return __builtin_amdgcn_rcpf(1.f + __expf(-v)); }

// A lane's features of block b in a row: natural order (slots arranged by gemm_nt_kernel), or packed rows (packed row 16 h + j = output 2 j + h).
template <bool PACKED> __device__ __forceinline__ void lane_values(const f32x4 (&acc)[2], float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = PACKED ? acc[i & 1][i >> 1] : acc[i >> 2][i & 3];
}

template <int KIND, int TR>
__device__ __forceinline__ void nt_finish(const NtArgs& a, const NtItem& it, const int* rinfo, const NtAcc<TR>& acc, int wm, int wn, int lane, int ni_on) {
    const int l16 = lane & 15, lq = lane >> 4;
    const int f0 = it.n0 + wm * 128;                       // this wavefront's first feature
    if (f0 >= a.N) return;
    const size_t row0 = (size_t)it.row0;
    const unsigned rc = (unsigned)it.rc;
    if constexpr (KIND == DX) {
        const __amdgpu_buffer_rsrc_t ro = make_rsrc(a.dx_perm + row0 * a.N, rc * (unsigned)a.N * 4u);
        const unsigned ld = (unsigned)a.N * 4u, row = (unsigned)(wn * 32 + l16);
#pragma unroll
        for (int ni = 0; ni < Nt<TR>::NI; ++ni) {
            if (ni >= ni_on) continue;
#pragma unroll
            for (int n16 = 0; n16 < 2; ++n16) {
                const unsigned down = (unsigned)(ni * 64 + n16 * 16);
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    if (f0 + b * 32 >= a.N) continue;
                    const unsigned col = (unsigned)(f0 + b * 32) * 4u;
                    if constexpr (TR == 256) {             // (no registers for the exchange: the caches put the lines together)
#pragma unroll
                        for (int h = 0; h < 2; ++h) store_b128(__builtin_bit_cast(u32x4, acc[ni][n16][b][h]), ro, (row + down) * ld + (unsigned)(lq * 32 + h * 16), col);
                    } else {
                        // a lane has 32 bytes of a row: the halves of lanes 32 apart change places, then rows' halves
                        u32x4 v[2];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const u32x2 p = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[ni][n16][b][0][i]), __float_as_uint(acc[ni][n16][b][1][i]), false, false);
                            v[0][i] = p[0];
                            v[1][i] = p[1];
                        }
                        to_lines(v[0], v[1]);
                        const unsigned at = (row - (unsigned)(l16 & 8) + down) * ld + (unsigned)((l16 >> 3) * 64 + (lq & 1) * 32 + (lq >> 1) * 16);
                        store_b128<STREAM>(v[0], ro, at, col);
                        store_b128<STREAM>(v[1], ro, at + 8u * ld, col);
                    }
                }
            }
        }
    } else if constexpr (KIND <= KEEP_SWIGLU) {
        const unsigned F = (unsigned)a.F, Z = (unsigned)a.Z;
        const __amdgpu_buffer_rsrc_t rh = make_rsrc(a.h + row0 * F, rc * F * 2u);
        const __amdgpu_buffer_rsrc_t rq = make_rsrc(a.q_out + row0 * Z, rc * Z);
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(a.scale_out + row0 * (Z / 64), rc * (Z / 64) * 4u);
#pragma unroll
        for (int ni = 0; ni < Nt<TR>::NI; ++ni) {
            if (ni >= ni_on) continue;
#pragma unroll
            for (int n16 = 0; n16 < 2; ++n16) {
                const unsigned row = (unsigned)((ni * 2 + wn) * 32 + n16 * 16 + l16);
                // two blocks of 64 kept columns: neighbouring features (ReLU), or the gates and the ups of the same 64 outputs
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    constexpr bool SW = KIND == KEEP_SWIGLU;
                    const int b0 = SW ? p : 2 * p, db = SW ? 2 : 1;
                    const int zc = SW ? f0 / 2 + p * a.F : f0 + p * 64;            // column of z
                    if (!SW && zc >= a.F) continue;
                    float v[2][8];
                    unsigned most = 0;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        lane_values<true>(acc[ni][n16][b0 + i * db], v[i]);
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            if (!SW) v[i][c] = relu_f(v[i][c]);
                            most = max_u32(most, magnitude(v[i][c]));
                        }
                    }
                    const KeepScale ks = keep_scale(quarter_max(most));
                    __builtin_amdgcn_sched_barrier(0);     // (one block's values at a time: there are no registers for more)
                    if (lq == 0) __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(ks.scale), rs, row * (Z / 64) * 4u, (unsigned)(zc / 64) * 4u, 0);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const u32x2 w = {keep_four<!SW>(v[i][0], v[i][1], v[i][2], v[i][3], ks.to_q), keep_four<!SW>(v[i][4], v[i][5], v[i][6], v[i][7], ks.to_q)};
                        __builtin_amdgcn_raw_buffer_store_b64(w, rq, row * Z + (unsigned)lq * 8u, (unsigned)(zc + i * 32), 0);
                    }
                    if (!SW || p == 1) {
                        u32x4 w[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            if (SW) {                      // (v holds the ups)
                                float g[8];
                                lane_values<true>(acc[ni][n16][2 * i], g);
#pragma unroll
                                for (int c = 0; c < 8; ++c) v[i][c] *= g[c] * sigmoid(g[c]);
                            }
                            w[i] = u32x4{half_bits(v[i][0], v[i][1]), half_bits(v[i][2], v[i][3]), half_bits(v[i][4], v[i][5]), half_bits(v[i][6], v[i][7])};
                        }
                        to_lines(w[0], w[1]);
                        const unsigned at = (row - (unsigned)(l16 & 8)) * F * 2u + (unsigned)((l16 >> 3) * 64 + lq * 16);
#pragma unroll
                        for (int i = 0; i < 2; ++i) store_b128(w[i], rh, at + (unsigned)i * F * 16u, (unsigned)(SW ? f0 / 2 : zc) * 2u);
                    }
                }
            }
        }
    } else {
        constexpr bool SW = KIND == HID_SWIGLU;
        constexpr int MATS = SW ? 2 : 1, NG = Nt<TR>::NI * 2;
        const unsigned F = (unsigned)a.F, Z = (unsigned)a.Z;
        const __amdgpu_buffer_rsrc_t rq = make_rsrc(a.q_in + row0 * Z, rc * Z);
        const __amdgpu_buffer_rsrc_t rs = make_rsrc(a.scale_in + row0 * (Z / 64), rc * (Z / 64) * 4u);
        const __amdgpu_buffer_rsrc_t rz = make_rsrc(a.dz + row0 * Z, rc * Z * 2u);
        const __amdgpu_buffer_rsrc_t rw = make_rsrc(a.wh + row0 * F, rc * F * 2u);
        const int on = a.N - f0 < 128 ? a.N - f0 : 128;    // features of this wavefront: 64 or 128
        const unsigned last = (unsigned)((on - 64) / 64);  // (where there are 64, the second 64 read the first's once more)
        // (group g: 16 rows, first_row + rows_of(g); what is added to a lane's offset is wave-uniform)
        const unsigned first_row = (unsigned)(wn * 32 + l16);
        auto rows_of = [](int g) { return (unsigned)((g >> 1) * 64 + (g & 1) * 16); };
        float gate[NG];
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const unsigned row = first_row + rows_of(g);
            gate[g] = a.gate_w && row < rc ? a.gate_w[rinfo[row]] : 1.f;
        }
        // What is kept is fetched AHEAD groups ahead: loads are counted together with the stores before them, so that a load issued
        // behind a group's stores would wait for their way to memory.
        constexpr int AHEAD = NG < 4 ? NG - 1 : 3;
        u32x2 q[AHEAD + 1][MATS][4];
        float sc[AHEAD + 1][MATS][2];
        unsigned q_at = first_row * Z + (unsigned)lq * 8u, s_at = first_row * (Z / 64) * 4u;
        auto fetch = [&](int g) {
            const int to = g % (AHEAD + 1);
            asm volatile("" : "+v"(q_at), "+v"(s_at));     // (keeps the groups' offsets from being formed, and held, up front)
            const unsigned qo = q_at + rows_of(g) * Z, so = s_at + rows_of(g) * (Z / 64) * 4u;
#pragma unroll
            for (int m = 0; m < MATS; ++m) {
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    q[to][m][b] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rq, qo, (unsigned)(f0 + m * a.F) + (b < 2 ? 0u : last * 64u) + (unsigned)(b & 1) * 32u, 0));
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    sc[to][m][j] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, so, ((unsigned)(f0 + m * a.F) / 64u + (j ? last : 0u)) * 4u, 0));
            }
        };
        const unsigned line_row = first_row - (unsigned)(l16 & 8), in_line = (unsigned)((l16 >> 3) * 64 + lq * 16);
        unsigned w_at = line_row * F * 2u + in_line, z_at = line_row * Z * 2u + in_line;
#pragma unroll
        for (int g = 0; g < AHEAD; ++g) fetch(g);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const int ni = g >> 1, n16 = g & 1, at = g % (AHEAD + 1);
            if (g + AHEAD < NG) fetch(g + AHEAD);
            __builtin_amdgcn_sched_barrier(0);
            if (ni >= ni_on) continue;
            const unsigned row = first_row + rows_of(g);
            asm volatile("" : "+v"(w_at), "+v"(z_at));
            const unsigned wo = w_at + rows_of(g) * F * 2u, zo = z_at + rows_of(g) * Z * 2u;
            float dgate = 0.f;
            u32x4 wh_b[2], dz0_b[2], dz1_b[2];             // of two blocks, for whole lines
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                if (b * 32 >= on) continue;
                float s[8], wh[8], dz0[8], dz1[8];
                lane_values<false>(acc[ni][n16][b], s);
                const unsigned zw[2] = {q[at][0][b][0], q[at][0][b][1]}, uw[2] = {q[at][MATS - 1][b][0], q[at][MATS - 1][b][1]};
                const float zs = sc[at][0][b >> 1], us = sc[at][MATS - 1][b >> 1];
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const float z = (float)(int8_t)(zw[c >> 2] >> (8 * (c & 3))) * zs;
                    const float dh = gate[g] * s[c];
                    float h;
                    if (SW) {
                        const float u = (float)(int8_t)(uw[c >> 2] >> (8 * (c & 3))) * us;
                        const float sig = sigmoid(z), silu = z * sig;
                        h = silu * u;
                        dz0[c] = dh * u * fmaf(silu, 1.f - sig, sig);
                        dz1[c] = dh * silu;
                    } else {
                        h = z;
                        dz0[c] = z > 0.f ? dh : z;         // (z is 0 else, or no number)
                    }
                    dgate = fmaf(h, s[c], dgate);
                    wh[c] = gate[g] * h;
                }
                wh_b[b & 1] = to_bf16(wh);
                dz0_b[b & 1] = to_bf16(dz0);
                if (SW) dz1_b[b & 1] = to_bf16(dz1);
                if (b & 1) {
                    const unsigned col = (unsigned)(f0 + (b - 1) * 32) * 2u;
                    to_lines(wh_b[0], wh_b[1]);
                    to_lines(dz0_b[0], dz0_b[1]);
                    if (SW) to_lines(dz1_b[0], dz1_b[1]);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        store_b128<STREAM>(wh_b[i], rw, wo + (unsigned)i * F * 16u, col);
                        store_b128<STREAM>(dz0_b[i], rz, zo + (unsigned)i * Z * 16u, col);
                        if (SW) store_b128<STREAM>(dz1_b[i], rz, zo + (unsigned)i * Z * 16u, col + F * 2u);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            dgate = quarter_sum(dgate);
            if (lq == 0 && row < rc) a.dgate_part[(row0 + row) * (size_t)a.parts + (unsigned)(f0 / 128)] = dgate;
        }
    }
}

template <int KIND, int TR>
__global__ __launch_bounds__(NTH) void gemm_nt_kernel(const NtArgs a) {
#ifdef __HIP_DEVICE_COMPILE__                              // (the host's pass makes the stub only: it has no buffer descriptors)
    extern __shared__ __attribute__((aligned(1024))) unsigned char ring[];
    const int* rinfo = (const int*)(ring + Nt<TR>::ROWS_AT);
    const int tid = threadIdx.x, lane = tid & 63, wave = sgpr(tid >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    const int l16 = lane & 15, lq = lane >> 4;
    const Sums tiles = sums_over_experts(a.offsets, a.E, lane, [](int n) { return (n + TR - 1) / TR; });
    NtWork w;
    w.ncb = (a.N + 255) / 256;
    // the XCDs take neighbouring runs of the items, so that an expert's matrix stays in few L2s
    const long long all = (long long)tiles.total() * w.ncb;
    const int xcd = (int)blockIdx.x % XCD;
    w.stride = (int)gridDim.x / XCD;
    w.end = sgpr((int)(all * (xcd + 1) / XCD));
    const int first = sgpr((int)(all * xcd / XCD) + (int)blockIdx.x / XCD);
    if (first >= w.end) return;
    w.ring = (unsigned)(uintptr_t)(lds_void_t*)ring;
    w.rinfo = w.ring + Nt<TR>::ROWS_AT;
    w.div = 0xFFFFFFFFu / (unsigned)a.k;
    w.wave = wave;
    w.lane = lane;
    w.ld_row = tid >> 3;
    w.piece = (unsigned)((tid & 7) ^ ((w.ld_row >> 1) & 7)) << 4;
    NtLane ln;
    const int frag = l16 * 128 + ((lq ^ (l16 >> 1)) << 4);
    ln.f_rd = wm * (128 * 128) + frag;
    ln.r_rd = Nt<TR>::F_BYTES + wn * (32 * 128) + frag;

    NtLoader<TR> L;
    // packed matrices: rows as they lie; else slot 16 h + j of a block of 32 holds feature 8 (j / 4) + 4 h + j % 4: the two halves give a lane
    // eight neighbours
    const int f = KIND <= KEEP_SWIGLU ? w.ld_row : ((w.ld_row & 12) << 1) + ((w.ld_row & 16) >> 2) + (w.ld_row & 3);
    L.vf = (unsigned)f * (unsigned)a.ld_w * 2u + w.piece;
#pragma unroll
    for (int q = 0; q < Nt<TR>::NRL; ++q) L.vr[q] = (unsigned)(q * 32 + w.ld_row) * (unsigned)a.ld_rows * 2u + w.piece;      // (DX)
    L.item = first;
    L.kt = L.buf = L.seq = 0;
    if constexpr (KIND != DX) {
        nt_fetch_rows<TR>(a, w, nt_locate<TR>(a, tiles, w.ncb, first), 0);
        MOE_WAIT_VMCNT(0);
        wg_barrier();
    }
    nt_turn<KIND, TR>(a, w, tiles, rinfo, L);
#pragma unroll
    for (int st = 0; st < Nt<TR>::RING; ++st) {
        nt_loads<KIND, TR, 0, Nt<TR>::LPS>(a, w, L, NtFrom{settled(L.rr), settled(L.rf)});
        if (st + 1 == Nt<TR>::RING) break;
        if (KIND != DX && a.KT < Nt<TR>::RING) {           // (the next item's rows may be wanted now)
            MOE_WAIT_VMCNT(0);
            wg_barrier();
        }
        nt_advance<KIND, TR>(a, w, tiles, rinfo, L);
    }
    MOE_WAIT_VMCNT((Nt<TR>::RING - 1) * Nt<TR>::LPS);
    wg_barrier();
    NtAcc<TR> acc;
    NtFrags<TR> fr[2];
#pragma unroll
    for (int j = 0; j < 8 + 2 * Nt<TR>::NI; ++j) nt_read<TR>(fr[0], ring, j, ln.f_rd, ln.r_rd);
    int buf = 0, stores = 0, seq = 0;
    for (int item = first; item < w.end; item += w.stride, ++seq) {
        const NtItem it = nt_locate<TR>(a, tiles, w.ncb, item);
#pragma unroll
        for (int ni = 0; ni < Nt<TR>::NI; ++ni)
#pragma unroll
            for (int j = 0; j < 16; ++j) acc[ni][j >> 3][(j >> 1) & 3][j & 1] = f32x4{0.f, 0.f, 0.f, 0.f};
        int ni_on = ((it.rc + 31) / 32 - wn + 1) / 2;      // 32-row blocks of this wavefront that hold rows
        ni_on = ni_on > Nt<TR>::NI ? Nt<TR>::NI : ni_on;
        if (ni_on == Nt<TR>::NI) nt_contract<KIND, TR, true>(a, w, tiles, rinfo, L, ln, ring, buf, acc, fr, stores, ni_on);
        else nt_contract<KIND, TR, false>(a, w, tiles, rinfo, L, ln, ring, buf, acc, fr, stores, ni_on);
        nt_finish<KIND, TR>(a, it, rinfo + (seq & 7) * TR, acc, wm, wn, lane, ni_on);
        // store instructions just issued, at least: two for every 32 rows x 32 features (SwiGLU: gates and ups make one block of outputs)
        int cols = (a.N - it.n0 - wm * 128 + 31) / 32;
        cols = cols < 0 ? 0 : cols > 4 ? 4 : cols;
        stores = ni_on * 2 * cols * (KIND == KEEP_SWIGLU ? 1 : 2);
    }
    MOE_WAIT_VMCNT(0);                                      // (the trailing empty loads still target this LDS)
#endif
}

// ------------------------------------------------------------------------------------------ products over the rows
// dW[m][n] = sum over an expert's rows r of M[r][m] N[r][n].  Both operands lie with the contraction outermost: LDS holds 64 rows of 256
// columns of each, and the reads that transpose (ds_read_b64_tr_b16: lane i of sixteen gets column i of four rows) bring the terms of a column together.
// One operand is gathered (x for dW_in, dy for dW_out), the other lies in the experts' order (dz, w h).
struct TnArgs {
    const uint16_t *x, *dy, *dz, *wh;
    const int32_t* offsets;
    const uint32_t* src;           // of each row in the experts' order, the bits of its token's byte offset in x and dy inverted
    int T, E, d, F, Z, mats;
    void *dwa, *dwb, *dwo;
};

// TS: the side of a tile of dW, 256 (a work-group a CU) or 128 (two).
template <int TS> struct Tn {
    static constexpr int PANELS = TS / 64, BLOCKS = TS / 32;          // of 64 columns; of 16 columns, a wavefront
    static constexpr int BUF = 32 * TS * 2;                // LDS: an operand's 32 rows; the N operand's four buffers, then the M operand's
    static constexpr int IDS = 8 * BUF;                    // behind them source rows: [8 halves][4 wavefronts][64 lanes]
    static constexpr int LOADS = 2 * PANELS;               // of a thread, for a half
    static constexpr int GROUPS = BLOCKS * BLOCKS / 4;     // of four matrix instructions a step
    static constexpr size_t SMEM = IDS + 8 * 4 * 256;
};

struct TnItem {
    int e, row0, n, m0, n0, M, N;
    bool out;                      // dW_out (M: w h, N: dy gathered); else dW_in (M: x gathered, N: dz from column zc)
    int zc;
    void* dw;
};

struct TnShape { int ta, tb, per_mat, per_expert; };       // tiles along d and F

template <int TS, int ES> __device__ __forceinline__ TnItem tn_locate(const TnArgs& a, const TnShape& sh, int item) {
    TnItem it;
    it.e = sgpr(item / sh.per_expert);
    const int local = item - it.e * sh.per_expert, mat = local / sh.per_mat, at = local - mat * sh.per_mat;
    it.out = mat == a.mats - 1;
    it.M = it.out ? a.F : a.d;
    it.N = it.out ? a.d : a.F;
    const int tm = it.out ? sh.tb : sh.ta, tn = it.out ? sh.ta : sh.tb;
    const int grp = at / (GROUP_ROWS * tn), rem = at - grp * GROUP_ROWS * tn;
    const int gs = tm - grp * GROUP_ROWS < GROUP_ROWS ? tm - grp * GROUP_ROWS : GROUP_ROWS;
    const int cb = rem / gs;
    it.n0 = sgpr(cb * TS);
    it.m0 = sgpr((grp * GROUP_ROWS + rem - cb * gs) * TS);
    it.row0 = sgpr(a.offsets[it.e]);
    it.n = sgpr(a.offsets[it.e + 1]) - it.row0;
    it.zc = mat == 1 ? a.F : 0;
    it.dw = (unsigned char*)(it.out ? a.dwo : mat == 1 ? a.dwb : a.dwa) + (size_t)it.e * a.d * a.F * ES;
    return it;
}

struct TnWork {
    TnShape sh;
    int end, stride;
    unsigned ring;                 // LDS address
    int wave;
};
// A lane's row among a load's 32, times 4; its place in the tables of source rows; the piece of 16 bytes that it fetches of a panel's row (rows 2 r and
// 2 r + 1 fill 256 bytes, and the transposing reads of 32 lanes, 32 bytes of eight rows, touch all 64 banks once).
struct TnThread {
    int wave;
    unsigned tables;
    __device__ __forceinline__ unsigned row4() const { return (unsigned)(wave * 8 + (lane_now() >> 3)) * 4u; }
    __device__ __forceinline__ unsigned ids() const { return tables + (unsigned)lane_now() * 4u; }
    __device__ __forceinline__ unsigned piece() const {
        const unsigned l = (unsigned)lane_now();
        return ((l & 7u) ^ ((l >> 4 & 3u) << 1)) << 4;
    }
};

// The contraction goes in stages of 64 rows, in halves of 32 through four buffers: the loads of a half are issued while the one four before is multiplied and
// are due two steps later.  An operand's 32 rows of 256 columns lie in LDS as four panels of 64 columns: a load of a wavefront fetches whole
// 128-byte lines of eight rows, load Q rows 8 wave + lane / 8 of panel Q.
//
// The loader's place in the stream of stages (items without rows have none).
struct TnLoads {
    int item, left;                // rows of the item from this stage on
    u32x4 rd, rg;                  // the direct operand's rows of this stage, the gathered one's matrix
    unsigned ld_d, cd, cg, to_d, to_g;
    unsigned vd;                   // this thread's row in the direct operand
};
// two stages ahead of it, the fetch of source rows
struct TnAhead {
    int item, left;
    u32x4 src;
};
__device__ __forceinline__ unsigned rows_of_stage(int left) { return (unsigned)(left < 0 ? 0 : left < 64 ? left : 64); }
// Turns to the first item with rows from L.item on.
template <int TS, int ES> __device__ __forceinline__ void tn_turn(const TnArgs& a, const TnWork& w, const TnThread& th, TnLoads& L) {
    for (; L.item < w.end; L.item += w.stride) {
        const TnItem it = tn_locate<TS, ES>(a, w.sh, L.item);
        if (it.n == 0) continue;
        const int ld = it.out ? a.F : a.Z;
        L.left = it.n;
        L.ld_d = (unsigned)ld * 2u;
        L.rd = descriptor((it.out ? a.wh : a.dz) + (size_t)it.row0 * ld, rows_of_stage(it.n) * L.ld_d);
        L.rg = descriptor(it.out ? a.dy : a.x, (unsigned)a.T * (unsigned)a.d * 2u);
        L.vd = (th.row4() >> 2) * L.ld_d + th.piece();
        L.cd = (unsigned)(it.out ? it.m0 : it.n0 + it.zc) * 2u;
        L.cg = (unsigned)(it.out ? it.n0 : it.m0) * 2u;
        const unsigned to = w.ring + (unsigned)(w.wave * 1024);
        L.to_d = to + (it.out ? 4 * Tn<TS>::BUF : 0);
        L.to_g = to + (it.out ? 0 : 4 * Tn<TS>::BUF);
        return;
    }
    L.left = 0;                                            // past the last item: nothing is fetched, the schedule stays
    L.ld_d = 0u;
    L.rd = L.rg = descriptor(a.dz, 0u);
}
// To the next stage of the item; at its end, which the caller sees to (left <= 0), to something that is not used.
__device__ __forceinline__ void tn_step_on(TnLoads& L) {
    const uint64_t at = ((uint64_t)L.rd[1] << 32 | L.rd[0]) + (uint64_t)L.ld_d * 64u;
    L.left -= 64;
    L.rd[0] = (unsigned)at;
    L.rd[1] = (unsigned)(at >> 32);
    L.rd[2] = rows_of_stage(L.left) * L.ld_d;
}
template <int TS, int ES> __device__ __forceinline__ void tn_next_item(const TnArgs& a, const TnWork& w, const TnThread& th, TnLoads& L) {
    if (L.item < w.end) L.item += w.stride;
    tn_turn<TS, ES>(a, w, th, L);
}
__device__ __forceinline__ void tn_turn(const TnArgs& a, const TnWork& w, TnAhead& p) {
    for (; p.item < w.end; p.item += w.stride) {
        const int e = sgpr(p.item / w.sh.per_expert), row0 = sgpr(a.offsets[e]);
        p.left = sgpr(a.offsets[e + 1]) - row0;
        p.src = descriptor(a.src + row0, (unsigned)p.left * 4u);
        if (p.left > 0) return;
    }
    p.left = 0;
    p.src = descriptor(a.src, 0u);
}
__device__ __forceinline__ void tn_step_on(TnAhead& p) {
    const uint64_t at = ((uint64_t)p.src[1] << 32 | p.src[0]) + 256u;
    p.left -= 64;
    p.src[0] = (unsigned)at;
    p.src[1] = (unsigned)(at >> 32);
    p.src[2] = (unsigned)(p.left < 0 ? 0 : p.left) * 4u;
}
__device__ __forceinline__ void tn_next_item(const TnArgs& a, const TnWork& w, TnAhead& p) {
    if (p.item < w.end) p.item += w.stride;
    tn_turn(a, w, p);
}
// Every lane's source row of half h of a stage, into one of eight tables of its wavefront's (behind the expert's last row: zeros).
template <int TS> __device__ __forceinline__ void tn_fetch_ids(const TnWork& w, const TnThread& th, const u32x4& src, int h, int slot) {
    load_to_lds4(src, w.ring + (unsigned)(Tn<TS>::IDS + slot * 1024 + w.wave * 256), th.row4() + (unsigned)h * 128u);
}
// Its offset.  (One that is not there has the largest offset, and keeps it: the range check reads zeros.)
__device__ __forceinline__ unsigned tn_row(const TnThread& th, int slot) {
    typedef __attribute__((address_space(3))) unsigned lds_word;
    return __builtin_elementwise_add_sat(~*(lds_word*)(uintptr_t)(th.ids() + (unsigned)slot * 1024u), th.piece());
}
// load Q of half H: the direct operand's first
struct TnFrom { u32x4 rd, rg, src; };
template <int TS, int H, int Q> __device__ __forceinline__ void tn_load(const TnLoads& L, const TnFrom& from, unsigned buf_at, unsigned row) {
    constexpr int N = Tn<TS>::PANELS, p = Q % N;
    if constexpr (Q < N) load_to_lds(from.rd, L.to_d + buf_at, p * 4096, L.vd, L.cd + (unsigned)(H * 32) * L.ld_d + (unsigned)p * 128u, 0u);
    else load_to_lds(from.rg, L.to_g + buf_at, p * 4096, row, L.cg + (unsigned)p * 128u, 0u);
}
template <int TS, int H, int FROM, int TO> __device__ __forceinline__ void tn_loads(const TnLoads& L, const TnFrom& from, unsigned buf_at, unsigned row) {
    if constexpr (FROM < TO) {
        tn_load<TS, H, FROM>(L, from, buf_at, row);
        tn_loads<TS, H, FROM + 1, TO>(L, from, buf_at, row);
    }
}

template <int TS> using TnAcc = f32x4[Tn<TS>::BLOCKS][Tn<TS>::BLOCKS];         // [16 rows of dW][16 columns of dW]
template <int TS> struct TnFrags { s16x4 n[Tn<TS>::BLOCKS][2], m[Tn<TS>::BLOCKS][2]; };

// Read j of the half in buffer `half` of two: four terms of a column of a 16-column block.  n[c]: this lane's place in block c of the N operand's
// first panel (pair of buffers included); the M operand's lie a wave-uniform distance behind.
struct TnLane { unsigned n[4], to_m; };
template <int TS> __device__ __forceinline__ void tn_read(TnFrags<TS>& fr, const TnLane& at, int half, int j) {
    constexpr int B = Tn<TS>::BLOCKS;
    const int c = j % (2 * B) >> 1, i = j & 1, off = half * Tn<TS>::BUF + (c >> 2) * 4096 + i * 2048;
    typedef __attribute__((address_space(3))) unsigned char lds_byte;
    if (j < 2 * B) fr.n[c][i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)((lds_byte*)(uintptr_t)at.n[c & 3] + off));
    else fr.m[c][i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)((lds_byte*)(uintptr_t)(at.n[c & 3] + at.to_m) + off));
}
__device__ __forceinline__ bf16x8 tn_frag(const s16x4 (&f)[2]) {
    typedef __attribute__((ext_vector_type(8))) short s16x8;
    const s16x8 v = __builtin_shufflevector(f[0], f[1], 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, v);
}

// Step S multiplies the half in buffer 2 pair + S (its fragments are in registers), reads the next one's fragments and issues the loads of the fourth one
// behind it into the same buffer, which everybody has read.  What moves the places on stands between the multiplications: a wavefront has
// its SIMD for itself, an instruction that none of them covers costs its whole time.
template <int TS, int S, int t>
__device__ __forceinline__ void tn_groups(const TnWork& w, const TnThread& th, TnLoads& L, TnFrom& from, TnAhead& ahead, const TnLane& ln, int pair, int slot,
                                          unsigned& row, TnAcc<TS>& acc, TnFrags<TS> (&fr)[2]) {
    constexpr int B = Tn<TS>::BLOCKS, G = Tn<TS>::GROUPS, READS = 4 * B, SPREAD = 3 * G / 4, LOADS = Tn<TS>::LOADS;
    if constexpr (t < G) {
        constexpr int m = t / (B / 4), n4 = t % (B / 4) * 4;
        if constexpr (t == 0) row = tn_row(th, (slot + 4) & 7);
        if constexpr (t == G - 2) from.src = pinned(ahead.src);
        if constexpr (t == G - 1) tn_fetch_ids<TS>(w, th, from.src, S, slot);
        static_assert(SPREAD <= G - 1, "the places move on behind the loads");
        if constexpr (S == 1 && t == (G > 4 ? G - 2 : G - 1)) tn_step_on(L);
        if constexpr (S == 1 && t == G - 1) tn_step_on(ahead);
#pragma unroll
        for (int n = n4; n < n4 + 4; ++n)
            acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(tn_frag(fr[S].n[n]), tn_frag(fr[S].m[m]), acc[m][n], 0, 0, 0);
        if (t < SPREAD) {
#pragma unroll
            for (int j = t * READS / SPREAD; j < (t + 1) * READS / SPREAD; ++j) tn_read<TS>(fr[S ^ 1], ln, S ^ 1, j);
        }
        if constexpr (t < SPREAD) tn_loads<TS, S, t * LOADS / SPREAD, (t + 1) * LOADS / SPREAD>(L, from, (unsigned)((pair * 2 + S) * Tn<TS>::BUF), row);
        __builtin_amdgcn_sched_barrier(0);
        tn_groups<TS, S, t + 1>(w, th, L, from, ahead, ln, pair, slot, row, acc, fr);
    }
}
template <int TS, int ES, int S>
__device__ __forceinline__ void tn_step(const TnArgs& a, const TnWork& w, const TnThread& th, TnLoads& L, TnAhead& ahead, TnLane& ln, int& slot, TnAcc<TS>& acc, TnFrags<TS> (&fr)[2],
                                        int stores) {
    const int pair = (slot >> 1) & 1;
    if (S == 1) {
#pragma unroll
        for (int c = 0; c < 4; ++c) ln.n[c] ^= 2 * Tn<TS>::BUF;
    }
    unsigned row;
    TnFrom from = {pinned(L.rd), scalars(L.rg)};
    tn_groups<TS, S, 0>(w, th, L, from, ahead, ln, pair, slot, row, acc, fr);
    slot = (slot + 1) & 7;
    // everybody has read the next half, and the one behind it is there: what was issued before the last two steps (their loads and a fetch of source
    // rows each) and an item's stores
    MOE_WAIT_LGKMCNT(0);
    wait_landed<2 * (Tn<TS>::LOADS + 1)>(stores);
    wg_barrier();
    if (S == 1) {
        if (L.left <= 0) tn_next_item<TS, ES>(a, w, th, L);
        if (ahead.left <= 0) tn_next_item(a, w, ahead);
    }
}

template <int TS, int ES>
__device__ __forceinline__ void tn_contract(const TnArgs& a, const TnWork& w, const TnThread& th, TnLoads& L, TnAhead& ahead, TnLane& ln, int KT, int& slot, TnAcc<TS>& acc,
                                            TnFrags<TS> (&fr)[2], int stores) {
    tn_step<TS, ES, 0>(a, w, th, L, ahead, ln, slot, acc, fr, stores);
    tn_step<TS, ES, 1>(a, w, th, L, ahead, ln, slot, acc, fr, stores);
#pragma clang loop unroll(disable)
    for (int kt = 1; kt < KT; ++kt) {
        tn_step<TS, ES, 0>(a, w, th, L, ahead, ln, slot, acc, fr, 0);
        tn_step<TS, ES, 1>(a, w, th, L, ahead, ln, slot, acc, fr, 0);
    }
}

template <int TS, typename O, bool ADD> __device__ __forceinline__ void tn_finish(const TnItem& it, TnAcc<TS>& acc, int wm, int wn) {
    constexpr unsigned ES = sizeof(O);
    const int lane = lane_now(), l16 = lane & 15, lq = lane >> 4;
    constexpr int B = Tn<TS>::BLOCKS;
    const int c0 = it.n0 + wm * (TS / 2);
    if (c0 >= it.N) return;
    const unsigned ld = (unsigned)it.N * ES;
    const __amdgpu_buffer_rsrc_t ro = make_rsrc((unsigned char*)it.dw + (size_t)it.m0 * ld, (unsigned)(it.M - it.m0 < TS ? it.M - it.m0 : TS) * ld);
#pragma unroll
    for (int m = 0; m < B; ++m) {
        // the lane's piece in a row: four fp32 columns of 16, or eight bf16 ones of 32 (below)
        const unsigned in_row = ES == 4 ? (unsigned)lq * 16u : (unsigned)((lq & 1) * 16 + (lq >> 1) * 8) * 2u;
        const unsigned from = (unsigned)(wn * (TS / 2) + m * 16 + l16) * ld + in_row;
        const unsigned to = (unsigned)(wn * (TS / 2) + m * 16 + (l16 & 7)) * ld + (unsigned)(l16 >> 3) * 64u + in_row, to8 = to + 8u * ld;
        __builtin_amdgcn_sched_barrier(0);                 // (16 rows at a time: there are no registers for more)
#pragma unroll
        for (int n = 0; n < B; n += 128 / (16 * (int)ES)) {
            if (c0 + n * 16 >= it.N) continue;             // (N is a multiple of 64)
            const unsigned col = (unsigned)(c0 + n * 16) * ES;
            u32x4 out[2];
            if constexpr (ES == 4) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    f32x4 v;                               // (a copy: the sums stay where the matrix instruction wants them)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float x = acc[m][n + i][r];
                        asm volatile("" : "+v"(x));
                        v[r] = x;
                    }
                    if (ADD) v += __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(ro, from, col + (unsigned)i * 64u, 0));
                    out[i] = __builtin_bit_cast(u32x4, v);
                }
            } else {
                // a lane has columns 4 lq + r of two blocks of 16; lanes 16 apart exchange them, so that each has eight neighbours:
                // columns 0, 16, 8, 24 .. + 7 for lq = 0 .. 3
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float v[8];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const u32x2 p = __builtin_amdgcn_permlane16_swap(__float_as_uint(acc[m][n + 2 * i][r]), __float_as_uint(acc[m][n + 2 * i + 1][r]), false, false);
                        v[r] = __uint_as_float(p[0]);
                        v[4 + r] = __uint_as_float(p[1]);
                    }
                    if (ADD) {
                        const u32x4 old = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(ro, from, col + (unsigned)i * 64u, 0));
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += __uint_as_float(e & 1 ? old[e >> 1] & 0xffff0000u : old[e >> 1] << 16);
                    }
                    out[i] = to_bf16(v);
                }
            }
            to_lines(out[0], out[1]);
            store_b128<STREAM>(out[0], ro, to, col);
            store_b128<STREAM>(out[1], ro, to8, col);
        }
    }
}

template <int TS, typename O, bool ADD>
__global__ __launch_bounds__(NTH, TS == 256 ? 1 : 2) void gemm_tn_kernel(const TnArgs a) {
#ifdef __HIP_DEVICE_COMPILE__
    extern __shared__ __attribute__((aligned(1024))) unsigned char ring[];
    constexpr int ES = sizeof(O);
    const int tid = threadIdx.x, lane = tid & 63, wave = sgpr(tid >> 6);
    const int wm = wave & 1, wn = wave >> 1, l16 = lane & 15, lq = lane >> 4;
    TnWork w;
    w.sh.ta = (a.d + TS - 1) / TS;
    w.sh.tb = (a.F + TS - 1) / TS;
    w.sh.per_mat = w.sh.ta * w.sh.tb;
    w.sh.per_expert = w.sh.per_mat * a.mats;
    // An item costs its stages and the store of its tile (about six stages' time).  The XCDs take neighbouring runs of equal cost.
    const Sums cost = sums_over_experts(a.offsets, a.E, lane, [](int n) { return 6 + (n + 63) / 64; });
    const int xcd = (int)blockIdx.x % XCD;
    auto bound = [&](int x) {
        const long long at = (long long)cost.total() * w.sh.per_expert * x / XCD;
        if (x == XCD) return a.E * w.sh.per_expert;
        const int e = cost.find((int)(at / w.sh.per_expert));
        const long long in = at - (long long)cost.before(e) * w.sh.per_expert;
        return sgpr(e * w.sh.per_expert + (int)(in / (cost.before(e + 1) - cost.before(e))));
    };
    w.stride = (int)gridDim.x / XCD;
    w.end = bound(xcd + 1);
    const int first = bound(xcd) + (int)blockIdx.x / XCD;
    if (first >= w.end) return;
    w.ring = (unsigned)(uintptr_t)(lds_void_t*)ring;
    w.wave = wave;
    TnLane ln;
    const int row = lq * 4 + (l16 >> 2);                   // lane (l16, lq) reads from rows 4 lq + l16 / 4 of sixteen
#pragma unroll
    for (int c = 0; c < 4; ++c) ln.n[c] = w.ring + (unsigned)(wm * (TS * 32) + row * 128 + (l16 & 3) * 8) + (unsigned)((c ^ (row >> 1 & 3)) * 32);
    ln.to_m = (unsigned)sgpr(4 * Tn<TS>::BUF + (wn - wm) * (TS * 32));

    TnThread th;
    th.wave = wave;
    th.tables = w.ring + (unsigned)(Tn<TS>::IDS + wave * 256);

    // two stages on their way, the source rows of the two behind them
    TnLoads L;
    L.item = first;
    L.vd = L.cd = L.cg = L.to_d = L.to_g = 0u;
    tn_turn<TS, ES>(a, w, th, L);
    TnAhead ahead;
    ahead.item = first;
    tn_turn(a, w, ahead);
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        tn_fetch_ids<TS>(w, th, settled(ahead.src), 0, 2 * st);
        tn_fetch_ids<TS>(w, th, settled(ahead.src), 1, 2 * st + 1);
        tn_step_on(ahead);
        if (ahead.left <= 0) tn_next_item(a, w, ahead);
    }
    MOE_WAIT_VMCNT(0);
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        tn_loads<TS, 0, 0, Tn<TS>::LOADS>(L, TnFrom{settled(L.rd), settled(L.rg)}, (unsigned)(2 * st * Tn<TS>::BUF), tn_row(th, 2 * st));
        tn_fetch_ids<TS>(w, th, settled(ahead.src), 0, 4 + 2 * st);
        tn_loads<TS, 1, 0, Tn<TS>::LOADS>(L, TnFrom{settled(L.rd), settled(L.rg)}, (unsigned)((2 * st + 1) * Tn<TS>::BUF), tn_row(th, 2 * st + 1));
        tn_fetch_ids<TS>(w, th, settled(ahead.src), 1, 5 + 2 * st);
        tn_step_on(L);
        if (L.left <= 0) tn_next_item<TS, ES>(a, w, th, L);
        tn_step_on(ahead);
        if (ahead.left <= 0) tn_next_item(a, w, ahead);
    }
    MOE_WAIT_VMCNT(2 * (Tn<TS>::LOADS + 1));
    wg_barrier();
    TnAcc<TS> acc;
    TnFrags<TS> fr[2];
#pragma unroll
    for (int j = 0; j < 4 * Tn<TS>::BLOCKS; ++j) tn_read<TS>(fr[0], ln, 0, j);
    int slot = 0, stores = 0;
    for (int item = first; item < w.end; item += w.stride) {
        const TnItem it = tn_locate<TS, ES>(a, w.sh, item);
        const int KT = (it.n + 63) / 64;
        if (ADD && KT == 0) continue;
        constexpr int B = Tn<TS>::BLOCKS;
        int n_on = (it.N - it.n0 - wm * (TS / 2)) / 16;    // 16-column blocks of this wavefront inside the matrix
        n_on = n_on < 0 ? 0 : n_on > B ? B : n_on;
#pragma unroll
        for (int m = 0; m < B; ++m)
#pragma unroll
            for (int n = 0; n < B; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (KT > 0) {
            tn_contract<TS, ES>(a, w, th, L, ahead, ln, KT, slot, acc, fr, stores);
            stores = 0;
        }
        tn_finish<TS, O, ADD>(it, acc, wm, wn);
        stores += B / 2 * n_on * (ES / 2);                 // store instructions just issued
    }
    MOE_WAIT_VMCNT(0);                                      // (the trailing empty loads still target this LDS)
#endif
}

// dgate_w[a] = the sum of its row's parts, in their order (an assignment without a row: 0), and for the kernel over the rows where each row comes
// from: the byte offset of its token, inverted.
__global__ __launch_bounds__(256) void dgate_kernel(const float* __restrict__ part, const int32_t* __restrict__ offsets, const int32_t* __restrict__ perm,
                                                    const int32_t* __restrict__ inv_perm, int A, int E, int k, unsigned row_bytes, int parts, float* __restrict__ dgate_w,
                                                    uint32_t* __restrict__ src) {
    const int a = (int)(blockIdx.x * 256 + threadIdx.x);
    if (a >= A) return;
    if (src && a < offsets[E]) src[a] = ~((unsigned)perm[a] / (unsigned)k * row_bytes);
    if (!dgate_w) return;
    const int r = inv_perm[a];
    float s = 0.f;
    if (r >= 0)
        for (int j = 0; j < parts; ++j) s += part[(size_t)r * parts + j];
    dgate_w[a] = s;
}

// dy in fp32, rounded once to the matrix instruction's type
__global__ __launch_bounds__(256) void narrow_kernel(const f32x4* __restrict__ from, u32x4* __restrict__ to, size_t n) {
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const f32x4 a = from[2 * i], b = from[2 * i + 1];
    const float v[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    to[i] = to_bf16(v);
}

template <typename K> int set_smem(K kern, size_t bytes) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return moe_fail(MOE_ERR_HIP, "moe_grouped_ffn (training): shared memory attribute: %s", hipGetErrorString(e));
    return MOE_OK;
}
template <int KIND, int TR> int launch_nt(const NtArgs& a, hipStream_t st) {
    auto kern = gemm_nt_kernel<KIND, TR>;
    const int ok = set_smem(kern, Nt<TR>::SMEM);
    if (ok != MOE_OK) return ok;
    hipLaunchKernelGGL(kern, dim3(MOE_GEMM_GRID), dim3(NTH), Nt<TR>::SMEM, st, a);
    MOE_CHECK_LAUNCH("moe_grouped_ffn (training, over rows)");
    return MOE_OK;
}
// Rows per tile by the mean rows of an expert.  Measured, us by tiles of 64 / 128 / 256 rows: first products that are finished in place (KEEP, HID), mean 34 of
// 2048 x 1408 152 / 166 / 219, mean 546 (32768 rows) 417 / 326 / 382, mean 2048 of 4096 x 14336 3225 / 2188 / 2256: three stages in LDS let an item's
// stores go on longer.  Plain results (DX), mean 16 22 / 25 / 43, mean 34 169 / 156 / 187, mean 136 226 / 196 / 266, mean 546 625 / 470 / 460,
// mean 2048 of 4096 x 14336 5675 / 3794 / 3640, of 512 x 512 (64 tiles of 256 rows x 256) 26 / 22 / 33.
template <int KIND> int launch_nt_rows(const NtArgs& a, int A, hipStream_t st) {
    const long long mean = (A + a.E - 1) / a.E;
    if (mean <= (KIND == DX ? 32 : 64)) return launch_nt<KIND, 64>(a, st);
    if constexpr (KIND == DX)
        if (mean >= 512 && (long long)A / 256 * ((a.N + 255) / 256) >= 2 * MOE_GEMM_GRID) return launch_nt<KIND, 256>(a, st);
    return launch_nt<KIND, 128>(a, st);
}
template <int TS, typename O, bool ADD> int launch_tn(const TnArgs& a, hipStream_t st) {
    auto kern = gemm_tn_kernel<TS, O, ADD>;
    const int ok = set_smem(kern, Tn<TS>::SMEM);
    if (ok != MOE_OK) return ok;
    hipLaunchKernelGGL(kern, dim3(MOE_GEMM_GRID * (TS == 256 ? 1 : 2)), dim3(NTH), Tn<TS>::SMEM, st, a);
    MOE_CHECK_LAUNCH("moe_grouped_ffn_backward (over the rows)");
    return MOE_OK;
}
// Tiles of 128 where those of 256 would leave CUs without one: four experts of 512 x 512 over 8192 rows 36 us instead of 67, one of 512 x 1024 88 instead of
// 174.  Elsewhere they fetch twice the bytes for a product: 128 experts of d = 768, F = 4 d, over 16384 rows 649 instead of 545.
template <typename O, bool ADD> int launch_tn_tile(const TnArgs& a, hipStream_t st) {
    const long long tiles = (long long)a.E * a.mats * ((a.d + 255) / 256) * ((a.F + 255) / 256);
    return tiles <= MOE_GEMM_GRID ? launch_tn<128, O, ADD>(a, st) : launch_tn<256, O, ADD>(a, st);
}

int check_shape(const char* what, int T, int d, int F, int E, int k, moe_act act, moe_dtype dt) {
    MOE_REQUIRE(T >= 0 && d >= 1 && F >= 1 && E >= 1 && k >= 1, MOE_ERR_ARG, "%s: T=%d d=%d F=%d E=%d k=%d", what, T, d, F, E, k);
    MOE_REQUIRE(act == MOE_RELU || act == MOE_SWIGLU, MOE_ERR_UNSUPPORTED, "%s: activation %d", what, (int)act);
    MOE_REQUIRE(dt == MOE_BF16, MOE_ERR_UNSUPPORTED, "%s: dtype %d (MOE_BF16 only)", what, (int)dt);
    MOE_REQUIRE(E <= MOE_MAX_EXPERTS, MOE_ERR_UNSUPPORTED, "%s: E=%d", what, E);
    MOE_REQUIRE(d % 64 == 0 && F % 64 == 0, MOE_ERR_UNSUPPORTED, "%s: d=%d, F=%d have to be multiples of 64", what, d, F);
    const long long limit = (1ll << 32) - (1 << 16);       // bytes that a 32-bit offset reaches, with the columns of a tile beside it
    MOE_REQUIRE((long long)T * d * 2 < limit && 256ll * d * 4 < limit && 256ll * F * 4 < limit, MOE_ERR_UNSUPPORTED, "%s: T=%d rows of d=%d, F=%d pass 4 GiB", what, T, d, F);
    MOE_REQUIRE((long long)T * k < (1ll << 30), MOE_ERR_UNSUPPORTED, "%s: T=%d k=%d", what, T, k);
    MOE_REQUIRE(((long long)T * k / 64 + E) * ((F + 63) / 64) * 2 < (1ll << 30) && ((long long)T * k / 64 + E) * ((d + 63) / 64) < (1ll << 30) &&
                    (long long)E * ((d + 127) / 128) * ((F + 127) / 128) * 3 < (1ll << 30),
                MOE_ERR_UNSUPPORTED, "%s: T=%d k=%d E=%d d=%d F=%d make too many tiles", what, T, k, E, d, F);
    return MOE_OK;
}

}  // namespace

extern "C" int moe_grouped_ffn_keep(const void* x, int T, int d, int F, int E, int k, moe_act act, moe_dtype dt, const void* const* w_in, const int32_t* offsets,
                                    const int32_t* perm, void* h_scratch, int8_t* z_q, float* z_scale, void* stream) {
    int ok = check_shape("moe_grouped_ffn_keep", T, d, F, E, k, act, dt);
    if (ok != MOE_OK) return ok;
    if (T == 0) return MOE_OK;
    MOE_REQUIRE(x && w_in && offsets && perm && h_scratch && z_q && z_scale, MOE_ERR_ARG, "moe_grouped_ffn_keep: null pointer");
    MOE_REQUIRE((((uintptr_t)x | (uintptr_t)h_scratch | (uintptr_t)z_q) & 15) == 0 && (((uintptr_t)z_scale | (uintptr_t)offsets | (uintptr_t)perm) & 3) == 0,
                MOE_ERR_UNSUPPORTED, "moe_grouped_ffn_keep: x, h_scratch and z_q have to be aligned to 16 bytes");
    ok = moe_check_gemm_device();
    if (ok != MOE_OK) return ok;
    NtArgs a = {};
    a.rows = (const uint16_t*)x;
    a.offsets = offsets;
    a.perm = perm;
    a.w_ptrs = w_in;
    a.T = T;
    a.k = k;
    a.E = E;
    a.F = F;
    a.Z = act == MOE_SWIGLU ? 2 * F : F;
    a.N = a.Z;
    a.KT = a.KT0 = d / 64;
    a.ld_rows = a.ld_w = d;
    a.h = (uint16_t*)h_scratch;
    a.q_out = z_q;
    a.scale_out = z_scale;
    return act == MOE_SWIGLU ? launch_nt_rows<KEEP_SWIGLU>(a, T * k, (hipStream_t)stream) : launch_nt_rows<KEEP_RELU>(a, T * k, (hipStream_t)stream);
}

// Workspace: dz [A,Z] and w h [A,F] in bf16, the parts of dgate_w [A, ceil(F / 128)] in fp32, the rows' sources [A], dy [T,d] in bf16 where it
// comes in fp32, each rounded up to 256 bytes.
static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
size_t moe_ffn_back_bytes(int T, int d, int F, int k) {
    if (T < 0 || d < 1 || F < 1 || k < 1) return 0;
    const size_t A = (size_t)T * k;
    return up256(A * 2 * F * 2) + up256(A * F * 2) + up256(A * ((F + 127) / 128) * 4) + up256(A * 4) + up256((size_t)T * d * 2);
}

extern "C" int moe_grouped_ffn_backward(const void* dy, moe_dtype dy_dt, const void* x, int T, int d, int F, int E, int k, moe_act act, moe_dtype dt,
                                        const void* w_a, const void* w_b, const void* w_o, const int32_t* offsets, const int32_t* perm,
                                        const int32_t* inv_perm, const float* gate_w, const int8_t* z_q, const float* z_scale, float* dx_perm,
                                        float* dgate_w, void* dw_a, void* dw_b, void* dw_o, moe_dtype dw_dt, int accumulate, void* ws, size_t ws_bytes,
                                        void* stream) {
    int ok = check_shape("moe_grouped_ffn_backward", T, d, F, E, k, act, dt);
    if (ok != MOE_OK) return ok;
    const bool sw = act == MOE_SWIGLU;
    MOE_REQUIRE(moe_dtype_ok(dy_dt) && moe_dtype_ok(dw_dt), MOE_ERR_UNSUPPORTED, "moe_grouped_ffn_backward: dy of dtype %d, gradients of dtype %d", (int)dy_dt, (int)dw_dt);
    const bool dw = dw_a || dw_b || dw_o;
    MOE_REQUIRE(!dw || (dw_a && dw_o && (dw_b != nullptr) == sw), MOE_ERR_ARG, "moe_grouped_ffn_backward: the matrices' gradients are wanted all or none");
    MOE_REQUIRE(offsets, MOE_ERR_ARG, "moe_grouped_ffn_backward: null pointer");
    if (T > 0)
        MOE_REQUIRE(dy && (x || !dw) && w_o && perm && z_q && z_scale && (inv_perm || !dgate_w) && (!dx_perm || (w_a && (w_b != nullptr) == sw)), MOE_ERR_ARG,
                    "moe_grouped_ffn_backward: null pointer, or w_b with MOE_RELU");
    const size_t A = (size_t)T * k, Z = sw ? 2 * (size_t)F : F;
    const int parts = (F + 127) / 128;
    const size_t n_dz = up256(A * Z * 2), n_wh = up256(A * F * 2), n_parts = up256(A * parts * 4);
    const size_t n_src = up256(A * 4), need = n_dz + n_wh + n_parts + n_src + (dy_dt == MOE_F32 ? up256((size_t)T * d * 2) : 0);
    MOE_REQUIRE(T == 0 || (ws && ws_bytes >= need), MOE_ERR_WORKSPACE, "moe_grouped_ffn_backward: workspace of %zu bytes, %zu needed", ws_bytes, need);
    MOE_REQUIRE((((uintptr_t)dy | (uintptr_t)x | (uintptr_t)w_a | (uintptr_t)w_b | (uintptr_t)w_o | (uintptr_t)z_q | (uintptr_t)dx_perm | (uintptr_t)dw_a |
                  (uintptr_t)dw_b | (uintptr_t)dw_o | (uintptr_t)ws) & 15) == 0, MOE_ERR_UNSUPPORTED, "moe_grouped_ffn_backward: pointers have to be aligned to 16 bytes");
    ok = moe_check_gemm_device();
    if (ok != MOE_OK) return ok;
    const hipStream_t st = (hipStream_t)stream;
    uint32_t* src = (uint32_t*)((unsigned char*)ws + n_dz + n_wh + n_parts);
    if (dy_dt == MOE_F32 && T > 0) {
        u32x4* to = (u32x4*)((unsigned char*)ws + n_dz + n_wh + n_parts + n_src);
        const size_t n = (size_t)T * d / 8;
        hipLaunchKernelGGL(narrow_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, (const f32x4*)dy, to, n);
        MOE_CHECK_LAUNCH("moe_grouped_ffn_backward (dy)");
        dy = to;
    }
    if (T > 0) {
        NtArgs a = {};
        a.rows = (const uint16_t*)dy;
        a.offsets = offsets;
        a.perm = perm;
        a.w0 = (const uint16_t*)w_o;
        a.w_stride = (size_t)d * F;
        a.T = T;
        a.k = k;
        a.E = E;
        a.F = a.N = F;
        a.Z = (int)Z;
        a.KT = a.KT0 = d / 64;
        a.ld_rows = a.ld_w = d;
        a.parts = parts;
        a.q_in = z_q;
        a.scale_in = z_scale;
        a.gate_w = gate_w;
        a.dz = (uint16_t*)ws;
        a.wh = (uint16_t*)((unsigned char*)ws + n_dz);
        a.dgate_part = (float*)((unsigned char*)ws + n_dz + n_wh);
        ok = sw ? launch_nt_rows<HID_SWIGLU>(a, (int)A, st) : launch_nt_rows<HID_RELU>(a, (int)A, st);
        if (ok != MOE_OK) return ok;
        if (dgate_w || dw) {
            hipLaunchKernelGGL(dgate_kernel, dim3((unsigned)((A + 255) / 256)), dim3(256), 0, st, a.dgate_part, offsets, perm, inv_perm, (int)A, E, k, (unsigned)d * 2u, parts,
                               dgate_w, dw ? src : nullptr);
            MOE_CHECK_LAUNCH("moe_grouped_ffn_backward (gate values)");
        }
        if (dx_perm) {
            NtArgs b = a;
            b.rows = a.dz;
            b.w0 = (const uint16_t*)w_a;
            b.w1 = (const uint16_t*)w_b;
            b.N = d;
            b.KT0 = F / 64;
            b.KT = (int)Z / 64;
            b.ld_rows = (int)Z;
            b.ld_w = F;
            b.dx_perm = dx_perm;
            ok = launch_nt_rows<DX>(b, (int)A, st);
            if (ok != MOE_OK) return ok;
        }
    }
    if (dw) {
        TnArgs t = {};
        t.x = (const uint16_t*)x;
        t.dy = (const uint16_t*)dy;
        t.dz = (const uint16_t*)ws;
        t.wh = (const uint16_t*)((unsigned char*)ws + n_dz);
        t.offsets = offsets;
        t.src = src;
        t.T = T;
        t.E = E;
        t.d = d;
        t.F = F;
        t.Z = (int)Z;
        t.mats = sw ? 3 : 2;
        t.dwa = dw_a;
        t.dwb = dw_b;
        t.dwo = dw_o;
        if (dw_dt == MOE_F32) ok = accumulate ? launch_tn_tile<float, true>(t, st) : launch_tn_tile<float, false>(t, st);
        else ok = accumulate ? launch_tn_tile<uint16_t, true>(t, st) : launch_tn_tile<uint16_t, false>(t, st);
        if (ok != MOE_OK) return ok;
    }
    return MOE_OK;
}
