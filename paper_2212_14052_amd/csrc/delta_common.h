// What the kernels of the chunked gated delta rule share (delta.hip,
// delta_bwd.hip): the chunk's matrices, operands cut into fp16 pieces, and
// the layouts that the matrix cores' operands are kept in.
//
// Precision.  States, decays, sums and all results before their one rounding
// are float32.  A float32 operand of a matrix product goes in as two fp16
// pieces, the rounding and the rounding of what it leaves: 22 bits; of the four products
// of pieces the smallest (2^-22 at most) is left out.  fp16 inputs are one piece
// as they are.  Everything else is scaled by a power of two that takes the
// largest value that shares it to 2^13 .. 2^14, so that nothing overflows and what
// fp16 cannot hold is below 2^-38 of that largest value; bf16 inputs are then one
// exact piece (down to 2^-31 of the largest).  Exponents are kept as integers
// and undone in float32.  Each column of a state has its own; keys and queries have one for a
// chunk, triangular matrices one each: what lies 2^-16 and more below the largest that shares its scale has fewer bits.  (Three bf16 pieces, which need no scales, cost 182
// matrix instructions a chunk of 16 columns where these cost 132.)
#pragma once
#include "common.h"
#include "internal.h"

namespace h3 {

constexpr int DC = kDeltaChunk;

typedef _Float16 dl_h8 __attribute__((ext_vector_type(8)));
typedef float dl_f4 __attribute__((ext_vector_type(4)));
typedef short dl_s4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) dl_s4 dl_lds_s4;
typedef __attribute__((address_space(3))) void dl_lds_void;

// pieces of the inputs by type
template <int DT> constexpr int pieces() { return DT == F32 ? 2 : 1; }
// Everything else is two, also what only a 16-bit output is made of: a value written under a key that held
// another makes terms cancel, and what one piece rounds away of the old value can be all of the new one.

// an operand of eight values a lane in N pieces
template <int N> struct Op {
    uint4 p[N];
};

__device__ __forceinline__ dl_f4 dl_mfma(uint4 a, uint4 b, dl_f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(dl_h8, a), __builtin_bit_cast(dl_h8, b), c, 0, 0, 0);
}
// c + a b, the smallest products first
template <int NA, int NB> __device__ __forceinline__ dl_f4 mm(const Op<NA> &a, const Op<NB> &b, dl_f4 c) {
    constexpr int N = NA > NB ? NA : NB;
#pragma unroll
    for (int s = N - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB) c = dl_mfma(a.p[i], b.p[s - i], c);
    return c;
}

// M sums at once, product by product, so that no instruction waits for the one
// before it: c(m) += a(m) b(m).
template <int NA, int NB, int M, typename A, typename B, typename C>
__device__ __forceinline__ void mm_each(A a, B b, C c) {
    constexpr int N = NA > NB ? NA : NB;
#pragma unroll
    for (int s = N - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB) {
#pragma unroll
                for (int m = 0; m < M; ++m) c(m) = dl_mfma(a(m).p[i], b(m).p[s - i], c(m));
            }
}

__device__ __forceinline__ float low_half(uint32_t w) { return f16_to_f32((uint16_t)(w & 0xffffu)); }
__device__ __forceinline__ float high_half(uint32_t w) { return f16_to_f32((uint16_t)(w >> 16)); }

// x s and y t as N pieces, a word each: the products rounded to half words, and what that leaves, which is exact
// to float32's rounding, from a mixed-precision instruction each.  (Six instructions a pair; five in inline assembly, but
// the compiler does not see assembly among the matrix instructions, whose operands must not be
// written for some cycles before and after.)
template <int N> __device__ __forceinline__ void split2(float x, float s, float y, float t, uint32_t (&w)[N]) {
    w[0] = pack_16x2<F16>(x * s, y * t);
    if constexpr (N == 2) w[1] = pack_16x2<F16>(__builtin_fmaf(x, s, -low_half(w[0])), __builtin_fmaf(y, t, -high_half(w[0])));
}
template <int N> __device__ __forceinline__ Op<N> split8(const float (&x)[8], float s) {
    Op<N> o;
    uint32_t w[4][N];
#pragma unroll
    for (int i = 0; i < 4; ++i) split2<N>(x[2 * i], s, x[2 * i + 1], s, w[i]);
#pragma unroll
    for (int n = 0; n < N; ++n) o.p[n] = make_uint4(w[0][n], w[1][n], w[2][n], w[3][n]);
    return o;
}
template <int N> __device__ __forceinline__ Op<N> split8(dl_f4 a, dl_f4 b, float s) {
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return split8<N>(x, s);
}

// -------------------------------------------------------------- scales -----
// The exponent e with largest 2^-e in 2^13 .. 2^14, from the largest magnitude's
// bits; 0 for Inf and NaN, -126 where 2^-e would leave float32 and for zero: a tile of
// zeros must not raise the exponent of what it is added to.
__device__ __forceinline__ int scale_exp(uint32_t bits) {
    if (bits >= 0x7f800000u) return 0;
    const int e = (int)(bits >> 23) - 127 - 13;
    return e < -126 ? -126 : e;
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }   // -126 .. 127
// the same for sums of exponents: 0 where it would leave float32 at the bottom.  Exponents of
// operands are kLeast at least, so that what this drops is no part of the sum it belongs to
// (of a value of 2^-67 or less fewer bits go in).
constexpr int kLeast = -80;
__device__ __forceinline__ float pow2_sum(int e) { return e < -126 ? 0.f : pow2(e > 127 ? 127 : e); }
// e with 2^e <= x < 2^(e + 1); -127 for zero
__device__ __forceinline__ int floor_exp(float x) { return (int)((__float_as_uint(x) >> 23) & 255u) - 127; }
// what the backward pass is told of a state: its exponent e in the registers and E of the registers
__device__ __forceinline__ int kept_exp(int e, int E) { return e <= -126 ? -126 : max(min(max(e, kLeast) + E, 114), -126); }
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
// the larger of m and the magnitudes of two values
__device__ __forceinline__ float max3_abs(float m, float x, float y) {
    asm("v_max3_f32 %0, %0, |%1|, |%2|" : "+v"(m) : "v"(x), "v"(y));
    return m;
}
// The exponent for x of this lane's column, whose rows four lanes share.  Columns of a state are
// independent: each has its own scales, so that none loses bits, or all of them, by another's size.
template <int N> __device__ __forceinline__ int col_exp(const dl_f4 (&x)[N]) {
    float m = 0.f;
#pragma unroll
    for (int t = 0; t < N; ++t) {
        m = max3_abs(m, x[t][0], x[t][1]);
        m = max3_abs(m, x[t][2], x[t][3]);
    }
    uint32_t b = __float_as_uint(m);
    const auto r = __builtin_amdgcn_permlane16_swap(b, b, false, false);
    b = umax(r[0], r[1]);
    const auto s = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    return scale_exp(umax(s[0], s[1]));
}
// the largest of the 16 columns' exponents
__device__ __forceinline__ int tile_exp(int e) { return (int)group_max<16>((uint32_t)(e + 1024)) - 1024; }

// Eight consecutive inputs as floats; zeros where !on.
template <int DT> __device__ __forceinline__ void ld8(const typename IO<DT>::T *p, bool on, float (&x)[8]) {
    if constexpr (DT == F32) {
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f), b = a;
        if (on) a = *(const float4 *)p, b = *(const float4 *)(p + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
        uint4 a = make_uint4(0u, 0u, 0u, 0u);
        if (on) a = *(const uint4 *)p;
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = DT == BF16 ? bf16_to_f32(w[i] & 0xffffu) : low_half(w[i]);
            x[2 * i + 1] = DT == BF16 ? bf16_to_f32(w[i] >> 16) : high_half(w[i]);
        }
    }
}
__device__ __forceinline__ uint4 or_zero(uint4 x, bool on) {
    return make_uint4(on ? x.x : 0u, on ? x.y : 0u, on ? x.z : 0u, on ? x.w : 0u);
}
// raw registers of eight inputs, fetched ahead of their use
template <int DT> struct Raw8 {
    uint4 a[DT == F32 ? 2 : 1];
};
template <int DT> __device__ __forceinline__ Raw8<DT> ld8_raw(const typename IO<DT>::T *p) {
    Raw8<DT> r;
#pragma unroll
    for (int i = 0; i < (DT == F32 ? 2 : 1); ++i) r.a[i] = ((const uint4 *)p)[i];
    return r;
}
template <int DT> __device__ __forceinline__ Raw8<DT> or_zero(Raw8<DT> r, bool on) {
#pragma unroll
    for (int i = 0; i < (DT == F32 ? 2 : 1); ++i) r.a[i] = or_zero(r.a[i], on);
    return r;
}
template <int DT> __device__ __forceinline__ void raw_floats(const Raw8<DT> &r, float (&x)[8]) {
    const uint32_t w[8] = {r.a[0].x, r.a[0].y, r.a[0].z, r.a[0].w, r.a[DT == F32].x, r.a[DT == F32].y, r.a[DT == F32].z, r.a[DT == F32].w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (DT == F32) x[i] = __uint_as_float(w[i]);
        else if constexpr (DT == BF16) x[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        else x[i] = i & 1 ? high_half(w[i / 2]) : low_half(w[i / 2]);
    }
}
template <int DT> __device__ __forceinline__ uint32_t raw_mag(const Raw8<DT> &r) {
    float x[8];
    raw_floats<DT>(r, x);
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = umax(m, mag(x[i]));
    return m;
}
// its pieces, times scale (fp16: as it is)
template <int DT> __device__ __forceinline__ Op<pieces<DT>()> op_of(const Raw8<DT> &r, float scale) {
    Op<pieces<DT>()> o;
    if constexpr (DT == F16) {
        o.p[0] = r.a[0];
    } else {
        float x[8];
        raw_floats<DT>(r, x);
        o = split8<pieces<DT>()>(x, scale);
    }
    return o;
}

// ------------------------------------------------------------- layouts -----
// Matrix-core tiles are 16 x 16 with 32 products a step: lane 16 g + n holds of
// the left operand row n, of the right one column n, eight of the 32 summands;
// of a result column n, rows 4 g .. 4 g + 3.  The summands' order is free as long
// as both operands share it.  With the order
//     slot j of lane group g = 32 s + 4 g + j (j < 4), 32 s + 16 + 4 g + j - 4
// ("token order") two result tiles, rows 32 s .. + 31, are an operand of the next
// product as they lie in the registers.  Rows of the state (key channels) are
// numbered so that the same holds with slot j = 32 s + 8 g + j, which is 16
// contiguous bytes of a key or query: tile 2 s + h, row r is channel
//     32 s + 8 (r / 4) + 4 h + r % 4.
//
// A triangular 64 x 64 matrix of a chunk (X, P and their transposes) is kept in
// global memory as the left operand's registers: six fragments (row tile, s) of
// 64 lanes of 16 bytes, the two that hold only zeros left out, each piece for itself.
constexpr int FRAG = 64;                 // uint4 a fragment
constexpr int MAT = 6 * FRAG;            // uint4 a piece of a matrix
constexpr int GATES = (int)sizeof(ChunkGates) / 16;
constexpr int lower_frag(int t, int s) { return t < 2 ? t : 2 * t - 2 + s; }       // s <= t / 2
constexpr int upper_frag(int t, int s) { return t < 2 ? 2 * t + s : 2 + t; }       // s >= t / 2

// The keys (queries) of a chunk, in memory and in LDS alike: 1 KB blocks of 16
// tokens by 32 channels, [piece][token block][channel block], in each the eight
// channels 8 g of token n at 16-byte place 4 n + (g ^ n / 4).  Sixteen tokens of one
// g are then on sixteen different places of a 256-byte bank row.
// (RB: blocks of 16 rows; the backward pass keeps other matrices so, too.)
template <int KS, int RB = 4> constexpr int kq_block(int piece, int t, int s) { return (piece * RB + t) * KS + s; }
__device__ __forceinline__ int kq_place(int n, int g) { return 4 * n + (g ^ (n >> 2)); }
template <int KS> constexpr int kq_words(int pieces) { return pieces * 4 * KS * 64; }   // uint4

// the left operand of token rows 16 t .. + 15, channels 32 s .. + 31
template <int NT, int KS> __device__ __forceinline__ Op<NT> lds_rows(const uint4 *m, int t, int s, int lane) {
    Op<NT> o;
#pragma unroll
    for (int n = 0; n < NT; ++n) o.p[n] = m[kq_block<KS>(n, t, s) * 64 + kq_place(lane & 15, lane >> 4)];
    return o;
}
// the left operand of the transpose: rows = channels of state tile T (or, with
// natural order, channels 16 T + 0 .. 15), summands = tokens 32 s .. + 31 in
// token order.  A transposing read gives lane j of 16 the four rows that lanes 4 i + c
// address, at the j-th of the 16 columns that lanes c = 0 .. 3 address four at a time.
template <int NT, int KS, bool STATE = true, int RB = 4>
__device__ __forceinline__ Op<NT> lds_cols(const uint4 *m, int T, int s, int lane) {
    const int c = lane & 3, row = 4 * (lane >> 4) + ((lane & 15) >> 2);   // and 16 rows on
    const int g = STATE ? c : 2 * (T & 1) + (c >> 1), half = STATE ? T & 1 : c & 1;
    const int at = kq_place(row, g) * 8 + 4 * half;   // 16-bit elements in a block
    Op<NT> o;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint16_t *p = (const uint16_t *)m + at;
        const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((dl_lds_s4 *)(p + kq_block<KS, RB>(n, 2 * s, T >> 1) * 512)));
        const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((dl_lds_s4 *)(p + kq_block<KS, RB>(n, 2 * s + 1, T >> 1) * 512)));
        o.p[n] = make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
    return o;
}
// fragment f of a matrix in N pieces
template <int N> __device__ __forceinline__ Op<N> ld_frag(const uint4 *m, int f, int lane) {
    Op<N> o;
#pragma unroll
    for (int n = 0; n < N; ++n) o.p[n] = m[n * MAT + f * FRAG + lane];
    return o;
}
// Nothing is moved over this point, so that what is asked for ahead of its use is
// (where a wave has a vector unit for itself; waves that share one need the registers).
template <bool ON> __device__ __forceinline__ void in_order() {
    if constexpr (ON) __builtin_amdgcn_sched_barrier(0);
}

// rows r0 .. r0 + 3 of this lane's column (c0 + lane % 16) of 16-bit or float32 values in LDS, r0 = a + 4 (lane / 16)
template <int DT>
__device__ __forceinline__ dl_f4 lds_column4(const typename IO<DT>::T *m, int row, int a, int c0, int lane) {
    const int g4 = lane >> 4, c16 = lane & 15;
    dl_f4 v;
    if constexpr (DT == F32) {
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = m[(a + 4 * g4 + r) * row + c0 + c16];
    } else {
        const typename IO<DT>::T *p = m + (a + 4 * g4 + (c16 >> 2)) * row + c0 + 4 * (lane & 3);
        const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((dl_lds_s4 *)p));
        const uint32_t y[2] = {x.x, x.y};
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if constexpr (DT == BF16) v[r] = __uint_as_float(r & 1 ? y[r / 2] & 0xffff0000u : y[r / 2] << 16);
            else v[r] = r & 1 ? high_half(y[r / 2]) : low_half(y[r / 2]);
        }
    }
    return v;
}

// the sum of x over the lanes up to and with this one, on the vector unit
template <int CTRL, int ROWS> __device__ __forceinline__ float from_lane(float x) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float lane_sums(float x) {
    x += from_lane<0x111, 0xf>(x);   // row_shr:1, 2, 4, 8
    x += from_lane<0x112, 0xf>(x);
    x += from_lane<0x114, 0xf>(x);
    x += from_lane<0x118, 0xf>(x);
    x += from_lane<0x142, 0xa>(x);   // lane 15 of rows 0 and 2 to the rows behind them
    x += from_lane<0x143, 0xc>(x);   // lane 31 to rows 2 and 3
    return x;
}

// ------------------------------------------------------- a chunk's decays ---
constexpr double kLog2e = 1.4426950408889634073599246810018921;
// a log decay below this is an exact zero in float32 whatever it is (also -inf,
// whose differences would not be numbers)
constexpr double kLowest = -1e6;

// The running sum over the wave's lanes, in units of log 2.
__device__ __forceinline__ double decay_sum(float g, bool on, int lane) {
    double x = on ? (double)g : 0.0;
    x = x < kLowest ? kLowest : x;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const double y = __shfl_up(x, m);
        if (lane >= m) x += y;
    }
    return x * kLog2e;
}

// ----------------------------------------------------------- arguments -----
// tokens of sequence b
__device__ __forceinline__ int tokens_of(const DeltaArgs &a, int b) {
    if (!a.lengths) return a.L;
    const int n = a.lengths[b];
    return n < 0 ? 0 : n > a.L ? a.L : n;
}

// ---------------------------------------------- bringing in a scan's chunk ---
// A workgroup of NW waves of 16 columns keeps in LDS a chunk's keys and
// queries, its record (two triangular matrices in two pieces each, the gates) and the
// workgroup's columns of V or do.  All of it is copied from memory as it lies there,
// 1 KB an instruction, without passing through registers, and, where two fit, while the
// chunk before is worked on.  Nothing is cleared: rows behind the end are copies of the
// last token (their beta is 0, their rows of X and P are 0, and what they would output is not
// stored), columns behind Dv copies of the first ones (not stored either).
// LEAN: no queries and no P (the first half of a forward record), one chunk at a
// time, small enough that two workgroups share a CU and wait for each other's turn.
template <int DT, int KS, int NW, bool LEAN = false> struct ScanLds {
    static constexpr int words = 4 * MAT + GATES, kq = kq_words<KS>(pieces<DT>());   // uint4
    static constexpr int vrow = 16 * NW, v16 = DC * vrow * (int)sizeof(typename IO<DT>::T) / 16;
    static constexpr int k = 0, q = kq, v = LEAN ? kq : 2 * kq, rec = v + v16, mats = (LEAN ? 2 : 4) * MAT, gates = rec + mats,
                         one = gates + GATES;
    static constexpr bool two = !LEAN && 2 * one * 16 <= 160 * 1024;
    static constexpr int total = (two ? 2 : 1) * one * 16;
    static_assert(total <= 160 * 1024, "LDS of a CU");
};

template <int DT, int KS, int NW, bool LEAN = false> struct ChunkCopy {
    typedef typename IO<DT>::T T;
    typedef ScanLds<DT, KS, NW, LEAN> Lds;
    const uint4 *kq, *rec;   // this key head's and this value head's chunks
    const T *v;              // this value head's row of the first token, at the workgroup's first column
    long vstride;            // elements from token to token
    int cols, len;           // columns from there, tokens
    uint32_t lds;

    static __device__ __forceinline__ void copy(const void *base, uint32_t off, uint32_t to) {
        copy_to_lds(base, off, __builtin_amdgcn_readfirstlane(to));
    }
    // n words from base to word `at` of the buffer
    template <int N> static __device__ __forceinline__ void copy_words(const uint4 *base, uint32_t to, int w, int lane) {
#pragma unroll
        for (int i = 0; i < (N + 64 * NW - 1) / (64 * NW); ++i) {
            const int at = (i * NW + w) * 64 + lane;
            if (N % (64 * NW) == 0 || at < N) copy(base, (uint32_t)at * 16, to + (i * NW + w) * 1024);
        }
    }
    __device__ __forceinline__ void issue(int n, int w, int lane) const {
        const uint32_t to = lds + (Lds::two ? (uint32_t)(n & 1) * Lds::one * 16 : 0u);
        const uint4 *kn = kq + (long)n * 2 * Lds::kq, *rn = rec + (long)n * Lds::words;
        copy_words<(LEAN ? 1 : 2) * Lds::kq>(kn, to + Lds::k * 16, w, lane);
        const T *vn = v + (long)n * DC * vstride;
        const int last = min(DC, len - n * DC) - 1;
        constexpr int VP = 16 / (int)sizeof(T), VR = Lds::vrow / VP;   // values, words a row
#pragma unroll
        for (int i = 0; i < Lds::v16 / (64 * NW); ++i) {
            const int at = (i * NW + w) * 64 + lane, t = min(at / VR, last), c = VP * (at % VR);
            copy(vn, (uint32_t)((t * vstride + (c < cols ? c : 0)) * sizeof(T)), to + (Lds::v + (i * NW + w) * 64) * 16);
        }
        if constexpr (LEAN) {
            copy_words<Lds::mats>(rn, to + Lds::rec * 16, w, lane);
            if (w == 0 && lane < GATES) copy(rn + 4 * MAT, (uint32_t)lane * 16, to + Lds::gates * 16);
        } else {
            copy_words<Lds::words>(rn, to + Lds::rec * 16, w, lane);
        }
    }
    // Chunk n is in LDS, for every wave, and chunk `next` (if `more`) under way.
    __device__ __forceinline__ const uint4 *arrive(const uint4 *base, int n, int next, bool more, int w, int lane) const {
        if constexpr (Lds::two) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (more) issue(next, w, lane);
            return base + (n & 1) * Lds::one;
        } else {
            __syncthreads();
            issue(n, w, lane);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            return base;
        }
    }
};

// ---------------------------------------------------------------- segments ---
// What a workgroup of a scan works on: a (b, h), a segment, its columns.  With MAPS
// there are the columns of V from a zero state, and then the unit matrix's
// from no values; no map is needed of the last segment (BACK: of the first).
template <int NW, bool MAPS, bool BACK = false> struct ScanPlace {
    long bh;
    int b, h, seg, cb, c0, width;   // width: columns there are
    bool unit;
    __device__ __forceinline__ ScanPlace(const DeltaArgs &a, const DeltaSegments &sg, unsigned block, int w) {
        const int v = delta_col_tiles(a.Dv, NW), tiles = v + (MAPS ? delta_col_tiles(a.Dk, NW) : 0), segs = sg.G - (MAPS ? 1 : 0);
        const int tile = (int)(block % tiles);
        seg = (int)(block / tiles % segs) + (MAPS && BACK ? 1 : 0);
        bh = block / tiles / segs;
        h = (int)(bh % a.H);
        b = (int)(bh / a.H);
        unit = tile >= v;
        width = unit ? a.Dk : a.Dv;
        cb = (unit ? tile - v : tile) * 16 * NW;
        c0 = cb + 16 * w;
    }
};

// S as columns of a segment's map: (32 KS, dvp + 32 KS) row-major, its
// second part with the exponent of its scale for every 16 columns.
template <int KS, typename P>
__device__ __forceinline__ void store_map(const DeltaArgs &a, const DeltaSegments &sg, const P &at, const dl_f4 (&S)[2 * KS], int lane) {
    const int dvp = (a.Dv + 15) & ~15, row = dvp + 32 * KS, e = tile_exp(col_exp(S));
    float *p = sg.maps + ((at.bh * sg.G + at.seg) * 32 * KS + 8 * (lane >> 4)) * row + (at.unit ? dvp : 0) + at.c0 + (lane & 15);
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) p[(32 * (t >> 1) + 4 * (t & 1) + r) * row] = S[t][r];
    if (at.unit && lane == 0) sg.exps[(at.bh * sg.G + at.seg) * 8 + at.c0 / 16] = e;
}

// dynamic LDS above 64 KB has to be asked for
template <typename K> hipError_t lds_room(K *kernel, int bytes) {
    return bytes > 65536 ? hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) : hipSuccess;
}

}  // namespace h3
