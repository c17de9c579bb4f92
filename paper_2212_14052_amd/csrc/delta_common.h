// What the kernels of the chunked gated delta rule share (delta.hip,
// delta_bwd.hip): the chunk's matrices, operands cut into bf16 pieces, and
// the layouts that the matrix cores' operands are kept in.
//
// Precision.  States, decays, sums and all results before their one rounding
// are float32.  A float32 operand of a matrix product goes in as a sum of bf16
// pieces, each the rounding of what is left: three hold all 24 bits, two are off by
// 2^-16 at most; a product of pieces i and j is formed where i + j is below the
// larger number of pieces (so two by two are off by 2^-15 at most, three by
// three by 2^-22).  bf16 has float32's exponents, so no value needs a scale.  bf16 inputs are one piece,
// fp16 inputs two, float32 inputs three, all exact.
#pragma once
#include "common.h"
#include "internal.h"

namespace h3 {

constexpr int DC = kDeltaChunk;

typedef __bf16 dl_b8 __attribute__((ext_vector_type(8)));
typedef float dl_f4 __attribute__((ext_vector_type(4)));
typedef short dl_s4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) dl_s4 dl_lds_s4;

// pieces of the inputs by type, and how far the products of two inputs are
// taken (both pieces of fp16 are exact: all four)
template <int DT> constexpr int pieces() { return DT == BF16 ? 1 : DT == F16 ? 2 : 3; }
template <int DT> constexpr int input_products() { return DT == BF16 ? 1 : 3; }

// an operand of eight values a lane in N pieces
template <int N> struct Op {
    uint4 p[N];
};

__device__ __forceinline__ dl_f4 dl_mfma(uint4 a, uint4 b, dl_f4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(dl_b8, a), __builtin_bit_cast(dl_b8, b), c, 0, 0, 0);
}
// c + a b, the smallest products first; N: how far products of pieces are taken
template <int NA, int NB, int N = (NA > NB ? NA : NB)>
__device__ __forceinline__ dl_f4 mm(const Op<NA> &a, const Op<NB> &b, dl_f4 c) {
#pragma unroll
    for (int s = N - 1; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB) c = dl_mfma(a.p[i], b.p[s - i], c);
    return c;
}

// Two floats as N pieces, a word each: each the rounding of what the pieces
// before it leave, so that piece n is at most 2^-8n of the value.
template <int N> __device__ __forceinline__ void split2(float x, float y, uint32_t (&w)[N]) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
        w[n] = pack_16x2<BF16>(x, y);
        x -= __uint_as_float(w[n] << 16);
        y -= __uint_as_float(w[n] & 0xffff0000u);
    }
}
template <int N> __device__ __forceinline__ Op<N> split8(const float (&x)[8]) {
    Op<N> o;
    uint32_t w[4][N];
#pragma unroll
    for (int i = 0; i < 4; ++i) split2<N>(x[2 * i], x[2 * i + 1], w[i]);
#pragma unroll
    for (int n = 0; n < N; ++n) o.p[n] = make_uint4(w[0][n], w[1][n], w[2][n], w[3][n]);
    return o;
}
template <int N> __device__ __forceinline__ Op<N> split8(dl_f4 a, dl_f4 b) {
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return split8<N>(x);
}

// Eight consecutive inputs as their pieces, or as floats; zeros where !on.
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
            x[2 * i] = DT == BF16 ? bf16_to_f32(w[i] & 0xffffu) : f16_to_f32(w[i] & 0xffffu);
            x[2 * i + 1] = DT == BF16 ? bf16_to_f32(w[i] >> 16) : f16_to_f32(w[i] >> 16);
        }
    }
}
// raw registers of eight inputs, fetched ahead of their use
template <int DT> struct Raw8 {
    uint4 a[DT == F32 ? 2 : 1];
};
template <int DT> __device__ __forceinline__ Raw8<DT> ld8_raw(const typename IO<DT>::T *p, bool on) {
    Raw8<DT> r;
#pragma unroll
    for (int i = 0; i < (DT == F32 ? 2 : 1); ++i) r.a[i] = on ? ((const uint4 *)p)[i] : make_uint4(0u, 0u, 0u, 0u);
    return r;
}
template <int DT> __device__ __forceinline__ Op<pieces<DT>()> op_of(const Raw8<DT> &r) {
    if constexpr (DT == BF16) {
        Op<1> o;
        o.p[0] = r.a[0];
        return o;
    } else {
        float x[8];
        const uint32_t *w = (const uint32_t *)&r;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (DT == F32) x[i] = __uint_as_float(w[i]);
            else x[i] = f16_to_f32((uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu));
        }
        return split8<pieces<DT>()>(x);
    }
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
constexpr int lower_frag(int t, int s) { return t < 2 ? t : 2 * t - 2 + s; }       // s <= t / 2
constexpr int upper_frag(int t, int s) { return t < 2 ? 2 * t + s : 2 + t; }       // s >= t / 2

// keys and queries of a chunk in LDS: [piece][token][channel], rows padded by
// 16 bytes, which spreads a tile's 16 rows over the banks
template <int KS> constexpr int lds_row() { return 32 * KS + 8; }   // elements

// the left operand of token rows 16 t .. + 15, channels 32 s .. + 31
template <int NT, int KS>
__device__ __forceinline__ Op<NT> lds_rows(const uint16_t *m, int t, int s, int lane) {
    Op<NT> o;
#pragma unroll
    for (int n = 0; n < NT; ++n)
        o.p[n] = *(const uint4 *)(m + ((n * DC + 16 * t + (lane & 15)) * lds_row<KS>() + 32 * s + 8 * (lane >> 4)));
    return o;
}
// the left operand of the transpose: rows = channels of state tile T (or, with
// natural order, channels 16 T + 0 .. 15), summands = tokens 32 s .. + 31 in
// token order.  A transposing read gives lane j of 16 the four rows that lanes 4 i + c
// address, at the j-th of the 16 columns that lanes c = 0 .. 3 address four at a time.
template <int NT, int KS, bool STATE = true>
__device__ __forceinline__ Op<NT> lds_cols(const uint16_t *m, int T, int s, int lane) {
    const int c = lane & 3, row = 32 * s + 4 * (lane >> 4) + ((lane & 15) >> 2);
    const int col = STATE ? 32 * (T >> 1) + 8 * c + 4 * (T & 1) : 16 * T + 4 * c;
    Op<NT> o;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const uint16_t *p = m + ((n * DC + row) * lds_row<KS>() + col);
        const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((dl_lds_s4 *)p));
        const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((dl_lds_s4 *)(p + 16 * lds_row<KS>())));
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
            const uint16_t z = (uint16_t)(r & 1 ? y[r / 2] >> 16 : y[r / 2] & 0xffffu);
            v[r] = DT == BF16 ? bf16_to_f32(z) : f16_to_f32(z);
        }
    }
    return v;
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

// Pieces of X and of the transposes that the backward pass reads: the states and the
// gates' gradients are float32 (with X in two pieces beta's gradient was 1.3e-6 off).
constexpr int kFullPieces = 3;
// pieces of P, which only o is made of: 16-bit results need 16 bits of it
template <int DT> constexpr int mat_pieces() { return DT == F32 ? 3 : 2; }

// LDS of a workgroup of NW waves: keys and queries in pieces, two
// triangular matrices of MP pieces together as fragments, its columns of V (or do) (rows padded by 16 bytes), the gates.
template <int DT, int KS, int NW, int MP> struct ScanLds {
    static constexpr int vrow = 16 * NW + 16 / (int)sizeof(typename IO<DT>::T);
    static constexpr int kq = pieces<DT>() * DC * lds_row<KS>() * 2;
    static constexpr int k = 0, q = kq, mats = 2 * kq, v = mats + MP * MAT * 16,
                         gates = v + DC * vrow * (int)sizeof(typename IO<DT>::T), total = gates + (int)sizeof(ChunkGates);
    static_assert(total <= 160 * 1024, "LDS of a CU");
};

}  // namespace h3
