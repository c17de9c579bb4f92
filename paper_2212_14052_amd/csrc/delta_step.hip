// The gated delta rule in its recurrent form, for generation: for each (b, h)
// with the state S (Dk, Dv) and T tokens,
//   S <- exp(g_t) S;  e = v_t - S^T k_t;  S <- S + k_t (beta_t e)^T;  o_t = scale S^T q_t.
//
// Columns of S are independent.  A wave takes 32 of them: lane 8 r + c holds
// the rows R r .. R r + R - 1 of columns 4 c .. 4 c + 3, so a load covers eight
// rows of 128 contiguous bytes, all of a wave's loads are in flight at once, a
// lane's keys and queries are R contiguous values, and the sums over rows are R
// additions and three exchanges between lanes.  The state stays in registers over
// the T tokens, the next token's inputs are fetched while one is worked on: each call
// reads and writes the state once and is bound by HBM, or by latency where there are few heads.
// 64 sequences of 20 heads of 128 x 128 bf16, one token: 30.0 us, 5.6 TB/s.  One sequence of 6 heads:
// 7 to 8 us of the kernel, less than the call on the host (10).  19 sequences of 5 tokens, 12 heads of 64 x 96: 10 us
// of the kernel, which asks for a token's inputs only one token ahead, as long as the call.
#include "common.h"
#include "internal.h"

namespace h3 {
namespace {

// the sum over the eight lanes that hold the same columns
__device__ __forceinline__ float rows_sum(float x) {
    x += __shfl_xor(x, 8);
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// N consecutive inputs as floats; VEC: aligned to all of them, or to 16 bytes
template <int DT, int N, bool VEC>
__device__ __forceinline__ void ld_n(const typename IO<DT>::T *__restrict__ p, float (&f)[N]) {
    constexpr int BYTES = N * (int)sizeof(typename IO<DT>::T);
    if constexpr (VEC && BYTES >= 4) {
        uint32_t w[BYTES / 4];
        if constexpr (BYTES % 16 == 0) {
#pragma unroll
            for (int i = 0; i < BYTES / 16; ++i) {
                const uint4 v = ((const uint4 *)p)[i];
                w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
            }
        } else if constexpr (BYTES == 8) {
            const uint2 v = *(const uint2 *)p;
            w[0] = v.x; w[1] = v.y;
        } else {
            w[0] = *(const uint32_t *)p;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (DT == F32) f[i] = __uint_as_float(w[i]);
            else if constexpr (DT == BF16) f[i] = __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
            else f[i] = f16_to_f32((uint16_t)(i & 1 ? w[i / 2] >> 16 : w[i / 2] & 0xffffu));
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) f[i] = IO<DT>::ld(p, i);
    }
}

template <int DT, int R, bool VEC>
__global__ __launch_bounds__(256) void delta_step_kernel(
    const typename IO<DT>::T *__restrict__ q, const typename IO<DT>::T *__restrict__ k,
    const typename IO<DT>::T *__restrict__ v, const float *__restrict__ g, const float *__restrict__ beta, float scale,
    int T, int H, int Hk, int Dk, int Dv, long waves, float *__restrict__ S, typename IO<DT>::T *__restrict__ o) {
    const long wave = (long)blockIdx.x * 4 + threadIdx.x / 64;
    if (wave >= waves) return;
    const int lane = threadIdx.x & 63, r = lane >> 3;
    const int tiles = (Dv + 31) / 32;
    const long bh = wave / tiles, b = bh / H;
    const int h = (int)(bh % H), hk = h / (H / Hk);
    const int col = (int)(wave % tiles) * 32 + 4 * (lane & 7);
    // Dk and Dv are multiples of 8: up to eight rows at a time are there or not
    constexpr int U = R < 8 ? R : 8, NU = R / U;
    const bool on = col < Dv;
    bool rows[NU];
#pragma unroll
    for (int n = 0; n < NU; ++n) rows[n] = r * R + n * U < Dk;
    float kf[NU][U], qf[NU][U], vf[4], a, be;
    auto fetch = [&](int t) {
        const long tok = b * T + t;
#pragma unroll
        for (int n = 0; n < NU; ++n)
            if (rows[n]) {
                ld_n<DT, U, VEC>(k + (tok * Hk + hk) * Dk + r * R + n * U, kf[n]);
                ld_n<DT, U, VEC>(q + (tok * Hk + hk) * Dk + r * R + n * U, qf[n]);
            }
        if (on) ld_n<DT, 4, VEC>(v + (tok * H + h) * Dv + col, vf);
        a = g[tok * H + h];
        be = beta[tok * H + h];
    };
#pragma unroll
    for (int i = 0; i < R; ++i) kf[i / U][i % U] = qf[i / U][i % U] = 0.f;
    vf[0] = vf[1] = vf[2] = vf[3] = 0.f;
    fetch(0);
    float *Sp = S + (bh * Dk + r * R) * Dv + col;
    float4 s[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        s[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (on && rows[i / U]) s[i] = *(const float4 *)(Sp + (long)i * Dv);
    }
    for (int t = 0; t < T; ++t) {
        float kt[R], qt[R], vt[4];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            kt[i] = kf[i / U][i % U];
            qt[i] = qf[i / U][i % U];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) vt[j] = vf[j];
        const float at = expf(a), bt = be;
        if (t + 1 < T) fetch(t + 1);
        float p[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < R; ++i) {
            s[i].x *= at; s[i].y *= at; s[i].z *= at; s[i].w *= at;
            p[0] += kt[i] * s[i].x; p[1] += kt[i] * s[i].y; p[2] += kt[i] * s[i].z; p[3] += kt[i] * s[i].w;
        }
        float u[4], z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = bt * (vt[j] - rows_sum(p[j]));
#pragma unroll
        for (int i = 0; i < R; ++i) {
            s[i].x += kt[i] * u[0]; s[i].y += kt[i] * u[1]; s[i].z += kt[i] * u[2]; s[i].w += kt[i] * u[3];
            z[0] += qt[i] * s[i].x; z[1] += qt[i] * s[i].y; z[2] += qt[i] * s[i].z; z[3] += qt[i] * s[i].w;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = scale * rows_sum(z[j]);
        if (on && r == 0) {
            typename IO<DT>::T *op = o + ((b * T + t) * H + h) * Dv + col;
            if constexpr (VEC && DT == F32) {
                *(float4 *)op = make_float4(z[0], z[1], z[2], z[3]);
            } else if constexpr (VEC) {
                *(uint2 *)op = make_uint2(pack_16x2<DT>(z[0], z[1]), pack_16x2<DT>(z[2], z[3]));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) IO<DT>::st(op, j, z[j]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (on && rows[i / U]) *(float4 *)(Sp + (long)i * Dv) = s[i];
}

template <int DT, bool VEC>
hipError_t step_of(const void *q, const void *k, const void *v, const float *g, const float *beta, float scale, int B,
                   int T, int H, int Hk, int Dk, int Dv, float *S, void *o, hipStream_t st) {
    typedef typename IO<DT>::T E;
    const long waves = (long)B * H * ((Dv + 31) / 32);
    const unsigned grid = (unsigned)((waves + 3) / 4);
#define H3_STEP(RV)                                                                                                       \
    delta_step_kernel<DT, RV, VEC><<<grid, 256, 0, st>>>((const E *)q, (const E *)k, (const E *)v, g, beta, scale, T, H, \
                                                         Hk, Dk, Dv, waves, S, (E *)o)
    if (Dk <= 8) H3_STEP(1);
    else if (Dk <= 16) H3_STEP(2);
    else if (Dk <= 32) H3_STEP(4);
    else if (Dk <= 64) H3_STEP(8);
    else H3_STEP(16);
#undef H3_STEP
    return hipGetLastError();
}

template <int DT>
hipError_t step_by(const void *q, const void *k, const void *v, const float *g, const float *beta, float scale, int B,
                   int T, int H, int Hk, int Dk, int Dv, float *S, void *o, hipStream_t st) {
    // 16-byte loads where all rows start on 16 bytes (Dk and Dv are multiples of 8)
    if ((((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)o) & 15) == 0)
        return step_of<DT, true>(q, k, v, g, beta, scale, B, T, H, Hk, Dk, Dv, S, o, st);
    return step_of<DT, false>(q, k, v, g, beta, scale, B, T, H, Hk, Dk, Dv, S, o, st);
}

}  // namespace

hipError_t launch_delta_step(const void *q, const void *k, const void *v, const float *g, const float *beta, float scale,
                             int B, int T, int H, int Hk, int Dk, int Dv, int dtype, float *S, void *o, hipStream_t s) {
    if (dtype == F32) return step_by<F32>(q, k, v, g, beta, scale, B, T, H, Hk, Dk, Dv, S, o, s);
    if (dtype == F16) return step_by<F16>(q, k, v, g, beta, scale, B, T, H, Hk, Dk, Dv, S, o, s);
    return step_by<BF16>(q, k, v, g, beta, scale, B, T, H, Hk, Dk, Dv, S, o, s);
}

}  // namespace h3
