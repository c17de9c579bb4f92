// The gated delta rule in its recurrent form, for generation: for each (b, h)
// with the state S (Dk, Dv) and T tokens,
//   S <- exp(g_t) S;  e = v_t - S^T k_t;  S <- S + k_t (beta_t e)^T;  o_t = scale S^T q_t.
//
// Columns of S are independent.  A wave takes 32 of them: lane 8 r + c holds
// the rows r + 8 i (i < R) of columns 4 c .. 4 c + 3, so a load covers eight
// rows of 128 contiguous bytes, all of a wave's loads are in flight at once, and the
// sums over rows are R additions and three exchanges between lanes.  The state
// stays in registers over the T tokens: each call reads and writes it once and
// is bound by HBM, or by latency where there are few heads.
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

template <int DT, int R>
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
    const bool on = col < Dv;   // Dv is a multiple of 8
    float *Sp = S + bh * Dk * Dv + col;
    float4 s[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
        s[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (on && r + 8 * i < Dk) s[i] = *(const float4 *)(Sp + (long)(r + 8 * i) * Dv);
    }
    for (int t = 0; t < T; ++t) {
        const long tok = b * T + t;
        const typename IO<DT>::T *kt = k + (tok * Hk + hk) * Dk, *qt = q + (tok * Hk + hk) * Dk;
        float kf[R], qf[R], vf[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const bool in = r + 8 * i < Dk;
            kf[i] = in ? IO<DT>::ld(kt, r + 8 * i) : 0.f;
            qf[i] = in ? IO<DT>::ld(qt, r + 8 * i) : 0.f;
        }
        if (on) {
#pragma unroll
            for (int j = 0; j < 4; ++j) vf[j] = IO<DT>::ld(v + (tok * H + h) * Dv, col + j);
        }
        const float a = expf(g[tok * H + h]), be = beta[tok * H + h];
        float p[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < R; ++i) {
            s[i].x *= a; s[i].y *= a; s[i].z *= a; s[i].w *= a;
            p[0] += kf[i] * s[i].x; p[1] += kf[i] * s[i].y; p[2] += kf[i] * s[i].z; p[3] += kf[i] * s[i].w;
        }
        float u[4], z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) u[j] = be * (vf[j] - rows_sum(p[j]));
#pragma unroll
        for (int i = 0; i < R; ++i) {
            s[i].x += kf[i] * u[0]; s[i].y += kf[i] * u[1]; s[i].z += kf[i] * u[2]; s[i].w += kf[i] * u[3];
            z[0] += qf[i] * s[i].x; z[1] += qf[i] * s[i].y; z[2] += qf[i] * s[i].z; z[3] += qf[i] * s[i].w;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = scale * rows_sum(z[j]);
        if (on && r == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) IO<DT>::st(o + (tok * H + h) * Dv, col + j, z[j]);
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i)
        if (on && r + 8 * i < Dk) *(float4 *)(Sp + (long)(r + 8 * i) * Dv) = s[i];
}

template <int DT>
hipError_t step_of(const void *q, const void *k, const void *v, const float *g, const float *beta, float scale, int B,
                   int T, int H, int Hk, int Dk, int Dv, float *S, void *o, hipStream_t st) {
    typedef typename IO<DT>::T E;
    const long waves = (long)B * H * ((Dv + 31) / 32);
    const unsigned grid = (unsigned)((waves + 3) / 4);
#define H3_STEP(RV)                                                                                                  \
    delta_step_kernel<DT, RV><<<grid, 256, 0, st>>>((const E *)q, (const E *)k, (const E *)v, g, beta, scale, T, H, \
                                                    Hk, Dk, Dv, waves, S, (E *)o)
    if (Dk <= 8) H3_STEP(1);
    else if (Dk <= 32) H3_STEP(4);
    else if (Dk <= 64) H3_STEP(8);
    else if (Dk <= 96) H3_STEP(12);
    else H3_STEP(16);
#undef H3_STEP
    return hipGetLastError();
}

}  // namespace

hipError_t launch_delta_step(const void *q, const void *k, const void *v, const float *g, const float *beta, float scale,
                             int B, int T, int H, int Hk, int Dk, int Dv, int dtype, float *S, void *o, hipStream_t s) {
    if (dtype == F32) return step_of<F32>(q, k, v, g, beta, scale, B, T, H, Hk, Dk, Dv, S, o, s);
    if (dtype == F16) return step_of<F16>(q, k, v, g, beta, scale, B, T, H, Hk, Dk, Dv, S, o, s);
    return step_of<BF16>(q, k, v, g, beta, scale, B, T, H, Hk, Dk, Dv, S, o, s);
}

}  // namespace h3
