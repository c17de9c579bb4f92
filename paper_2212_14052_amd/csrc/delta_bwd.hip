// Backward pass of the gated delta rule, chunk by chunk.
//
// With a chunk's G, A, X, P, e, u, S of the forward pass (delta.hip), f_i = exp(G_i), t_i =
// exp(G_63 - G_i), do the output's gradient times the scale, and dS' the gradient of the state
// behind the chunk:
//     du = P^T do + t (K dS'),   z = du - X^T (beta du),   y = beta z = dv,
//     dS = exp(G_63) dS' + Q^T (f do) - K^T (f y)
// is again a scan whose columns do not meet, in the order from the end
// (delta_bwd_scan_kernel); it leaves z and dS' of every chunk.  Then every chunk for itself
// (delta_bwd_chunk_kernel), with
//     D = lower part of (do u^T) exp(G_i - G_j),  E = -(strictly lower part of (y u^T) exp(G_i - G_j)):
//     dq = f (do S^T) + D K,   dk = reads + writes,  reads = E K - f (y S^T),
//     writes = D^T Q + E^T K + t (u dS'^T),   dbeta_i = z_i . e_i,
//     dG_i = q_i . dq_i + k_i . (reads_i - writes_i),   dg_t = sum_{i >= t} dG_i + <S', dS'>,
// where <S', dS'> = exp(G_63) <S, dS'> + sum_i k_i . t_i (u dS'^T)_i.
#include "delta_common.h"

namespace h3 {
namespace {

template <int DT, int KS, int NW>
__global__ __launch_bounds__(64 * NW, 1) void delta_bwd_scan_kernel(DeltaArgs a, const uint4 *__restrict__ XTF,
                                                                   const uint4 *__restrict__ PTF,
                                                                   const ChunkGates *__restrict__ gates, DeltaGrads d) {
    typedef typename IO<DT>::T T;
    constexpr int NT = pieces<DT>(), NM = kFullPieces;
    typedef ScanLds<DT, KS, NW, 2 * NM> Lds;
    constexpr int NTH = 64 * NW, ITEMS = 4 * KS / NW, MATS = 2 * NM * MAT / NTH, VALS = 2, GATES = (3 * DC + NTH - 1) / NTH;
    static_assert(2 * NM * MAT % NTH == 0 && 4 * KS % NW == 0 && DC * 2 * NW == VALS * NTH, "whole shares");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    uint16_t *ks = (uint16_t *)(lds + Lds::k), *qs = (uint16_t *)(lds + Lds::q);
    uint4 *ms = (uint4 *)(lds + Lds::mats);
    T *vs = (T *)(lds + Lds::v);
    ChunkGates *gt = (ChunkGates *)(lds + Lds::gates);
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g4 = lane >> 4, c16 = lane & 15;
    const int tiles = (a.Dv + 16 * NW - 1) / (16 * NW);
    const long bh = blockIdx.x / tiles;
    const int h = (int)(bh % a.H), b = (int)(bh / a.H), hk = h / (a.H / a.Hk);
    const int c0 = ((int)(blockIdx.x % tiles) * NW + w) * 16, cb = c0 - 16 * w;
    const bool here = c0 < a.Dv;
    const int col = c0 + c16;
    const bool on = col < a.Dv;
    const int len = tokens_of(a, b), nb = (len + DC - 1) / DC;
    const T *kp = (const T *)a.k, *qp = (const T *)a.q, *vp = (const T *)d.dout;

    Raw8<DT> pk[ITEMS], pq[ITEMS], pv[VALS];
    uint4 pm[MATS];
    float pg[GATES];
    auto fetch = [&](int n) {
        const long tok0 = (long)b * a.L + n * DC;
        const int nt = len - n * DC;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int it = i * NTH + tid, t = it / (4 * KS), c = 8 * (it % (4 * KS));
            const long at = ((tok0 + t) * a.Hk + hk) * a.Dk + c;
            pk[i] = ld8_raw<DT>(kp + at, t < nt && c < a.Dk);
            pq[i] = ld8_raw<DT>(qp + at, t < nt && c < a.Dk);
        }
#pragma unroll
        for (int i = 0; i < VALS; ++i) {
            const int it = i * NTH + tid, t = it / (2 * NW), c = cb + 8 * (it % (2 * NW));
            pv[i] = ld8_raw<DT>(vp + ((tok0 + t) * a.H + h) * a.Dv + c, t < nt && c < a.Dv);
        }
        const long ch = bh * a.N + n;
        const uint4 *xp = XTF + ch * NM * MAT, *pp = PTF + ch * NM * MAT;
#pragma unroll
        for (int i = 0; i < MATS; ++i) {
            const int it = i * NTH + tid;
            pm[i] = it < NM * MAT ? xp[it] : pp[it - NM * MAT];
        }
        const float *gp = (const float *)(gates + ch);
#pragma unroll
        for (int i = 0; i < GATES; ++i)
            if (i * NTH + tid < 3 * DC) pg[i] = gp[i * NTH + tid];
    };

    dl_f4 S[2 * KS];   // dS'
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r;
            S[t][r] = d.dS && on && dk < a.Dk ? d.dS[(bh * a.Dk + dk) * a.Dv + col] : 0.f;
        }
    if (nb > 0) fetch(nb - 1);
    for (int n = nb - 1; n >= 0; --n) {
        const long ch = bh * a.N + n;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int it = i * NTH + tid, t = it / (4 * KS), c = 8 * (it % (4 * KS));
            const Op<NT> ko = op_of<DT>(pk[i]), qo = op_of<DT>(pq[i]);
#pragma unroll
            for (int p = 0; p < NT; ++p) {
                *(uint4 *)(ks + (p * DC + t) * lds_row<KS>() + c) = ko.p[p];
                *(uint4 *)(qs + (p * DC + t) * lds_row<KS>() + c) = qo.p[p];
            }
        }
#pragma unroll
        for (int i = 0; i < VALS; ++i) {
            const int it = i * NTH + tid;
            T *p = vs + it / (2 * NW) * Lds::vrow + 8 * (it % (2 * NW));
#pragma unroll
            for (int j = 0; j < (DT == F32 ? 2 : 1); ++j) ((uint4 *)p)[j] = pv[i].a[j];
        }
#pragma unroll
        for (int i = 0; i < MATS; ++i) ms[i * NTH + tid] = pm[i];
#pragma unroll
        for (int i = 0; i < GATES; ++i)
            if (i * NTH + tid < 3 * DC) ((float *)gt)[i * NTH + tid] = pg[i];
        __syncthreads();
        if (n > 0) fetch(n - 1);
        if (!here) continue;
        if (on) {
#pragma unroll
            for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r;
                    if (dk < a.Dk) d.dends[(ch * a.Dk + dk) * a.Dv + col] = S[t][r];
                }
        }
        // du = t (K dS') + P^T do
        dl_f4 u[4], dd[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            u[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
            dd[t] = lds_column4<DT>(vs, Lds::vrow, 16 * t, 16 * w, lane);
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const Op<3> so = split8<3>(S[2 * s], S[2 * s + 1]);
#pragma unroll
            for (int t = 0; t < 4; ++t) u[t] = mm(lds_rows<NT, KS>(ks, t, s, lane), so, u[t]);
        }
        Op<NM> bu[2];
        dl_f4 be[4];
        {
            Op<NT> od[2];   // exact: do as it came
#pragma unroll
            for (int s = 0; s < 2; ++s) od[s] = split8<NT>(dd[2 * s], dd[2 * s + 1]);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                dl_f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = t / 2; s < 2; ++s) x = mm(ld_frag<NM>(ms + NM * MAT, upper_frag(t, s), lane), od[s], x);
                const dl_f4 f = *(const dl_f4 *)(gt->toend + 16 * t + 4 * g4);
                be[t] = *(const dl_f4 *)(gt->beta + 16 * t + 4 * g4);
#pragma unroll
                for (int r = 0; r < 4; ++r) u[t][r] = f[r] * u[t][r] + a.scale * x[r];
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                dl_f4 p, q;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    p[r] = be[2 * s][r] * u[2 * s][r];
                    q[r] = be[2 * s + 1][r] * u[2 * s + 1][r];
                }
                bu[s] = split8<NM>(p, q);
            }
        }
        // z = du - X^T (beta du); then f y and f do for the state
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            dl_f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = t / 2; s < 2; ++s) x = mm(ld_frag<NM>(ms, upper_frag(t, s), lane), bu[s], x);
            const dl_f4 f = *(const dl_f4 *)(gt->from0 + 16 * t + 4 * g4);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float z = u[t][r] - x[r];
                if (on) d.zs[(ch * DC + 16 * t + 4 * g4 + r) * a.Dv + col] = z;
                u[t][r] = -f[r] * be[t][r] * z;
                dd[t][r] *= f[r] * a.scale;
            }
        }
        Op<3> yo[2], qo[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            yo[s] = split8<3>(u[2 * s], u[2 * s + 1]);
            qo[s] = split8<3>(dd[2 * s], dd[2 * s + 1]);
        }
        const float f = gt->from0[DC - 1];
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t) {
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] *= f;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                S[t] = mm(lds_cols<NT, KS>(ks, t, s, lane), yo[s], S[t]);
                S[t] = mm(lds_cols<NT, KS>(qs, t, s, lane), qo[s], S[t]);
            }
        }
    }
    if (here && on && d.dS0) {
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r;
                if (dk < a.Dk) d.dS0[(bh * a.Dk + dk) * a.Dv + col] = S[t][r];
            }
    }
}

constexpr int AROW = DC + 4;   // floats a row of a 64 x 64 matrix in LDS

template <int DT, int KS> struct GradLds {
    static constexpr int kq = pieces<DT>() * DC * lds_row<KS>() * 2;
    static constexpr int k = 0, q = kq, D = 2 * kq, E = D + DC * AROW * 4, gd = E + DC * AROW * 4, gates = gd + DC * 8,
                         red = gates + (int)sizeof(ChunkGates), total = red + (4 * DC + 4) * 4;
    static_assert(total <= 160 * 1024, "LDS of a CU");
};

// A workgroup of four waves takes a chunk of a key head and goes through the
// value heads that share it.  Every wave has KS / 2 (rounded up) of the key channels' tiles
// for all tokens: results are transposed (rows are channels), so that a lane
// holds four consecutive channels of one token.
template <int DT, int KS>
__global__ __launch_bounds__(256, 1) void delta_bwd_chunk_kernel(DeltaArgs a, const ChunkGates *__restrict__ gates,
                                                              const float *__restrict__ es,
                                                              const float *__restrict__ states, DeltaGrads d) {
    typedef typename IO<DT>::T T;
    constexpr int NT = pieces<DT>(), TT = (KS + 1) / 2;
    typedef GradLds<DT, KS> Lds;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    uint16_t *ks = (uint16_t *)(lds + Lds::k), *qs = (uint16_t *)(lds + Lds::q);
    float *D = (float *)(lds + Lds::D), *E = (float *)(lds + Lds::E);
    double *gd = (double *)(lds + Lds::gd);
    ChunkGates *gt = (ChunkGates *)(lds + Lds::gates);
    float *red = (float *)(lds + Lds::red);   // 4 x 64 partial sums of dG, 4 of <S', dS'>
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g4 = lane >> 4, c16 = lane & 15;
    const int n = (int)(blockIdx.x % a.N), hk = (int)(blockIdx.x / a.N % a.Hk), b = (int)(blockIdx.x / a.N / a.Hk);
    const int per = a.H / a.Hk;
    const int nt = min(DC, tokens_of(a, b) - n * DC), room = min(DC, a.L - n * DC);   // tokens, and places, of this chunk
    const long tok0 = (long)b * a.L + n * DC;
    const T *kp = (const T *)a.k, *qp = (const T *)a.q, *op = (const T *)d.dout;
    T *dqp = (T *)d.dq, *dkp = (T *)d.dk, *dvp = (T *)d.dv;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        const int it = i * 256 + tid, t = it / (4 * KS), c = 8 * (it % (4 * KS));
        const long at = ((tok0 + t) * a.Hk + hk) * a.Dk + c;
        const bool on = t < nt && c < a.Dk;
        const Op<NT> ko = op_of<DT>(ld8_raw<DT>(kp + at, on)), qo = op_of<DT>(ld8_raw<DT>(qp + at, on));
#pragma unroll
        for (int p = 0; p < NT; ++p) {
            *(uint4 *)(ks + (p * DC + t) * lds_row<KS>() + c) = ko.p[p];
            *(uint4 *)(qs + (p * DC + t) * lds_row<KS>() + c) = qo.p[p];
        }
    }
    dl_f4 tq[4][TT], tk[4][TT];   // sums over the value heads
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < TT; ++j) tq[t][j] = tk[t][j] = dl_f4{0.f, 0.f, 0.f, 0.f};

    for (int hh = 0; hh < per; ++hh) {
        const int h = hk * per + hh;
        const long ch = ((long)b * a.H + h) * a.N + n;
        __syncthreads();   // keys and queries are there; the last head's matrices are read
        if (nt <= 0) {     // nothing behind a sequence's end has a gradient
            for (int it = tid; it < room * a.Dv; it += 256) IO<DT>::st(dvp + ((tok0 + it / a.Dv) * a.H + h) * a.Dv, it % a.Dv, 0.f);
            if (tid < room) d.dg[(tok0 + tid) * a.H + h] = d.dbeta[(tok0 + tid) * a.H + h] = 0.f;
            continue;
        }
        if (w == 0) gd[lane] = decay_sum(lane < nt ? a.g[(tok0 + lane) * a.H + h] : 0.f, lane < nt, lane);
        if (tid < 3 * DC) ((float *)gt)[tid] = ((const float *)(gates + ch))[tid];
        __syncthreads();
        const float *ep = es + ch * DC * a.Dv, *zp = d.zs + ch * DC * a.Dv;
        const float *Sp = states + ch * a.Dk * a.Dv, *Ep = d.dends + ch * a.Dk * a.Dv;
        // row tile w of D and E; dv and dbeta of its tokens
        {
            dl_f4 ad[4], ae[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) ad[j] = ae[j] = dl_f4{0.f, 0.f, 0.f, 0.f};
            const int row = 16 * w + c16;
            const float be = gt->beta[row];
            float dot = 0.f;
            for (int c = 8 * g4; c < ((a.Dv + 31) & ~31); c += 32) {
                const bool on = c < a.Dv;
                float z[8], e[8], y[8];
                ld8<F32>(zp + (long)row * a.Dv + c, on, z);
                ld8<F32>(ep + (long)row * a.Dv + c, on, e);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dot += z[i] * e[i];
                    y[i] = row < nt ? be * z[i] : 0.f;
                }
                if (on && row < room) {
                    T *p = dvp + ((tok0 + row) * a.H + h) * a.Dv + c;
                    if constexpr (DT == F32) {
                        *(float4 *)p = make_float4(y[0], y[1], y[2], y[3]);
                        *(float4 *)(p + 4) = make_float4(y[4], y[5], y[6], y[7]);
                    } else {
                        *(uint4 *)p = make_uint4(pack_16x2<DT>(y[0], y[1]), pack_16x2<DT>(y[2], y[3]),
                                                 pack_16x2<DT>(y[4], y[5]), pack_16x2<DT>(y[6], y[7]));
                    }
                }
                const Op<3> yo = split8<3>(y);
                const Op<NT> oo = op_of<DT>(ld8_raw<DT>(op + ((tok0 + row) * a.H + h) * a.Dv + c, on && row < nt));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j > w) break;
                    float u[8];
                    const int r = 16 * j + c16;
                    ld8<F32>(ep + (long)r * a.Dv + c, on, u);
                    const float bj = gt->beta[r];
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[i] *= bj;
                    const Op<3> uo = split8<3>(u);
                    ad[j] = mm(oo, uo, ad[j]);
                    ae[j] = mm(yo, uo, ae[j]);
                }
            }
            dot += __shfl_xor(dot, 16);
            dot += __shfl_xor(dot, 32);
            if (g4 == 0 && row < room) d.dbeta[(tok0 + row) * a.H + h] = row < nt ? dot : 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = 16 * j + c16;
                const double gj = gd[col];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * w + 4 * g4 + r;
                    float f = 0.f;
                    if (i >= col) f = __builtin_amdgcn_exp2f((float)(gd[i] - gj));
                    D[i * AROW + col] = i >= col ? a.scale * ad[j][r] * f : 0.f;
                    E[i * AROW + col] = i > col ? -ae[j][r] * f : 0.f;
                }
            }
        }
        // products with the states
        dl_f4 dq[4][TT], kr[4][TT], kw[4][TT];
        float inner = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < TT; ++j) dq[t][j] = kr[t][j] = kw[t][j] = dl_f4{0.f, 0.f, 0.f, 0.f};
        for (int c = 8 * g4; c < ((a.Dv + 31) & ~31); c += 32) {
            const bool on = c < a.Dv;
            Op<3> so[TT], eo[TT];
#pragma unroll
            for (int j = 0; j < TT; ++j) {
                const int dk = 16 * (w * TT + j) + c16;
                float x[8], y[8];
                ld8<F32>(Sp + (long)dk * a.Dv + c, on && dk < a.Dk, x);
                ld8<F32>(Ep + (long)dk * a.Dv + c, on && dk < a.Dk, y);
#pragma unroll
                for (int i = 0; i < 8; ++i) inner += x[i] * y[i];
                so[j] = split8<3>(x);
                eo[j] = split8<3>(y);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int row = 16 * t + c16;
                const float be = gt->beta[row];
                float y[8], u[8];
                ld8<F32>(zp + (long)row * a.Dv + c, on, y);
                ld8<F32>(ep + (long)row * a.Dv + c, on, u);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    y[i] *= be;
                    u[i] *= be;
                }
                const Op<3> yo = split8<3>(y), uo = split8<3>(u);
                const Op<NT> oo = op_of<DT>(ld8_raw<DT>(op + ((tok0 + row) * a.H + h) * a.Dv + c, on && row < nt));
#pragma unroll
                for (int j = 0; j < TT; ++j) {
                    dq[t][j] = mm(so[j], oo, dq[t][j]);
                    kr[t][j] = mm(so[j], yo, kr[t][j]);
                    kw[t][j] = mm(eo[j], uo, kw[t][j]);
                }
            }
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) inner += __shfl_xor(inner, m);
        inner *= gt->from0[DC - 1];
        float kx = 0.f;   // sum of k . t (u dS'^T)
        __syncthreads();  // D and E are there
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int row = 16 * t + c16;
            const float f = gt->from0[row], e = gt->toend[row];
            Op<3> dr[2], er[2], dc[2], ec[2];   // rows and columns `row` of D and E
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int o = 32 * s + 4 * g4;
                if (s <= t / 2) {
                    dr[s] = split8<3>(*(const dl_f4 *)(D + row * AROW + o), *(const dl_f4 *)(D + row * AROW + o + 16));
                    er[s] = split8<3>(*(const dl_f4 *)(E + row * AROW + o), *(const dl_f4 *)(E + row * AROW + o + 16));
                }
                if (s >= t / 2) {
                    float x[8], y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[i] = D[(o + (i & 3) + 16 * (i >> 2)) * AROW + row];
                        y[i] = E[(o + (i & 3) + 16 * (i >> 2)) * AROW + row];
                    }
                    dc[s] = split8<3>(x);
                    ec[s] = split8<3>(y);
                }
            }
            float dG = 0.f;
#pragma unroll
            for (int j = 0; j < TT; ++j) {
                const int ct = w * TT + j;   // this wave's channel tile
                if (ct >= 2 * KS) break;
                float kv[4] = {0.f, 0.f, 0.f, 0.f}, qv[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int p = NT - 1; p >= 0; --p) {
                    const int at = (p * DC + row) * lds_row<KS>() + 16 * ct + 4 * g4;
                    const uint2 x = *(const uint2 *)(ks + at), y = *(const uint2 *)(qs + at);
                    kv[0] += __uint_as_float(x.x << 16); kv[1] += __uint_as_float(x.x & 0xffff0000u);
                    kv[2] += __uint_as_float(x.y << 16); kv[3] += __uint_as_float(x.y & 0xffff0000u);
                    qv[0] += __uint_as_float(y.x << 16); qv[1] += __uint_as_float(y.x & 0xffff0000u);
                    qv[2] += __uint_as_float(y.y << 16); qv[3] += __uint_as_float(y.y & 0xffff0000u);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    dq[t][j][r] *= f * a.scale;
                    kr[t][j][r] *= -f;
                    kw[t][j][r] *= e;
                    kx += kv[r] * kw[t][j][r];
                }
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const Op<NT> kc = lds_cols<NT, KS, false>(ks, ct, s, lane);
                    if (s <= t / 2) {
                        dq[t][j] = mm(kc, dr[s], dq[t][j]);
                        kr[t][j] = mm(kc, er[s], kr[t][j]);
                    }
                    if (s >= t / 2) {
                        kw[t][j] = mm(lds_cols<NT, KS, false>(qs, ct, s, lane), dc[s], kw[t][j]);
                        kw[t][j] = mm(kc, ec[s], kw[t][j]);
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    dG += qv[r] * dq[t][j][r] + kv[r] * (kr[t][j][r] - kw[t][j][r]);
                    tq[t][j][r] += dq[t][j][r];
                    tk[t][j][r] += kr[t][j][r] + kw[t][j][r];
                }
            }
            dG += __shfl_xor(dG, 16);
            dG += __shfl_xor(dG, 32);
            if (g4 == 0) red[w * DC + row] = dG;
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) kx += __shfl_xor(kx, m);
        if (lane == 0) red[4 * DC + w] = inner + kx;
        __syncthreads();
        if (w == 0) {
            // suffix sums in float64: many terms, of both signs
            double x = (double)red[lane] + red[DC + lane] + red[2 * DC + lane] + red[3 * DC + lane];
#pragma unroll
            for (int m = 1; m < 64; m *= 2) {
                const double y = __shfl_down(x, m);
                if (lane + m < 64) x += y;
            }
            x += (double)red[4 * DC] + red[4 * DC + 1] + red[4 * DC + 2] + red[4 * DC + 3];
            if (lane < room) d.dg[(tok0 + lane) * a.H + h] = lane < nt ? (float)x : 0.f;
        }
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int row = 16 * t + c16;
        if (row >= room) continue;
        const bool real = row < nt;
#pragma unroll
        for (int j = 0; j < TT; ++j) {
            const int dk = 16 * (w * TT + j) + 4 * g4;
            if (dk >= a.Dk) continue;
            const long at = ((tok0 + row) * a.Hk + hk) * a.Dk + dk;
            dl_f4 x = tq[t][j], y = tk[t][j];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = real ? x[r] : 0.f;
                y[r] = real ? y[r] : 0.f;
            }
            if constexpr (DT == F32) {
                *(float4 *)(dqp + at) = make_float4(x[0], x[1], x[2], x[3]);
                *(float4 *)(dkp + at) = make_float4(y[0], y[1], y[2], y[3]);
            } else {
                *(uint2 *)(dqp + at) = make_uint2(pack_16x2<DT>(x[0], x[1]), pack_16x2<DT>(x[2], x[3]));
                *(uint2 *)(dkp + at) = make_uint2(pack_16x2<DT>(y[0], y[1]), pack_16x2<DT>(y[2], y[3]));
            }
        }
    }
}

template <int DT, int KS> hipError_t bwd_of(const DeltaArgs &a, const DeltaBuffers &w, const DeltaGrads &d, hipStream_t st) {
    constexpr int NW = 4;
    constexpr int lds = ScanLds<DT, KS, NW, 2 * kFullPieces>::total, lds2 = GradLds<DT, KS>::total;
    if (lds > 65536)
        (void)hipFuncSetAttribute((const void *)delta_bwd_scan_kernel<DT, KS, NW>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    if (lds2 > 65536)
        (void)hipFuncSetAttribute((const void *)delta_bwd_chunk_kernel<DT, KS>, hipFuncAttributeMaxDynamicSharedMemorySize, lds2);
    const int tiles = (a.Dv + 16 * NW - 1) / (16 * NW);
    delta_bwd_scan_kernel<DT, KS, NW><<<(unsigned)((long)a.B * a.H * tiles), 64 * NW, lds, st>>>(a, w.XT, w.PT, w.gates, d);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    delta_bwd_chunk_kernel<DT, KS><<<(unsigned)((long)a.B * a.Hk * a.N), 256, lds2, st>>>(a, w.gates, w.es, w.states, d);
    return hipGetLastError();
}

template <int DT> hipError_t bwd_by(const DeltaArgs &a, const DeltaBuffers &w, const DeltaGrads &d, hipStream_t st) {
    switch ((a.Dk + 31) / 32) {
        case 1: return bwd_of<DT, 1>(a, w, d, st);
        case 2: return bwd_of<DT, 2>(a, w, d, st);
        case 3: return bwd_of<DT, 3>(a, w, d, st);
        default: return bwd_of<DT, 4>(a, w, d, st);
    }
}

}  // namespace

hipError_t launch_delta_rule_bwd(const DeltaArgs &a, int dtype, const DeltaBuffers &w, const DeltaGrads &d, hipStream_t s) {
    if (dtype == F32) return bwd_by<F32>(a, w, d, s);
    if (dtype == F16) return bwd_by<F16>(a, w, d, s);
    return bwd_by<BF16>(a, w, d, s);
}

}  // namespace h3
