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

template <int DT, int KS, int NW, bool MAPS>
__global__ __launch_bounds__(64 * NW, 1) void delta_bwd_scan_kernel(DeltaArgs a, DeltaSegments sg, const uint4 *__restrict__ rec,
                                                                   const uint4 *__restrict__ kq, DeltaGrads d) {
    typedef typename IO<DT>::T T;
    constexpr int NT = pieces<DT>(), NM = 2;
    typedef ChunkCopy<DT, KS, NW, 2 * NM> Copy;
    typedef typename Copy::Lds Lds;
    extern __shared__ uint4 lds[];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g4 = lane >> 4, c16 = lane & 15;
    const int dvp = (a.Dv + 15) & ~15;
    const ScanPlace<NW, MAPS, true> at_(a, sg, blockIdx.x, w);
    const long bh = at_.bh;
    const int h = at_.h, b = at_.b, hk = h / (a.H / a.Hk), seg = at_.seg, cb = at_.cb, c0 = at_.c0;
    const bool here = c0 < at_.width;
    const int col = c0 + c16;
    const bool on = col < at_.width;
    const int len = tokens_of(a, b), nb = (len + DC - 1) / DC;
    const int first = seg * sg.Ns, last = min(first + sg.Ns, nb);   // chunks from, and before
    if (MAPS ? first >= last : first >= last && seg > 0) return;
    const Copy in{kq + ((long)b * a.Hk + hk) * a.N * 2 * Lds::kq, rec + bh * a.N * Lds::words,
                  (const T *)d.dout + ((long)b * a.L * a.H + h) * a.Dv + (at_.unit ? 0 : cb), (long)a.H * a.Dv,
                  a.Dv - (at_.unit ? 0 : cb), len, (uint32_t)(uintptr_t)(dl_lds_void *)lds};

    dl_f4 S[2 * KS];   // dS' 2^-E
    int E = 0;
    const float *dS = MAPS ? nullptr : sg.G > 1 ? sg.in + ((long)seg * a.B * a.H) * a.Dk * a.Dv : d.dS;
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r;
            S[t][r] = dS && on && dk < a.Dk ? dS[(bh * a.Dk + dk) * a.Dv + col] : 0.f;
            if (MAPS && at_.unit && on && dk == col) S[t][r] = 1.f;
        }
    if (Lds::two && first < last) in.issue(last - 1, w, lane);
    for (int n = last - 1; n >= first; --n) {
        const long ch = bh * a.N + n;
        const uint4 *at = in.arrive(lds, n, n - 1, n > first, w, lane);
        if (!here) continue;
        const uint4 *ks = at + Lds::k, *qs = at + Lds::q, *xs = at + Lds::rec, *ps = xs + NM * MAT;   // X^T, P^T
        const T *vs = (const T *)(at + Lds::v);
        const ChunkGates *gt = (const ChunkGates *)(ps + NM * MAT);
        const int nt = min(DC, len - n * DC);
        if constexpr (!MAPS) {
            float *p = d.dends + (ch * 32 * KS + 8 * g4) * dvp + col;
#pragma unroll
            for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) p[(32 * (t >> 1) + 4 * (t & 1) + r) * dvp] = __builtin_amdgcn_ldexpf(S[t][r], E);
        }
        const int ek = __builtin_amdgcn_readfirstlane(gt->ek), eq = __builtin_amdgcn_readfirstlane(gt->eq),
                  ex = __builtin_amdgcn_readfirstlane(gt->ex), ep = __builtin_amdgcn_readfirstlane(gt->ep),
                  ef = __builtin_amdgcn_readfirstlane(gt->ef);
        // du = t (K dS') + P^T do
        dl_f4 u[4], dd[4], te[4], be[4];
        Op<NM> pf[6], xf[6];
        Op<NT> kf[2][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            u[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
            kf[0][t] = lds_rows<NT, KS>(ks, t, 0, lane);
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            dd[t] = lds_column4<DT>(vs, Lds::vrow, 16 * t, 16 * w, lane);
            if (MAPS && at_.unit) dd[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
        }
        const int em = wave_exp(S), eS = em + E;   // of the registers, of dS'
        const float sc = pow2(-em);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (s + 1 < KS) {
#pragma unroll
                for (int t = 0; t < 4; ++t) kf[(s + 1) & 1][t] = lds_rows<NT, KS>(ks, t, s + 1, lane);
            } else {
#pragma unroll
                for (int f = 0; f < 6; ++f) pf[f] = ld_frag<NM>(ps, f, lane);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    te[t] = *(const dl_f4 *)(gt->toend + 16 * t + 4 * g4);
                    be[t] = *(const dl_f4 *)(gt->beta + 16 * t + 4 * g4);
                }
            }
            in_order();
            const Op<2> so = split8<2>(S[2 * s], S[2 * s + 1], sc);
#pragma unroll
            for (int t = 0; t < 4; ++t) u[t] = mm(kf[s & 1][t], so, u[t]);
            in_order();
        }
        if (nt < DC) {   // the last chunk: nothing comes from behind the end
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) dd[t][r] = 16 * t + 4 * g4 + r < nt ? dd[t][r] : 0.f;
        }
        const int ed = wave_exp(dd);
#pragma unroll
        for (int f = 0; f < 6; ++f) xf[f] = ld_frag<NM>(xs, f, lane);
        in_order();
        dl_f4 y[4];
        {
            const int e = DT == F16 ? 0 : ed;
            const float py = __builtin_amdgcn_ldexpf(a.scale, ep + e);
            Op<NT> od[2];   // do as it came
#pragma unroll
            for (int s = 0; s < 2; ++s) od[s] = split8<NT>(dd[2 * s], dd[2 * s + 1], pow2(-e));
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                dl_f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = t / 2; s < 2; ++s) x = mm(pf[upper_frag(t, s)], od[s], x);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    u[t][r] = __builtin_amdgcn_ldexpf(te[t][r], ek + eS) * u[t][r] + py * x[r];
                    y[t][r] = be[t][r] * u[t][r];
                }
            }
        }
        // z = du - X^T (beta du); then f y and f do for the state
        const int eu = wave_exp(y);
        Op<NT> kc[2][2], qc[2][2];
        dl_f4 f0[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) f0[t] = *(const dl_f4 *)(gt->from0 + 16 * t + 4 * g4);
        const float fl = gt->from0[DC - 1];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            kc[0][s] = lds_cols<NT, KS>(ks, 0, s, lane);
            qc[0][s] = lds_cols<NT, KS>(qs, 0, s, lane);
        }
        in_order();
        {
            Op<NM> bu[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) bu[s] = split8<NM>(y[2 * s], y[2 * s + 1], pow2(-eu));
            float *p = d.zs + (ch * DC + 4 * g4) * dvp + col;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                dl_f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = t / 2; s < 2; ++s) x = mm(xf[upper_frag(t, s)], bu[s], x);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float z = u[t][r] - __builtin_amdgcn_ldexpf(x[r], eu + ex);
                    if constexpr (!MAPS) p[(16 * t + r) * dvp] = z;
                    y[t][r] = be[t][r] * z;
                    u[t][r] = -f0[t][r] * y[t][r];
                    dd[t][r] *= f0[t][r] * a.scale;
                }
            }
        }
        const int ez = wave_exp(y), esc = scale_exp(mag(a.scale)) + 13;   // 2^esc: at most the scale
        if (!MAPS && lane == 0) d.exps[ch * kDeltaTiles + c0 / 16] = make_int4(ez, max(min(eS, 114), -126), ed, 0);
        // dS <- exp(G_63) dS' + Q^T (f do) - K^T (f y), both in units of the larger one's scale; of
        // 2^-60 of dS' where both are smaller than that
        const int En = max(max(ek + ez + ef, eq + ed + ef + esc + 1), max(eS - 60, E - 100));
        const float fs = fl * pow2(max(E - En, -126)), sy = pow2(max(min(ek - En, 127), -126)), so_ = pow2(max(min(eq - En, 127), -126));
        E = En;
        Op<2> yo[2], qo[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            yo[s] = split8<2>(u[2 * s], u[2 * s + 1], sy);
            qo[s] = split8<2>(dd[2 * s], dd[2 * s + 1], so_);
        }
        dl_f4 x[2];
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t) {
            if (t + 1 < 2 * KS) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    kc[(t + 1) & 1][s] = lds_cols<NT, KS>(ks, t + 1, s, lane);
                    qc[(t + 1) & 1][s] = lds_cols<NT, KS>(qs, t + 1, s, lane);
                }
            }
            in_order();
            x[t & 1] = dl_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                x[t & 1] = mm(kc[t & 1][s], yo[s], x[t & 1]);
                x[t & 1] = mm(qc[t & 1][s], qo[s], x[t & 1]);
            }
            if (t > 0) {
#pragma unroll
                for (int r = 0; r < 4; ++r) S[t - 1][r] = S[t - 1][r] * fs + x[(t - 1) & 1][r];
            }
            in_order();
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) S[2 * KS - 1][r] = S[2 * KS - 1][r] * fs + x[1][r];
    }
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[t][r] = __builtin_amdgcn_ldexpf(S[t][r], E);
    if constexpr (MAPS) {
        if (here) store_map<KS>(a, sg, at_, S, E, lane);
        return;
    }
    if (here && on && d.dS0 && seg == 0) {
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
    static constexpr int kq = kq_words<KS>(pieces<DT>());
    static constexpr int k = 0, q = kq * 16, D = 2 * kq * 16, E = D + DC * AROW * 4, gd = E + DC * AROW * 4, gates = gd + DC * 8,
                         red = gates + (int)sizeof(ChunkGates), total = red + (4 * DC + 16) * 4;
    static_assert(total <= 160 * 1024, "LDS of a CU");
};

// A workgroup of four waves takes a chunk of a key head and goes through the
// value heads that share it.  Every wave has KS / 2 (rounded up) of the key channels' tiles
// for all tokens: results are transposed (rows are channels), so that a lane
// holds four consecutive channels of one token.
template <int DT, int KS>
__global__ __launch_bounds__(256, 1) void delta_bwd_chunk_kernel(DeltaArgs a, const uint4 *__restrict__ rec,
                                                              const uint4 *__restrict__ kq,
                                                              const float *__restrict__ es,
                                                              const float *__restrict__ states,
                                                              const int2 *__restrict__ exps, DeltaGrads d) {
    typedef typename IO<DT>::T T;
    constexpr int NT = pieces<DT>(), TT = (KS + 1) / 2;
    typedef GradLds<DT, KS> Lds;
    extern __shared__ uint4 lds[];
    char *l8 = (char *)lds;
    uint4 *ks = (uint4 *)(l8 + Lds::k), *qs = (uint4 *)(l8 + Lds::q);
    float *D = (float *)(l8 + Lds::D), *E = (float *)(l8 + Lds::E);
    double *gd = (double *)(l8 + Lds::gd);
    ChunkGates *gt = (ChunkGates *)(l8 + Lds::gates);
    float *red = (float *)(l8 + Lds::red);        // the waves' sums of dG
    double *rin = (double *)(red + 4 * DC);       // and of <S', dS'>
    uint32_t *big = (uint32_t *)(rin + 4);   // the waves' largest magnitudes of D and of E
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g4 = lane >> 4, c16 = lane & 15;
    const int n = (int)(blockIdx.x % a.N), hk = (int)(blockIdx.x / a.N % a.Hk), b = (int)(blockIdx.x / a.N / a.Hk);
    const int per = a.H / a.Hk, dvp = (a.Dv + 15) & ~15;
    const int nt = min(DC, tokens_of(a, b) - n * DC), room = min(DC, a.L - n * DC);   // tokens, and places, of this chunk
    const long tok0 = (long)b * a.L + n * DC;
    const T *op = (const T *)d.dout;
    T *dqp = (T *)d.dq, *dkp = (T *)d.dk, *dvo = (T *)d.dv;
    int ek = 0, eq = 0;
    if (nt > 0) {
        const ChunkGates *g = (const ChunkGates *)(rec + ((((long)b * a.H + hk * per) * a.N + n) * (4 * MAT + GATES) + 4 * MAT));
        ek = g->ek;   // the same for every value head
        eq = g->eq;
        const uint4 *in = kq + (((long)b * a.Hk + hk) * a.N + n) * 2 * Lds::kq;
#pragma unroll
        for (int i = 0; i < 2 * Lds::kq / 256; ++i) ks[i * 256 + tid] = in[i * 256 + tid];
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
            for (int it = tid; it < room * a.Dv; it += 256) IO<DT>::st(dvo + ((tok0 + it / a.Dv) * a.H + h) * a.Dv, it % a.Dv, 0.f);
            if (tid < room) d.dg[(tok0 + tid) * a.H + h] = d.dbeta[(tok0 + tid) * a.H + h] = 0.f;
            continue;
        }
        if (w == 0) gd[lane] = decay_sum(lane < nt ? a.g[(tok0 + lane) * a.H + h] : 0.f, lane < nt, lane);
        if (tid < GATES) ((uint4 *)gt)[tid] = rec[(ch + 1) * (4 * MAT + GATES) - GATES + tid];
        // scales over all columns
        int eu = -126, eS = -126, ey = -126, eE = -126, eo = -126;
        for (int i = 0; i < (a.Dv + 15) / 16; ++i) {
            const int2 f = exps[ch * kDeltaTiles + i];
            const int4 g = d.exps[ch * kDeltaTiles + i];
            eu = max(eu, f.x); eS = max(eS, f.y);
            ey = max(ey, g.x); eE = max(eE, g.y); eo = max(eo, DT == F16 ? 0 : g.z);   // fp16 goes in as it is
        }
        const float su = pow2(-eu), sS = pow2(-eS), sy = pow2(-ey), sE = pow2(-eE), sd = pow2(-eo);
        __syncthreads();
        const float *ep = es + ch * DC * dvp, *zp = d.zs + ch * DC * dvp;
        const float *Sp = states + ch * 32 * KS * dvp, *Ep = d.dends + ch * 32 * KS * dvp;
        // row tile w of D and E; dv and dbeta of its tokens
        {
            dl_f4 ad[4], ae[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) ad[j] = ae[j] = dl_f4{0.f, 0.f, 0.f, 0.f};
            const int row = 16 * w + c16;
            const float be = gt->beta[row];
            float dot = 0.f;
            uint32_t md = 0, me = 0;
            for (int c = 8 * g4; c < ((a.Dv + 31) & ~31); c += 32) {
                const bool on = c < a.Dv;
                float z[8], e[8], y[8];
                ld8<F32>(zp + (long)row * dvp + c, on, z);
                ld8<F32>(ep + (long)row * dvp + c, on, e);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    dot += z[i] * e[i];
                    y[i] = row < nt ? be * z[i] : 0.f;
                }
                if (on && row < room) {
                    T *p = dvo + ((tok0 + row) * a.H + h) * a.Dv + c;
                    if constexpr (DT == F32) {
                        *(float4 *)p = make_float4(y[0], y[1], y[2], y[3]);
                        *(float4 *)(p + 4) = make_float4(y[4], y[5], y[6], y[7]);
                    } else {
                        *(uint4 *)p = make_uint4(pack_16x2<DT>(y[0], y[1]), pack_16x2<DT>(y[2], y[3]),
                                                 pack_16x2<DT>(y[4], y[5]), pack_16x2<DT>(y[6], y[7]));
                    }
                }
                const Op<2> yo = split8<2>(y, sy);
                const Op<NT> oo = op_of<DT>(or_zero<DT>(ld8_raw<DT>(op + ((tok0 + min(row, nt - 1)) * a.H + h) * a.Dv + (on ? c : 0)), on && row < nt), sd);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j > w) break;
                    float u[8];
                    const int r = 16 * j + c16;
                    ld8<F32>(ep + (long)r * dvp + c, on, u);
                    const float bj = gt->beta[r];
#pragma unroll
                    for (int i = 0; i < 8; ++i) u[i] *= bj;
                    const Op<2> uo = split8<2>(u, su);
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
                    const float x = i >= col ? a.scale * __builtin_amdgcn_ldexpf(ad[j][r], eo + eu) * f : 0.f;
                    const float y = i > col ? -__builtin_amdgcn_ldexpf(ae[j][r], ey + eu) * f : 0.f;
                    D[i * AROW + col] = x;
                    E[i * AROW + col] = y;
                    md = umax(md, mag(x));
                    me = umax(me, mag(y));
                }
            }
            md = group_max<64>(md);
            me = group_max<64>(me);
            if (lane == 0) {
                big[w] = md;
                big[4 + w] = me;
            }
        }
        // products with the states
        dl_f4 dq[4][TT], kr[4][TT], kw[4][TT];
        float inner[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};   // short sums: <S, dS'> cancels
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int j = 0; j < TT; ++j) dq[t][j] = kr[t][j] = kw[t][j] = dl_f4{0.f, 0.f, 0.f, 0.f};
        for (int c = 8 * g4; c < ((a.Dv + 31) & ~31); c += 32) {
            const bool on = c < a.Dv;
            Op<2> so[TT], to[TT];
#pragma unroll
            for (int j = 0; j < TT; ++j) {
                const int dk = 16 * (w * TT + j) + c16;
                float x[8], y[8];
                ld8<F32>(Sp + (long)dk * dvp + c, on && dk < a.Dk, x);
                ld8<F32>(Ep + (long)dk * dvp + c, on && dk < a.Dk, y);
#pragma unroll
                for (int i = 0; i < 8; ++i) inner[i] += x[i] * y[i];
                so[j] = split8<2>(x, sS);
                to[j] = split8<2>(y, sE);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int row = 16 * t + c16;
                const float be = gt->beta[row];
                float y[8], u[8];
                ld8<F32>(zp + (long)row * dvp + c, on, y);
                ld8<F32>(ep + (long)row * dvp + c, on, u);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    y[i] *= be;
                    u[i] *= be;
                }
                const Op<2> yo = split8<2>(y, sy), uo = split8<2>(u, su);
                const Op<NT> oo = op_of<DT>(or_zero<DT>(ld8_raw<DT>(op + ((tok0 + min(row, nt - 1)) * a.H + h) * a.Dv + (on ? c : 0)), on && row < nt), sd);
#pragma unroll
                for (int j = 0; j < TT; ++j) {
                    dq[t][j] = mm(so[j], oo, dq[t][j]);
                    kr[t][j] = mm(so[j], yo, kr[t][j]);
                    kw[t][j] = mm(to[j], uo, kw[t][j]);
                }
            }
        }
        double in64 = 0.0;
#pragma unroll
        for (int i = 0; i < 8; ++i) in64 += inner[i];
        in64 *= gt->from0[DC - 1];
        float kx = 0.f;   // sum of k . t (u dS'^T)
        __syncthreads();  // D and E are there
        const int eD = scale_exp(umax(umax(big[0], big[1]), umax(big[2], big[3])));
        const int eF = scale_exp(umax(umax(big[4], big[5]), umax(big[6], big[7])));
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int row = 16 * t + c16;
            const float f = gt->from0[row], e = gt->toend[row];
            Op<2> dr[2], er[2], dc[2], ec[2];   // rows and columns `row` of D and E
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int o = 32 * s + 4 * g4;
                if (s <= t / 2) {
                    dr[s] = split8<2>(*(const dl_f4 *)(D + row * AROW + o), *(const dl_f4 *)(D + row * AROW + o + 16), pow2(-eD));
                    er[s] = split8<2>(*(const dl_f4 *)(E + row * AROW + o), *(const dl_f4 *)(E + row * AROW + o + 16), pow2(-eF));
                }
                if (s >= t / 2) {
                    float x[8], y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        x[i] = D[(o + (i & 3) + 16 * (i >> 2)) * AROW + row];
                        y[i] = E[(o + (i & 3) + 16 * (i >> 2)) * AROW + row];
                    }
                    dc[s] = split8<2>(x, pow2(-eD));
                    ec[s] = split8<2>(y, pow2(-eF));
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
                    // channels 16 ct + 4 g .. + 3 of token `row`
                    const int at = (kq_block<KS>(p, t, ct >> 1) * 64 + kq_place(c16, 2 * (ct & 1) + (g4 >> 1))) * 2 + (g4 & 1);
                    const uint2 x = ((const uint2 *)ks)[at], y = ((const uint2 *)qs)[at];
                    kv[0] += low_half(x.x); kv[1] += high_half(x.x); kv[2] += low_half(x.y); kv[3] += high_half(x.y);
                    qv[0] += low_half(y.x); qv[1] += high_half(y.x); qv[2] += low_half(y.y); qv[3] += high_half(y.y);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    kv[r] = __builtin_amdgcn_ldexpf(kv[r], ek);
                    qv[r] = __builtin_amdgcn_ldexpf(qv[r], eq);
                    dq[t][j][r] = __builtin_amdgcn_ldexpf(dq[t][j][r], eS + eo) * (f * a.scale);
                    kr[t][j][r] = __builtin_amdgcn_ldexpf(kr[t][j][r], eS + ey) * -f;
                    kw[t][j][r] = __builtin_amdgcn_ldexpf(kw[t][j][r], eE + eu) * e;
                    kx += kv[r] * kw[t][j][r];
                }
                dl_f4 p = {0.f, 0.f, 0.f, 0.f}, q = p, x = p, y = p;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const Op<NT> kc = lds_cols<NT, KS, false>(ks, ct, s, lane);
                    if (s <= t / 2) {
                        p = mm(kc, dr[s], p);
                        q = mm(kc, er[s], q);
                    }
                    if (s >= t / 2) {
                        x = mm(lds_cols<NT, KS, false>(qs, ct, s, lane), dc[s], x);
                        y = mm(kc, ec[s], y);
                    }
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    dq[t][j][r] += __builtin_amdgcn_ldexpf(p[r], ek + eD);
                    kr[t][j][r] += __builtin_amdgcn_ldexpf(q[r], ek + eF);
                    kw[t][j][r] += __builtin_amdgcn_ldexpf(x[r], eq + eD) + __builtin_amdgcn_ldexpf(y[r], ek + eF);
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
        in64 += kx;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) in64 += __shfl_xor(in64, m);
        if (lane == 0) rin[w] = in64;
        __syncthreads();
        if (w == 0) {
            // suffix sums in float64: many terms, of both signs
            double x = (double)red[lane] + red[DC + lane] + red[2 * DC + lane] + red[3 * DC + lane];
#pragma unroll
            for (int m = 1; m < 64; m *= 2) {
                const double y = __shfl_down(x, m);
                if (lane + m < 64) x += y;
            }
            x += (rin[0] + rin[1]) + (rin[2] + rin[3]);
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
    constexpr int lds = ScanLds<DT, KS, NW, 4>::total, lds2 = GradLds<DT, KS>::total;
    const DeltaSegments sg = w.seg;
    const long bh = (long)a.B * a.H;
    hipError_t e;
    if (sg.G > 1) {
        if ((e = lds_room(delta_bwd_scan_kernel<DT, KS, NW, true>, lds)) != hipSuccess) return e;
        delta_bwd_scan_kernel<DT, KS, NW, true><<<(unsigned)(bh * (sg.G - 1) * (col_tiles(a.Dv, NW) + col_tiles(a.Dk, NW))), 64 * NW, lds, st>>>(
            a, sg, w.back, w.kq, d);
        if ((e = launch_delta_join(a, sg, d.dS, true, st)) != hipSuccess) return e;
    }
    if ((e = lds_room(delta_bwd_scan_kernel<DT, KS, NW, false>, lds)) != hipSuccess) return e;
    delta_bwd_scan_kernel<DT, KS, NW, false><<<(unsigned)(bh * sg.G * col_tiles(a.Dv, NW)), 64 * NW, lds, st>>>(a, sg, w.back, w.kq, d);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if ((e = lds_room(delta_bwd_chunk_kernel<DT, KS>, lds2)) != hipSuccess) return e;
    delta_bwd_chunk_kernel<DT, KS><<<(unsigned)((long)a.B * a.Hk * a.N), 256, lds2, st>>>(a, w.back, w.kq, w.es, w.states, w.exps, d);
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
