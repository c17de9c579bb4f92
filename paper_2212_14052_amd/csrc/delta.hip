// The gated delta rule over whole sequences, chunk by chunk.
//
// Per (b, h), with the state S (Dk, Dv):  S <- exp(g_t) S;  e_t = v_t - S^T k_t;
// S <- S + k_t (beta_t e_t)^T;  o_t = scale S^T q_t.  With G the running sum of g
// inside a chunk of 64 tokens, S the state at its start, K, Q, V its rows and
//     A = strictly lower part of (K K^T)_ij exp(G_i - G_j),   P = lower part of (Q K^T)_ij exp(G_i - G_j)
// the chunk's errors e solve (I + A diag(beta)) e = R with R = V - diag(exp G) K S, so
//     e = R - X (beta R),  X = (I + A diag(beta))^-1 A  (strictly lower),  u = beta e,
//     o = scale (diag(exp G) Q S + P u),   S' = exp(G_63) S + K^T diag(exp(G_63 - G)) u.
// No decay is ever divided by, and differences of G are taken in float64.
//
// Two kernels.  delta_chunk_kernel forms X and P, independent for every chunk,
// and leaves them as operand fragments.  delta_scan_kernel goes through the
// chunks in order.  The columns of S, V and o do not meet, so each wave takes 16
// of them and needs nothing from another wave: the state stays in its result
// registers for the whole sequence, and each product's result is, as it lies
// in the registers, the right operand of the next.  The waves of a workgroup share
// the chunk's keys and queries in LDS, fetched one chunk ahead.
#include "delta_common.h"

namespace h3 {
namespace {

constexpr int AROW = DC + 4;   // floats a row of a 64 x 64 matrix in LDS

template <int DT, int KS>
__global__ __launch_bounds__(256) void delta_chunk_kernel(DeltaArgs a, uint4 *__restrict__ XF, uint4 *__restrict__ PF,
                                                          uint4 *__restrict__ XTF, uint4 *__restrict__ PTF,
                                                          ChunkGates *__restrict__ gates) {
    typedef typename IO<DT>::T T;
    constexpr int NT = pieces<DT>(), NM = mat_pieces<DT>(), NX = kFullPieces;
    __shared__ __attribute__((aligned(16))) uint16_t ks[NT * DC * lds_row<KS>()];
    __shared__ __attribute__((aligned(16))) float A[DC * AROW], P[DC * AROW];
    __shared__ double gd[DC];
    __shared__ float be[DC];
    const long ch = blockIdx.x;
    const int n = (int)(ch % a.N), h = (int)(ch / a.N % a.H), b = (int)(ch / a.N / a.H);
    const int nt = min(DC, tokens_of(a, b) - n * DC);   // tokens of this chunk
    if (nt <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g4 = lane >> 4, c16 = lane & 15;
    const long tok0 = (long)b * a.L + n * DC;
    const int hk = h / (a.H / a.Hk);
    if (w == 0) {
        const bool on = lane < nt;
        const double x = decay_sum(on ? a.g[(tok0 + lane) * a.H + h] : 0.f, on, lane);
        const float bt = on ? a.beta[(tok0 + lane) * a.H + h] : 0.f;
        gd[lane] = x;
        be[lane] = bt;
        gates[ch].from0[lane] = __builtin_amdgcn_exp2f((float)x);
        gates[ch].toend[lane] = __builtin_amdgcn_exp2f((float)(__shfl(x, 63) - x));
        gates[ch].beta[lane] = bt;
    }
    const T *kp = (const T *)a.k, *qp = (const T *)a.q;
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        const int it = i * 256 + tid, t = it / (4 * KS), c = 8 * (it % (4 * KS));
        const Op<NT> o = op_of<DT>(ld8_raw<DT>(kp + ((tok0 + t) * a.Hk + hk) * a.Dk + c, t < nt && c < a.Dk));
#pragma unroll
        for (int p = 0; p < NT; ++p) *(uint4 *)(ks + (p * DC + t) * lds_row<KS>() + c) = o.p[p];
    }
    Op<NT> qo[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int t = 16 * w + c16, c = 32 * s + 8 * g4;
        qo[s] = op_of<DT>(ld8_raw<DT>(qp + ((tok0 + t) * a.Hk + hk) * a.Dk + c, t < nt && c < a.Dk));
    }
    __syncthreads();
    // row tile w of A and P
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        dl_f4 ka = {0.f, 0.f, 0.f, 0.f}, pa = ka;
        if (j <= w) {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const Op<NT> kj = lds_rows<NT, KS>(ks, j, s, lane);
                ka = mm<NT, NT, input_products<DT>()>(lds_rows<NT, KS>(ks, w, s, lane), kj, ka);
                pa = mm<NT, NT, input_products<DT>()>(qo[s], kj, pa);
            }
        }
        const int col = 16 * j + c16;
        const double gj = gd[col];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * w + 4 * g4 + r;
            float f = 0.f;
            if (row >= col) f = __builtin_amdgcn_exp2f((float)(gd[row] - gj));
            A[row * AROW + col] = row > col ? ka[r] * f : 0.f;
            P[row * AROW + col] = row >= col ? pa[r] * f : 0.f;
        }
    }
    __syncthreads();
    // X in place of A, row by row: x_i = A_i - sum_m<i A_im beta_m x_m, a column a lane
    if (w == 0) {
        float bx[DC];
#pragma unroll
        for (int i = 0; i < DC; ++i) {
            float x[4] = {A[i * AROW + lane], 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < i; m += 4) {
                const float4 am = *(const float4 *)(A + i * AROW + m);
                x[0] -= am.x * bx[m];
                if (m + 1 < i) x[1] -= am.y * bx[m + 1];
                if (m + 2 < i) x[2] -= am.z * bx[m + 2];
                if (m + 3 < i) x[3] -= am.w * bx[m + 3];
            }
            const float xi = (x[0] + x[1]) + (x[2] + x[3]);
            A[i * AROW + lane] = xi;
            bx[i] = be[i] * xi;
        }
    }
    __syncthreads();
    const long at = ch * NM * MAT, xat = ch * NX * MAT;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int row = 16 * w + c16, c0 = 32 * s + 4 * g4;
        if (s <= w / 2) {
            const int f = lower_frag(w, s) * FRAG + lane;
            const float *ar = A + row * AROW + c0, *pr = P + row * AROW + c0;
            const Op<NX> x = split8<NX>(*(const dl_f4 *)ar, *(const dl_f4 *)(ar + 16));
            const Op<NM> p = split8<NM>(*(const dl_f4 *)pr, *(const dl_f4 *)(pr + 16));
#pragma unroll
            for (int i = 0; i < NX; ++i) XF[xat + i * MAT + f] = x.p[i];
#pragma unroll
            for (int i = 0; i < NM; ++i) PF[at + i * MAT + f] = p.p[i];
        }
        if (XTF && s >= w / 2) {   // the transposes, for the backward pass
            const int f = upper_frag(w, s) * FRAG + lane;
            float xt[8], pt[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int r = c0 + (j & 3) + 16 * (j >> 2);
                xt[j] = A[r * AROW + row];
                pt[j] = P[r * AROW + row];
            }
            const Op<NX> xo = split8<NX>(xt), po = split8<NX>(pt);
#pragma unroll
            for (int i = 0; i < NX; ++i) {
                XTF[xat + i * MAT + f] = xo.p[i];
                PTF[xat + i * MAT + f] = po.p[i];
            }
        }
    }
}

// NW waves of 16 columns.  es, states: the chunks' errors (64, Dv) and first
// states (Dk, Dv), for the backward pass, or null.
template <int DT, int KS, int NW>
__global__ __launch_bounds__(64 * NW, 1) void delta_scan_kernel(DeltaArgs a, const uint4 *__restrict__ XF,
                                                               const uint4 *__restrict__ PF,
                                                               const ChunkGates *__restrict__ gates,
                                                               typename IO<DT>::T *__restrict__ o, float *S_final,
                                                               float *__restrict__ es, float *__restrict__ states) {
    typedef typename IO<DT>::T T;
    constexpr int NT = pieces<DT>(), NX = kFullPieces, NM = mat_pieces<DT>(), NO = DT == F32 ? 3 : 2;
    typedef ScanLds<DT, KS, NW, kFullPieces + mat_pieces<DT>()> Lds;
    // what a thread brings in: groups of eight channels of keys and of queries, 16-byte
    // words of X and P, groups of eight values, words of the gates
    constexpr int NTH = 64 * NW, ITEMS = 4 * KS / NW, WORDS = (NX + NM) * MAT, MATS = (WORDS + NTH - 1) / NTH, VALS = 2, GATES = (3 * DC + NTH - 1) / NTH;
    static_assert(4 * KS % NW == 0 && DC * 2 * NW == VALS * NTH, "whole shares");
    extern __shared__ __attribute__((aligned(16))) char lds[];
    uint16_t *ks = (uint16_t *)(lds + Lds::k), *qs = (uint16_t *)(lds + Lds::q);
    uint4 *ms = (uint4 *)(lds + Lds::mats);
    T *vs = (T *)(lds + Lds::v);
    ChunkGates *gt = (ChunkGates *)(lds + Lds::gates);
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g4 = lane >> 4, c16 = lane & 15;
    const int tiles = (a.Dv + 16 * NW - 1) / (16 * NW);
    const long bh = blockIdx.x / tiles;
    const int h = (int)(bh % a.H), b = (int)(bh / a.H), hk = h / (a.H / a.Hk);
    const int c0 = ((int)(blockIdx.x % tiles) * NW + w) * 16;
    const bool here = c0 < a.Dv;            // a wave without columns only helps to fetch
    const int col = c0 + c16;
    const bool on = col < a.Dv, on4 = c0 + 4 * g4 < a.Dv;
    const int len = tokens_of(a, b), nb = (len + DC - 1) / DC;
    const T *kp = (const T *)a.k, *qp = (const T *)a.q, *vp = (const T *)a.v;

    Raw8<DT> pk[ITEMS], pq[ITEMS], pv[VALS];
    uint4 pm[MATS];
    float pg[GATES];
    const int cb = c0 - 16 * w;   // the workgroup's first column
    auto fetch = [&](int n) {
        const long tok0 = (long)b * a.L + n * DC;
        const int nt = len - n * DC;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int it = i * 64 * NW + tid, t = it / (4 * KS), c = 8 * (it % (4 * KS));
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
        const uint4 *xp = XF + ch * NX * MAT, *pp = PF + ch * NM * MAT;
#pragma unroll
        for (int i = 0; i < MATS; ++i) {
            const int it = i * NTH + tid;
            if (it < WORDS) pm[i] = it < NX * MAT ? xp[it] : pp[it - NX * MAT];
        }
        const float *gp = (const float *)(gates + ch);
#pragma unroll
        for (int i = 0; i < GATES; ++i)
            if (i * NTH + tid < 3 * DC) pg[i] = gp[i * NTH + tid];
    };

    dl_f4 S[2 * KS];
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r;
            S[t][r] = a.S0 && on && dk < a.Dk ? a.S0[(bh * a.Dk + dk) * a.Dv + col] : 0.f;
        }
    if (nb > 0) fetch(0);
    for (int n = 0; n < nb; ++n) {
        const int nt = min(DC, len - n * DC);
        const long ch = bh * a.N + n, tok0 = (long)b * a.L + n * DC;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            const int it = i * 64 * NW + tid, t = it / (4 * KS), c = 8 * (it % (4 * KS));
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
        for (int i = 0; i < MATS; ++i)
            if (i * NTH + tid < WORDS) ms[i * NTH + tid] = pm[i];
#pragma unroll
        for (int i = 0; i < GATES; ++i)
            if (i * NTH + tid < 3 * DC) ((float *)gt)[i * NTH + tid] = pg[i];
        __syncthreads();
        if (n + 1 < nb) fetch(n + 1);
        if (!here) continue;
        if (states && on) {
#pragma unroll
            for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r;
                    if (dk < a.Dk) states[(ch * a.Dk + dk) * a.Dv + col] = S[t][r];
                }
        }
        // R = V - exp(G) K S
        Op<3> so[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) so[s] = split8<3>(S[2 * s], S[2 * s + 1]);
        dl_f4 R[4], u[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) R[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int t = 0; t < 4; ++t) R[t] = mm(lds_rows<NT, KS>(ks, t, s, lane), so[s], R[t]);
        dl_f4 be[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const dl_f4 f = *(const dl_f4 *)(gt->from0 + 16 * t + 4 * g4);
            be[t] = *(const dl_f4 *)(gt->beta + 16 * t + 4 * g4);
            const dl_f4 v = lds_column4<DT>(vs, Lds::vrow, 16 * t, 16 * w, lane);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                R[t][r] = v[r] - f[r] * R[t][r];
                u[t][r] = be[t][r] * R[t][r];
            }
        }
        // e = R - X (beta R), u = beta e
        {
            Op<NX> br[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) br[s] = split8<NX>(u[2 * s], u[2 * s + 1]);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                dl_f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s <= t / 2; ++s) x = mm(ld_frag<NX>(ms, lower_frag(t, s), lane), br[s], x);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    R[t][r] -= x[r];
                    u[t][r] = be[t][r] * R[t][r];
                }
            }
        }
        if (es && on) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) es[(ch * DC + 16 * t + 4 * g4 + r) * a.Dv + col] = R[t][r];
        }
        // o, transposed: rows are columns of S, so that a lane holds four consecutive values of one token
        {
            Op<NO> uo[2], sh[KS];
#pragma unroll
            for (int s = 0; s < 2; ++s) uo[s] = split8<NO>(u[2 * s], u[2 * s + 1]);
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int p = 0; p < NO; ++p) sh[s].p[p] = so[s].p[p];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                dl_f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < KS; ++s) x = mm(sh[s], lds_rows<NT, KS>(qs, t, s, lane), x);
                const float f = gt->from0[16 * t + c16];
#pragma unroll
                for (int r = 0; r < 4; ++r) x[r] *= f;
#pragma unroll
                for (int s = 0; s <= t / 2; ++s) x = mm(uo[s], ld_frag<NM>(ms + NX * MAT, lower_frag(t, s), lane), x);
                const int tt = 16 * t + c16;
                if (on4 && n * DC + tt < a.L) {
                    const bool real = tt < nt;
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[r] = real ? x[r] * a.scale : 0.f;
                    T *op = o + ((tok0 + tt) * a.H + h) * a.Dv + c0 + 4 * g4;
                    if constexpr (DT == F32) *(float4 *)op = make_float4(x[0], x[1], x[2], x[3]);
                    else *(uint2 *)op = make_uint2(pack_16x2<DT>(x[0], x[1]), pack_16x2<DT>(x[2], x[3]));
                }
            }
        }
        // S <- exp(G_63) S + K^T (exp(G_63 - G) u)
        {
            Op<3> wo[2];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const dl_f4 f = *(const dl_f4 *)(gt->toend + 16 * t + 4 * g4);
#pragma unroll
                for (int r = 0; r < 4; ++r) u[t][r] *= f[r];
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) wo[s] = split8<3>(u[2 * s], u[2 * s + 1]);
            const float f = gt->from0[DC - 1];
#pragma unroll
            for (int t = 0; t < 2 * KS; ++t) {
#pragma unroll
                for (int r = 0; r < 4; ++r) S[t][r] *= f;
#pragma unroll
                for (int s = 0; s < 2; ++s) S[t] = mm(lds_cols<NT, KS>(ks, t, s, lane), wo[s], S[t]);
            }
        }
    }
    if (!here) return;
    // tokens of chunks behind the end
    if (on4)
        for (int t = nb * DC + c16; t < a.L; t += 16) {
            T *op = o + (((long)b * a.L + t) * a.H + h) * a.Dv + c0 + 4 * g4;
            if constexpr (DT == F32) *(float4 *)op = make_float4(0.f, 0.f, 0.f, 0.f);
            else *(uint2 *)op = make_uint2(0u, 0u);
        }
    if (on && S_final) {
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r;
                if (dk < a.Dk) S_final[(bh * a.Dk + dk) * a.Dv + col] = S[t][r];
            }
    }
}

template <int DT, int KS>
hipError_t fwd_of(const DeltaArgs &a, const DeltaBuffers &w, void *o, float *S_final, hipStream_t st) {
    typedef typename IO<DT>::T T;
    constexpr int NW = 4;
    const long bh = (long)a.B * a.H;
    delta_chunk_kernel<DT, KS><<<(unsigned)(bh * a.N), 256, 0, st>>>(a, w.X, w.P, w.XT, w.PT, w.gates);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    constexpr int lds = ScanLds<DT, KS, NW, kFullPieces + mat_pieces<DT>()>::total;
    const int tiles = (a.Dv + 16 * NW - 1) / (16 * NW);
    if (lds > 65536)
        (void)hipFuncSetAttribute((const void *)delta_scan_kernel<DT, KS, NW>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    delta_scan_kernel<DT, KS, NW><<<(unsigned)(bh * tiles), 64 * NW, lds, st>>>(a, w.X, w.P, w.gates, (T *)o, S_final, w.es,
                                                                               w.states);
    return hipGetLastError();
}

template <int DT> hipError_t fwd_by(const DeltaArgs &a, const DeltaBuffers &w, void *o, float *S_final, hipStream_t st) {
    switch ((a.Dk + 31) / 32) {
        case 1: return fwd_of<DT, 1>(a, w, o, S_final, st);
        case 2: return fwd_of<DT, 2>(a, w, o, S_final, st);
        case 3: return fwd_of<DT, 3>(a, w, o, S_final, st);
        default: return fwd_of<DT, 4>(a, w, o, S_final, st);
    }
}

}  // namespace

hipError_t launch_delta_rule(const DeltaArgs &a, int dtype, const DeltaBuffers &w, void *o, float *S_final, hipStream_t s) {
    if (dtype == F32) return fwd_by<F32>(a, w, o, S_final, s);
    if (dtype == F16) return fwd_by<F16>(a, w, o, S_final, s);
    return fwd_by<BF16>(a, w, o, S_final, s);
}

}  // namespace h3
