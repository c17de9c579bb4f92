// The gated delta rule over whole sequences, chunk by chunk.
//
// Per (b, h), with the state S (Dk, Dv):  S <- exp(g_t) S;  e_t = v_t - S^T k_t;
// S <- S + k_t (beta_t e_t)^T;  o_t = scale S^T q_t.  With G the running sum of g
// inside a chunk of 64 tokens, S the state at its start, K, Q, V its rows and
//     A = strictly lower part of (K K^T)_ij exp(G_i - G_j),   P = lower part of (Q K^T)_ij exp(G_i - G_j)
// the chunk's errors e solve (I + A diag(beta)) e = R with R = V - diag(exp G) K S, so
//     e = R - X diag(beta) R,  X = (I + A diag(beta))^-1 A  (strictly lower),  u = beta e,
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
//
// At 8 sequences of 2048 tokens, 6 heads of 128 x 128, fp16: chunks 33 us (141 MB through
// memory, 4.2 TB/s), scan 115: 32 chunks after one another at 3.6 us, whose 132 matrix instructions of a
// wave would take 0.9.  What is left is the chain inside a chunk: K S, then R, its largest values,
// X R, the errors' and their decayed ones' largest values, P u and the new state, each waiting for the one before, and
// the vector instructions between them.
#include <math.h>

#include "delta_common.h"

namespace h3 {
namespace {

constexpr int AROW = DC + 4, TROW = 20;   // floats a row of a 64 x 64, a 16 x 16 matrix in LDS

template <int DT, int KS>
__global__ __launch_bounds__(256) void delta_chunk_kernel(DeltaArgs a, uint4 *__restrict__ rec, uint4 *__restrict__ back,
                                                          uint4 *__restrict__ kq) {
    typedef typename IO<DT>::T T;
    constexpr int NT = pieces<DT>(), NX = 2;
    constexpr int KQ = kq_words<KS>(NT);
    // the keys, then A and P in their place; the inverses of the diagonal blocks
    __shared__ uint4 ks[KQ > 2 * DC * AROW / 4 ? KQ : 2 * DC * AROW / 4];
    float *A = (float *)ks, *P = A + DC * AROW;
    __shared__ __attribute__((aligned(16))) float inv[4][16 * TROW];
    __shared__ double gd[DC];
    __shared__ __attribute__((aligned(16))) float be[DC];
    __shared__ uint32_t red[2][4];
    const long ch = blockIdx.x;
    const int n = (int)(ch % a.N), h = (int)(ch / a.N % a.H), b = (int)(ch / a.N / a.H);
    const int nt = min(DC, tokens_of(a, b) - n * DC);   // tokens of this chunk
    if (nt <= 0) return;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g4 = lane >> 4, c16 = lane & 15;
    const long tok0 = (long)b * a.L + n * DC;
    const int hk = h / (a.H / a.Hk);
    uint4 *xf = rec + ch * (2 * NX * MAT + GATES), *pf = xf + NX * MAT;
    uint4 *xt = back + ch * (2 * NX * MAT + GATES), *pt = xt + NX * MAT;
    ChunkGates *gf = (ChunkGates *)(pf + NX * MAT), *gb = (ChunkGates *)(pt + NX * MAT);
    const T *kp = (const T *)a.k + (tok0 * a.Hk + hk) * a.Dk, *qp = (const T *)a.q + (tok0 * a.Hk + hk) * a.Dk;
    Raw8<DT> kr[KS], qr[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        const int it = i * 256 + tid, t = it / (4 * KS), c = 8 * (it % (4 * KS));
        kr[i] = ld8_raw<DT>(kp + (long)min(t, nt - 1) * a.Hk * a.Dk + (c < a.Dk ? c : 0));
        kr[i] = or_zero<DT>(kr[i], t < nt && c < a.Dk);
    }
#pragma unroll
    for (int s = 0; s < KS; ++s) {   // the left operand of row tile w
        const int t = 16 * w + c16, c = 32 * s + 8 * g4;
        qr[s] = ld8_raw<DT>(qp + (long)min(t, nt - 1) * a.Hk * a.Dk + (c < a.Dk ? c : 0));
        qr[s] = or_zero<DT>(qr[s], t < nt && c < a.Dk);
    }
    if (w == 0) {
        const bool on = lane < nt;
        const double x = decay_sum(on ? a.g[(tok0 + lane) * a.H + h] : 0.f, on, lane);
        const float bt = on ? a.beta[(tok0 + lane) * a.H + h] : 0.f;
        gd[lane] = x;
        be[lane] = bt;
        const float f = __builtin_amdgcn_exp2f((float)x), e = __builtin_amdgcn_exp2f((float)(__shfl(x, 63) - x));
        gf->from0[lane] = f;
        gf->toend[lane] = e;
        gf->beta[lane] = bt;
        if (back) {
            gb->from0[lane] = f;
            gb->toend[lane] = e;
            gb->beta[lane] = bt;
        }
    }
    // the largest of two magnitudes over the workgroup
    auto largest = [&](uint32_t x, uint32_t y) {
        x = group_max<64>(x);
        y = group_max<64>(y);
        __syncthreads();
        if (lane == 0) {
            red[0][w] = x;
            red[1][w] = y;
        }
        __syncthreads();
        return make_int2(scale_exp(umax(umax(red[0][0], red[0][1]), umax(red[0][2], red[0][3]))),
                         scale_exp(umax(umax(red[1][0], red[1][1]), umax(red[1][2], red[1][3]))));
    };
    int ek = 0, eq = 0;
    if constexpr (DT != F16) {
        uint32_t mk = 0, mq = 0;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            mk = umax(mk, raw_mag<DT>(kr[i]));
            mq = umax(mq, raw_mag<DT>(qr[i]));
        }
        const int2 e = largest(mk, mq);
        ek = max(e.x, kLeast);
        eq = max(e.y, kLeast);
    }
    // the first value head of a key head leaves its keys and queries for the scans
    uint4 *ki = h % (a.H / a.Hk) == 0 ? kq + (((long)b * a.Hk + hk) * a.N + n) * 2 * KQ : nullptr;
    Op<NT> qo[KS];
#pragma unroll
    for (int i = 0; i < KS; ++i) {
        const int it = i * 256 + tid, t = it / (4 * KS), c = it % (4 * KS);
        const Op<NT> o = op_of<DT>(kr[i], pow2(-ek));
        qo[i] = op_of<DT>(qr[i], pow2(-eq));
#pragma unroll
        for (int p = 0; p < NT; ++p) {
            const int at = kq_block<KS>(p, t >> 4, c >> 2) * 64 + kq_place(t & 15, c & 3);
            ks[at] = o.p[p];
            if (ki) {
                ki[at] = o.p[p];
                ki[KQ + kq_block<KS>(p, w, i) * 64 + kq_place(c16, g4)] = qo[i].p[p];
            }
        }
    }
    __syncthreads();
    // row tile w of A and P
    dl_f4 ka[4], pa[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        ka[j] = pa[j] = dl_f4{0.f, 0.f, 0.f, 0.f};
        if (j <= w) {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const Op<NT> kj = lds_rows<NT, KS>(ks, j, s, lane);
                ka[j] = mm(lds_rows<NT, KS>(ks, w, s, lane), kj, ka[j]);
                pa[j] = mm(qo[s], kj, pa[j]);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int col = 16 * j + c16;
        const double gj = gd[col];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int row = 16 * w + 4 * g4 + r;
            float f = 0.f;
            if (row >= col) f = __builtin_amdgcn_exp2f((float)(gd[row] - gj));
            A[row * AROW + col] = row > col ? __builtin_amdgcn_ldexpf(ka[j][r], 2 * ek) * f : 0.f;
            P[row * AROW + col] = row >= col ? __builtin_amdgcn_ldexpf(pa[j][r], ek + eq) * f : 0.f;
        }
    }
    __syncthreads();
    // X = (I + A diag(beta))^-1 A by blocks of 16.  Wave w: the diagonal block w row
    // by row, x_i = A_i - sum_m<i A_im beta_m x_m, a column a lane (four times over), and
    // (I + A_ww diag(beta))^-1 = I - X_ww diag(beta).
    {
        float *D = A + 16 * w * (AROW + 1);
        float bx[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float x[4] = {D[i * AROW + c16], 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < i; m += 4) {
                const dl_f4 am = *(const dl_f4 *)(D + i * AROW + m);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (m + j < i) x[j] -= am[j] * bx[m + j];
            }
            const float xi = (x[0] + x[1]) + (x[2] + x[3]);
            bx[i] = be[16 * w + i] * xi;
            if (g4 == 0) {
                D[i * AROW + c16] = xi;
                inv[w][i * TROW + c16] = (i == c16 ? 1.f : 0.f) - xi * be[16 * w + c16];
            }
        }
    }
    __syncthreads();
    // Wave J: the blocks under diagonal block J, X_IJ = (I + A_II diag(beta))^-1 (A_IJ - sum_{J <= M < I}
    // A_IM diag(beta) X_MJ), float32 products whose results are, as they lie, the next right
    // operands (summand 4 g + s in step s).  A is overwritten when all are done.
    dl_f4 X[4], bX[4];
#pragma unroll
    for (int I = 0; I < 4; ++I) {
        if (I < w) continue;
        const float *AI = A + 16 * I * AROW + 16 * w + c16;
#pragma unroll
        for (int r = 0; r < 4; ++r) X[I][r] = AI[(4 * g4 + r) * AROW];
        if (I > w) {
            dl_f4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int M = 0; M < I; ++M) {
                if (M < w) continue;
                const dl_f4 am = *(const dl_f4 *)(A + (16 * I + c16) * AROW + 16 * M + 4 * g4);
#pragma unroll
                for (int s = 0; s < 4; ++s) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(am[s], bX[M][s], sum, 0, 0, 0);
            }
            const dl_f4 rhs = X[I] - sum, ti = *(const dl_f4 *)(inv[I] + c16 * TROW + 4 * g4);
            X[I] = dl_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 4; ++s) X[I] = __builtin_amdgcn_mfma_f32_16x16x4f32(ti[s], rhs[s], X[I], 0, 0, 0);
        }
        const dl_f4 bt = *(const dl_f4 *)(be + 16 * I + 4 * g4);
        bX[I] = bt * X[I];
    }
    __syncthreads();
#pragma unroll
    for (int I = 0; I < 4; ++I)
        if (I > w) {
#pragma unroll
            for (int r = 0; r < 4; ++r) A[(16 * I + 4 * g4 + r) * AROW + 16 * w + c16] = X[I][r];
        }
    __syncthreads();
    // the lower halves' fragments; the transposes for the backward pass
    float xv[2][8], pv[2][8];
    uint32_t mx = 0, mp = 0, mb = 0;
    const int row = 16 * w + c16;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int at = row * AROW + 32 * s + 4 * g4 + (j & 3) + 16 * (j >> 2);
            const float x = A[at];
            xv[s][j] = x * be[32 * s + 4 * g4 + (j & 3) + 16 * (j >> 2)];   // X diag(beta)
            pv[s][j] = P[at];
            mx = umax(mx, mag(xv[s][j]));
            mp = umax(mp, mag(pv[s][j]));
            mb = umax(mb, mag(x * be[row]));                                // diag(beta) X, whose transpose it is backward
        }
    const int2 em = largest(mx, mp);
    const int eb = back ? max(largest(mb, 0).x, kLeast) : 0, ex = max(em.x, kLeast), ep = max(em.y, kLeast);
    const float sx = pow2(-ex), sp = pow2(-ep), sb = pow2(-eb);
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        if (s <= w / 2) {
            const int f = lower_frag(w, s) * FRAG + lane;
            const Op<NX> x = split8<NX>(xv[s], sx);
            const Op<NX> p = split8<NX>(pv[s], sp);
#pragma unroll
            for (int i = 0; i < NX; ++i) {
                xf[i * MAT + f] = x.p[i];
                pf[i * MAT + f] = p.p[i];
            }
        }
        if (back && s >= w / 2) {
            const int f = upper_frag(w, s) * FRAG + lane;
            float x[8], p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int at = (32 * s + 4 * g4 + (j & 3) + 16 * (j >> 2)) * AROW + row;
                x[j] = A[at] * be[32 * s + 4 * g4 + (j & 3) + 16 * (j >> 2)];
                p[j] = P[at];
            }
            const Op<NX> xo = split8<NX>(x, sb), po = split8<NX>(p, sp);
#pragma unroll
            for (int i = 0; i < NX; ++i) {
                xt[i * MAT + f] = xo.p[i];
                pt[i * MAT + f] = po.p[i];
            }
        }
    }
    if (tid == 0) {
        gf->ek = ek;
        gf->eq = eq;
        gf->ex = ex;
        gf->ep = ep;
        if (back) {
            gb->ek = ek;
            gb->eq = eq;
            gb->ex = eb;
            gb->ep = ep;
        }
    }
}

// NW waves of 16 columns.  es, states, exps: for the backward pass, or null.
//
// A wave's vector instructions take longer than its matrix instructions here,
// so scales cost next to nothing of their own: they ride on the rounding to pieces, on the
// decays, or on a sum's multiplication.  The registers hold S 2^-E with an exponent
// E for each column, that of the last chunk's keys times errors, so that a chunk is
// added in the same instruction that decays them.
//
// What the backward pass reads is stored between the last products, and past the caches: a CU takes
// 1 KB of stores or copies every 16 cycles, and a wave waits where it asks for many at once, as for
// the state at a chunk's start, behind the next chunk's copies (both kernels for 4 x 2048
// tokens of 20 heads of 128 bf16: 212 us as it is, 169 with nothing kept; with P and u in one piece 204, then 234 at a
// chunk's start past the caches, and 244 through them).
//
// Sequences may be cut into segments (see DeltaSegments).  In mode MAP a workgroup
// does not produce outputs but its segment's map from state to state.
enum ScanMode { OUT, OUT_SAVE, MAP };   // outputs; outputs and what the backward pass reads; a segment's map

template <int DT, int KS, int NW, ScanMode MODE>
__global__ __launch_bounds__(64 * NW, MODE == MAP ? NW / 2 : NW / 4) void delta_scan_kernel(DeltaArgs a, DeltaSegments sg, const uint4 *__restrict__ rec,
                                                               const uint4 *__restrict__ kq,
                                                               typename IO<DT>::T *__restrict__ o, float *S_final,
                                                               float *__restrict__ es, float *__restrict__ states,
                                                               int2 *__restrict__ exps) {
    typedef typename IO<DT>::T T;
    constexpr int NT = pieces<DT>(), NX = 2;
    constexpr bool MAPS = MODE == MAP, SAVE = MODE == OUT_SAVE;
    typedef ChunkCopy<DT, KS, NW, MAPS> Copy;
    typedef typename Copy::Lds Lds;
    extern __shared__ uint4 lds[];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g4 = lane >> 4, c16 = lane & 15;
    const ScanPlace<NW, MAPS> at_(a, sg, blockIdx.x, w);
    const long bh = at_.bh;
    const int h = at_.h, b = at_.b, hk = h / (a.H / a.Hk), seg = at_.seg, cb = at_.cb, c0 = at_.c0;
    const bool here = c0 < at_.width;       // a wave without columns only helps to copy
    const int len = tokens_of(a, b), nb = (len + DC - 1) / DC;
    const int first = seg * sg.Ns, last = min(first + sg.Ns, nb);   // chunks from, and before
    if (MAPS && last >= nb) return;         // nothing starts behind it
    const Copy in{kq + ((long)b * a.Hk + hk) * a.N * 2 * Lds::kq, rec + bh * a.N * Lds::words,
                  (const T *)a.v + ((long)b * a.L * a.H + h) * a.Dv + (at_.unit ? 0 : cb), (long)a.H * a.Dv,
                  a.Dv - (at_.unit ? 0 : cb), len, (uint32_t)(uintptr_t)(dl_lds_void *)lds};

    dl_f4 S[2 * KS];
    int E = 0;
    const float *S0 = MAPS ? nullptr : sg.G > 1 ? sg.in + ((long)seg * a.B * a.H) * a.Dk * a.Dv : a.S0;
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r, col = c0 + c16;
            S[t][r] = S0 && col < a.Dv && dk < a.Dk ? S0[(bh * a.Dk + dk) * a.Dv + col] : 0.f;
            if (MAPS && at_.unit && dk < a.Dk && dk == col) S[t][r] = 1.f;
        }
    if (Lds::two && first < last) in.issue(first, w, lane);
    for (int n = first; n < last; ++n) {
        const int nt = min(DC, len - n * DC);
        const long ch = bh * a.N + n;
        const uint4 *at = in.arrive(lds, n, n + 1, n + 1 < last, w, lane);
        if (!here) continue;
        const uint4 *ks = at + Lds::k, *qs = at + Lds::q, *xs = at + Lds::rec, *ps = xs + NX * MAT;
        const T *vs = (const T *)(at + Lds::v);
        const ChunkGates *gt = (const ChunkGates *)(at + Lds::gates);
        dl_f4 *kept = (dl_f4 *)states + (ch * delta_col_tiles(a.Dv, 1) + c0 / 16) * 2 * KS * 64 + lane;   // where this state is left
        const int ek = __builtin_amdgcn_readfirstlane(gt->ek), eq = __builtin_amdgcn_readfirstlane(gt->eq),
                  ex = __builtin_amdgcn_readfirstlane(gt->ex), ep = __builtin_amdgcn_readfirstlane(gt->ep);
        // K S and, transposed (rows are columns of S, so that a lane will hold four
        // consecutive values of one token), Q S
        dl_f4 R[4], u[4], x[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) R[t] = x[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
        Op<NT> kf[2][4], qf[2][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) kf[0][t] = lds_rows<NT, KS>(ks, t, 0, lane);
#pragma unroll
        for (int t = 0; t < (MAPS ? 0 : 4); ++t) qf[0][t] = lds_rows<NT, KS>(qs, t, 0, lane);
        const int e0 = col_exp(S), em = max(e0, kLeast), eS = em + E;   // of the registers, of S
        const float sc = pow2(-em);
        Op<NX> xo[6];
        dl_f4 be[4], v[4], f0[4];
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (s + 1 < KS) {
#pragma unroll
                for (int t = 0; t < 4; ++t) kf[(s + 1) & 1][t] = lds_rows<NT, KS>(ks, t, s + 1, lane);
#pragma unroll
                for (int t = 0; t < (MAPS ? 0 : 4); ++t) qf[(s + 1) & 1][t] = lds_rows<NT, KS>(qs, t, s + 1, lane);
            } else {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    f0[t] = *(const dl_f4 *)(gt->from0 + 16 * t + 4 * g4);
                    be[t] = *(const dl_f4 *)(gt->beta + 16 * t + 4 * g4);
                    v[t] = lds_column4<DT>(vs, Lds::vrow, 16 * t, 16 * w, lane);
                    if (MAPS && at_.unit) v[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
                }
#pragma unroll
                for (int f = 0; f < 6; ++f) xo[f] = ld_frag<NX>(xs, f, lane);
            }
            in_order<NW == 4>();
            const Op<2> so = split8<2>(S[2 * s], S[2 * s + 1], sc);
            mm_each<NT, 2, 4>([&](int m) -> const Op<NT> & { return kf[s & 1][m]; }, [&](int) -> const Op<2> & { return so; },
                                   [&](int m) -> dl_f4 & { return R[m]; });
            if constexpr (!MAPS)
                mm_each<NX, NT, 4>([&](int) -> const Op<2> & { return so; }, [&](int m) -> const Op<NT> & { return qf[s & 1][m]; },
                                        [&](int m) -> dl_f4 & { return x[m]; });
            in_order<NW == 4>();
        }
        // R = V - exp(G) K S
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const float f = __builtin_amdgcn_ldexpf(f0[t][r], ek + eS);
                R[t][r] = v[t][r] - f * R[t][r];
            }
        // e = R - (X diag(beta)) R, u = beta e
        const int er = max(col_exp(R), kLeast);
        const float px = pow2_sum(er + ex), sr = pow2(-er);
        Op<NX> po[6];
#pragma unroll
        for (int f = 0; f < (MAPS ? 0 : 6); ++f) po[f] = ld_frag<NX>(ps, f, lane);
        in_order<NW == 4>();
        {
            Op<NX> br[2];
            dl_f4 y[4];
#pragma unroll
            for (int s = 0; s < 2; ++s) br[s] = split8<NX>(R[2 * s], R[2 * s + 1], sr);
#pragma unroll
            for (int t = 0; t < 4; ++t) y[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
            mm_each<NX, NX, 4>([&](int m) -> const Op<NX> & { return xo[lower_frag(m, 0)]; }, [&](int) -> const Op<NX> & { return br[0]; },
                                    [&](int m) -> dl_f4 & { return y[m]; });
            mm_each<NX, NX, 2>([&](int m) -> const Op<NX> & { return xo[lower_frag(2 + m, 1)]; }, [&](int) -> const Op<NX> & { return br[1]; },
                                    [&](int m) -> dl_f4 & { return y[2 + m]; });
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    R[t][r] -= px * y[t][r];
                    u[t][r] = be[t][r] * R[t][r];
                }
        }
        const int eu = max(col_exp(u), kLeast);
        if constexpr (SAVE) {
            dl_f4 *p = (dl_f4 *)es + (ch * delta_col_tiles(a.Dv, 1) + c0 / 16) * 4 * 64 + lane;
#pragma unroll
            for (int t = 0; t < 4; ++t) store_stream(p + t * 64, __builtin_bit_cast(uint4, R[t]));
            const int2 e = make_int2(tile_exp(eu), tile_exp(kept_exp(e0, E)));
            if (lane == 0) exps[ch * kDeltaTiles + c0 / 16] = e;
        }
        constexpr int TG = KS % 2 == 0 ? 4 : 2;   // state tiles at a time
        Op<NT> kc[2][TG][2];
        dl_f4 te[4];
        float fo[4];
#pragma unroll
        for (int t = 0; t < TG; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) kc[0][t][s] = lds_cols<NT, KS>(ks, t, s, lane);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            te[t] = *(const dl_f4 *)(gt->toend + 16 * t + 4 * g4);
            fo[t] = gt->from0[16 * t + c16];
        }
        const float fl = gt->from0[DC - 1];
        in_order<NW == 4>();
        // o = scale (exp(G) Q S + P u)
        if constexpr (!MAPS) {
            const float su = pow2(-eu);
            float px[4], py[4];   // rows are columns of S and u here: their exponents come from those columns' lanes
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int e = __shfl(eS * 65536 + eu, 4 * g4 + r);   // |eu| < 2^15
                px[r] = __builtin_amdgcn_ldexpf(a.scale, eq + ((e + 32768) >> 16));
                py[r] = __builtin_amdgcn_ldexpf(a.scale, ep + (int)(int16_t)e);
            }
            T *oc = o + (((long)b * a.L + n * DC) * a.H + h) * a.Dv + c0;
            const int room = a.L - n * DC;
            Op<NX> uo[2];
            dl_f4 y[4];
#pragma unroll
            for (int s = 0; s < 2; ++s) uo[s] = split8<NX>(u[2 * s], u[2 * s + 1], su);
#pragma unroll
            for (int t = 0; t < 4; ++t) y[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
            mm_each<NX, NX, 4>([&](int) -> const Op<NX> & { return uo[0]; }, [&](int m) -> const Op<NX> & { return po[lower_frag(m, 0)]; },
                                    [&](int m) -> dl_f4 & { return y[m]; });
            mm_each<NX, NX, 2>([&](int) -> const Op<NX> & { return uo[1]; }, [&](int m) -> const Op<NX> & { return po[lower_frag(2 + m, 1)]; },
                                    [&](int m) -> dl_f4 & { return y[2 + m]; });
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) x[t][r] = x[t][r] * fo[t] * px[r] + y[t][r] * py[r];
            if (nt < DC) {   // the last chunk: places behind the end are 0
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) x[t][r] = 16 * t + c16 < nt ? x[t][r] : 0.f;
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (c0 + 4 * g4 < a.Dv && 16 * t + c16 < room) {
                    T *op = oc + (uint32_t)((16 * t + c16) * a.H * a.Dv + 4 * g4);
                    if constexpr (DT == F32) *(float4 *)op = make_float4(x[t][0], x[t][1], x[t][2], x[t][3]);
                    else *(uint2 *)op = make_uint2(pack_16x2<DT>(x[t][0], x[t][1]), pack_16x2<DT>(x[t][2], x[t][3]));
                }
        }
        // S <- exp(G_63) S + K^T w, w = exp(G_63 - G) u, in units of the keys' times w's scale (w's own: where the
        // chunk decays, its largest value is far below that of u); of 2^-60 of exp(G_63) S where w is smaller than that
#pragma unroll
        for (int t = 0; t < 4; ++t) te[t] *= u[t];
        const int En = max(ek + col_exp(te), max(eS - 60, E - 100) + floor_exp(fl));
        const float fs = __builtin_amdgcn_ldexpf(fl, E - En), sw = pow2(max(min(ek - En, 127), -126));
        const int Eo = E;
        E = En;
        Op<2> wo[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) wo[s] = split8<2>(te[2 * s], te[2 * s + 1], sw);
        dl_f4 y[2][TG];   // summed from zero: added to S step by step, each step would round it
        auto add = [&](int q) {
#pragma unroll
            for (int t = 0; t < TG; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[q * TG + t][r] = S[q * TG + t][r] * fs + y[q & 1][t][r];
        };
#pragma unroll
        for (int q = 0; q < 2 * KS / TG; ++q) {
            if (q + 1 < 2 * KS / TG) {
#pragma unroll
                for (int t = 0; t < TG; ++t)
#pragma unroll
                    for (int s = 0; s < 2; ++s) kc[(q + 1) & 1][t][s] = lds_cols<NT, KS>(ks, (q + 1) * TG + t, s, lane);
            }
            in_order<NW == 4>();
#pragma unroll
            for (int t = 0; t < TG; ++t)
                y[q & 1][t] = dl_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 2; ++s)
                mm_each<NT, 2, TG>([&](int m) -> const Op<NT> & { return kc[q & 1][m][s]; }, [&](int) -> const Op<2> & { return wo[s]; },
                                        [&](int m) -> dl_f4 & { return y[q & 1][m]; });
            if (q > 0) add(q - 1);
            if constexpr (SAVE) {
#pragma unroll
                for (int t = q * TG; t < q * TG + TG; ++t) {
                    dl_f4 y;
#pragma unroll
                    for (int r = 0; r < 4; ++r) y[r] = __builtin_amdgcn_ldexpf(S[t][r], Eo);
                    store_stream(kept + t * 64, __builtin_bit_cast(uint4, y));
                }
            }
            in_order<NW == 4>();
        }
        add(2 * KS / TG - 1);
    }
    if (!here) return;
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[t][r] = __builtin_amdgcn_ldexpf(S[t][r], E);
    if constexpr (MAPS) {
        store_map<KS>(a, sg, at_, S, lane);
        return;
    }
    const bool write = S_final && last == nb && (first < last || seg == 0);
    // tokens of this segment's chunks behind the end
    if (c0 + 4 * g4 < a.Dv)
        for (int t = max(first, nb) * DC + c16; t < min(a.L, (first + sg.Ns) * DC); t += 16) {
            T *op = o + (((long)b * a.L + t) * a.H + h) * a.Dv + c0 + 4 * g4;
            if constexpr (DT == F32) *(float4 *)op = make_float4(0.f, 0.f, 0.f, 0.f);
            else *(uint2 *)op = make_uint2(0u, 0u);
        }
    const int col = c0 + c16;
    if (write && col < a.Dv) {
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r;
                if (dk < a.Dk) S_final[(bh * a.Dk + dk) * a.Dv + col] = S[t][r];
            }
    }
}

// The state in front of every segment from the segments' maps, in order (or the
// gradient of the state behind each, in reverse): S <- F S + D.  A workgroup takes 16
// columns, its four waves share the rows: each holds its part of the next map while
// the states go round through LDS.  Bound by latency: 11 steps of 20 heads of 128 x 128 take 51 us,
// a load, a product and two barriers each, against 276 for the scan that they let run at once.
template <int KS>
__global__ __launch_bounds__(256, 1) void delta_join_kernel(DeltaArgs a, DeltaSegments sg, const float *__restrict__ S0, bool back) {
    constexpr int TW = (KS + 1) / 2;   // row tiles a wave
    __shared__ dl_f4 st[2 * KS][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, g4 = lane >> 4, c16 = lane & 15;
    const int tiles = (a.Dv + 15) / 16, dvp = 16 * tiles, row = dvp + 32 * KS;
    const long bh = blockIdx.x / tiles, n = (long)a.B * a.H;
    const int col = (int)(blockIdx.x % tiles) * 16 + c16;
    const bool on = col < a.Dv;
    const int nb = (tokens_of(a, (int)(bh / a.H)) + DC - 1) / DC, segs = max((nb + sg.Ns - 1) / sg.Ns, 1);
    float fx[TW][KS][8];
    dl_f4 dx[TW];
    int ef = 0;
    auto fetch = [&](int seg) {
        const float *m = sg.maps + (bh * sg.G + seg) * 32 * KS * row;
#pragma unroll
        for (int j = 0; j < TW; ++j) {
            const int t = w * TW + j;
            if (t >= 2 * KS) break;
            const float *f = m + (long)(32 * (t >> 1) + 8 * (c16 >> 2) + 4 * (t & 1) + (c16 & 3)) * row + dvp + 8 * g4;
#pragma unroll
            for (int s = 0; s < KS; ++s) ld8<F32>(f + 32 * s, 32 * s + 8 * g4 < a.Dk, fx[j][s]);
#pragma unroll
            for (int r = 0; r < 4; ++r) dx[j][r] = m[(long)(32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r) * row + col];
        }
        ef = -126;
        for (int j = 0; j < (a.Dk + 15) / 16; ++j) ef = max(ef, sg.exps[(bh * sg.G + seg) * 8 + j]);
    };
    auto put = [&](int seg, int t, dl_f4 x) {
        st[t][lane] = x;
        float *to = sg.in + (seg * n + bh) * a.Dk * a.Dv + col;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r;
            if (on && dk < a.Dk) to[(long)dk * a.Dv] = x[r];
        }
    };
    if (segs > 1) fetch(back ? segs - 1 : 0);
    // the first state too: the last result may go where it came from
#pragma unroll
    for (int j = 0; j < TW; ++j) {
        const int t = w * TW + j;
        if (t >= 2 * KS) break;
        dl_f4 x;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r;
            x[r] = S0 && on && dk < a.Dk ? S0[(bh * a.Dk + dk) * a.Dv + col] : 0.f;
        }
        put(back ? segs - 1 : 0, t, x);
    }
    for (int i = 0; i + 1 < segs; ++i) {
        const int seg = back ? segs - 1 - i : i;
        __syncthreads();
        dl_f4 S[2 * KS], y[TW];
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t) S[t] = st[t][lane];
        const int es = col_exp(S), e = es + ef;
        Op<2> so[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) so[s] = split8<2>(S[2 * s], S[2 * s + 1], pow2(-es));
#pragma unroll
        for (int j = 0; j < TW; ++j) {
            y[j] = dl_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < KS; ++s) y[j] = mm(split8<2>(fx[j][s], pow2(-ef)), so[s], y[j]);
#pragma unroll
            for (int r = 0; r < 4; ++r) y[j][r] = __builtin_amdgcn_ldexpf(y[j][r], e) + dx[j][r];
        }
        if (i + 2 < segs) fetch(back ? seg - 1 : seg + 1);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < TW; ++j) {
            if (w * TW + j >= 2 * KS) break;
            put(back ? seg - 1 : seg + 1, w * TW + j, y[j]);
        }
    }
}

}  // namespace

// How a launch's scans are cut.  32768 tokens of 20 heads of 128 bf16 take 743 us in the 12
// segments of eight waves that this gives, 1920 uncut, 800 with four waves, 1355 in four segments, 817 in 24; 8 x 2048
// tokens of 6 heads fp16 take 139 uncut with four waves, 182 with eight, 176 in four segments.  Heads of
// 8 x 8 to 128 x 256, fp16 and float32, 1536 to 32768 tokens of 2 to 512 heads (52 shapes), against the best of 1, 2, 4, 8, 16 and 32 segments
// of four and of eight waves: at worst 1.17 times it, where a chunk of narrow heads takes less than the units
// assumed and more segments would do (4096 tokens of 4 heads of 8 x 8 float32: 62 us, 53 in 16 segments, 151 uncut).
// A workgroup of four waves takes about one time
// unit (4 us) a chunk on a CU of its own, one of eight 1.5; two workgroups of eight that form
// maps share a CU and take kMaps; joining takes about 1.3 units a segment.
DeltaCut delta_cut(int B, int H, int N, int Dk, int Dv, int dtype) {
    constexpr double kMaps = 1.3;
    const double bh = (double)B * H;
    DeltaCut best{1, 4};
    double least = 0;
    for (int NW = 4; NW <= (dtype == F32 ? 4 : 8); NW += 4)
        for (int G = 1; G <= 64 && (G == 1 || 4 * G <= N); ++G) {
            const double Ns = (N + G - 1) / G;
            double t = (NW == 4 ? 1.0 : 1.5) * ceil(bh * delta_col_tiles(Dv, NW) * G / 256) * Ns;
            if (G > 1) t += kMaps * ceil(bh * (delta_col_tiles(Dv, 8) + delta_col_tiles(Dk, 8)) * (G - 1) / 512) * Ns + 1.3 * G + 5;
            if ((NW == 4 && G == 1) || t < 0.95 * least) {
                best = DeltaCut{G, NW};
                least = t;
            }
        }
    return best;
}

namespace {

template <int DT, int KS, int NW, ScanMode MODE>
hipError_t scan_of(const DeltaArgs &a, const DeltaBuffers &w, void *o, float *S_final, hipStream_t st) {
    typedef typename IO<DT>::T T;
    constexpr int lds = ScanLds<DT, KS, NW>::total;
    const hipError_t e = lds_room(delta_scan_kernel<DT, KS, NW, MODE>, lds);
    if (e != hipSuccess) return e;
    delta_scan_kernel<DT, KS, NW, MODE><<<(unsigned)((long)a.B * a.H * w.seg.G * delta_col_tiles(a.Dv, NW)), 64 * NW, lds, st>>>(
        a, w.seg, w.rec, w.kq, (T *)o, S_final, w.es, w.states, w.exps);
    return hipGetLastError();
}

template <int DT, int KS>
hipError_t fwd_of(const DeltaArgs &a, const DeltaBuffers &w, void *o, float *S_final, hipStream_t st) {
    const long bh = (long)a.B * a.H;
    delta_chunk_kernel<DT, KS><<<(unsigned)(bh * a.N), 256, 0, st>>>(a, w.rec, w.back, w.kq);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const DeltaSegments sg = w.seg;
    if (sg.G > 1) {
        constexpr int NW = 8, lds = ScanLds<DT, KS, NW, true>::total;
        if ((e = lds_room(delta_scan_kernel<DT, KS, NW, MAP>, lds)) != hipSuccess) return e;
        delta_scan_kernel<DT, KS, NW, MAP><<<(unsigned)(bh * (sg.G - 1) * (delta_col_tiles(a.Dv, NW) + delta_col_tiles(a.Dk, NW))), 64 * NW, lds, st>>>(
            a, sg, w.rec, w.kq, nullptr, nullptr, nullptr, nullptr, nullptr);
        if ((e = launch_delta_join(a, sg, a.S0, false, st)) != hipSuccess) return e;
    }
    if constexpr (DT != F32)
        if (sg.NW == 8) return w.es ? scan_of<DT, KS, 8, OUT_SAVE>(a, w, o, S_final, st) : scan_of<DT, KS, 8, OUT>(a, w, o, S_final, st);
    return w.es ? scan_of<DT, KS, 4, OUT_SAVE>(a, w, o, S_final, st) : scan_of<DT, KS, 4, OUT>(a, w, o, S_final, st);
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

hipError_t launch_delta_join(const DeltaArgs &a, const DeltaSegments &sg, const float *S0, bool back, hipStream_t st) {
    const unsigned grid = (unsigned)((long)a.B * a.H * ((a.Dv + 15) / 16));
    switch ((a.Dk + 31) / 32) {
        case 1: delta_join_kernel<1><<<grid, 256, 0, st>>>(a, sg, S0, back); break;
        case 2: delta_join_kernel<2><<<grid, 256, 0, st>>>(a, sg, S0, back); break;
        case 3: delta_join_kernel<3><<<grid, 256, 0, st>>>(a, sg, S0, back); break;
        default: delta_join_kernel<4><<<grid, 256, 0, st>>>(a, sg, S0, back);
    }
    return hipGetLastError();
}

hipError_t launch_delta_rule(const DeltaArgs &a, int dtype, const DeltaBuffers &w, void *o, float *S_final, hipStream_t s) {
    if (dtype == F32) return fwd_by<F32>(a, w, o, S_final, s);
    if (dtype == F16) return fwd_by<F16>(a, w, o, S_final, s);
    return fwd_by<BF16>(a, w, o, S_final, s);
}

}  // namespace h3
