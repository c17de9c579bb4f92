// Backward pass of the gated delta rule, chunk by chunk.
//
// With a chunk's G, A, X, P, e, u, S of the forward pass (delta.hip), f_i = exp(G_i), t_i =
// exp(G_63 - G_i), do the output's gradient times the scale, and dS' the gradient of the state
// behind the chunk:
//     du = P^T do + t (K dS'),   z = du - (diag(beta) X)^T du,   y = beta z = dv,
//     dS = exp(G_63) dS' + Q^T (f do) - K^T (f y)
// is again a scan whose columns do not meet, in the order from the end
// (delta_bwd_scan_kernel, bound by the same chain inside a chunk as the forward pass's: 141 us for 4 x 2048
// tokens of 20 heads of 128 bf16; with dS' stored at a chunk's start it took 186 where it took 142); it leaves z and dS' of every chunk.  Then every chunk for itself
// (delta_bwd_chunk_kernel), with
//     D = lower part of (do u^T) exp(G_i - G_j),  E = -(strictly lower part of (y u^T) exp(G_i - G_j)):
//     dq = f (do S^T) + D K,   dk = reads + writes,  reads = E K - f (y S^T),
//     writes = D^T Q + E^T K + t (u dS'^T),   dbeta_i = z_i . e_i.
// The decay of token t lies in what passes from a token j < t to a token i >= t, M_ij = D_ij q_i . k_j + E_ij k_i . k_j, in
// what tokens i >= t read of S, in what tokens j < t leave to S', and in what S leaves to it:
//     dg_t = sum_{i >= t > j} M_ij + sum_{i >= t} (q_i . f_i (do S^T)_i - k_i . f_i (y S^T)_i)
//          + sum_{j < t} k_j . t_j (u dS'^T)_j + exp(G_63) <S, dS'>.
// Every term has token t's decay in it (the difference of the sums of q . dq and k . dk does not, and is rounding alone
// where gates are nearly closed: off by 1e-3 of dg at decays of exp(-5) to exp(-60), all of it where the last tokens only have gradients).
#include "delta_common.h"

namespace h3 {
namespace {

template <int DT, int KS, int NW, bool MAPS>
__global__ __launch_bounds__(64 * NW, NW / 4) void delta_bwd_scan_kernel(DeltaArgs a, DeltaSegments sg, const uint4 *__restrict__ rec,
                                                                   const uint4 *__restrict__ kq, DeltaGrads d) {
    typedef typename IO<DT>::T T;
    constexpr int NT = pieces<DT>(), NM = 2;
    typedef ChunkCopy<DT, KS, NW> Copy;
    typedef typename Copy::Lds Lds;
    extern __shared__ uint4 lds[];
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g4 = lane >> 4, c16 = lane & 15;
    const ScanPlace<NW, MAPS, true> at_(a, sg, blockIdx.x, w);
    const long bh = at_.bh;
    const int h = at_.h, b = at_.b, hk = h / (a.H / a.Hk), seg = at_.seg, cb = at_.cb, c0 = at_.c0;
    const bool here = c0 < at_.width;
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
            const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r, col = c0 + c16;
            S[t][r] = dS && col < a.Dv && dk < a.Dk ? dS[(bh * a.Dk + dk) * a.Dv + col] : 0.f;
            if (MAPS && at_.unit && dk < a.Dk && dk == col) S[t][r] = 1.f;
        }
    if (Lds::two && first < last) in.issue(last - 1, w, lane);
    for (int n = last - 1; n >= first; --n) {
        const long ch = bh * a.N + n;
        const uint4 *at = in.arrive(lds, n, n - 1, n > first, w, lane);
        if (!here) continue;
        const uint4 *ks = at + Lds::k, *qs = at + Lds::q, *xs = at + Lds::rec, *ps = xs + NM * MAT;   // (diag(beta) X)^T, P^T
        const T *vs = (const T *)(at + Lds::v);
        const ChunkGates *gt = (const ChunkGates *)(at + Lds::gates);
        const int nt = min(DC, len - n * DC);
        dl_f4 *kept = (dl_f4 *)d.dends + (ch * delta_col_tiles(a.Dv, 1) + c0 / 16) * 2 * KS * 64 + lane;   // where this state is left
        const int ek = __builtin_amdgcn_readfirstlane(gt->ek), eq = __builtin_amdgcn_readfirstlane(gt->eq),
                  ex = __builtin_amdgcn_readfirstlane(gt->ex), ep = __builtin_amdgcn_readfirstlane(gt->ep);
        // du = t (K dS') + P^T do
        dl_f4 u[4], dd[4], te[4], be[4];
        Op<NM> pf[6], xf[6];
        Op<NT> kf[2][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) kf[0][t] = lds_rows<NT, KS>(ks, t, 0, lane);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            u[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
            dd[t] = lds_column4<DT>(vs, Lds::vrow, 16 * t, 16 * w, lane);
            if (MAPS && at_.unit) dd[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
        }
        const int e0 = col_exp(S), em = max(e0, kLeast), eS = em + E;   // of the registers, of dS'
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
            in_order<NW == 4>();
            const Op<2> so = split8<2>(S[2 * s], S[2 * s + 1], sc);
            mm_each<NT, 2, 4>([&](int m) -> const Op<NT> & { return kf[s & 1][m]; }, [&](int) -> const Op<2> & { return so; },
                                   [&](int m) -> dl_f4 & { return u[m]; });
            in_order<NW == 4>();
        }
        if (nt < DC) {   // the last chunk: nothing comes from behind the end
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) dd[t][r] = 16 * t + 4 * g4 + r < nt ? dd[t][r] : 0.f;
        }
        const int ed = max(col_exp(dd), kLeast);
#pragma unroll
        for (int f = 0; f < 6; ++f) xf[f] = ld_frag<NM>(xs, f, lane);
        in_order<NW == 4>();
        dl_f4 y[4];
        {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) te[t][r] = __builtin_amdgcn_ldexpf(te[t][r], ek + eS);
            const int e = DT == F16 ? 0 : ed;
            const float py = __builtin_amdgcn_ldexpf(a.scale, ep + e);
            Op<NT> od[2];   // do as it came
            dl_f4 x[4];
#pragma unroll
            for (int s = 0; s < 2; ++s) od[s] = split8<NT>(dd[2 * s], dd[2 * s + 1], pow2(-e));
#pragma unroll
            for (int t = 0; t < 4; ++t) x[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
            mm_each<NM, NT, 4>([&](int m) -> const Op<NM> & { return pf[upper_frag(m, 1)]; }, [&](int) -> const Op<NT> & { return od[1]; },
                                    [&](int m) -> dl_f4 & { return x[m]; });
            mm_each<NM, NT, 2>([&](int m) -> const Op<NM> & { return pf[upper_frag(m, 0)]; }, [&](int) -> const Op<NT> & { return od[0]; },
                                    [&](int m) -> dl_f4 & { return x[m]; });
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) u[t][r] = te[t][r] * u[t][r] + py * x[t][r];
        }
        // z = du - (diag(beta) X)^T du; then y for the state
        const int eu = max(col_exp(u), kLeast);
        const float px = pow2_sum(eu + ex), su = pow2(-eu);
        Op<NT> kc[2][2][2], qc[2][2][2];   // two state tiles at a time
        dl_f4 f0[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) f0[t] = *(const dl_f4 *)(gt->from0 + 16 * t + 4 * g4);
        const float fl = gt->from0[DC - 1];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                kc[0][t][s] = lds_cols<NT, KS>(ks, t, s, lane);
                qc[0][t][s] = lds_cols<NT, KS>(qs, t, s, lane);
            }
        in_order<NW == 4>();
        {
            Op<NM> bu[2];
            dl_f4 x[4];
#pragma unroll
            for (int s = 0; s < 2; ++s) bu[s] = split8<NM>(u[2 * s], u[2 * s + 1], su);
#pragma unroll
            for (int t = 0; t < 4; ++t) x[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
            mm_each<NM, NM, 4>([&](int m) -> const Op<NM> & { return xf[upper_frag(m, 1)]; }, [&](int) -> const Op<NM> & { return bu[1]; },
                                    [&](int m) -> dl_f4 & { return x[m]; });
            mm_each<NM, NM, 2>([&](int m) -> const Op<NM> & { return xf[upper_frag(m, 0)]; }, [&](int) -> const Op<NM> & { return bu[0]; },
                                    [&](int m) -> dl_f4 & { return x[m]; });
            dl_f4 *p = (dl_f4 *)d.zs + (ch * delta_col_tiles(a.Dv, 1) + c0 / 16) * 4 * 64 + lane;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                dl_f4 z;
#pragma unroll
                for (int r = 0; r < 4; ++r) z[r] = u[t][r] - px * x[t][r];
                if (!MAPS) store_stream(p + t * 64, __builtin_bit_cast(uint4, z));
#pragma unroll
                for (int r = 0; r < 4; ++r) y[t][r] = be[t][r] * z[r];
            }
        }
        const int ez = max(col_exp(y), kLeast);
        if constexpr (!MAPS) {
            const int4 e = make_int4(tile_exp(ez), tile_exp(kept_exp(e0, E)), tile_exp(ed), 0);
            if (lane == 0) d.exps[ch * kDeltaTiles + c0 / 16] = e;
        }
        // dS <- exp(G_63) dS' + Q^T (f do) - K^T (f y), both in units of the larger product's scale; of
        // 2^-60 of exp(G_63) dS' where both are smaller than that
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            y[t] *= f0[t];
            dd[t] *= f0[t] * a.scale;
        }
        const int En = max(max(ek + col_exp(y), eq + col_exp(dd)), max(eS - 60, E - 100) + floor_exp(fl));
        const float fs = __builtin_amdgcn_ldexpf(fl, E - En), sy = -pow2(max(min(ek - En, 127), -126)), so_ = pow2(max(min(eq - En, 127), -126));
        const int Eo = E;
        E = En;
        Op<2> yo[2], qo[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            yo[s] = split8<2>(y[2 * s], y[2 * s + 1], sy);
            qo[s] = split8<2>(dd[2 * s], dd[2 * s + 1], so_);
        }
        dl_f4 x[2][2];
        auto add = [&](int q) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[2 * q + t][r] = S[2 * q + t][r] * fs + x[q & 1][t][r];
        };
#pragma unroll
        for (int q = 0; q < KS; ++q) {
            if (q + 1 < KS) {
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        kc[(q + 1) & 1][t][s] = lds_cols<NT, KS>(ks, 2 * q + 2 + t, s, lane);
                        qc[(q + 1) & 1][t][s] = lds_cols<NT, KS>(qs, 2 * q + 2 + t, s, lane);
                    }
            }
            in_order<NW == 4>();
#pragma unroll
            for (int t = 0; t < 2; ++t)
                x[q & 1][t] = dl_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                mm_each<NT, 2, 2>([&](int m) -> const Op<NT> & { return kc[q & 1][m][s]; }, [&](int) -> const Op<2> & { return yo[s]; },
                                       [&](int m) -> dl_f4 & { return x[q & 1][m]; });
                mm_each<NT, 2, 2>([&](int m) -> const Op<NT> & { return qc[q & 1][m][s]; }, [&](int) -> const Op<2> & { return qo[s]; },
                                       [&](int m) -> dl_f4 & { return x[q & 1][m]; });
            }
            if (q > 0) add(q - 1);
            if constexpr (!MAPS) {
#pragma unroll
                for (int t = q * 2; t < q * 2 + 2; ++t) {
                    dl_f4 y;
#pragma unroll
                    for (int r = 0; r < 4; ++r) y[r] = __builtin_amdgcn_ldexpf(S[t][r], Eo);
                    store_stream(kept + t * 64, __builtin_bit_cast(uint4, y));
                }
            }
            in_order<NW == 4>();
        }
        add(KS - 1);
    }
    if (!here) return;
#pragma unroll
    for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[t][r] = __builtin_amdgcn_ldexpf(S[t][r], E);
    if constexpr (MAPS) {
        store_map<KS>(a, sg, at_, S, lane);
    } else if (d.dS0 && seg == 0) {
        const int col = c0 + c16;
        if (col >= a.Dv) return;
#pragma unroll
        for (int t = 0; t < 2 * KS; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int dk = 32 * (t >> 1) + 8 * g4 + 4 * (t & 1) + r;
                if (dk < a.Dk) d.dS0[(bh * a.Dk + dk) * a.Dv + col] = S[t][r];
            }
    }
}

template <int KS> constexpr int grad_waves = KS > 2 ? 8 : 4;   // one for each of the key channels' tiles

// LDS of delta_bwd_chunk_kernel, in 16-byte words: first 32 columns at a time of the states, of y and u, and of do,
// then keys, queries, D and E in the same place.
template <int DT, int KS> struct GradLds {
    static constexpr int NT = pieces<DT>(), NW = grad_waves<KS>;
    static constexpr int S = 0, dS = S + 4 * KS * 64, y = dS + 4 * KS * 64, u = y + 8 * 64, o = u + 8 * 64, stage = o + NT * 4 * 64;
    static constexpr int kq = kq_words<KS>(NT), k = 0, q = kq, D = 2 * kq, E = D + kq_words<2>(2), after = E + kq_words<2>(2);
    static constexpr int rest = stage > after ? stage : after;
    static constexpr int gd = rest, gates = gd + DC / 2, red = gates + GATES, dot = red + 2 * NW * DC / 4, rin = dot + DC / 4, big = rin + NW / 2,
                         below = big + 2, across = below + 2 * DC / 4, total = (across + 2 * 4 * DC / 4) * 16;
    static_assert(total <= 160 * 1024, "LDS of a CU");
};

// A workgroup of NW waves takes a chunk of a key head and goes through the
// value heads that share it (ONE: there is one).  It brings in, 32 columns at a time, the
// states, z and e of a chunk as the scans left them, cuts them into pieces once for all
// waves, and reads operands whose summands are columns with transposing reads.  Every wave
// has one of the key channels' tiles for all tokens: results are transposed
// (rows are channels), so that a lane holds four consecutive channels of one token; and a row tile
// of D and E, of eight waves the first four of D, the others of E.
//
// 4 x 2048 tokens of 20 heads of 128 bf16: 272 us for 783 MB, 2.9 TB/s; 17 of them for the sums of dg.  The states alone are as many
// bytes as the chunk's inputs and gradients together, and a CU holds one workgroup, whose
// loads run beside its products but not beside its splits.  With four waves, D and E split by every
// wave for itself and keys and queries asked for only then it took 293; in the 128 registers a
// lane that two workgroups a CU would leave it spills.
template <int DT, int KS, bool ONE>
__global__ __launch_bounds__(64 * grad_waves<KS>, (KS > 2 || ONE ? 2 : 1)) void delta_bwd_chunk_kernel(
    DeltaArgs a, const uint4 *__restrict__ rec, const uint4 *__restrict__ kq, const float *__restrict__ es,
    const float *__restrict__ states, const int2 *__restrict__ exps, DeltaGrads d) {
    typedef typename IO<DT>::T T;
    typedef GradLds<DT, KS> Lds;
    constexpr int NT = pieces<DT>(), NW = Lds::NW, NS = (4 * KS + NW - 1) / NW, NI = 8 / NW;   // tiles of states, of e and z, a wave
    extern __shared__ uint4 lds[];
    double *gd = (double *)(lds + Lds::gd);
    ChunkGates *gt = (ChunkGates *)(lds + Lds::gates);
    float *red = (float *)(lds + Lds::red);        // the waves' sums of what tokens read of S; of what they leave to S'
    float *dots = (float *)(lds + Lds::dot);       // z . e over the later columns
    double *rin = (double *)(lds + Lds::rin);      // the waves' sums of <S, dS'>
    float *below = (float *)(lds + Lds::below);    // of D and of E: sums of M over j < t and i >= t in t's row tile
    float *across = (float *)(lds + Lds::across);  // of D and of E, a row tile: its rows' sums for every column left of it
    uint32_t *big = (uint32_t *)(lds + Lds::big);  // the waves' largest magnitudes of D and of E
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g4 = lane >> 4, c16 = lane & 15;
    const int wt = w & 3, half = w >> 2;   // token tile; which columns of 32, which of D and E
    // chunks from the front first: the scan wrote theirs last
    const int hk = (int)(blockIdx.x % a.Hk), b = (int)(blockIdx.x / a.Hk % a.B), n = (int)(blockIdx.x / a.Hk / a.B);
    const int per = ONE ? 1 : a.H / a.Hk, ct16 = delta_col_tiles(a.Dv, 1);
    const int nt = min(DC, tokens_of(a, b) - n * DC), room = min(DC, a.L - n * DC);   // tokens, and places, of this chunk
    const long tok0 = (long)b * a.L + n * DC;
    const T *op = (const T *)d.dout;
    T *dqp = (T *)d.dq, *dkp = (T *)d.dk, *dvo = (T *)d.dv;
    dl_f4 tq[ONE ? 1 : 4], tk[ONE ? 1 : 4];   // sums over the value heads
#pragma unroll
    for (int t = 0; t < (ONE ? 1 : 4); ++t) tq[t] = tk[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
    auto store = [&](int t, dl_f4 x, dl_f4 y) {   // dq and dk of this wave's channel tile, token tile t
        const int row = 16 * t + c16, dk = 16 * w + 4 * g4;
        if (row >= room || dk >= a.Dk) return;
        const bool real = row < nt;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            x[r] = real ? x[r] : 0.f;
            y[r] = real ? y[r] : 0.f;
        }
        const long at = ((tok0 + row) * a.Hk + hk) * a.Dk + dk;
        if constexpr (DT == F32) {
            *(float4 *)(dqp + at) = make_float4(x[0], x[1], x[2], x[3]);
            *(float4 *)(dkp + at) = make_float4(y[0], y[1], y[2], y[3]);
        } else {
            *(uint2 *)(dqp + at) = make_uint2(pack_16x2<DT>(x[0], x[1]), pack_16x2<DT>(x[2], x[3]));
            *(uint2 *)(dkp + at) = make_uint2(pack_16x2<DT>(y[0], y[1]), pack_16x2<DT>(y[2], y[3]));
        }
    };

    for (int hh = 0; hh < per; ++hh) {
        const int h = hk * per + hh;
        const long ch = ((long)b * a.H + h) * a.N + n;
        // (offsets into LDS are formed where they are used: kept over the loop they take more registers than there are)
        int lane = tid & 63;
        asm volatile("" : "+v"(lane));
        int g4 = lane >> 4, c16 = lane & 15;
        __syncthreads();   // the last head's matrices are read
        if (nt <= 0) {     // nothing behind a sequence's end has a gradient
            for (int it = tid; it < room * a.Dv; it += 64 * NW) IO<DT>::st(dvo + ((tok0 + it / a.Dv) * a.H + h) * a.Dv, it % a.Dv, 0.f);
            if (tid < room) d.dg[(tok0 + tid) * a.H + h] = d.dbeta[(tok0 + tid) * a.H + h] = 0.f;
            continue;
        }
        const dl_f4 *Sp = (const dl_f4 *)states + ch * ct16 * 2 * KS * 64, *Ep = (const dl_f4 *)d.dends + ch * ct16 * 2 * KS * 64;
        const dl_f4 *ep = (const dl_f4 *)es + ch * ct16 * 4 * 64, *zp = (const dl_f4 *)d.zs + ch * ct16 * 4 * 64;
        // 32 columns: states of NS (column tile, row tile)s a wave, e, z and do of token tile wt
        dl_f4 xs[NS], xe[NS], x_e[NI], x_z[NI], xo[NI];
        auto fetch = [&](int c2) {
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const int at = min(i * NW + w, 4 * KS - 1), ct = min(c2 + at / (2 * KS), ct16 - 1);
                xs[i] = Sp[(ct * 2 * KS + at % (2 * KS)) * 64 + lane];
                xe[i] = Ep[(ct * 2 * KS + at % (2 * KS)) * 64 + lane];
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int ct = min(c2 + half + i, ct16 - 1);
                x_e[i] = ep[(ct * 4 + wt) * 64 + lane];
                x_z[i] = zp[(ct * 4 + wt) * 64 + lane];
                const int c = 16 * (c2 + half + i) + 4 * g4;
                const T *p = op + ((tok0 + min(16 * wt + c16, nt - 1)) * a.H + h) * a.Dv + (c < a.Dv ? c : 0);
                if constexpr (DT == F32) {
                    xo[i] = *(const dl_f4 *)p;
                } else {
                    const uint2 v = *(const uint2 *)p;
                    xo[i] = dl_f4{__uint_as_float(v.x), __uint_as_float(v.y), 0.f, 0.f};
                }
            }
        };
        fetch(0);
        if (w == 0) gd[lane] = decay_sum(lane < nt ? a.g[(tok0 + lane) * a.H + h] : 0.f, lane < nt, lane);
        if (tid < GATES) ((uint4 *)gt)[tid] = rec[(ch + 1) * (4 * MAT + GATES) - GATES + tid];
        // scales over all columns
        int eu = -126, eS = -126, ey = -126, eE = -126, eo = -126;
        for (int i = 0; i < ct16; ++i) {
            const int2 f = exps[ch * kDeltaTiles + i];
            const int4 g = d.exps[ch * kDeltaTiles + i];
            eu = max(eu, f.x); eS = max(eS, f.y);
            ey = max(ey, g.x); eE = max(eE, g.y); eo = max(eo, DT == F16 ? 0 : g.z);   // fp16 goes in as it is
        }
        const float su = pow2(-eu), sS = pow2(-eS), sy = pow2(-ey), sE = pow2(-eE), sd = pow2(-eo);
        dl_f4 dq[4], kr[4], kw[4], ad[NI][4];   // ad: a row tile of D (of E), or of both
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            dq[t] = kr[t] = kw[t] = dl_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < NI; ++i) ad[i][t] = dl_f4{0.f, 0.f, 0.f, 0.f};
        }
        float inner[4] = {0.f, 0.f, 0.f, 0.f}, dot[4] = {0.f, 0.f, 0.f, 0.f};   // short sums: <S, dS'> cancels
        __syncthreads();
        const dl_f4 be = *(const dl_f4 *)(gt->beta + 16 * wt + 4 * g4);
        for (int c2 = 0; c2 < ct16; c2 += 2) {
            if (c2) __syncthreads();   // the columns before are read
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                const bool once = 4 * KS % NW == 0 || i * NW + w < 4 * KS;   // else the last tile again
                const int at = min(i * NW + w, 4 * KS - 1), ct = at / (2 * KS), t = at % (2 * KS);
                const bool on = 16 * (c2 + ct) + c16 < a.Dv;
                const int to = (kq_block<KS, 2>(0, ct, t >> 1) * 64 + kq_place(c16, g4)) * 2 + (t & 1);
                dl_f4 x, y;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x[r] = on ? xs[i][r] : 0.f;
                    y[r] = on ? xe[i][r] : 0.f;
                    inner[r] += once ? x[r] * y[r] : 0.f;
                }
                uint32_t p[2][2], q[2][2];
                split2<2>(x[0], sS, x[1], sS, p[0]); split2<2>(x[2], sS, x[3], sS, p[1]);
                split2<2>(y[0], sE, y[1], sE, q[0]); split2<2>(y[2], sE, y[3], sE, q[1]);
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    ((uint2 *)(lds + Lds::S))[to + m * 2 * KS * 128] = make_uint2(p[0][m], p[1][m]);
                    ((uint2 *)(lds + Lds::dS))[to + m * 2 * KS * 128] = make_uint2(q[0][m], q[1][m]);
                }
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const int c = 16 * (c2 + half + i) + c16;
                const bool on = c < a.Dv;
                const int to = (kq_block<2, 2>(0, half + i, wt >> 1) * 64 + kq_place(c16, 2 * (wt & 1) + (g4 >> 1))) * 2 + (g4 & 1);
                dl_f4 x, y;
                T *p = dvo + ((tok0 + 16 * wt + 4 * g4) * a.H + h) * a.Dv + c;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    dot[r] += on ? x_z[i][r] * x_e[i][r] : 0.f;
                    x[r] = on ? be[r] * x_z[i][r] : 0.f;
                    y[r] = on ? be[r] * x_e[i][r] : 0.f;
                    const int row = 16 * wt + 4 * g4 + r;
                    if (on && row < room) IO<DT>::st(p, (long)r * a.H * a.Dv, row < nt ? x[r] : 0.f);
                }
                uint32_t f[2][2], q[2][2];
                split2<2>(x[0], sy, x[1], sy, f[0]); split2<2>(x[2], sy, x[3], sy, f[1]);
                split2<2>(y[0], su, y[1], su, q[0]); split2<2>(y[2], su, y[3], su, q[1]);
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    ((uint2 *)(lds + Lds::y))[to + m * 4 * 128] = make_uint2(f[0][m], f[1][m]);
                    ((uint2 *)(lds + Lds::u))[to + m * 4 * 128] = make_uint2(q[0][m], q[1][m]);
                }
            }
#pragma unroll
            for (int i = 0; i < NI; ++i) {   // four columns of a token as the first half of an operand
                Raw8<DT> v{};
                v.a[0] = or_zero(__builtin_bit_cast(uint4, xo[i]), 16 * wt + c16 < nt && 16 * (c2 + half + i) + 4 * g4 < a.Dv);
                const Op<NT> oo = op_of<DT>(v, sd);
#pragma unroll
                for (int m = 0; m < NT; ++m)
                    ((uint2 *)(lds + Lds::o + (m * 4 + wt) * 64 + lane))[half + i] = make_uint2(__builtin_bit_cast(uint4, oo.p[m]).x, __builtin_bit_cast(uint4, oo.p[m]).y);
            }
            if (c2 + 2 < ct16) fetch(c2 + 2);
            __syncthreads();
            const int ct = min(w, 2 * KS - 1);   // a tile too many is not stored
            const Op<2> so = lds_cols<2, KS, false, 2>(lds + Lds::S, ct, 0, lane), to = lds_cols<2, KS, false, 2>(lds + Lds::dS, ct, 0, lane);
            Op<NT> ow;
            const Op<2> yw = lds_cols<2, 2, false, 2>(lds + Lds::y, wt, 0, lane);
#pragma unroll
            for (int m = 0; m < NT; ++m) ow.p[m] = lds[Lds::o + (m * 4 + wt) * 64 + lane];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const Op<2> yo = lds_cols<2, 2, false, 2>(lds + Lds::y, t, 0, lane), uo = lds_cols<2, 2, false, 2>(lds + Lds::u, t, 0, lane);
                Op<NT> oo;
#pragma unroll
                for (int m = 0; m < NT; ++m) oo.p[m] = lds[Lds::o + (m * 4 + t) * 64 + lane];
                dq[t] = mm(so, oo, dq[t]);
                mm_each<2, 2, 2>([&](int j) -> const Op<2> & { return j ? to : so; }, [&](int j) -> const Op<2> & { return j ? uo : yo; },
                                 [&](int j) -> dl_f4 & { return j ? kw[t] : kr[t]; });
                if (t <= wt) {
                    if (NW == 4 || half == 0) ad[0][t] = mm(ow, uo, ad[0][t]);
                    if (NW == 4 || half == 1) ad[NI - 1][t] = mm(yw, uo, ad[NI - 1][t]);
                }
            }
        }
        // dbeta of token tile wt: the sum over a row's 16 lanes
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
            for (int m = 1; m < 16; m *= 2) dot[r] += __shfl_xor(dot[r], m);
            if (half == 1 && c16 == 0) dots[16 * wt + 4 * g4 + r] = dot[r];
        }
        double in64 = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) in64 += inner[i];
        in64 *= gt->from0[DC - 1];
        // keys and queries are under way while D and E are formed
        constexpr int NQ = 2 * Lds::kq / (64 * NW);
        dl_f4 x_k[NQ];
        {
            const dl_f4 *in = (const dl_f4 *)kq + (((long)b * a.Hk + hk) * a.N + n) * 2 * Lds::kq;
#pragma unroll
            for (int i = 0; i < NQ; ++i) x_k[i] = in[i * 64 * NW + tid];
        }
        asm volatile("" : "+v"(lane));
        g4 = lane >> 4;
        c16 = lane & 15;
#pragma unroll
        for (int m = 0; m < NI; ++m) {
            const bool of_d = NW == 4 ? m == 0 : half == 0;
            const float f = of_d ? a.scale : -1.f;
            const int e = eu + (of_d ? eo : ey);
            uint32_t md = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int col = 16 * j + c16;
                const double gj = gd[col];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * wt + 4 * g4 + r;
                    const float x = __builtin_amdgcn_ldexpf(ad[m][j][r], e) * f * __builtin_amdgcn_exp2f((float)(gd[i] - gj));
                    ad[m][j][r] = i > col || (of_d && i == col) ? x : 0.f;
                    md = umax(md, mag(ad[m][j][r]));
                }
            }
            md = group_max<64>(md);
            if (lane == 0) big[4 * (NW == 4 ? m : half) + wt] = md;
        }
        __syncthreads();   // the columns are read: keys, queries, D and E take their place
#pragma unroll
        for (int i = 0; i < NQ; ++i) ((dl_f4 *)lds)[i * 64 * NW + tid] = x_k[i];
        if (half == 0 && c16 == 0)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * wt + 4 * g4 + r;
                if (row < room) d.dbeta[(tok0 + row) * a.H + h] = row < nt ? dot[r] + (NW == 8 ? dots[row] : 0.f) : 0.f;
            }
        const uint4 *ks = lds + Lds::k, *qs = lds + Lds::q, *Ds = lds + Lds::D, *Es = lds + Lds::E;
        const int ek = gt->ek, eq = gt->eq;
        const int eD = scale_exp(umax(umax(big[0], big[1]), umax(big[2], big[3])));
        const int eF = scale_exp(umax(umax(big[4], big[5]), umax(big[6], big[7])));
#pragma unroll
        for (int m = 0; m < NI; ++m) {
            const bool of_d = NW == 4 ? m == 0 : half == 0;
            const float f = pow2(-(of_d ? eD : eF));
            uint2 *to = (uint2 *)(lds + (of_d ? Lds::D : Lds::E)) + (kq_block<2>(0, 0, wt >> 1) * 64 + kq_place(c16, 2 * (wt & 1) + (g4 >> 1))) * 2 + (g4 & 1);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t x[2][2];
                split2<2>(ad[m][j][0], f, ad[m][j][1], f, x[0]);
                split2<2>(ad[m][j][2], f, ad[m][j][3], f, x[1]);
#pragma unroll
                for (int i = 0; i < 2; ++i) to[kq_block<2>(i, j, 0) * 128] = make_uint2(x[0][i], x[1][i]);
            }
        }
        __syncthreads();  // D and E are there
        // M's row tile wt, from D and E as they are in the registers
        {
            float T[4] = {0.f, 0.f, 0.f, 0.f}, A[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < NI; ++m) {
                const bool of_d = NW == 4 ? m == 0 : half == 0;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (j > wt) continue;
                    dl_f4 p = {0.f, 0.f, 0.f, 0.f}, y = p;
#pragma unroll
                    for (int s = 0; s < KS; ++s)
                        p = mm(lds_rows<NT, KS>(of_d ? qs : ks, wt, s, lane), lds_rows<NT, KS>(ks, j, s, lane), p);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        p[r] = ad[m][j][r] * __builtin_amdgcn_ldexpf(p[r], ek + (of_d ? eq : ek));
                        if (j == wt) p[r] = 4 * g4 + r > c16 ? p[r] : 0.f;
                    }
                    // rows t: the sums over rows i >= t of the tile
#pragma unroll
                    for (int s = 0; s < 4; ++s) y = __builtin_amdgcn_mfma_f32_16x16x4f32(4 * g4 + s >= c16 ? 1.f : 0.f, p[s], y, 0, 0, 0);
#pragma unroll
                    for (int r = 0; r < 4; ++r) T[r] += j < wt || c16 < 4 * g4 + r ? y[r] : 0.f;
                    A[j] += y[0];
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int m = 1; m < 16; m *= 2) T[r] += __shfl_xor(T[r], m);
            float *b = below + (NW == 4 ? 0 : half) * DC, *a = across + (NW == 4 ? 0 : half) * 4 * DC + wt * DC;
            if (c16 == 0) *(dl_f4 *)(b + 16 * wt + 4 * g4) = dl_f4{T[0], T[1], T[2], T[3]};
            if (g4 == 0)
#pragma unroll
                for (int j = 0; j < 3; ++j)
                    if (j < wt) a[16 * j + c16] = A[j];
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            __builtin_amdgcn_sched_barrier(0);   // a token tile's operands at a time: the registers
            const int row = 16 * t + c16;
            const float f = gt->from0[row], e = gt->toend[row];
            Op<2> dr[2], er[2], dc[2], ec[2];   // rows and columns `row` of D and E
            const int at = (kq_place(c16, g4 >> 1) * 2 + (g4 & 1)), at2 = kq_place(c16, 2 + (g4 >> 1)) * 2 + (g4 & 1);
            auto column = [&](const uint4 *M, int s) {
                Op<2> x;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const uint2 *p = (const uint2 *)(M + kq_block<2>(i, t, s) * 64), lo = p[at], hi = p[at2];
                    x.p[i] = make_uint4(lo.x, lo.y, hi.x, hi.y);
                }
                return x;
            };
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                if (s <= t / 2) {
                    dr[s] = lds_cols<2, 2, false>(Ds, t, s, lane);
                    er[s] = lds_cols<2, 2, false>(Es, t, s, lane);
                }
                if (s >= t / 2) {
                    dc[s] = column(Ds, s);
                    ec[s] = column(Es, s);
                }
            }
            float rs = 0.f, ws = 0.f;
            const int ct = w;   // this wave's channel tile
            if (ct < 2 * KS) {
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
                    dq[t][r] = __builtin_amdgcn_ldexpf(dq[t][r], eS + eo) * (f * a.scale);
                    kr[t][r] = __builtin_amdgcn_ldexpf(kr[t][r], eS + ey) * -f;
                    kw[t][r] = __builtin_amdgcn_ldexpf(kw[t][r], eE + eu) * e;
                    rs += qv[r] * dq[t][r] + kv[r] * kr[t][r];
                    ws += kv[r] * kw[t][r];
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
                    dq[t][r] += __builtin_amdgcn_ldexpf(p[r], ek + eD);
                    kr[t][r] += __builtin_amdgcn_ldexpf(q[r], ek + eF);
                    kw[t][r] += __builtin_amdgcn_ldexpf(x[r], eq + eD) + __builtin_amdgcn_ldexpf(y[r], ek + eF);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) kr[t][r] += kw[t][r];
                if constexpr (ONE) {
                    store(t, dq[t], kr[t]);
                } else {
                    tq[t] += dq[t];
                    tk[t] += kr[t];
                }
            }
            rs += __shfl_xor(rs, 16);
            ws += __shfl_xor(ws, 16);
            rs += __shfl_xor(rs, 32);
            ws += __shfl_xor(ws, 32);
            if (g4 == 0) {
                red[w * DC + row] = rs;
                red[(NW + w) * DC + row] = ws;
            }
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) in64 += __shfl_xor(in64, m);
        if (lane == 0) rin[w] = in64;
        __syncthreads();
        if (w == 0) {
            // Sums over the lanes up to this one, token t = lane: of reads from the last token on, of what the tokens
            // before t leave, and of the rows below each row tile over the columns before t.
            const int tile = lane >> 4, j = max(lane - 1, 0);   // column: the token before
            float x = 0.f, y = 0.f, left[3] = {0.f, 0.f, 0.f};
            double c = 0.0;
#pragma unroll
            for (int i = 0; i < NW; ++i) {
                x += red[i * DC + 63 - lane];
                y += red[(NW + i) * DC + j];
                c += rin[i];
            }
#pragma unroll
            for (int i = 0; i < NW / 4; ++i) {
                c += (double)below[i * DC + lane];
#pragma unroll
                for (int t = 0; t < 3; ++t)
#pragma unroll
                    for (int q = t + 1; q < 4; ++q) left[t] += j >> 4 <= t ? across[(4 * i + q) * DC + j] : 0.f;
            }
#pragma unroll
            for (int t = 0; t < 3; ++t) left[t] = lane_sums(lane > 0 ? left[t] : 0.f);
            c += __shfl(lane_sums(x), 63 - lane) + lane_sums(lane > 0 ? y : 0.f);
            c += tile == 0 ? left[0] : tile == 1 ? left[1] : tile == 2 ? left[2] : 0.f;
            if (lane < room) d.dg[(tok0 + lane) * a.H + h] = lane < nt ? (float)c : 0.f;
        }
    }
    if (ONE && nt > 0) return;
    const dl_f4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 4; ++t) store(t, ONE ? zero : tq[ONE ? 0 : t], ONE ? zero : tk[ONE ? 0 : t]);
}

template <int DT, int KS, int NW>
hipError_t scans_of(const DeltaArgs &a, const DeltaBuffers &w, const DeltaGrads &d, hipStream_t st) {
    constexpr int lds = ScanLds<DT, KS, NW>::total;
    const DeltaSegments sg = w.seg;
    const long bh = (long)a.B * a.H;
    hipError_t e;
    if (sg.G > 1) {
        if ((e = lds_room(delta_bwd_scan_kernel<DT, KS, NW, true>, lds)) != hipSuccess) return e;
        delta_bwd_scan_kernel<DT, KS, NW, true><<<(unsigned)(bh * (sg.G - 1) * (delta_col_tiles(a.Dv, NW) + delta_col_tiles(a.Dk, NW))), 64 * NW, lds, st>>>(
            a, sg, w.back, w.kq, d);
        if ((e = launch_delta_join(a, sg, d.dS, true, st)) != hipSuccess) return e;
    }
    if ((e = lds_room(delta_bwd_scan_kernel<DT, KS, NW, false>, lds)) != hipSuccess) return e;
    delta_bwd_scan_kernel<DT, KS, NW, false><<<(unsigned)(bh * sg.G * delta_col_tiles(a.Dv, NW)), 64 * NW, lds, st>>>(a, sg, w.back, w.kq, d);
    return hipGetLastError();
}

template <int DT, int KS> hipError_t bwd_of(const DeltaArgs &a, const DeltaBuffers &w, const DeltaGrads &d, hipStream_t st) {
    constexpr int lds2 = GradLds<DT, KS>::total;
    hipError_t e;
    if constexpr (DT != F32)
        e = w.seg.NW == 8 ? scans_of<DT, KS, 8>(a, w, d, st) : scans_of<DT, KS, 4>(a, w, d, st);
    else
        e = scans_of<DT, KS, 4>(a, w, d, st);
    if (e != hipSuccess) return e;
    const unsigned grid = (unsigned)((long)a.B * a.Hk * a.N);
    if (a.H == a.Hk) {
        if ((e = lds_room(delta_bwd_chunk_kernel<DT, KS, true>, lds2)) != hipSuccess) return e;
        delta_bwd_chunk_kernel<DT, KS, true><<<grid, 64 * grad_waves<KS>, lds2, st>>>(a, w.back, w.kq, w.es, w.states, w.exps, d);
    } else {
        if ((e = lds_room(delta_bwd_chunk_kernel<DT, KS, false>, lds2)) != hipSuccess) return e;
        delta_bwd_chunk_kernel<DT, KS, false><<<grid, 64 * grad_waves<KS>, lds2, st>>>(a, w.back, w.kq, w.es, w.states, w.exps, d);
    }
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
