// Layer norm over the last dimension of (rows, d), forward and backward.
//
//   mu = mean(x),  r = (mean((x - mu)^2) + eps)^-1/2,  y = (x - mu) r w + b
//   xh = (x - mu) r,  t = dy w:
//   dx = r (t - mean(t) - xh mean(t xh)),  dw = sum_rows dy xh,  db = sum_rows dy
//
// Both are bound by HBM: forward reads x and writes y, backward reads x and dy
// and writes dx.  A row stays in registers between its sums and its output, so
// it is read once; the variance is a second sum over the registers (of squared
// deviations, not of squares, which would cancel where a row sits far from
// zero).  A row is held by TPR threads, VEC elements (16 bytes where the width
// and the pointers allow it) at a time, NV times.  Workgroups walk over rows: the
// weight and bias, in float32 twice a 16-bit row's bytes each, stay in registers (read again
// for every row they were most of the traffic: forward 17.3 us instead of 8.7 at 16384 x 768 fp16), and the
// next row is under way while this one is summed.  The backward pass keeps the column
// sums of dw and db in registers, too; each
// workgroup writes one float32 partial row of each to the workspace and a
// second kernel sums those in a fixed order, so results do not depend on timing.
// Rows too wide for the registers are read again for each sum.  Outputs are streamed
// past the caches (8192 x 2560 bf16: 17.7 us with ordinary stores, 16.7 so).
//
// Forward at 8192 x 2560 bf16: 16.9 us, 4.97 TB/s, what a large copy reaches (4.99).
// At 16384 x 768 fp16: forward 8.4 us (6.0 TB/s: part of it stays in the last cache),
// backward 19.8, the second kernel 6.2 (3 MB by 48 workgroups, which is few).  At 4999 x 1031 float32: forward 11,
// backward 16.3, the second kernel 6.4; rows that do not start on 16 bytes are read 4 bytes at a time.
#include <type_traits>

#include "common.h"
#include "internal.h"

namespace h3 {
namespace {

// the sum of x over the wave's 64 lanes, in every lane
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int m = 1; m < 64; m *= 2) x += __shfl_xor(x, m);
    return x;
}

// sums of v[0..N) over the TPR threads of a row; lds: N floats per wave
template <int TPR, int N> __device__ __forceinline__ void row_sum(float (&v)[N], float *lds) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = wave_sum(v[j]);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        const int w = threadIdx.x / 64;
        __syncthreads();   // the sums before are read
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int j = 0; j < N; ++j) lds[j * W + w] = v[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < W; ++i) s += lds[j * W + i];
            v[j] = s;
        }
    }
}

// VEC elements as stored, and as float32
template <int DT, int VEC> struct Raw { typename IO<DT>::T v[VEC]; } ;
template <int DT, int VEC>
__device__ __forceinline__ Raw<DT, VEC> ld_raw(const typename IO<DT>::T *p) {
    Raw<DT, VEC> r;
    if constexpr (VEC == 1) {
        r.v[0] = *p;
    } else {
        static_assert(sizeof(r) == 16, "16-byte vectors");
        r = __builtin_bit_cast(Raw<DT, VEC>, *(const uint4 *)p);
    }
    return r;
}
template <int DT> __device__ __forceinline__ float to_f(typename IO<DT>::T t) { return IO<DT>::ld(&t, 0); }
template <int DT, int VEC>
__device__ __forceinline__ void st_vec(typename IO<DT>::T *p, const float (&f)[VEC]) {
    if constexpr (VEC == 1) {
        IO<DT>::st(p, 0, f[0]);
    } else if constexpr (DT == F32) {
        store_stream(p, __builtin_bit_cast(uint4, make_float4(f[0], f[1], f[2], f[3])));
    } else {
        store_stream(p, make_uint4(pack_16x2<DT>(f[0], f[1]), pack_16x2<DT>(f[2], f[3]), pack_16x2<DT>(f[4], f[5]),
                                   pack_16x2<DT>(f[6], f[7])));
    }
}
// VEC float32 parameters at p (any alignment of 4), or `other` where p is null
template <int VEC> __device__ __forceinline__ void ld_par(const float *p, int c, float other, float (&f)[VEC]) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) f[j] = p ? p[c + j] : other;
}

constexpr int threads_of(int TPR) { return TPR < 256 ? 256 : TPR; }

template <int DT, int VEC, int NV, int TPR>
__global__ __launch_bounds__(threads_of(TPR)) void layernorm_kernel(
    const typename IO<DT>::T *x, const float *__restrict__ w, const float *__restrict__ b, int rows, int d,
    float eps, typename IO<DT>::T *y, float *__restrict__ mean, float *__restrict__ rstd) {
    constexpr int RPB = threads_of(TPR) / TPR;   // rows at a time
    __shared__ float lds[TPR > 64 ? TPR / 64 : 1];
    const int t = threadIdx.x % TPR;
    const long step = (long)gridDim.x * RPB;
    long row = (long)blockIdx.x * RPB + threadIdx.x / TPR;
    if (row >= rows) return;   // whole waves; with TPR >= 256 the grid is at most the rows
    Raw<DT, VEC> v[NV], next[NV];
    float wf[NV][VEC], bf[NV][VEC];
    auto fetch = [&](long r) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * VEC;
            if (c < d) next[i] = ld_raw<DT, VEC>(x + r * d + c);
        }
    };
    fetch(row);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * VEC;
        if (c < d) {
            ld_par<VEC>(w, c, 1.f, wf[i]);
            ld_par<VEC>(b, c, 0.f, bf[i]);
        }
    }
    for (; row < rows; row += step) {
#pragma unroll
        for (int i = 0; i < NV; ++i) v[i] = next[i];
        if (row + step < rows) fetch(row + step);
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((i * TPR + t) * VEC < d) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) s[0] += to_f<DT>(v[i].v[j]);
            }
        row_sum<TPR>(s, lds);
        const float mu = s[0] / (float)d;
        s[0] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((i * TPR + t) * VEC < d) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float e = to_f<DT>(v[i].v[j]) - mu;
                    s[0] += e * e;
                }
            }
        row_sum<TPR>(s, lds);
        const float r = 1.f / sqrtf(s[0] / (float)d + eps);
        if (t == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * VEC;
            if (c >= d) continue;
            float o[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) o[j] = (to_f<DT>(v[i].v[j]) - mu) * r * wf[i][j] + bf[i][j];
            st_vec<DT, VEC>(y + row * d + c, o);
        }
    }
}

// Rows wider than the registers of a workgroup: x is read for each sum and for
// the output, which may lie over it (as in the other kernels: no __restrict__).
template <int DT>
__global__ __launch_bounds__(1024) void layernorm_wide_kernel(
    const typename IO<DT>::T *x, const float *__restrict__ w, const float *__restrict__ b, int rows, int d,
    float eps, typename IO<DT>::T *y, float *__restrict__ mean, float *__restrict__ rstd) {
    __shared__ float lds[16];
    const long row = blockIdx.x;
    const typename IO<DT>::T *xr = x + row * d;
    float s[1] = {0.f};
    for (int c = threadIdx.x; c < d; c += 1024) s[0] += IO<DT>::ld(xr, c);
    row_sum<1024>(s, lds);
    const float mu = s[0] / (float)d;
    s[0] = 0.f;
    for (int c = threadIdx.x; c < d; c += 1024) {
        const float e = IO<DT>::ld(xr, c) - mu;
        s[0] += e * e;
    }
    row_sum<1024>(s, lds);
    const float r = 1.f / sqrtf(s[0] / (float)d + eps);
    if (threadIdx.x == 0) {
        if (mean) mean[row] = mu;
        if (rstd) rstd[row] = r;
    }
    for (int c = threadIdx.x; c < d; c += 1024)
        IO<DT>::st(y + row * d, c, (IO<DT>::ld(xr, c) - mu) * r * (w ? w[c] : 1.f) + (b ? b[c] : 0.f));
}

// part: (gridDim.x, 2, d) float32, or null where neither dw nor db is asked
template <int DT, int VEC, int NV, int TPR>
__global__ __launch_bounds__(threads_of(TPR)) void layernorm_bwd_kernel(
    const typename IO<DT>::T *dy, const typename IO<DT>::T *x, const float *__restrict__ w,
    const float *__restrict__ mean, const float *__restrict__ rstd, int rows, int d, typename IO<DT>::T *dx,
    float *__restrict__ part) {
    constexpr int RPB = threads_of(TPR) / TPR;   // rows at a time
    __shared__ float lds[TPR > 64 ? 2 * TPR / 64 : 1];
    __shared__ float comb[RPB > 1 ? RPB - 1 : 1][RPB > 1 ? 2 * TPR * VEC : 1];
    const int t = threadIdx.x % TPR, sub = threadIdx.x / TPR;
    float wf[NV][VEC], aw[NV][VEC], ab[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * VEC;
#pragma unroll
        for (int j = 0; j < VEC; ++j) aw[i][j] = ab[i][j] = 0.f, wf[i][j] = 1.f;
        if (c < d) ld_par<VEC>(w, c, 1.f, wf[i]);
    }
    const float inv = 1.f / (float)d;
    const long step = (long)gridDim.x * RPB;
    Raw<DT, VEC> vx[NV], vy[NV], nx[NV], ny[NV];
    float nmu = 0.f, nr = 0.f;
    auto fetch = [&](long row) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * VEC;
            if (c < d) {
                nx[i] = ld_raw<DT, VEC>(x + row * d + c);
                ny[i] = ld_raw<DT, VEC>(dy + row * d + c);
            }
        }
        nmu = mean[row];
        nr = rstd[row];
    };
    long row = (long)blockIdx.x * RPB + sub;
    if (row < rows) fetch(row);
    for (; row < rows; row += step) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            vx[i] = nx[i];
            vy[i] = ny[i];
        }
        const float mu = nmu, r = nr;
        if (row + step < rows) fetch(row + step);
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if ((i * TPR + t) * VEC < d) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float g = to_f<DT>(vy[i].v[j]), h = (to_f<DT>(vx[i].v[j]) - mu) * r;
                    const float tw = g * wf[i][j];
                    s[0] += tw;
                    s[1] += tw * h;
                    aw[i][j] += g * h;
                    ab[i][j] += g;
                }
            }
        if (!dx) continue;
        row_sum<TPR>(s, lds);
        const float m0 = s[0] * inv, m1 = s[1] * inv;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + t) * VEC;
            if (c >= d) continue;
            float o[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float h = (to_f<DT>(vx[i].v[j]) - mu) * r;
                o[j] = (to_f<DT>(vy[i].v[j]) * wf[i][j] - m0 - h * m1) * r;
            }
            st_vec<DT, VEC>(dx + row * d + c, o);
        }
    }
    if (!part) return;
    float *pw = part + (long)blockIdx.x * 2 * d, *pb = pw + d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * TPR + t) * VEC;
        if constexpr (RPB > 1) {   // the rows' sums of this workgroup, in their order
            __syncthreads();
            if (sub > 0) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    comb[sub - 1][j * TPR + t] = aw[i][j];
                    comb[sub - 1][(VEC + j) * TPR + t] = ab[i][j];
                }
            }
            __syncthreads();
            if (sub == 0) {
#pragma unroll
                for (int q = 0; q < RPB - 1; ++q)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        aw[i][j] += comb[q][j * TPR + t];
                        ab[i][j] += comb[q][(VEC + j) * TPR + t];
                    }
            }
        }
        if (sub == 0 && c < d) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                pw[c + j] = aw[i][j];
                pb[c + j] = ab[i][j];
            }
        }
    }
}

// The two halves of the backward pass for rows wider than the registers.
template <int DT>
__global__ __launch_bounds__(1024) void layernorm_bwd_wide_dx_kernel(
    const typename IO<DT>::T *dy, const typename IO<DT>::T *x, const float *__restrict__ w,
    const float *__restrict__ mean, const float *__restrict__ rstd, int rows, int d, typename IO<DT>::T *dx) {
    __shared__ float lds[32];
    const long row = blockIdx.x;
    const float mu = mean[row], r = rstd[row];
    float s[2] = {0.f, 0.f};
    for (int c = threadIdx.x; c < d; c += 1024) {
        const float tw = IO<DT>::ld(dy + row * d, c) * (w ? w[c] : 1.f);
        s[0] += tw;
        s[1] += tw * (IO<DT>::ld(x + row * d, c) - mu) * r;
    }
    row_sum<1024>(s, lds);
    const float m0 = s[0] / (float)d, m1 = s[1] / (float)d;
    for (int c = threadIdx.x; c < d; c += 1024) {
        const float h = (IO<DT>::ld(x + row * d, c) - mu) * r;
        IO<DT>::st(dx + row * d, c, (IO<DT>::ld(dy + row * d, c) * (w ? w[c] : 1.f) - m0 - h * m1) * r);
    }
}
template <int DT>
__global__ __launch_bounds__(256) void layernorm_bwd_wide_dw_kernel(
    const typename IO<DT>::T *__restrict__ dy, const typename IO<DT>::T *__restrict__ x, const float *__restrict__ mean,
    const float *__restrict__ rstd, int rows, int d, float *__restrict__ part, int groups) {
    const int c = (blockIdx.x / groups) * 256 + threadIdx.x, gr = blockIdx.x % groups;
    if (c >= d) return;
    float aw = 0.f, ab = 0.f;
    for (long row = gr; row < rows; row += groups) {
        const float g = IO<DT>::ld(dy + row * d, c);
        aw += g * (IO<DT>::ld(x + row * d, c) - mean[row]) * rstd[row];
        ab += g;
    }
    part[((long)gr * 2) * d + c] = aw;
    part[((long)gr * 2 + 1) * d + c] = ab;
}

// dw, db = sums over the G partial rows: 32 columns a workgroup, 32 threads
// along the rows, then those 32 in order.
__global__ __launch_bounds__(1024) void layernorm_reduce_kernel(const float *__restrict__ part, int G, int d,
                                                                float *__restrict__ dw, float *__restrict__ db) {
    __shared__ float lds[32][33];
    const int c = threadIdx.x & 31, q = threadIdx.x >> 5;
    const long n = 2L * d, col = (long)blockIdx.x * 32 + c;
    float s = 0.f;
    if (col < n)
        for (int g = q; g < G; g += 32) s += part[g * n + col];
    lds[q][c] = s;
    __syncthreads();
    if (q == 0 && col < n) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) s += lds[i][c];
        if (col < d) {
            if (dw) dw[col] = s;
        } else if (db) {
            db[col - d] = s;
        }
    }
}

// How a row is laid over threads: 16-byte vectors where every row starts on 16
// bytes; a wave where `most` vectors a lane hold the row (no barrier in its sums), else 256
// threads, else 1024; tpr 0 where those do not hold it.  With up to eight vectors a lane a
// wave also takes rows of 2560 16-bit values, with too few rows under way: 19.6 us instead of
// 16.9 at 8192 x 2560; with one the rows of 768 go to workgroups and their barriers: 66.7 us
// instead of 34.0 at 16384 x 768, forward and backward.
struct Shape {
    int vec, nv, tpr;
};
Shape shape_of(int d, int dtype, bool aligned) {
    const int full = dtype == F32 ? 4 : 8;
    Shape s{aligned && d % full == 0 ? full : 1, 0, 0};
    const int most = s.vec == 1 ? 8 : 4;
    for (int tpr : {64, 256, 1024}) {
        const int nv = (d + tpr * s.vec - 1) / (tpr * s.vec);
        if (nv <= most) {
            s.nv = nv;
            s.tpr = tpr;
            break;
        }
    }
    return s;
}

// Workgroups that walk over the rows: fewer leave the card empty, more read the weights (and
// write partial sums) once more each.  8192 x 2560 bf16 forward: 23.5 us with a quarter of
// them, 19.1 with four times as many, 16.9 so; forward and backward of 16384 x 768 fp16 with 512
// and 256 (of 2048 and 512): 37.7, with 8192 and 1024: 40.6, so 34.0; of 4999 x 1031 float32
// 42.3, 35.2 and 31.5.
int fwd_groups(int rows, int tpr) {
    const int rpb = threads_of(tpr) / tpr, most = tpr == 1024 ? 512 : 2048, want = (rows - 1) / rpb + 1;
    return want < most ? want : most;
}
int bwd_groups(int rows, int tpr) {
    const int rpb = tpr == 0 ? 1 : threads_of(tpr) / tpr;
    const int most = tpr == 64 ? 512 : tpr == 256 ? 512 : 256;
    const int want = (rows - 1) / rpb + 1;
    return want < most ? want : most;
}

template <int DT, int VEC, typename F> hipError_t by_shape(const Shape &s, F f) {
    auto nv = [&](auto tpr) {
        switch (s.nv) {
            case 1: return f(std::integral_constant<int, 1>(), tpr);
            case 2: return f(std::integral_constant<int, 2>(), tpr);
            case 3: return f(std::integral_constant<int, 3>(), tpr);
            case 4: return f(std::integral_constant<int, 4>(), tpr);
        }
        if constexpr (VEC == 1) {
            if (s.nv == 5) return f(std::integral_constant<int, 5>(), tpr);
            return s.nv == 6 ? f(std::integral_constant<int, 6>(), tpr) : f(std::integral_constant<int, 8>(), tpr);
        }
        return hipErrorInvalidValue;
    };
    if (s.tpr == 64) return nv(std::integral_constant<int, 64>());
    if (s.tpr == 256) return nv(std::integral_constant<int, 256>());
    return nv(std::integral_constant<int, 1024>());
}

constexpr int kWideRows = 1 << 21;          // rows a launch with a workgroup of 1024 for each (under 2^32 threads)

template <int DT, int VEC>
hipError_t ln_fwd(const Shape &s, const void *x, const float *w, const float *b, int rows, int d, float eps, void *y,
                  float *mean, float *rstd, hipStream_t st) {
    typedef typename IO<DT>::T T;
    return by_shape<DT, VEC>(s, [&](auto nv, auto tpr) {
        constexpr int NV = decltype(nv)::value, TPR = decltype(tpr)::value;
        layernorm_kernel<DT, VEC, NV, TPR><<<(unsigned)fwd_groups(rows, TPR), threads_of(TPR), 0, st>>>(
            (const T *)x, w, b, rows, d, eps, (T *)y, mean, rstd);
        return hipGetLastError();
    });
}

template <int DT, int VEC>
hipError_t ln_bwd(const Shape &s, const void *dy, const void *x, const float *w, const float *mean, const float *rstd,
                  int rows, int d, void *dx, float *part, int G, hipStream_t st) {
    typedef typename IO<DT>::T T;
    return by_shape<DT, VEC>(s, [&](auto nv, auto tpr) {
        constexpr int NV = decltype(nv)::value, TPR = decltype(tpr)::value;
        layernorm_bwd_kernel<DT, VEC, NV, TPR><<<(unsigned)G, threads_of(TPR), 0, st>>>(
            (const T *)dy, (const T *)x, w, mean, rstd, rows, d, (T *)dx, part);
        return hipGetLastError();
    });
}

template <int DT>
hipError_t fwd_of(const void *x, const float *w, const float *b, int rows, int d, float eps, void *y, float *mean,
                  float *rstd, hipStream_t st) {
    typedef typename IO<DT>::T T;
    const Shape s = shape_of(d, DT, (((uintptr_t)x | (uintptr_t)y) & 15) == 0);
    if (s.tpr == 0) {
        for (int r = 0; r < rows; r += kWideRows) {
            const int n = rows - r < kWideRows ? rows - r : kWideRows;
            layernorm_wide_kernel<DT><<<(unsigned)n, 1024, 0, st>>>((const T *)x + (long)r * d, w, b, n, d, eps, (T *)y + (long)r * d,
                                                                   mean ? mean + r : nullptr, rstd ? rstd + r : nullptr);
            if (rows - r <= kWideRows) break;
        }
        return hipGetLastError();
    }
    if (s.vec == 1) return ln_fwd<DT, 1>(s, x, w, b, rows, d, eps, y, mean, rstd, st);
    return ln_fwd<DT, DT == F32 ? 4 : 8>(s, x, w, b, rows, d, eps, y, mean, rstd, st);
}

template <int DT>
hipError_t bwd_of(const void *dy, const void *x, const float *w, const float *mean, const float *rstd, int rows, int d,
                  void *dx, float *dw, float *db, float *part, hipStream_t st) {
    typedef typename IO<DT>::T T;
    const Shape s = shape_of(d, DT, (((uintptr_t)x | (uintptr_t)dy | (uintptr_t)dx) & 15) == 0);
    if (!dw && !db) part = nullptr;
    int G = bwd_groups(rows, s.tpr);
    hipError_t e = hipSuccess;
    if (s.tpr == 0) {
        for (int r = 0; dx && r < rows; r += kWideRows) {
            const int n = rows - r < kWideRows ? rows - r : kWideRows;
            layernorm_bwd_wide_dx_kernel<DT><<<(unsigned)n, 1024, 0, st>>>((const T *)dy + (long)r * d, (const T *)x + (long)r * d, w,
                                                                          mean + r, rstd + r, n, d, (T *)dx + (long)r * d);
            if (rows - r <= kWideRows) break;
        }
        if (part)
            layernorm_bwd_wide_dw_kernel<DT><<<(unsigned)(((d + 255) / 256) * G), 256, 0, st>>>(
                (const T *)dy, (const T *)x, mean, rstd, rows, d, part, G);
        e = hipGetLastError();
    } else if (s.vec == 1) {
        e = ln_bwd<DT, 1>(s, dy, x, w, mean, rstd, rows, d, dx, part, G, st);
    } else {
        e = ln_bwd<DT, DT == F32 ? 4 : 8>(s, dy, x, w, mean, rstd, rows, d, dx, part, G, st);
    }
    if (e != hipSuccess || !part) return e;
    layernorm_reduce_kernel<<<(unsigned)((2L * d + 31) / 32), 1024, 0, st>>>(part, G, d, dw, db);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_layernorm(const void *x, const float *w, const float *b, int rows, int d, float eps, int dtype, void *y,
                            float *mean, float *rstd, hipStream_t s) {
    if (dtype == F32) return fwd_of<F32>(x, w, b, rows, d, eps, y, mean, rstd, s);
    if (dtype == F16) return fwd_of<F16>(x, w, b, rows, d, eps, y, mean, rstd, s);
    return fwd_of<BF16>(x, w, b, rows, d, eps, y, mean, rstd, s);
}

// for the most groups that any layout of these rows takes (see bwd_groups)
size_t layernorm_bwd_workspace(int rows, int d) { return (size_t)(rows < 512 ? rows : 512) * 2 * d * sizeof(float); }

hipError_t launch_layernorm_bwd(const void *dy, const void *x, const float *w, const float *mean, const float *rstd,
                                int rows, int d, int dtype, void *dx, float *dw, float *db, float *ws, hipStream_t s) {
    if (dtype == F32) return bwd_of<F32>(dy, x, w, mean, rstd, rows, d, dx, dw, db, ws, s);
    if (dtype == F16) return bwd_of<F16>(dy, x, w, mean, rstd, rows, d, dx, dw, db, ws, s);
    return bwd_of<BF16>(dy, x, w, mean, rstd, rows, d, dx, dw, db, ws, s);
}

}  // namespace h3
