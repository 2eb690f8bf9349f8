// Group normalization (Wu and He 2018), NHWC, with the residual add and the activation behind it.  Image n's group g is H*W rows
// of Cg = C/G neighbouring channels, C apart.
#include "common.h"

namespace rn50 {

struct GnShape {
    int HW, C, G, Cg;
    __device__ long at(int n, int g) const { return (long)n * HW * C + (long)g * Cg; }  // first element of a group
};

constexpr int kGnThreads = 256;

__device__ inline float gn_ld(const float *p) { return *p; }
__device__ inline float gn_ld(const bf16_t *p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ inline void gn_st(float *p, float v) { *p = v; }
__device__ inline void gn_st(bf16_t *p, float v) { *p = (bf16_t)bf16_rne(v); }

// The sum over the workgroup, in every thread.
__device__ inline double gn_block_sum(double v, double *red)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();  // red is free again
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.;
    for (unsigned i = 0; i < blockDim.x / 64; ++i) v += red[i];
    return v;
}

// What the forward pass feeds its activation, and the backward pass forms again: the same roundings in both.
__device__ inline float gn_pre(float x, float mean, float scale, float beta) { return fmaf(x - mean, scale, beta); }

template <int ACT> __device__ inline float gn_act(float u)
{
    if (ACT == RN50_ACT_RELU) return u <= 0.f ? 0.f : u;  // a NaN stays one
    if (ACT == RN50_ACT_SILU) return u / (1.f + expf(-u));
    return u;
}
// act'(u)
template <int ACT> __device__ inline float gn_slope(float u)
{
    if (ACT == RN50_ACT_RELU) return u > 0.f ? 1.f : 0.f;
    if (ACT == RN50_ACT_SILU) {
        const float s = 1.f / (1.f + expf(-u));
        return s * (1.f + u * (1.f - s));
    }
    return 1.f;
}

template <class T, int ACT>
__global__ __launch_bounds__(kGnThreads) void gn_fwd_kernel(GnShape s, const T *__restrict__ x, const float *__restrict__ gamma,
                                                            const float *__restrict__ beta, float eps, const T *__restrict__ res,
                                                            T *__restrict__ y, float *__restrict__ save_mean, float *__restrict__ save_invstd)
{
    __shared__ double red[kGnThreads / 64];
    const int n = blockIdx.x / s.G, g = blockIdx.x % s.G;
    const long base = s.at(n, g);
    const int m = s.HW * s.Cg;
    double a = 0.;
    for (int i = threadIdx.x; i < m; i += kGnThreads) a += gn_ld(x + base + (long)(i / s.Cg) * s.C + i % s.Cg);
    const float mean = (float)(gn_block_sum(a, red) / m);
    a = 0.;
    for (int i = threadIdx.x; i < m; i += kGnThreads) {
        const float d = gn_ld(x + base + (long)(i / s.Cg) * s.C + i % s.Cg) - mean;
        a += (double)d * d;
    }
    const float invstd = 1.f / sqrtf((float)(gn_block_sum(a, red) / m) + eps);
    for (int i = threadIdx.x; i < m; i += kGnThreads) {
        const int c = g * s.Cg + i % s.Cg;
        const long at = base + (long)(i / s.Cg) * s.C + i % s.Cg;
        float u = gn_pre(gn_ld(x + at), mean, gamma[c] * invstd, beta[c]);
        if (res) u += gn_ld(res + at);
        gn_st(y + at, gn_act<ACT>(u));
    }
    if (save_mean && threadIdx.x == 0) {
        save_mean[blockIdx.x] = mean;
        save_invstd[blockIdx.x] = invstd;
    }
}

// dz of one element
template <class T, int ACT>
__device__ inline float gn_dz(const T *x, const T *dy, const T *dy2, const T *res, long at, float mean, float scale, float beta)
{
    float d = gn_ld(dy + at);
    if (dy2) d += gn_ld(dy2 + at);
    if (ACT == RN50_ACT_NONE) return d;
    float u = gn_pre(gn_ld(x + at), mean, scale, beta);
    if (res) u += gn_ld(res + at);
    return ACT == RN50_ACT_RELU ? (u > 0.f ? d : 0.f) : d * gn_slope<ACT>(u);
}

// sums[0][n][c] = sum of dz over the image, sums[1][n][c] = sum of dz*xhat
template <class T, int ACT>
__global__ __launch_bounds__(kGnThreads) void gn_bwd_sums_kernel(GnShape s, int NC, const T *__restrict__ x, const T *__restrict__ dy,
                                                                 const T *__restrict__ dy2, const T *__restrict__ res,
                                                                 const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                 const float *__restrict__ mean, const float *__restrict__ invstd,
                                                                 float *__restrict__ sums)
{
    __shared__ double red[kGnThreads / 64];
    const int n = blockIdx.x / s.C, c = blockIdx.x % s.C, ng = n * s.G + c / s.Cg;
    const float mu = mean[ng], is = invstd[ng], scale = gamma[c] * is, b = beta[c];
    double a0 = 0., a1 = 0.;
    for (int i = threadIdx.x; i < s.HW; i += kGnThreads) {
        const long at = ((long)n * s.HW + i) * s.C + c;
        const float dz = gn_dz<T, ACT>(x, dy, dy2, res, at, mu, scale, b);
        a0 += dz;
        a1 += (double)dz * ((gn_ld(x + at) - mu) * is);
    }
    a0 = gn_block_sum(a0, red);
    a1 = gn_block_sum(a1, red);
    if (threadIdx.x == 0) {
        sums[blockIdx.x] = (float)a0;
        sums[NC + blockIdx.x] = (float)a1;
    }
}

template <class T, int ACT>
__global__ __launch_bounds__(kGnThreads) void gn_bwd_apply_kernel(GnShape s, int NC, const T *__restrict__ x, const T *__restrict__ dy,
                                                                  const T *__restrict__ dy2, const T *__restrict__ res,
                                                                  const float *__restrict__ gamma, const float *__restrict__ beta,
                                                                  const float *__restrict__ mean, const float *__restrict__ invstd,
                                                                  const float *__restrict__ sums, T *__restrict__ dx, T *__restrict__ dres)
{
    __shared__ double red[kGnThreads / 64];
    const int n = blockIdx.x / s.G, g = blockIdx.x % s.G;
    const float mu = mean[blockIdx.x], is = invstd[blockIdx.x];
    const int m = s.HW * s.Cg;
    double a0 = 0., a1 = 0.;
    for (int i = threadIdx.x; i < s.Cg; i += kGnThreads) {
        const int c = g * s.Cg + i;
        a0 += (double)gamma[c] * sums[(long)n * s.C + c];
        a1 += (double)gamma[c] * sums[NC + (long)n * s.C + c];
    }
    const float A = (float)(gn_block_sum(a0, red) / m), B = (float)(gn_block_sum(a1, red) / m);
    const long base = s.at(n, g);
    for (int i = threadIdx.x; i < m; i += kGnThreads) {
        const int c = g * s.Cg + i % s.Cg;
        const long at = base + (long)(i / s.Cg) * s.C + i % s.Cg;
        const float dz = gn_dz<T, ACT>(x, dy, dy2, res, at, mu, gamma[c] * is, beta[c]);
        gn_st(dx + at, is * (fmaf(gamma[c], dz, -A) - (gn_ld(x + at) - mu) * is * B));
        if (dres) gn_st(dres + at, dz);
    }
}

// dgamma and dbeta: the images' sums in image order
__global__ __launch_bounds__(kGnThreads) void gn_bwd_params_kernel(int N, int C, const float *__restrict__ sums, float *__restrict__ dgamma,
                                                                   float *__restrict__ dbeta)
{
    const int c = blockIdx.x * kGnThreads + threadIdx.x;
    if (c >= C) return;
    float b = 0.f, g = 0.f;
    for (int n = 0; n < N; ++n) {
        b += sums[(long)n * C + c];
        g += sums[(long)(N + n) * C + c];
    }
    dbeta[c] = b;
    dgamma[c] = g;
}

static size_t gn_ws_floats(int n, int c) { return (size_t)2 * n * c; }

static int gn_check(const char *who, int n, int c, int h, int w, int layout, int groups, int act)
{
    RN50_REQUIRE(n > 0 && c > 0 && h > 0 && w > 0 && groups > 0, RN50_EINVAL, "%s: non-positive dimension", who);
    RN50_REQUIRE(layout == RN50_LAYOUT_NHWC, RN50_EUNSUPPORTED, "%s: only the NHWC layout has kernels", who);
    RN50_REQUIRE(c % 4 == 0, RN50_EUNSUPPORTED, "%s: channel count must be a multiple of 4", who);
    RN50_REQUIRE(c % groups == 0, RN50_EINVAL, "%s: groups must divide the channel count", who);
    RN50_REQUIRE(act >= RN50_ACT_NONE && act <= RN50_ACT_SILU, RN50_EINVAL, "%s: unknown activation", who);
    RN50_REQUIRE((long)h * w < (1L << 31) && (long)h * w * c < (1L << 31) && (long)n * c < (1L << 31), RN50_EUNSUPPORTED,
                 "%s: H*W*C and N*C must be below 2^31", who);
    return RN50_OK;
}

template <class F> static void gn_with_act(int act, F f)
{
    if (act == RN50_ACT_RELU) f(std::integral_constant<int, RN50_ACT_RELU>{});
    else if (act == RN50_ACT_SILU) f(std::integral_constant<int, RN50_ACT_SILU>{});
    else f(std::integral_constant<int, RN50_ACT_NONE>{});
}

template <class T>
static int gn_fwd_impl(const char *who, int n, int c, int h, int w, int layout, int groups, const T *x, const float *gamma, const float *beta,
                       float eps, const T *res, int act, T *y, float *save_mean, float *save_invstd, void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = gn_check(who, n, c, h, w, layout, groups, act)) return rc;
    RN50_REQUIRE(x && gamma && beta && y && ws, RN50_EINVAL, "%s: null pointer", who);
    RN50_REQUIRE(!save_mean == !save_invstd, RN50_EINVAL, "%s: the statistics are saved together", who);
    RN50_REQUIRE(aligned16(x) && aligned16(gamma) && aligned16(beta) && aligned16(res) && aligned16(y) && aligned16(save_mean) &&
                     aligned16(save_invstd) && aligned16(ws),
                 RN50_EINVAL, "%s: pointers must be 16-byte aligned", who);
    RN50_REQUIRE(y != x && y != res, RN50_EINVAL, "%s: not in place", who);
    RN50_REQUIRE(eps >= 0.f, RN50_EINVAL, "%s: negative eps", who);
    RN50_REQUIRE(ws_bytes >= gn_ws_floats(n, c) * sizeof(float), RN50_EWORKSPACE, "%s: workspace too small", who);
    const GnShape s{h * w, c, groups, c / groups};
    hipStream_t st = (hipStream_t)stream;
    gn_with_act(act, [&](auto a) {
        hipLaunchKernelGGL((gn_fwd_kernel<T, decltype(a)::value>), dim3(n * groups), dim3(kGnThreads), 0, st, s, x, gamma, beta, eps, res, y,
                           save_mean, save_invstd);
    });
    return launch_status(who);
}

template <class T>
static int gn_bwd_impl(const char *who, int n, int c, int h, int w, int layout, int groups, const T *x, const T *dy, const T *dy2, const T *res,
                       const float *gamma, const float *beta, const float *mean, const float *invstd, int act, T *dx, T *dres, float *dgamma,
                       float *dbeta, void *ws, size_t ws_bytes, void *stream)
{
    if (int rc = gn_check(who, n, c, h, w, layout, groups, act)) return rc;
    RN50_REQUIRE(x && dy && gamma && beta && mean && invstd && dx && dgamma && dbeta && ws, RN50_EINVAL, "%s: null pointer", who);
    RN50_REQUIRE(aligned16(x) && aligned16(dy) && aligned16(dy2) && aligned16(res) && aligned16(gamma) && aligned16(beta) && aligned16(mean) &&
                     aligned16(invstd) && aligned16(dx) && aligned16(dres) && aligned16(dgamma) && aligned16(dbeta) && aligned16(ws),
                 RN50_EINVAL, "%s: pointers must be 16-byte aligned", who);
    RN50_REQUIRE(dx != x && dx != dy && dx != dy2 && dx != res && dx != dres, RN50_EINVAL, "%s: not in place", who);
    RN50_REQUIRE(!dres || (dres != x && dres != dy && dres != dy2 && dres != res), RN50_EINVAL, "%s: not in place", who);
    RN50_REQUIRE(ws_bytes >= gn_ws_floats(n, c) * sizeof(float), RN50_EWORKSPACE, "%s: workspace too small", who);
    const GnShape s{h * w, c, groups, c / groups};
    float *sums = (float *)ws;
    hipStream_t st = (hipStream_t)stream;
    gn_with_act(act, [&](auto a) {
        constexpr int ACT = decltype(a)::value;
        hipLaunchKernelGGL((gn_bwd_sums_kernel<T, ACT>), dim3(n * c), dim3(kGnThreads), 0, st, s, n * c, x, dy, dy2, res, gamma, beta, mean, invstd,
                           sums);
        hipLaunchKernelGGL((gn_bwd_apply_kernel<T, ACT>), dim3(n * groups), dim3(kGnThreads), 0, st, s, n * c, x, dy, dy2, res, gamma, beta, mean,
                           invstd, sums, dx, dres);
    });
    hipLaunchKernelGGL(gn_bwd_params_kernel, dim3(ceil_div(c, kGnThreads)), dim3(kGnThreads), 0, st, n, c, sums, dgamma, dbeta);
    return launch_status(who);
}

}  // namespace rn50

using namespace rn50;

extern "C" size_t rn50_gn_workspace_bytes(int n, int c, int h, int w, int groups)
{
    if (n <= 0 || c <= 0 || h <= 0 || w <= 0 || groups <= 0 || c % 4 || c % groups || (long)h * w >= (1L << 31) || (long)h * w * c >= (1L << 31) ||
        (long)n * c >= (1L << 31))
        return 0;
    return gn_ws_floats(n, c) * sizeof(float);
}

extern "C" int gn_fwd(int n, int c, int h, int w, int layout, int groups, const float *x, const float *gamma, const float *beta, float eps,
                      const float *residual_or_null, int act, float *y, float *save_mean_or_null, float *save_invstd_or_null, void *ws,
                      size_t ws_bytes, void *stream)
{
    return gn_fwd_impl<float>("gn_fwd", n, c, h, w, layout, groups, x, gamma, beta, eps, residual_or_null, act, y, save_mean_or_null,
                              save_invstd_or_null, ws, ws_bytes, stream);
}
extern "C" int gn_fwd_bf16(int n, int c, int h, int w, int layout, int groups, const uint16_t *x, const float *gamma, const float *beta, float eps,
                           const uint16_t *residual_or_null, int act, uint16_t *y, float *save_mean_or_null, float *save_invstd_or_null, void *ws,
                           size_t ws_bytes, void *stream)
{
    return gn_fwd_impl<bf16_t>("gn_fwd_bf16", n, c, h, w, layout, groups, x, gamma, beta, eps, residual_or_null, act, y, save_mean_or_null,
                               save_invstd_or_null, ws, ws_bytes, stream);
}

extern "C" int gn_bwd(int n, int c, int h, int w, int layout, int groups, const float *x, const float *dy, const float *dy2_or_null,
                      const float *residual_or_null, const float *gamma, const float *beta, const float *save_mean, const float *save_invstd,
                      int act, float *dx, float *dresidual_or_null, float *dgamma, float *dbeta, void *ws, size_t ws_bytes, void *stream)
{
    return gn_bwd_impl<float>("gn_bwd", n, c, h, w, layout, groups, x, dy, dy2_or_null, residual_or_null, gamma, beta, save_mean, save_invstd, act,
                              dx, dresidual_or_null, dgamma, dbeta, ws, ws_bytes, stream);
}
extern "C" int gn_bwd_bf16(int n, int c, int h, int w, int layout, int groups, const uint16_t *x, const uint16_t *dy, const uint16_t *dy2_or_null,
                           const uint16_t *residual_or_null, const float *gamma, const float *beta, const float *save_mean,
                           const float *save_invstd, int act, uint16_t *dx, uint16_t *dresidual_or_null, float *dgamma, float *dbeta, void *ws,
                           size_t ws_bytes, void *stream)
{
    return gn_bwd_impl<bf16_t>("gn_bwd_bf16", n, c, h, w, layout, groups, x, dy, dy2_or_null, residual_or_null, gamma, beta, save_mean,
                               save_invstd, act, dx, dresidual_or_null, dgamma, dbeta, ws, ws_bytes, stream);
}
