// Learning from a teacher's largest logits (Hinton et al. 2015): the cross-entropy with the label and with them, with its gradient.
#include "rows.h"

namespace rn50 {

constexpr int kRowThreads = 256;

template <class Op>
__device__ inline float row_reduce(float v, float *red, Op op)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = op(v, __shfl_xor(v, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = red[0];
    for (int w = 1; w < kRowThreads / 64; ++w) v = op(v, red[w]);
    return v;
}
struct Sum { __device__ float operator()(float a, float b) const { return a + b; } };
// a NaN stays one
struct Max { __device__ float operator()(float a, float b) const { return a > b || a != a ? a : b; } };

struct DistillArgs {
    int K, t;
    size_t ld, ld_d;
    const int32_t *labels;  // null: no hard term
    const int32_t *idx;     // null: no soft term
    const float *val;
    float alpha, tau, scale;
};

template <class T>
__global__ __launch_bounds__(kRowThreads) void distill_kernel(DistillArgs a, const T *__restrict__ z, T *__restrict__ dz, float *__restrict__ row_loss)
{
    __shared__ float red[kRowThreads / 64], p[RN50_TOPK_MAX];
    __shared__ int at[RN50_TOPK_MAX];
    const int K = a.K, tid = threadIdx.x, n = blockIdx.x;
    const T *row = z + n * a.ld;
    T *out = dz + n * a.ld_d;
    const float nan = __builtin_nanf("");
    // the teacher's entry tid (t <= kRowThreads)
    int k = -1;
    float v = -INFINITY;
    if (a.idx && tid < a.t) {
        k = a.idx[(size_t)n * a.t + tid];
        v = k != -1 ? a.val[(size_t)n * a.t + tid] : -INFINITY;
    }
    const bool kept = v > -INFINITY || v != v, class_ok = (unsigned)k < (unsigned)K;
    const float vmx = row_reduce(v, red, Max());
    const bool some = vmx > -INFINITY || vmx != vmx;
    const int label = a.labels ? a.labels[n] : -1;
    const bool has = label != -1, label_ok = (unsigned)label < (unsigned)K;
    if (!has && !some) {  // a row that counts for nothing, whatever its logits
        if (tid == 0) row_loss[2 * n] = row_loss[2 * n + 1] = 0.f;
        if (dz)
            for (int c = tid; c < K; c += kRowThreads) row_st(out, c, 0.f);
        return;
    }
    float mx = -INFINITY;
    for (int k = tid; k < K; k += kRowThreads) mx = Max()(mx, row_ld(row, k));
    mx = row_reduce(mx, red, Max());
    float s1 = 0.f, st = 0.f;
    for (int k = tid; k < K; k += kRowThreads) {
        const float d = row_ld(row, k) - mx;
        s1 += expf(d);
        st += expf(d / a.tau);
    }
    s1 = row_reduce(s1, red, Sum());
    st = row_reduce(st, red, Sum());

    float hard = 0.f, soft = 0.f;
    bool bad = false;
    if (has) {
        if (label_ok) hard = logf(s1) - (row_ld(row, label) - mx);
        else bad = true;
    }
    const float d = (v - vmx) / a.tau, e = kept ? expf(d) : 0.f;
    const float se = row_reduce(e, red, Sum());
    const float pt = kept ? e / se : 0.f;
    float term = 0.f;
    if (kept && class_ok && pt != 0.f) term = pt * ((d - logf(se)) - ((row_ld(row, k) - mx) / a.tau - logf(st)));
    if (kept && !class_ok) term = nan;
    if (some) soft = a.tau * a.tau * row_reduce(term, red, Sum());
    if (tid == 0) {
        row_loss[2 * n] = bad || s1 != s1 ? nan : hard;
        row_loss[2 * n + 1] = s1 != s1 ? nan : soft;
    }
    if (!dz) return;
    __syncthreads();
    p[tid] = pt;
    at[tid] = kept && class_ok ? k : -1;
    __syncthreads();
    const float w1 = has ? (1.f - a.alpha) * a.scale : 0.f, wt = some ? a.alpha * a.tau * a.scale : 0.f;
    auto grad = [&](int c) {
        const float x = row_ld(row, c) - mx;
        float g = 0.f;
        if (has) g += w1 * (expf(x) / s1 - (c == label ? 1.f : 0.f));
        if (some) g += wt * (expf(x / a.tau) / st);
        return s1 != s1 ? nan : g;
    };
    for (int c = tid; c < K; c += kRowThreads) row_st(out, c, grad(c));
    __syncthreads();
    // the teacher's classes again, less their probabilities; the first entry of a class writes for all of it
    if (at[tid] >= 0 && tid < a.t) {
        float sum = 0.f;
        bool first = true;
        for (int i = 0; i < a.t; ++i)
            if (at[i] == at[tid]) {
                first = first && i >= tid;
                sum += p[i];
            }
        if (first) row_st(out, at[tid], grad(at[tid]) - wt * sum);
    }
}

// loss[0..2] from the rows' terms; each thread adds every 256th row, in 64 bits
__global__ __launch_bounds__(kRowThreads) void distill_loss_kernel(int N, float alpha, float scale, const float *__restrict__ row_loss,
                                                                   float *__restrict__ loss)
{
    __shared__ double part[2][kRowThreads];
    double h = 0., s = 0.;
    for (int n = threadIdx.x; n < N; n += kRowThreads) {
        h += row_loss[2 * (size_t)n];
        s += row_loss[2 * (size_t)n + 1];
    }
    part[0][threadIdx.x] = h;
    part[1][threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        h = s = 0.;
        for (int i = 0; i < kRowThreads; ++i) {
            h += part[0][i];
            s += part[1][i];
        }
        h *= scale;
        s *= scale;
        loss[1] = (float)h;
        loss[2] = (float)s;
        // a term of weight 0 has no part in it, whatever it is
        loss[0] = (float)((alpha < 1.f ? (1. - alpha) * h : 0.) + (alpha > 0.f ? alpha * s : 0.));
    }
}

static size_t distill_ws_bytes(int n) { return (size_t)2 * n * sizeof(float); }

template <class T>
static int distill_impl(const char *who, int n, int k, int t, const T *logits, size_t ld, const int32_t *labels, const int32_t *teacher_idx,
                        const float *teacher_val, float alpha, float tau, float scale, float *loss, T *dlogits, size_t ld_d, void *ws,
                        size_t ws_bytes, void *stream)
{
    RN50_REQUIRE(n > 0 && k > 0, RN50_EINVAL, "%s: non-positive dimension", who);
    RN50_REQUIRE(n < kMaxRows, RN50_EUNSUPPORTED, "%s: 2^22 rows and more", who);
    RN50_REQUIRE(alpha >= 0.f && alpha <= 1.f, RN50_EINVAL, "%s: alpha must be in [0, 1]", who);
    RN50_REQUIRE(tau >= 1.f / 1024 && tau <= 1024.f, RN50_EINVAL, "%s: the temperature must be in [1/1024, 1024]", who);
    RN50_REQUIRE(fabsf(scale) < INFINITY, RN50_EINVAL, "%s: scale is not finite", who);
    RN50_REQUIRE(t >= (alpha > 0.f ? 1 : 0), RN50_EINVAL, "%s: no kept logits", who);
    RN50_REQUIRE(t <= RN50_TOPK_MAX, RN50_EUNSUPPORTED, "%s: at most %d kept logits of a row", who, RN50_TOPK_MAX);
    RN50_REQUIRE(ld >= (size_t)k && ld < (1ull << 31), RN50_EINVAL, "%s: rows of logits overlap or are 2^31 elements apart and more", who);
    RN50_REQUIRE(!dlogits || (ld_d >= (size_t)k && ld_d < (1ull << 31)), RN50_EINVAL,
                 "%s: rows of dlogits overlap or are 2^31 elements apart and more", who);
    RN50_REQUIRE(logits && loss && ws, RN50_EINVAL, "%s: null pointer", who);
    RN50_REQUIRE(labels || alpha == 1.f, RN50_EINVAL, "%s: no labels", who);
    RN50_REQUIRE((teacher_idx && teacher_val) || alpha == 0.f, RN50_EINVAL, "%s: no teacher", who);
    RN50_REQUIRE(aligned16(logits) && aligned16(labels) && aligned16(teacher_idx) && aligned16(teacher_val) && aligned16(loss) &&
                     aligned16(dlogits) && aligned16(ws),
                 RN50_EINVAL, "%s: pointers must be 16-byte aligned", who);
    RN50_REQUIRE(dlogits != logits, RN50_EINVAL, "%s: not in place", who);
    RN50_REQUIRE(ws_bytes >= distill_ws_bytes(n), RN50_EWORKSPACE, "%s: workspace too small", who);
    const DistillArgs a{k, t, ld, dlogits ? ld_d : 0, alpha < 1.f ? labels : nullptr, alpha > 0.f ? teacher_idx : nullptr, teacher_val, alpha, tau, scale};
    float *row_loss = (float *)ws;
    hipLaunchKernelGGL((distill_kernel<T>), dim3(n), dim3(kRowThreads), 0, (hipStream_t)stream, a, logits, dlogits, row_loss);
    hipLaunchKernelGGL(distill_loss_kernel, dim3(1), dim3(kRowThreads), 0, (hipStream_t)stream, n, alpha, scale, row_loss, loss);
    return launch_status(who);
}

}  // namespace rn50

using namespace rn50;

extern "C" size_t rn50_distill_workspace_bytes(int n, int k, int t)
{
    return n > 0 && k > 0 && t >= 0 ? distill_ws_bytes(n) : 0;
}

extern "C" int distill_ce(int n, int k, int t, const float *logits, size_t ld, const int32_t *labels_or_null, const int32_t *teacher_idx,
                          const float *teacher_val, float alpha, float tau, float scale, float *loss, float *dlogits_or_null, size_t ld_dlogits,
                          void *ws, size_t ws_bytes, void *stream)
{
    return distill_impl<float>("distill_ce", n, k, t, logits, ld, labels_or_null, teacher_idx, teacher_val, alpha, tau, scale, loss,
                               dlogits_or_null, ld_dlogits, ws, ws_bytes, stream);
}
extern "C" int distill_ce_bf16(int n, int k, int t, const uint16_t *logits, size_t ld, const int32_t *labels_or_null, const int32_t *teacher_idx,
                               const float *teacher_val, float alpha, float tau, float scale, float *loss, uint16_t *dlogits_or_null,
                               size_t ld_dlogits, void *ws, size_t ws_bytes, void *stream)
{
    return distill_impl<bf16_t>("distill_ce_bf16", n, k, t, logits, ld, labels_or_null, teacher_idx, teacher_val, alpha, tau, scale, loss,
                                dlogits_or_null, ld_dlogits, ws, ws_bytes, stream);
}
