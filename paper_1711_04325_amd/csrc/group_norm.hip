// Group normalization (Wu and He 2018), NHWC, with the residual add and the activation behind it.  Image n's group g is H*W rows
// of Cg = C/G neighbouring channels, C apart.  Bound by memory: what counts is how often x (and dy) are read.
//
// A group that fits the registers of one workgroup is read once: a workgroup takes W channels (whole groups, 64 bytes of a row or
// more where that fits) of all the image's rows, keeps them, and goes over them again in registers (gn_fwd_kernel, gn_bwd_kernel).
// Larger groups take two passes over memory: partial results of bands of rows (gn_stats_kernel, gn_sums_kernel), their merge, and
// the element-wise pass.  All sums run in an order that the sizes alone decide.
#include <type_traits>

#include "common.h"

namespace rn50 {

// ---- vectors of V channels of a row, as they lie in memory -----------------------------------------------------------------
template <class T, int V> struct GnVec;
template <> struct GnVec<float, 4> {
    typedef float4 Raw;
    static __device__ void unpack(const Raw &r, float *f) { f[0] = r.x; f[1] = r.y; f[2] = r.z; f[3] = r.w; }
    static __device__ Raw pack(const float *f) { return make_float4(f[0], f[1], f[2], f[3]); }
};
template <> struct GnVec<bf16_t, 4> {
    typedef uint2 Raw;
    static __device__ void unpack(const Raw &r, float *f) { f[0] = bf16_lo(r.x); f[1] = bf16_hi(r.x); f[2] = bf16_lo(r.y); f[3] = bf16_hi(r.y); }
    static __device__ Raw pack(const float *f) { return make_uint2(bf16_pack2(f[0], f[1]), bf16_pack2(f[2], f[3])); }
};
template <> struct GnVec<bf16_t, 8> {
    typedef uint4 Raw;
    static __device__ void unpack(const Raw &r, float *f)
    {
        f[0] = bf16_lo(r.x); f[1] = bf16_hi(r.x); f[2] = bf16_lo(r.y); f[3] = bf16_hi(r.y);
        f[4] = bf16_lo(r.z); f[5] = bf16_hi(r.z); f[6] = bf16_lo(r.w); f[7] = bf16_hi(r.w);
    }
    static __device__ Raw pack(const float *f)
    {
        return make_uint4(bf16_pack2(f[0], f[1]), bf16_pack2(f[2], f[3]), bf16_pack2(f[4], f[5]), bf16_pack2(f[6], f[7]));
    }
};
template <class T, int V> __device__ inline typename GnVec<T, V>::Raw gn_load(const T *p) { return *reinterpret_cast<const typename GnVec<T, V>::Raw *>(p); }
template <class T, int V> __device__ inline void gn_store(T *p, const float *f) { *reinterpret_cast<typename GnVec<T, V>::Raw *>(p) = GnVec<T, V>::pack(f); }
template <int V> __device__ inline void gn_load_floats(const float *p, float *f)
{
#pragma unroll
    for (int v = 0; v < V; v += 4) GnVec<float, 4>::unpack(reinterpret_cast<const float4 *>(p)[v / 4], f + v);
}

// ---- the activation --------------------------------------------------------------------------------------------------------
// What the forward pass feeds its activation, and the backward pass forms again: the same roundings in both.
__device__ inline float gn_pre(float x, float mean, float scale, float beta) { return fmaf(x - mean, scale, beta); }

// 1 / (1 + exp(-u)) from the hardware's 2^x and reciprocal (a rounding or two each; with expf and a division the element-wise pass of
// the smooth activation is bound by its arithmetic)
__device__ inline float gn_sigmoid(float u) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * u)); }

template <int ACT> __device__ inline float gn_act(float u)
{
    if (ACT == RN50_ACT_RELU) return u <= 0.f ? 0.f : u;  // a NaN stays one
    if (ACT == RN50_ACT_SILU) return u * gn_sigmoid(u);
    return u;
}
// d * act'(u)
template <int ACT> __device__ inline float gn_act_bwd(float d, float u)
{
    if (ACT == RN50_ACT_RELU) return u > 0.f ? d : 0.f;
    if (ACT == RN50_ACT_SILU) {
        const float s = gn_sigmoid(u);
        return d * (s * fmaf(u, 1.f - s, 1.f));
    }
    return d;
}

// ---- how threads lie over rows and channels ----------------------------------------------------------------------------------
// A workgroup's rows have `cols` vectors.  Up to 64 of them: a wavefront has 64/cols rows side by side (lanes left over idle), and adds
// them up with shuffles.  More: thread = row lane * cols + column.  Either way a thread stays in its column, and `slots` partial rows
// per workgroup meet in LDS.
struct GnMap {
    int cols, row_lanes, slots;
    static GnMap of(int cols, int threads)
    {
        GnMap m;
        m.cols = cols;
        m.row_lanes = cols <= 64 ? 64 / cols * (threads / 64) : threads / cols;
        m.slots = cols <= 64 ? threads / 64 : m.row_lanes;
        return m;
    }
};
struct GnThread {
    int col, row, slot, lane_row;
    bool active;
    __device__ GnThread(const GnMap &m)
    {
        if (m.cols <= 64) {
            const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per = 64 / m.cols;
            lane_row = lane / m.cols;
            col = lane - lane_row * m.cols;
            active = lane_row < per;
            row = wave * per + lane_row;
            slot = wave;
        } else {
            row = slot = threadIdx.x / m.cols;
            col = threadIdx.x - row * m.cols;
            active = row < m.row_lanes;
            lane_row = 0;
        }
    }
};
// Adds v over the rows of a wavefront; valid in its row 0.
template <int V> __device__ inline void gn_wave_rows_sum(const GnMap &m, const GnThread &t, float *v)
{
    if (m.cols > 32) return;
    const int per = 64 / m.cols, lane = threadIdx.x & 63;
    for (int off = 32; off > 0; off >>= 1)
        if (off < per) {
            const bool take = t.lane_row + off < per;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float o = __shfl(v[i], (lane + off * m.cols) & 63, 64);
                if (take) v[i] += o;
            }
        }
}
// Leaves the workgroup's sums of a thread's V values by column in out[W], W = cols*V (part: slots * W floats); threads beyond the
// active ones bring zeros.  Ends with a barrier.
template <int V> __device__ inline void gn_column_sums(const GnMap &m, const GnThread &t, float *v, float *part, float *out)
{
    const int W = m.cols * V;
    gn_wave_rows_sum<V>(m, t, v);
    if (t.active && t.lane_row == 0)
#pragma unroll
        for (int i = 0; i < V; ++i) part[t.slot * W + t.col * V + i] = v[i];
    __syncthreads();
    for (int c = threadIdx.x; c < W; c += blockDim.x) {
        float s = part[c];
        for (int k = 1; k < m.slots; ++k) s += part[k * W + c];
        out[c] = s;
    }
    __syncthreads();
}
// Sums of runs of Cg channels: groups[i] = sum of chan[i*Cg ..].  One group: the whole workgroup's work.  Ends with a barrier.
__device__ inline void gn_group_sums(int W, int Cg, const float *chan, float *groups, float *red)
{
    if (W == Cg && Cg > 32) {
        float s = 0.f;
        for (int c = threadIdx.x; c < W; c += blockDim.x) s += chan[c];
        s = wave_sum(s);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (unsigned k = 1; k < blockDim.x / 64; ++k) s += red[k];
            groups[0] = s;
        }
    } else {
        for (int g = threadIdx.x; g < W / Cg; g += blockDim.x) {
            float s = 0.f;
            for (int i = 0; i < Cg; ++i) s += chan[g * Cg + i];
            groups[g] = s;
        }
    }
    __syncthreads();
}

struct GnShape {
    int HW, C, G, Cg;
    int n0;  // first image of the launch
};

// ---- a group in one workgroup ----------------------------------------------------------------------------------------------
struct GnResident {
    GnMap map;
    int W, chunks;  // channels of a workgroup, and how many such to an image
};

// LDS: slots*W partial sums, W sums by channel, sums by group
static size_t gn_lds_floats(const GnMap &m, int W, int planes) { return (size_t)planes * (m.slots * W + W) + 16 + planes * (size_t)W; }

template <class T, int V, int E, int TH, int ACT, bool RES>
__global__ __launch_bounds__(TH) void gn_fwd_kernel(GnShape s, GnResident p, const T *__restrict__ x, const float *__restrict__ gamma,
                                                    const float *__restrict__ beta, float eps, const T *__restrict__ res, T *__restrict__ y,
                                                    float *__restrict__ save_mean, float *__restrict__ save_invstd)
{
    typedef GnVec<T, V> Vec;
    extern __shared__ float lds[];
    float *part = lds, *chan = part + p.map.slots * p.W, *red = chan + p.W, *grp = red + 16;
    const int id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int n = s.n0 + id / p.chunks, c0 = id % p.chunks * p.W;
    const GnThread t(p.map);
    const int c = c0 + t.col * V, RL = p.map.row_lanes;
    const long base = (long)n * s.HW * s.C + c;
    typename Vec::Raw raw[E];
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e * RL < s.HW && t.active) raw[e] = gn_load<T, V>(x + base + (long)min(t.row + e * RL, s.HW - 1) * s.C);
    float a[V];
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (t.active && t.row + e * RL < s.HW) {
            float f[V];
            Vec::unpack(raw[e], f);
#pragma unroll
            for (int i = 0; i < V; ++i) a[i] += f[i];
        }
    gn_column_sums<V>(p.map, t, a, part, chan);
    gn_group_sums(p.W, s.Cg, chan, grp, red);
    const float m = (float)s.HW * (float)s.Cg;  // a division: the mean of equal values is that value, whatever their number
    float mean[V];
    const int col = t.active ? t.col * V : 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        mean[i] = grp[(col + i) / s.Cg] / m;
        a[i] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (t.active && t.row + e * RL < s.HW) {
            float f[V];
            Vec::unpack(raw[e], f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = f[i] - mean[i];
                a[i] = fmaf(d, d, a[i]);
            }
        }
    gn_column_sums<V>(p.map, t, a, part, chan);  // its first barrier: every thread has read grp
    gn_group_sums(p.W, s.Cg, chan, grp, red);
    float scale[V], b[V];
    if (t.active) {
        gn_load_floats<V>(gamma + c, scale);
        gn_load_floats<V>(beta + c, b);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float invstd = 1.f / sqrtf(grp[(col + i) / s.Cg] / m + eps);
            if (save_mean && t.row == 0 && (c + i) % s.Cg == 0) {
                save_mean[(long)n * s.G + (c + i) / s.Cg] = mean[i];
                save_invstd[(long)n * s.G + (c + i) / s.Cg] = invstd;
            }
            scale[i] *= invstd;
        }
    }
    constexpr int B = E < 4 ? E : 4;  // rows whose residuals are in flight together
#pragma unroll
    for (int e0 = 0; e0 < E; e0 += B) {
        typename Vec::Raw rr[B];
        if (RES)
#pragma unroll
            for (int u = 0; u < B; ++u)
                if (t.active && t.row + (e0 + u) * RL < s.HW) rr[u] = gn_load<T, V>(res + base + (long)(t.row + (e0 + u) * RL) * s.C);
#pragma unroll
        for (int u = 0; u < B; ++u)
            if (t.active && t.row + (e0 + u) * RL < s.HW) {
                float f[V], q[V];
                Vec::unpack(raw[e0 + u], f);
                if (RES) Vec::unpack(rr[u], q);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float v = gn_pre(f[i], mean[i], scale[i], b[i]);
                    if (RES) v += q[i];
                    f[i] = gn_act<ACT>(v);
                }
                gn_store<T, V>(y + base + (long)(t.row + (e0 + u) * RL) * s.C, f);
            }
    }
}

// The operands of dz of one vector.
template <class T> struct GnBwdIn {
    const T *x, *dy, *dy2, *res;
    const float *gamma, *beta, *mean, *invstd;
};
// A column's constants: mean, 1/sigma, scale and beta as the forward pass had them.
template <int V> struct GnColumn {
    float mean[V], inv[V], scale[V], beta[V], gamma[V];
    template <class T> __device__ GnColumn(const GnShape &s, const GnBwdIn<T> &in, int n, int c)
    {
        gn_load_floats<V>(in.gamma + c, gamma);
        gn_load_floats<V>(in.beta + c, beta);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const long at = (long)n * s.G + (c + i) / s.Cg;
            mean[i] = in.mean[at];
            inv[i] = in.invstd[at];
            scale[i] = gamma[i] * inv[i];
        }
    }
};
template <class T, int V, int ACT, bool RES, bool DY2> struct GnDz {
    typename GnVec<T, V>::Raw x, dy, dy2, res;
    __device__ void load(const GnBwdIn<T> &in, long at)
    {
        x = gn_load<T, V>(in.x + at);
        dy = gn_load<T, V>(in.dy + at);
        if (DY2) dy2 = gn_load<T, V>(in.dy2 + at);
        if (RES) res = gn_load<T, V>(in.res + at);
    }
    // dz, and x - mean
    __device__ void form(const GnColumn<V> &k, float *dz, float *d) const
    {
        float f[V], g[V], q[V];
        GnVec<T, V>::unpack(x, f);
        GnVec<T, V>::unpack(dy, g);
        if (DY2) {
            GnVec<T, V>::unpack(dy2, q);
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] += q[i];
        }
        if (RES) GnVec<T, V>::unpack(res, q);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float u = gn_pre(f[i], k.mean[i], k.scale[i], k.beta[i]);
            if (RES) u += q[i];
            dz[i] = gn_act_bwd<ACT>(g[i], u);
            d[i] = f[i] - k.mean[i];
        }
    }
};
// dx from dz, x - mean and the group's two means
template <int V> __device__ inline void gn_dx(const GnColumn<V> &k, const float *dz, const float *d, const float *A, const float *B, float *out)
{
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = k.inv[i] * (fmaf(k.gamma[i], dz[i], -A[i]) - d[i] * k.inv[i] * B[i]);
}

// sums[0][n][c] = sum of dz over the image, sums[1][n][c] = sum of dz*xhat (NC = N*C apart)
template <class T, int V, int E, int TH, int ACT, bool RES, bool DY2>
__global__ __launch_bounds__(TH) void gn_bwd_kernel(GnShape s, GnResident p, long NC, GnBwdIn<T> in, float *__restrict__ sums, T *__restrict__ dx,
                                                    T *__restrict__ dres)
{
    typedef GnVec<T, V> Vec;
    extern __shared__ float lds[];
    const int plane = p.map.slots * p.W;
    float *part0 = lds, *part1 = part0 + plane, *chan0 = part1 + plane, *chan1 = chan0 + p.W, *red = chan1 + p.W, *grp0 = red + 16, *grp1 = grp0 + p.W;
    const int id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int n = s.n0 + id / p.chunks, c0 = id % p.chunks * p.W;
    const GnThread t(p.map);
    const int col = t.active ? t.col * V : 0, c = c0 + col, RL = p.map.row_lanes;
    const long base = (long)n * s.HW * s.C + c;
    const GnColumn<V> k(s, in, n, c);
    typename Vec::Raw xr[E];
    float dz[E][V], a0[V], a1[V];
#pragma unroll
    for (int i = 0; i < V; ++i) a0[i] = a1[i] = 0.f;
    constexpr int B = E < 2 ? E : 2;
#pragma unroll
    for (int e0 = 0; e0 < E; e0 += B) {
        GnDz<T, V, ACT, RES, DY2> q[B];
#pragma unroll
        for (int u = 0; u < B; ++u)
            if (t.active && t.row + (e0 + u) * RL < s.HW) q[u].load(in, base + (long)(t.row + (e0 + u) * RL) * s.C);
#pragma unroll
        for (int u = 0; u < B; ++u)
            if (t.active && t.row + (e0 + u) * RL < s.HW) {
                float d[V];
                q[u].form(k, dz[e0 + u], d);
                xr[e0 + u] = q[u].x;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    a0[i] += dz[e0 + u][i];
                    a1[i] = fmaf(dz[e0 + u][i], d[i] * k.inv[i], a1[i]);
                }
            }
    }
    gn_column_sums<V>(p.map, t, a0, part0, chan0);
    gn_column_sums<V>(p.map, t, a1, part1, chan1);
    for (int i = threadIdx.x; i < p.W; i += TH) {
        const float s0 = chan0[i], s1 = chan1[i], g = in.gamma[c0 + i];
        sums[(long)n * s.C + c0 + i] = s0;
        sums[NC + (long)n * s.C + c0 + i] = s1;
        chan0[i] = s0 * g;
        chan1[i] = s1 * g;
    }
    __syncthreads();
    gn_group_sums(p.W, s.Cg, chan0, grp0, red);
    gn_group_sums(p.W, s.Cg, chan1, grp1, red);
    const float m = (float)s.HW * (float)s.Cg;
    float A[V], Bm[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        A[i] = grp0[(col + i) / s.Cg] / m;
        Bm[i] = grp1[(col + i) / s.Cg] / m;
    }
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (t.active && t.row + e * RL < s.HW) {
            float f[V];
            Vec::unpack(xr[e], f);
#pragma unroll
            for (int i = 0; i < V; ++i) f[i] -= k.mean[i];
            const long at = base + (long)(t.row + e * RL) * s.C;
            if (dres) gn_store<T, V>(dres + at, dz[e]);
            gn_dx<V>(k, dz[e], f, A, Bm, f);
            gn_store<T, V>(dx + at, f);
        }
}

// ---- two passes over memory ------------------------------------------------------------------------------------------------
// A workgroup takes a band of rows of a run of columns, whatever groups they are in; partial results by channel lie at [image][band][C],
// a second plane behind the first.
constexpr int kGnThreads = 512, kGnRows = 8;  // rows of a thread in a band
struct GnBands {
    GnMap map;
    int W, chunks;   // channels of a workgroup (the last run of an image may be short), runs of an image
    int rows, bands; // rows of a band (the last may be short), bands of an image
    long plane;      // floats of a plane of partial results
};
__device__ inline int gn_band_rows(const GnShape &s, const GnBands &p, int band) { return min(p.rows, s.HW - band * p.rows); }

// mean and sum of squared deviations of every channel over a band
template <class T, int V>
__global__ __launch_bounds__(kGnThreads) void gn_stats_kernel(GnShape s, GnBands p, const T *__restrict__ x, float *__restrict__ part_out)
{
    typedef GnVec<T, V> Vec;
    extern __shared__ float lds[];
    float *part = lds, *chan = part + p.map.slots * p.W;
    int id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int chunk = id % p.chunks;
    id /= p.chunks;
    const int band = id % p.bands, image = id / p.bands;
    GnThread t(p.map);
    const int c = chunk * p.W + t.col * V, r0 = band * p.rows, rows = gn_band_rows(s, p, band), RL = p.map.row_lanes;
    t.active = t.active && c < s.C;
    const T *from = x + ((long)(s.n0 + image) * s.HW + r0) * s.C + c;
    typename Vec::Raw raw[kGnRows];
#pragma unroll
    for (int e = 0; e < kGnRows; ++e)
        if (e * RL < rows && t.active) raw[e] = gn_load<T, V>(from + (long)min(t.row + e * RL, rows - 1) * s.C);
    float a[V], mean[V];
#pragma unroll
    for (int i = 0; i < V; ++i) a[i] = 0.f;
#pragma unroll
    for (int e = 0; e < kGnRows; ++e)
        if (t.active && t.row + e * RL < rows) {
            float f[V];
            Vec::unpack(raw[e], f);
#pragma unroll
            for (int i = 0; i < V; ++i) a[i] += f[i];
        }
    gn_column_sums<V>(p.map, t, a, part, chan);
    const int col = t.active ? t.col * V : 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        mean[i] = chan[col + i] / (float)rows;
        a[i] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < kGnRows; ++e)
        if (t.active && t.row + e * RL < rows) {
            float f[V];
            Vec::unpack(raw[e], f);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = f[i] - mean[i];
                a[i] = fmaf(d, d, a[i]);
            }
        }
    gn_column_sums<V>(p.map, t, a, part, chan);  // its first barrier: every thread has its mean
    float *out = part_out + ((long)image * p.bands + band) * s.C + c;
    if (t.active && t.row == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            *reinterpret_cast<float4 *>(out + i) = make_float4(mean[i], mean[i + 1], mean[i + 2], mean[i + 3]);
            *reinterpret_cast<float4 *>(out + p.plane + i) = make_float4(chan[col + i], chan[col + i + 1], chan[col + i + 2], chan[col + i + 3]);
        }
    }
}

constexpr int kGnMergeThreads = 256;
__device__ inline double gn_block_sum(double v, double *red)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    __syncthreads();  // red is free again
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.;
#pragma unroll
    for (int i = 0; i < kGnMergeThreads / 64; ++i) v += red[i];
    return v;
}

// A group's statistics from its channels' in all bands; in 64 bits, since there may be thousands.
__global__ __launch_bounds__(kGnMergeThreads) void gn_stats_merge_kernel(GnShape s, GnBands p, const float *__restrict__ part, float eps,
                                                                         float *__restrict__ mean_out, float *__restrict__ invstd_out)
{
    __shared__ double red[kGnMergeThreads / 64];
    const int image = blockIdx.x / s.G, g = blockIdx.x % s.G;
    const float *from = part + (long)image * p.bands * s.C + g * s.Cg;
    const int count = p.bands * s.Cg;
    double a = 0.;
    for (int i = threadIdx.x; i < count; i += kGnMergeThreads) {
        const int b = i / s.Cg;
        a += (double)gn_band_rows(s, p, b) * from[(long)b * s.C + i - b * s.Cg];
    }
    const double m = (double)s.HW * s.Cg, mean = gn_block_sum(a, red) / m;
    a = 0.;
    for (int i = threadIdx.x; i < count; i += kGnMergeThreads) {
        const int b = i / s.Cg;
        const long at = (long)b * s.C + i - b * s.Cg;
        const double d = from[at] - mean;
        a += from[p.plane + at] + gn_band_rows(s, p, b) * d * d;
    }
    const float var = (float)(gn_block_sum(a, red) / m);
    if (threadIdx.x == 0) {
        const long at = (long)(s.n0 + image) * s.G + g;
        mean_out[at] = (float)mean;
        invstd_out[at] = 1.f / sqrtf(var + eps);
    }
}

template <class T, int V, int ACT, bool RES>
__global__ __launch_bounds__(kGnThreads) void gn_apply_kernel(GnShape s, GnBands p, const T *__restrict__ x, const float *__restrict__ gamma,
                                                              const float *__restrict__ beta, const float *__restrict__ mean_in,
                                                              const float *__restrict__ invstd, const T *__restrict__ res, T *__restrict__ y)
{
    typedef GnVec<T, V> Vec;
    int id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int chunk = id % p.chunks;
    id /= p.chunks;
    const int band = id % p.bands, n = s.n0 + id / p.bands;
    const GnThread t(p.map);
    const int c = chunk * p.W + t.col * V, rows = gn_band_rows(s, p, band), RL = p.map.row_lanes;
    if (!t.active || c >= s.C) return;
    const long base = ((long)n * s.HW + (long)band * p.rows) * s.C + c;
    float mean[V], scale[V], b[V];
    gn_load_floats<V>(gamma + c, scale);
    gn_load_floats<V>(beta + c, b);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const long at = (long)n * s.G + (c + i) / s.Cg;
        mean[i] = mean_in[at];
        scale[i] *= invstd[at];
    }
    constexpr int B = 4;
    for (int r0 = t.row; r0 < rows; r0 += B * RL) {
        typename Vec::Raw xr[B], rr[B];
#pragma unroll
        for (int u = 0; u < B; ++u)
            if (r0 + u * RL < rows) {
                xr[u] = gn_load<T, V>(x + base + (long)(r0 + u * RL) * s.C);
                if (RES) rr[u] = gn_load<T, V>(res + base + (long)(r0 + u * RL) * s.C);
            }
#pragma unroll
        for (int u = 0; u < B; ++u)
            if (r0 + u * RL < rows) {
                float f[V], q[V];
                Vec::unpack(xr[u], f);
                if (RES) Vec::unpack(rr[u], q);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float v = gn_pre(f[i], mean[i], scale[i], b[i]);
                    if (RES) v += q[i];
                    f[i] = gn_act<ACT>(v);
                }
                gn_store<T, V>(y + base + (long)(r0 + u * RL) * s.C, f);
            }
    }
}

// sums of dz and dz*xhat of every channel over a band
template <class T, int V, int ACT, bool RES, bool DY2>
__global__ __launch_bounds__(kGnThreads) void gn_sums_kernel(GnShape s, GnBands p, GnBwdIn<T> in, float *__restrict__ part_out)
{
    extern __shared__ float lds[];
    float *part = lds, *chan0 = part + p.map.slots * p.W, *chan1 = chan0 + p.W;
    int id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int chunk = id % p.chunks;
    id /= p.chunks;
    const int band = id % p.bands, image = id / p.bands, n = s.n0 + image;
    GnThread t(p.map);
    t.active = t.active && chunk * p.W + t.col * V < s.C;
    const int col = t.active ? t.col * V : 0, c = chunk * p.W + col, rows = gn_band_rows(s, p, band), RL = p.map.row_lanes;
    const long base = ((long)n * s.HW + (long)band * p.rows) * s.C + c;
    const GnColumn<V> k(s, in, n, c);
    float a0[V], a1[V];
#pragma unroll
    for (int i = 0; i < V; ++i) a0[i] = a1[i] = 0.f;
    constexpr int B = 4;
    if (t.active)
        for (int r0 = t.row; r0 < rows; r0 += B * RL) {
            GnDz<T, V, ACT, RES, DY2> q[B];
#pragma unroll
            for (int u = 0; u < B; ++u)
                if (r0 + u * RL < rows) q[u].load(in, base + (long)(r0 + u * RL) * s.C);
#pragma unroll
            for (int u = 0; u < B; ++u)
                if (r0 + u * RL < rows) {
                    float dz[V], d[V];
                    q[u].form(k, dz, d);
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        a0[i] += dz[i];
                        a1[i] = fmaf(dz[i], d[i] * k.inv[i], a1[i]);
                    }
                }
        }
    gn_column_sums<V>(p.map, t, a0, part, chan0);
    gn_column_sums<V>(p.map, t, a1, part, chan1);
    float *out = part_out + ((long)image * p.bands + band) * s.C + c;
    if (t.active && t.row == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            *reinterpret_cast<float4 *>(out + i) = make_float4(chan0[col + i], chan0[col + i + 1], chan0[col + i + 2], chan0[col + i + 3]);
            *reinterpret_cast<float4 *>(out + p.plane + i) = make_float4(chan1[col + i], chan1[col + i + 1], chan1[col + i + 2], chan1[col + i + 3]);
        }
    }
}

// The bands' sums, by image and channel, and the group's two means of gamma*dz and gamma*dz*xhat
__global__ __launch_bounds__(kGnMergeThreads) void gn_sums_merge_kernel(GnShape s, GnBands p, const float *__restrict__ part,
                                                                        const float *__restrict__ gamma, long NC, float *__restrict__ sums,
                                                                        float *__restrict__ means)
{
    __shared__ double red[kGnMergeThreads / 64], acc[2][kGnMergeThreads];
    const int image = blockIdx.x / s.G, g = blockIdx.x % s.G, n = s.n0 + image;
    const float *from = part + (long)image * p.bands * s.C + g * s.Cg;
    const int wide = min(s.Cg, kGnMergeThreads), slices = kGnMergeThreads / wide, ci = threadIdx.x % wide, sl = threadIdx.x / wide;
    double A = 0., B = 0.;
    for (int c0 = 0; c0 < s.Cg; c0 += wide) {
        double a0 = 0., a1 = 0.;
        if (sl < slices && c0 + ci < s.Cg)
            for (int b = sl; b < p.bands; b += slices) {
                a0 += from[(long)b * s.C + c0 + ci];
                a1 += from[p.plane + (long)b * s.C + c0 + ci];
            }
        __syncthreads();
        acc[0][threadIdx.x] = a0;
        acc[1][threadIdx.x] = a1;
        __syncthreads();
        if (sl == 0 && c0 + ci < s.Cg) {
            for (int k = 1; k < slices; ++k) {
                a0 += acc[0][k * wide + ci];
                a1 += acc[1][k * wide + ci];
            }
            const int c = g * s.Cg + c0 + ci;
            sums[(long)n * s.C + c] = (float)a0;
            sums[NC + (long)n * s.C + c] = (float)a1;
            A += gamma[c] * a0;
            B += gamma[c] * a1;
        }
    }
    const double m = (double)s.HW * s.Cg;
    A = gn_block_sum(A, red) / m;
    B = gn_block_sum(B, red) / m;
    if (threadIdx.x == 0) {
        means[2 * ((long)image * s.G + g)] = (float)A;
        means[2 * ((long)image * s.G + g) + 1] = (float)B;
    }
}

template <class T, int V, int ACT, bool RES, bool DY2>
__global__ __launch_bounds__(kGnThreads) void gn_bwd_apply_kernel(GnShape s, GnBands p, GnBwdIn<T> in, const float *__restrict__ means,
                                                                  T *__restrict__ dx, T *__restrict__ dres)
{
    int id = xcd_contiguous(blockIdx.x, gridDim.x);
    const int chunk = id % p.chunks;
    id /= p.chunks;
    const int band = id % p.bands, image = id / p.bands, n = s.n0 + image;
    const GnThread t(p.map);
    const int c = chunk * p.W + t.col * V, rows = gn_band_rows(s, p, band), RL = p.map.row_lanes;
    if (!t.active || c >= s.C) return;
    const long base = ((long)n * s.HW + (long)band * p.rows) * s.C + c;
    const GnColumn<V> k(s, in, n, c);
    float A[V], Bm[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const long at = 2 * ((long)image * s.G + (c + i) / s.Cg);
        A[i] = means[at];
        Bm[i] = means[at + 1];
    }
    constexpr int B = 4;
    for (int r0 = t.row; r0 < rows; r0 += B * RL) {
        GnDz<T, V, ACT, RES, DY2> q[B];
#pragma unroll
        for (int u = 0; u < B; ++u)
            if (r0 + u * RL < rows) q[u].load(in, base + (long)(r0 + u * RL) * s.C);
#pragma unroll
        for (int u = 0; u < B; ++u)
            if (r0 + u * RL < rows) {
                float dz[V], d[V];
                q[u].form(k, dz, d);
                const long at = base + (long)(r0 + u * RL) * s.C;
                if (dres) gn_store<T, V>(dres + at, dz);
                gn_dx<V>(k, dz, d, A, Bm, d);
                gn_store<T, V>(dx + at, d);
            }
    }
}

// dgamma and dbeta: the images' sums; a workgroup takes 64 channels, a wavefront every 16th image
constexpr int kGnParamWaves = 16;
__global__ __launch_bounds__(64 * kGnParamWaves) void gn_params_kernel(int N, int C, const float *__restrict__ sums, float *__restrict__ dgamma,
                                                                       float *__restrict__ dbeta)
{
    __shared__ float part[2][kGnParamWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = min(blockIdx.x * 64 + lane, (unsigned)C - 1);
    const long NC = (long)N * C;
    float b[4] = {0.f, 0.f, 0.f, 0.f}, g[4] = {0.f, 0.f, 0.f, 0.f};
    for (int n0 = wave; n0 < N; n0 += 4 * kGnParamWaves)
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (n0 + u * kGnParamWaves < N) {
                b[u] += sums[(long)(n0 + u * kGnParamWaves) * C + c];
                g[u] += sums[NC + (long)(n0 + u * kGnParamWaves) * C + c];
            }
    part[0][wave][lane] = (b[0] + b[1]) + (b[2] + b[3]);
    part[1][wave][lane] = (g[0] + g[1]) + (g[2] + g[3]);
    __syncthreads();
    if (threadIdx.x < 128) {
        float v[kGnParamWaves];
#pragma unroll
        for (int w = 0; w < kGnParamWaves; ++w) v[w] = part[wave][w][lane];
#pragma unroll
        for (int half = kGnParamWaves / 2; half; half /= 2)
#pragma unroll
            for (int w = 0; w < half; ++w) v[w] += v[w + half];
        if (blockIdx.x * 64 + lane < (unsigned)C) (wave == 0 ? dbeta : dgamma)[c] = v[0];
    }
}

// ---- host side -------------------------------------------------------------------------------------------------------------
static int gcd(int a, int b) { return b ? gcd(b, a % b) : a; }

// Channels of a workgroup: whole groups and whole vectors, of at least `bytes` of a row where the image has them.  0: groups and
// vectors of V do not meet below C.
static int gn_run(int C, int Cg, int V, int size, int bytes)
{
    if (C % V) return 0;
    const int unit = Cg / gcd(Cg, V) * V;
    if (C % unit) return 0;
    for (int j = 1; j <= C / unit; ++j)
        if (C / unit % j == 0 && (j * unit * size >= bytes || j == C / unit)) return j * unit;
    return C;
}

constexpr int kGnSegment = 64;
// The two-pass kernels' cut.
template <class T> static GnBands gn_bands(int n, int HW, int C, int V)
{
    GnBands p;
    const int cols = C / V;
    p.chunks = ceil_div(cols, kGnThreads);
    p.W = ceil_div(cols, p.chunks) * V;
    p.map = GnMap::of(p.W / V, kGnThreads);
    p.rows = p.map.row_lanes * kGnRows;
    p.bands = ceil_div(HW, p.rows);
    p.plane = (long)n * p.bands * C;
    return p;
}

// Workspace: sums by image and channel (two planes), statistics or means by image and group (two values), partial results (two planes).
struct GnRoom { size_t sums, pairs, parts; size_t floats() const { return sums + pairs + parts; } };
static GnRoom gn_room(int n, int c, int HW, int groups)
{
    const GnBands p = gn_bands<float>(n, HW, c, 4);  // vectors of four channels: the most bands
    const GnBands q = c % 8 == 0 ? gn_bands<float>(n, HW, c, 8) : p;
    const long plane = p.plane > q.plane ? p.plane : q.plane;
    return {((size_t)2 * n * c + 3) & ~(size_t)3, ((size_t)2 * n * groups + 3) & ~(size_t)3, (size_t)2 * plane};
}

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
template <class F> static void gn_with(bool b, F f)
{
    if (b) f(std::true_type{});
    else f(std::false_type{});
}
// f(V) with the widest vectors that runs of whole groups are made of
template <class T, class F> static void gn_with_vector(int c, int Cg, F f)
{
    if constexpr (std::is_same<T, bf16_t>::value) {
        if (c % 8 == 0) return f(std::integral_constant<int, 8>{});
    }
    f(std::integral_constant<int, 4>{});
}

// Images of one launch: below 2^31 threads of it.
static int gn_images(int n, long workgroups_each, int threads)
{
    const long most = (1L << 31) / threads / workgroups_each;
    return (int)(most < 1 ? 1 : most < n ? most : n);
}

template <int TH, int E> struct GnSize { static constexpr int threads = TH, rows = E; };
// Tries sizes in turn: f(size) for the first whose threads hold all rows.
template <class S, class... More, class F> static bool gn_first_fit_of(int HW, int cols, F f)
{
    if (cols <= S::threads && (long)GnMap::of(cols, S::threads).row_lanes * S::rows >= HW) {
        f(S{});
        return true;
    }
    if constexpr (sizeof...(More) > 0) return gn_first_fit_of<More...>(HW, cols, f);
    return false;
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
    const int HW = h * w, Cg = c / groups;
    const GnRoom room = gn_room(n, c, HW, groups);
    RN50_REQUIRE(ws_bytes >= room.floats() * sizeof(float), RN50_EWORKSPACE, "%s: workspace too small", who);
    hipStream_t st = (hipStream_t)stream;
    gn_with_vector<T>(c, Cg, [&](auto vec) {
        constexpr int V = decltype(vec)::value;
        const int W = gn_run(c, Cg, V, sizeof(T), kGnSegment);
        bool done = false;
        if (W)
            done = gn_first_fit_of<GnSize<256, 4>, GnSize<256, 8>, GnSize<512, 8>, GnSize<512, 16>, GnSize<1024, 16>>(HW, W / V, [&](auto size) {
                constexpr int TH = decltype(size)::threads, E = decltype(size)::rows;
                const GnResident p{GnMap::of(W / V, TH), W, c / W};
                const size_t lds = gn_lds_floats(p.map, W, 1) * sizeof(float);
                const int each = gn_images(n, p.chunks, TH);
                for (int n0 = 0; n0 < n; n0 += each) {
                    const GnShape s{HW, c, groups, Cg, n0};
                    const dim3 grid((unsigned)((n - n0 < each ? n - n0 : each) * p.chunks));
                    gn_with_act(act, [&](auto a) {
                        gn_with(res != nullptr, [&](auto r) {
                            hipLaunchKernelGGL((gn_fwd_kernel<T, V, E, TH, decltype(a)::value, decltype(r)::value>), grid, dim3(TH), lds, st, s, p, x,
                                               gamma, beta, eps, res, y, save_mean, save_invstd);
                        });
                    });
                }
            });
        if (done) return;
        const GnBands p = gn_bands<T>(n, HW, c, V);
        float *mean = save_mean ? save_mean : (float *)ws + room.sums, *invstd = save_invstd ? save_invstd : mean + (size_t)n * groups;
        float *part = (float *)ws + room.sums + room.pairs;
        const size_t lds = (size_t)(p.map.slots + 1) * p.W * sizeof(float);
        const int each = gn_images(n, (long)p.bands * p.chunks, kGnThreads);
        for (int n0 = 0; n0 < n; n0 += each) {
            const int images = n - n0 < each ? n - n0 : each;
            const GnShape s{HW, c, groups, Cg, n0};
            const dim3 grid((unsigned)(images * p.bands * p.chunks));
            hipLaunchKernelGGL((gn_stats_kernel<T, V>), grid, dim3(kGnThreads), lds, st, s, p, x, part);
            hipLaunchKernelGGL(gn_stats_merge_kernel, dim3(images * groups), dim3(kGnMergeThreads), 0, st, s, p, part, eps, mean, invstd);
            gn_with_act(act, [&](auto a) {
                gn_with(res != nullptr, [&](auto r) {
                    hipLaunchKernelGGL((gn_apply_kernel<T, V, decltype(a)::value, decltype(r)::value>), grid, dim3(kGnThreads), 0, st, s, p, x, gamma,
                                       beta, mean, invstd, res, y);
                });
            });
        }
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
    const int HW = h * w, Cg = c / groups;
    const GnRoom room = gn_room(n, c, HW, groups);
    RN50_REQUIRE(ws_bytes >= room.floats() * sizeof(float), RN50_EWORKSPACE, "%s: workspace too small", who);
    const long NC = (long)n * c;
    float *sums = (float *)ws;
    hipStream_t st = (hipStream_t)stream;
    const GnBwdIn<T> in{x, dy, dy2, act == RN50_ACT_NONE ? nullptr : res, gamma, beta, mean, invstd};
    auto with_kind = [&](auto f) {  // f(ACT, RES, DY2)
        gn_with_act(act, [&](auto a) {
            gn_with(dy2 != nullptr, [&](auto d) {
                if constexpr (decltype(a)::value == RN50_ACT_NONE) f(a, std::false_type{}, d);
                else gn_with(in.res != nullptr, [&](auto r) { f(a, r, d); });
            });
        });
    };
    gn_with_vector<T>(c, Cg, [&](auto vec) {
        constexpr int V = decltype(vec)::value;
        const int W = gn_run(c, Cg, V, sizeof(T), kGnSegment);
        bool done = false;
        if (W)
            done = gn_first_fit_of<GnSize<256, 4>, GnSize<256, 8>, GnSize<512, 8>, GnSize<V == 4 ? 1024 : 512, 8>>(HW, W / V, [&](auto size) {
                constexpr int TH = decltype(size)::threads, E = decltype(size)::rows;
                const GnResident p{GnMap::of(W / V, TH), W, c / W};
                const size_t lds = gn_lds_floats(p.map, W, 2) * sizeof(float);
                const int each = gn_images(n, p.chunks, TH);
                for (int n0 = 0; n0 < n; n0 += each) {
                    const GnShape s{HW, c, groups, Cg, n0};
                    const dim3 grid((unsigned)((n - n0 < each ? n - n0 : each) * p.chunks));
                    with_kind([&](auto a, auto r, auto d) {
                        hipLaunchKernelGGL((gn_bwd_kernel<T, V, E, TH, decltype(a)::value, decltype(r)::value, decltype(d)::value>), grid, dim3(TH), lds,
                                           st, s, p, NC, in, sums, dx, dres);
                    });
                }
            });
        if (!done) {
            const GnBands p = gn_bands<T>(n, HW, c, V);
            float *means = sums + room.sums, *part = means + room.pairs;
            const size_t lds = (size_t)(p.map.slots + 2) * p.W * sizeof(float);
            const int each = gn_images(n, (long)p.bands * p.chunks, kGnThreads);
            for (int n0 = 0; n0 < n; n0 += each) {
                const int images = n - n0 < each ? n - n0 : each;
                const GnShape s{HW, c, groups, Cg, n0};
                const dim3 grid((unsigned)(images * p.bands * p.chunks));
                with_kind([&](auto a, auto r, auto d) {
                    constexpr int ACT = decltype(a)::value;
                    constexpr bool RES = decltype(r)::value, DY2 = decltype(d)::value;
                    hipLaunchKernelGGL((gn_sums_kernel<T, V, ACT, RES, DY2>), grid, dim3(kGnThreads), lds, st, s, p, in, part);
                    hipLaunchKernelGGL(gn_sums_merge_kernel, dim3(images * groups), dim3(kGnMergeThreads), 0, st, s, p, part, gamma, NC, sums, means);
                    hipLaunchKernelGGL((gn_bwd_apply_kernel<T, V, ACT, RES, DY2>), grid, dim3(kGnThreads), 0, st, s, p, in, means, dx, dres);
                });
            }
        }
    });
    hipLaunchKernelGGL(gn_params_kernel, dim3(ceil_div(c, 64)), dim3(64 * kGnParamWaves), 0, st, n, c, sums, dgamma, dbeta);
    return launch_status(who);
}

}  // namespace rn50

using namespace rn50;

extern "C" size_t rn50_gn_workspace_bytes(int n, int c, int h, int w, int groups)
{
    if (n <= 0 || c <= 0 || h <= 0 || w <= 0 || groups <= 0 || c % 4 || c % groups || (long)h * w >= (1L << 31) || (long)h * w * c >= (1L << 31) ||
        (long)n * c >= (1L << 31))
        return 0;
    return gn_room(n, c, h * w, groups).floats() * sizeof(float);
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
