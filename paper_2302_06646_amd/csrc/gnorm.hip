// Group norm with an activation, channels last: x [B,S,C], groups of C / G neighbouring channels over all S positions,
//     xhat = (x - mean) rstd,   z = gamma xhat + beta,   y = act(z)
// and its backward pass, with dz = dy act'(z) and m = S C / G:
//     dbeta = sum dz,   dgamma = sum dz xhat (over b and positions),   dx = rstd (gamma dz - (s1 + xhat s2) / m),
//     s1 = sum gamma dz,   s2 = sum gamma dz xhat over the group.
//
// Sums go by channel first: a thread keeps eight channels and walks over positions, so a group may be of any width, and dgamma, dbeta
// and the group's sums come from the same numbers.  Mean and variance are carried as (mean, sum of squared differences), merged
// pairwise, so a mean that is large against the deviation costs nothing.  All in fp32, in a fixed order.
#include "vec8.hpp"

namespace lc {
namespace {

constexpr int GT = 512;              // threads
constexpr int SLAB = 64;             // pieces of eight channels of a workgroup, at most
constexpr int GROUPS_WANTED = 1024;  // workgroups of a pass over the tensor
constexpr int AHEAD = 4;             // pieces that a thread asks for before it uses the first

// The normal distribution function, and e = exp(-z^2 / 2) beside it.  erfc(x) exp(x^2) is t Q(t), t = 1 / (1 + 0.4 x), for x >= 0, Q the
// polynomial of degree eight of the least largest relative error (fitted by weighted least squares): 1.3e-7, and 2.2e-7 absolute in
// fp32.  Below zero the result is not a difference, so its relative error is that of e, 8e-7 down to z = -4.
__device__ __forceinline__ float normal_cdf(float z, float& e)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.28284271247461901f, fabsf(z), 1.f));
    float q = 0.0502542145550251f;
    q = __builtin_fmaf(q, t, -0.18287357687950134f);
    q = __builtin_fmaf(q, t, 0.16904595494270325f);
    q = __builtin_fmaf(q, t, -0.0055788299068808556f);
    q = __builtin_fmaf(q, t, 0.14142005145549774f);
    q = __builtin_fmaf(q, t, 0.16854438185691833f);
    q = __builtin_fmaf(q, t, 0.20784245431423187f);
    q = __builtin_fmaf(q, t, 0.22566960752010345f);
    q = __builtin_fmaf(q, t, 0.22567586600780487f);
    e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
    const float h = 0.5f * q * t * e;
    return z < 0.f ? h : 1.f - h;
}

template <int ACT>
__device__ __forceinline__ float act_of(float z)
{
    if constexpr (ACT == LONGCONV_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f));
    if constexpr (ACT == LONGCONV_ACT_GELU) {
        float e;
        return z * normal_cdf(z, e);
    }
    if constexpr (ACT == LONGCONV_ACT_RELU) return z > 0.f ? z : z != z ? z : 0.f;
    return z;
}
template <int ACT>
__device__ __forceinline__ float slope_of(float z)
{
    if constexpr (ACT == LONGCONV_ACT_SILU) {
        const float q = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f));
        return q * (1.f + z * (1.f - q));
    }
    if constexpr (ACT == LONGCONV_ACT_GELU) {
        float e;
        const float c = normal_cdf(z, e);
        return __builtin_fmaf(z * 0.39894228040143268f, e, c);
    }
    if constexpr (ACT == LONGCONV_ACT_RELU) return z > 0.f ? 1.f : 0.f;
    return 1.f;
}

// (n, mean, m2) <- both sets together
__device__ __forceinline__ void merge(float& n, float& mean, float& m2, float n2, float mean2, float m22)
{
    if (n2 == 0.f) return;
    const float all = n + n2, d = mean2 - mean, f = n2 * __builtin_amdgcn_rcpf(all);
    mean = __builtin_fmaf(d, f, mean);
    m2 += m22 + d * d * n * f;
    n = all;
}

// How a pass walks over a tensor: workgroup (b, part, slab) takes `slices` pieces of eight channels of `per` positions; its threads
// are `rows` positions by `slices`.
struct Walk {
    uint32_t P, slices, slabs, rows, parts;
    int64_t per;
};
Walk walk(int64_t B, int64_t S, int64_t C)
{
    Walk w;
    w.P = (uint32_t)((C + VE - 1) / VE);
    w.slices = w.P < SLAB ? w.P : SLAB;
    w.slabs = (w.P + w.slices - 1) / w.slices;
    w.rows = GT / w.slices;
    int64_t parts = GROUPS_WANTED / (B * w.slabs);
    const int64_t most = (S + 4 * w.rows - 1) / (4 * w.rows);      // four positions of a thread at least
    if (parts > most) parts = most;
    if (parts < 1) parts = 1;
    w.per = (S + parts - 1) / parts;
    w.parts = (uint32_t)((S + w.per - 1) / w.per);
    return w;
}
// most rows (b, part) of partial results there can be: does not fall as B grows
size_t part_rows(int64_t B, int64_t S, int64_t C)
{
    const Walk w = walk(1, S, C);
    const int64_t most = (S + 4 * w.rows - 1) / (4 * w.rows), wanted = GROUPS_WANTED / w.slabs;
    const int64_t all = B * most;
    return (size_t)(all < wanted ? all : B > wanted ? B : wanted);
}

struct Place {
    uint32_t b, part, slab, s, r;
    int64_t from, to;
    int c, wide;          // first channel of the thread's piece, channels it has there (0: none)
    bool on;
};
__device__ __forceinline__ Place place(const Walk& w, int64_t S, int64_t C)
{
    Place p;
    p.slab = blockIdx.x % w.slabs;
    p.part = blockIdx.x / w.slabs % w.parts;
    p.b = blockIdx.x / w.slabs / w.parts;
    p.s = threadIdx.x % w.slices;
    p.r = threadIdx.x / w.slices;
    p.from = p.part * w.per;
    p.to = p.from + w.per < S ? p.from + w.per : S;
    p.c = (int)(p.slab * w.slices + p.s) * VE;
    p.on = p.r < w.rows && p.c < C;
    p.wide = p.on ? (int)(C - p.c < VE ? C - p.c : VE) : 0;
    return p;
}

// mean and sum of squared differences of every channel over the part's positions -> part[(b, part)][2][C]
template <class IO>
__global__ void __launch_bounds__(GT)
gnorm_stats_kernel(const typename IO::T* __restrict__ x, float* __restrict__ part, int64_t S, int64_t C, Walk w)
{
    __shared__ float sm[GT * VE], s2[GT * VE], sn[GT];
    const Place p = place(w, S, C);
    float mean[VE] = {}, m2[VE] = {}, n = 0.f;
    if (p.on)
        for (int64_t i = p.from + p.r; i < p.to; i += (int64_t)AHEAD * w.rows) {
            Raw8<IO> raw[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                load_raw<IO>(x + ((int64_t)p.b * S + i + u * w.rows) * C + p.c, i + u * w.rows < p.to ? p.wide : 0, raw[u]);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (i + u * w.rows >= p.to) break;
                float v[VE];
                raw[u].get(v);
                n += 1.f;
                const float f = __builtin_amdgcn_rcpf(n);
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const float d = v[j] - mean[j];
                    mean[j] = __builtin_fmaf(d, f, mean[j]);
                    m2[j] = __builtin_fmaf(d, v[j] - mean[j], m2[j]);
                }
            }
        }
    const int t = threadIdx.x;
#pragma unroll
    for (int j = 0; j < VE; ++j) {
        sm[t * VE + j] = mean[j];
        s2[t * VE + j] = m2[j];
    }
    sn[t] = n;
    __syncthreads();
    const int wide = (int)w.slices * VE;
    for (int i = t; i < wide; i += GT) {
        const int64_t c = (int64_t)p.slab * wide + i;
        if (c >= C) break;
        float an = 0.f, am = 0.f, a2 = 0.f;
        for (uint32_t r = 0; r < w.rows; ++r) {
            const int from = (int)(r * w.slices);
            merge(an, am, a2, sn[from + i / VE], sm[from * VE + i], s2[from * VE + i]);
        }
        float* q = part + ((size_t)p.b * w.parts + p.part) * 2 * C;
        q[c] = am;
        q[C + c] = a2;
    }
}

// a wave for each group: its channels' and parts' results together
__global__ void __launch_bounds__(64)
gnorm_group_kernel(const float* __restrict__ part, float* __restrict__ mean, float* __restrict__ rstd, int64_t S, int64_t C, uint32_t G,
                   uint32_t parts, int64_t per, float eps)
{
    const uint32_t b = blockIdx.x / G, g = blockIdx.x % G, D = (uint32_t)(C / G);
    float n = 0.f, m = 0.f, m2 = 0.f;
    for (uint64_t i = threadIdx.x; i < (uint64_t)parts * D; i += 64) {
        const uint32_t q = (uint32_t)(i / D), c = g * D + (uint32_t)(i - (uint64_t)q * D);
        const float* row = part + ((size_t)b * parts + q) * 2 * C;
        const int64_t here = S - q * per < per ? S - q * per : per;
        merge(n, m, m2, (float)here, row[c], row[C + c]);
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        // the lower lane of a pair first, on both sides: every lane ends with the same numbers
        float n2 = __shfl_xor(n, s), a2 = __shfl_xor(m, s), b2 = __shfl_xor(m2, s);
        if (threadIdx.x & s) {
            float t;
            t = n; n = n2; n2 = t;
            t = m; m = a2; a2 = t;
            t = m2; m2 = b2; b2 = t;
        }
        if (n == 0.f) { n = n2; m = a2; m2 = b2; }
        else merge(n, m, m2, n2, a2, b2);
    }
    if (threadIdx.x == 0) {
        mean[blockIdx.x] = m;
        rstd[blockIdx.x] = 1.f / sqrtf(m2 / n + eps);
    }
}

// eight parameters of the channels from c on (those beyond a tensor's last as `or_else`); p may be null
__device__ __forceinline__ void load_params(const float* p, int c, int wide, float or_else, float (&v)[VE])
{
#pragma unroll
    for (int j = 0; j < VE; ++j) v[j] = or_else;
    if (!p || wide < 1) return;
    load8<IoF32>(p + c, wide, v);
}

struct Channels {      // of a thread's piece
    float mean[VE], rstd[VE], gamma[VE], beta[VE];
    __device__ __forceinline__ void load(const Place& p, const float* mn, const float* rs, const float* ga, const float* be, uint32_t G, uint32_t D)
    {
        load_params(ga, p.c, p.wide, 1.f, gamma);
        load_params(be, p.c, p.wide, 0.f, beta);
        each_group(p, G, D, [&](int j, size_t g) {
            mean[j] = mn[g];
            rstd[j] = rs[g];
        });
    }
    // f(j, number of the group of channel j): one division for the eight
    template <class F>
    static __device__ __forceinline__ void each_group(const Place& p, uint32_t G, uint32_t D, F&& f)
    {
        uint32_t g = (uint32_t)p.c / D, at = (uint32_t)p.c - g * D;
        if (at + VE <= D) {
#pragma unroll
            for (int j = 0; j < VE; ++j) f(j, (size_t)p.b * G + g);
            return;
        }
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            f(j, (size_t)p.b * G + (g < G ? g : G - 1));
            if (++at == D) { at = 0; ++g; }
        }
    }
};

template <class IO, int ACT>
__global__ void __launch_bounds__(GT)
gnorm_apply_kernel(const typename IO::T* __restrict__ x, typename IO::T* __restrict__ y, const float* __restrict__ mean,
                   const float* __restrict__ rstd, const float* __restrict__ gamma, const float* __restrict__ beta, int64_t S, int64_t C,
                   uint32_t G, Walk w)
{
    const Place p = place(w, S, C);
    if (!p.on) return;
    Channels k;
    k.load(p, mean, rstd, gamma, beta, G, (uint32_t)(C / G));
    for (int64_t i = p.from + p.r; i < p.to; i += (int64_t)AHEAD * w.rows) {
        const size_t e = ((size_t)p.b * S + i) * C + p.c, more = (size_t)w.rows * C;
        Raw8<IO> raw[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) load_raw<IO>(x + e + u * more, i + u * w.rows < p.to ? p.wide : 0, raw[u]);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (i + u * w.rows >= p.to) break;
            float v[VE];
            raw[u].get(v);
#pragma unroll
            for (int j = 0; j < VE; ++j)
                v[j] = act_of<ACT>(__builtin_fmaf((v[j] - k.mean[j]) * k.rstd[j], k.gamma[j], k.beta[j]));
            store8<IO, true>(y + e + u * more, p.wide, v);
        }
    }
}

// sums of dz and dz xhat of every channel over the part's positions -> part[(b, part)][2][C]
template <class IO, int ACT>
__global__ void __launch_bounds__(GT)
gnorm_sums_kernel(const typename IO::T* __restrict__ dy, const typename IO::T* __restrict__ x, const float* __restrict__ mean,
                  const float* __restrict__ rstd, const float* __restrict__ gamma, const float* __restrict__ beta, float* __restrict__ part,
                  int64_t S, int64_t C, uint32_t G, Walk w)
{
    __shared__ float sa[GT * VE], sb[GT * VE];
    const Place p = place(w, S, C);
    float a[VE] = {}, b[VE] = {};
    if (p.on) {
        Channels k;
        k.load(p, mean, rstd, gamma, beta, G, (uint32_t)(C / G));
        for (int64_t i = p.from + p.r; i < p.to; i += (int64_t)AHEAD / 2 * w.rows) {
            const size_t e = ((size_t)p.b * S + i) * C + p.c, more = (size_t)w.rows * C;
            Raw8<IO> rx[AHEAD / 2], rg[AHEAD / 2];
#pragma unroll
            for (int u = 0; u < AHEAD / 2; ++u) {
                const int n = i + u * w.rows < p.to ? p.wide : 0;
                load_raw<IO>(x + e + u * more, n, rx[u]);
                load_raw<IO>(dy + e + u * more, n, rg[u]);
            }
#pragma unroll
            for (int u = 0; u < AHEAD / 2; ++u) {
                if (i + u * w.rows >= p.to) break;
                float v[VE], g[VE];
                rx[u].get(v);
                rg[u].get(g);
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const float h = (v[j] - k.mean[j]) * k.rstd[j];
                    const float dz = g[j] * slope_of<ACT>(__builtin_fmaf(h, k.gamma[j], k.beta[j]));
                    a[j] += dz;
                    b[j] = __builtin_fmaf(dz, h, b[j]);
                }
            }
        }
    }
    const int t = threadIdx.x;
#pragma unroll
    for (int j = 0; j < VE; ++j) {
        sa[t * VE + j] = a[j];
        sb[t * VE + j] = b[j];
    }
    __syncthreads();
    const int wide = (int)w.slices * VE;
    for (int i = t; i < wide; i += GT) {
        const int64_t c = (int64_t)p.slab * wide + i;
        if (c >= C) break;
        float ta = 0.f, tb = 0.f;
        for (uint32_t r = 0; r < w.rows; ++r) {
            ta += sa[r * wide + i];
            tb += sb[r * wide + i];
        }
        float* q = part + ((size_t)p.b * w.parts + p.part) * 2 * C;
        q[c] = ta;
        q[C + c] = tb;
    }
}

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) v += __shfl_xor(v, s);
    return v;
}

constexpr int RT = 1024, RC = 16;      // threads of a workgroup that sums channels, and channels of it

// workgroups 0 .. ceil(C / 16) - 1: dgamma and dbeta of sixteen channels, the rows of partial results spread over the threads; behind
// them sixteen groups each, s1 and s2 by a wave for every group
__global__ void __launch_bounds__(RT)
gnorm_gather_kernel(const float* __restrict__ part, const float* __restrict__ gamma, float* __restrict__ s1, float* __restrict__ s2,
                    float* __restrict__ dgamma, float* __restrict__ dbeta, int64_t B, int64_t C, uint32_t G, uint32_t parts)
{
    __shared__ float sa[RT], sh[RT];
    const uint32_t D = (uint32_t)(C / G), blocks = (uint32_t)((C + RC - 1) / RC);
    float a = 0.f, h = 0.f;
    if (blockIdx.x >= blocks) {
        const uint32_t id = (blockIdx.x - blocks) * (RT / 64) + threadIdx.x / 64;
        if (id >= (uint32_t)B * G) return;
        const uint32_t b = id / G, g = id % G;
        for (uint32_t i = threadIdx.x % 64; i < parts * D; i += 64) {
            const uint32_t q = i / D, c = g * D + (i - q * D);
            const float* row = part + ((size_t)b * parts + q) * 2 * C;
            const float ga = gamma ? gamma[c] : 1.f;
            a = __builtin_fmaf(ga, row[c], a);
            h = __builtin_fmaf(ga, row[C + c], h);
        }
        a = wave_sum(a);
        h = wave_sum(h);
        if (threadIdx.x % 64 == 0) {
            s1[id] = a;
            s2[id] = h;
        }
        return;
    }
    const uint32_t c = blockIdx.x * RC + threadIdx.x % RC, rows = (uint32_t)B * parts;
    if (c < C) {
#pragma unroll 8
        for (uint32_t i = threadIdx.x / RC; i < rows; i += RT / RC) {
            a += part[(size_t)i * 2 * C + c];
            h += part[(size_t)i * 2 * C + C + c];
        }
    }
    sa[threadIdx.x] = a;
    sh[threadIdx.x] = h;
    for (int s = RT / 2; s >= RC; s >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < s) {
            sa[threadIdx.x] += sa[threadIdx.x + s];
            sh[threadIdx.x] += sh[threadIdx.x + s];
        }
    }
    if (threadIdx.x < RC && c < C) {
        if (dbeta) dbeta[c] = sa[threadIdx.x];
        if (dgamma) dgamma[c] = sh[threadIdx.x];
    }
}

template <class IO, int ACT>
__global__ void __launch_bounds__(GT)
gnorm_dx_kernel(const typename IO::T* __restrict__ dy, const typename IO::T* __restrict__ x, const float* __restrict__ mean,
                const float* __restrict__ rstd, const float* __restrict__ gamma, const float* __restrict__ beta, const float* __restrict__ s1,
                const float* __restrict__ s2, typename IO::T* __restrict__ dx, int64_t S, int64_t C, uint32_t G, float inv, Walk w)
{
    const Place p = place(w, S, C);
    if (!p.on) return;
    const uint32_t D = (uint32_t)(C / G);
    Channels k;
    k.load(p, mean, rstd, gamma, beta, G, D);
    float c1[VE], c2[VE];
    Channels::each_group(p, G, D, [&](int j, size_t g) {
        c1[j] = s1[g] * inv;
        c2[j] = s2[g] * inv;
    });
    for (int64_t i = p.from + p.r; i < p.to; i += (int64_t)AHEAD / 2 * w.rows) {
        const size_t e = ((size_t)p.b * S + i) * C + p.c, more = (size_t)w.rows * C;
        Raw8<IO> rx[AHEAD / 2], rg[AHEAD / 2];
#pragma unroll
        for (int u = 0; u < AHEAD / 2; ++u) {
            const int n = i + u * w.rows < p.to ? p.wide : 0;
            load_raw<IO>(x + e + u * more, n, rx[u]);
            load_raw<IO>(dy + e + u * more, n, rg[u]);
        }
#pragma unroll
        for (int u = 0; u < AHEAD / 2; ++u) {
            if (i + u * w.rows >= p.to) break;
            float v[VE], g[VE];
            rx[u].get(v);
            rg[u].get(g);
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const float h = (v[j] - k.mean[j]) * k.rstd[j];
                const float dz = g[j] * slope_of<ACT>(__builtin_fmaf(h, k.gamma[j], k.beta[j]));
                v[j] = k.rstd[j] * (__builtin_fmaf(dz, k.gamma[j], -c1[j]) - h * c2[j]);
            }
            store8<IO, true>(dx + e + u * more, p.wide, v);
        }
    }
}

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

template <class IO, int ACT>
hipError_t forward(const GnormArgs& a, const void* x, void* y, float* mean, float* rstd, float eps, void* ws, hipStream_t st)
{
    using T = typename IO::T;
    const Walk w = walk(a.B, a.S, a.C);
    dim3 g, gg;
    hipError_t e = launch_grid((uint64_t)a.B * w.parts * w.slabs, GT, &g);
    if (e == hipSuccess) e = launch_grid((uint64_t)a.B * a.G, 64, &gg);
    if (e != hipSuccess) return e;
    float* part = (float*)ws;
    hipLaunchKernelGGL(gnorm_stats_kernel<IO>, g, dim3(GT), 0, st, (const T*)x, part, a.S, a.C, w);
    hipLaunchKernelGGL(gnorm_group_kernel, gg, dim3(64), 0, st, (const float*)part, mean, rstd, a.S, a.C, (uint32_t)a.G, w.parts, w.per, eps);
    hipLaunchKernelGGL((gnorm_apply_kernel<IO, ACT>), g, dim3(GT), 0, st, (const T*)x, (T*)y, (const float*)mean, (const float*)rstd, a.gamma,
                       a.beta, a.S, a.C, (uint32_t)a.G, w);
    return hipGetLastError();
}

template <class IO, int ACT>
hipError_t backward(const GnormArgs& a, const void* dy, const void* x, const float* mean, const float* rstd, void* dx, float* dgamma,
                    float* dbeta, void* ws, hipStream_t st)
{
    using T = typename IO::T;
    const Walk w = walk(a.B, a.S, a.C);
    dim3 g, gg;
    hipError_t e = launch_grid((uint64_t)a.B * w.parts * w.slabs, GT, &g);
    if (e == hipSuccess) e = launch_grid((uint64_t)(a.C + RC - 1) / RC + ((uint64_t)a.B * a.G + RT / 64 - 1) / (RT / 64), RT, &gg);
    if (e != hipSuccess) return e;
    float* part = (float*)ws;
    float* s1 = (float*)((char*)ws + up256(part_rows(a.B, a.S, a.C) * 2 * a.C * sizeof(float)));
    float* s2 = s1 + a.B * a.G;
    hipLaunchKernelGGL((gnorm_sums_kernel<IO, ACT>), g, dim3(GT), 0, st, (const T*)dy, (const T*)x, mean, rstd, a.gamma, a.beta, part, a.S,
                       a.C, (uint32_t)a.G, w);
    hipLaunchKernelGGL(gnorm_gather_kernel, gg, dim3(RT), 0, st, (const float*)part, a.gamma, s1, s2, dgamma, dbeta, a.B, a.C, (uint32_t)a.G,
                       w.parts);
    if (dx)
        hipLaunchKernelGGL((gnorm_dx_kernel<IO, ACT>), g, dim3(GT), 0, st, (const T*)dy, (const T*)x, mean, rstd, a.gamma, a.beta,
                           (const float*)s1, (const float*)s2, (T*)dx, a.S, a.C, (uint32_t)a.G, (float)(1.0 / ((double)a.S * (a.C / a.G))), w);
    return hipGetLastError();
}

template <class IO, class F>
hipError_t by_act(int act, F&& f)
{
    switch (act) {
        case LONGCONV_ACT_SILU: return f(std::integral_constant<int, LONGCONV_ACT_SILU>());
        case LONGCONV_ACT_GELU: return f(std::integral_constant<int, LONGCONV_ACT_GELU>());
        case LONGCONV_ACT_RELU: return f(std::integral_constant<int, LONGCONV_ACT_RELU>());
        default: return f(std::integral_constant<int, LONGCONV_ACT_NONE>());
    }
}

}  // namespace

size_t gnorm_workspace_bytes(int64_t B, int64_t S, int64_t C, int64_t G, int io, int backward)
{
    return up256(part_rows(B, S, C) * 2 * C * sizeof(float)) + (backward ? up256((size_t)B * G * 2 * sizeof(float)) : 0);
}

hipError_t gnorm_fwd(const GnormArgs& a, const void* x, void* y, float* mean, float* rstd, float eps, void* ws, hipStream_t st)
{
    const auto run = [&](auto io) {
        using IO = decltype(io);
        return by_act<IO>(a.act, [&](auto act) { return forward<IO, decltype(act)::value>(a, x, y, mean, rstd, eps, ws, st); });
    };
    return a.io == LONGCONV_F32 ? run(IoF32()) : a.io == LONGCONV_F16 ? run(IoF16()) : run(IoBF16());
}

hipError_t gnorm_bwd(const GnormArgs& a, const void* dy, const void* x, const float* mean, const float* rstd, void* dx, float* dgamma,
                     float* dbeta, void* ws, hipStream_t st)
{
    const auto run = [&](auto io) {
        using IO = decltype(io);
        return by_act<IO>(a.act,
                          [&](auto act) { return backward<IO, decltype(act)::value>(a, dy, x, mean, rstd, dx, dgamma, dbeta, ws, st); });
    };
    return a.io == LONGCONV_F32 ? run(IoF32()) : a.io == LONGCONV_F16 ? run(IoF16()) : run(IoBF16());
}

}  // namespace lc
