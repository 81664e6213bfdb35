// Short causal convolution of each head with its own few taps, with bias and activation, in the convolution's layout [B,H,N]:
//     z[t] = bias + sum_{j < taps} k[j] x[t - j],      y = act(z)
// with the `taps - 1` inputs before a sequence's first as its state (zeros without one), its backward pass
//     dz = dy act'(z),   dx[t] = sum_j k[j] dz[t + j],   dk[j] = sum_{b,t} dz[t] x[t - j],   dbias = sum_{b,t} dz,
// z made again from x, and the form for one new input of each sequence.
//
// A thread makes a piece of eight neighbouring outputs from its own piece and the neighbours' (which lie in the cache: their threads ask
// for them too).  Places at and behind a sequence's end read as zeros, whatever lies there.
#include "act.hpp"
#include "vec8.hpp"

namespace lc {
namespace {

constexpr int ST = 256;                   // threads of a workgroup
constexpr int SUMS = SHORT_TAPS + 1;      // of dk and dbias

__device__ __forceinline__ float act_by(int act, float z)
{
    switch (act) {
        case LONGCONV_ACT_SILU: return act_of<LONGCONV_ACT_SILU>(z);
        case LONGCONV_ACT_GELU: return act_of<LONGCONV_ACT_GELU>(z);
        case LONGCONV_ACT_RELU: return act_of<LONGCONV_ACT_RELU>(z);
        default: return z;
    }
}
__device__ __forceinline__ float slope_by(int act, float z)
{
    switch (act) {
        case LONGCONV_ACT_SILU: return slope_of<LONGCONV_ACT_SILU>(z);
        case LONGCONV_ACT_GELU: return slope_of<LONGCONV_ACT_GELU>(z);
        case LONGCONV_ACT_RELU: return slope_of<LONGCONV_ACT_RELU>(z);
        default: return 1.f;
    }
}

__device__ __forceinline__ int64_t length_of(const int64_t* lengths, int64_t b, int64_t N)
{
    if (!lengths) return N;
    const int64_t n = lengths[b];
    return n < 0 ? 0 : n > N ? N : n;
}

// v[8 - d] <- the input d places before t0, d = 1 .. taps - 1 (the others are not looked at)
template <class IO>
__device__ __forceinline__ void before(const typename IO::T* row, const typename IO::T* state, int taps, int64_t t0, float* v)
{
    if (t0 > 0) {
        float w[VE];
        load8<IO>(row + t0 - VE, VE, w);
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = w[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < VE; ++i) v[i] = 0.f;
    if (state)
#pragma unroll
        for (int d = 1; d < SHORT_TAPS; ++d)
            if (d < taps) v[VE - d] = IO::ld(state, taps - 1 - d);
}

// eight elements of a row from place t0 on, zero from place `len` on
template <class IO>
__device__ __forceinline__ void inside(const typename IO::T* row, int64_t t0, int64_t N, int64_t len, float* v)
{
    float w[VE];
    const int64_t n = N - t0;
    load8<IO>(row + t0, n < VE ? (int)n : VE, w);
#pragma unroll
    for (int i = 0; i < VE; ++i) v[i] = t0 + i < len ? w[i] : 0.f;
}

// W: taps are at most W.  P: pieces of a row
template <class IO, int W, class I>
__global__ __launch_bounds__(ST) void short_fwd_kernel(ShortArgs a, const typename IO::T* __restrict__ x, const typename IO::T* state,
                                                       typename IO::T* __restrict__ y, typename IO::T* last, I pieces, I P)
{
    using T = typename IO::T;
    const I id = (I)blockIdx.x * ST + threadIdx.x;
    if (id >= pieces) return;
    const I row = id / P;
    const int64_t t0 = (int64_t)(id - row * P) * VE;
    const uint32_t h = (uint32_t)(row % (I)a.H);
    const int64_t len = length_of(a.lengths, (int64_t)(row / (I)a.H), a.N);
    const T* xr = x + (size_t)row * a.N;
    const T* sr = state ? state + (size_t)row * (a.taps - 1) : nullptr;
    float v[2 * VE];
    before<IO>(xr, sr, a.taps, t0, v);
    inside<IO>(xr, t0, a.N, len, v + VE);
    const float bias = a.bias ? a.bias[h] : 0.f;
    float z[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) z[i] = bias;
#pragma unroll
    for (int j = 0; j < W; ++j)
        if (j < a.taps) {
            const float k = a.k[(size_t)h * a.taps + j];
#pragma unroll
            for (int i = 0; i < VE; ++i) z[i] = __builtin_fmaf(k, v[VE + i - j], z[i]);
        }
#pragma unroll
    for (int i = 0; i < VE; ++i) z[i] = t0 + i < len ? act_by(a.act, z[i]) : 0.f;
    const int64_t n = a.N - t0;
    store8<IO, true>(y + (size_t)row * a.N + t0, n < VE ? (int)n : VE, z);
    if (t0 == 0 && last) {      // (read before any is written: `last` may be `state`)
        T w[SHORT_TAPS];
#pragma unroll
        for (int j = 0; j < SHORT_TAPS - 1; ++j)
            if (j < a.taps - 1) {
                const int64_t at = len + j - (a.taps - 1);
                if (at >= 0) w[j] = xr[at];
                else if (sr) w[j] = sr[len + j];
                else IO::st(w, j, 0.f);
            }
#pragma unroll
        for (int j = 0; j < SHORT_TAPS - 1; ++j)
            if (j < a.taps - 1) last[(size_t)row * (a.taps - 1) + j] = w[j];
    }
}

// A workgroup takes part blockIdx.x % parts of head blockIdx.x / parts: `per` pieces of the B P of that head.
template <class IO, int W>
__global__ __launch_bounds__(ST) void short_bwd_kernel(ShortArgs a, const typename IO::T* __restrict__ dy, const typename IO::T* __restrict__ x,
                                                       const typename IO::T* __restrict__ state, const typename IO::T* __restrict__ dlast,
                                                       typename IO::T* __restrict__ dx, typename IO::T* __restrict__ dstate,
                                                       float* __restrict__ part, uint32_t parts, int64_t per, int64_t P)
{
    using T = typename IO::T;
    const uint32_t h = blockIdx.x / parts, q = blockIdx.x - h * parts;
    float k[W], sum[W], sum_bias = 0.f;
    const float bias = a.bias ? a.bias[h] : 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) {
        k[j] = j < a.taps ? a.k[(size_t)h * a.taps + j] : 0.f;
        sum[j] = 0.f;
    }
    const int64_t first = (int64_t)q * per, end = first + per < a.B * P ? first + per : a.B * P;
    for (int64_t id = first + threadIdx.x; id < end; id += ST) {
        const int64_t b = id / P, t0 = (id - b * P) * VE, len = length_of(a.lengths, b, a.N);
        const size_t row = (size_t)b * a.H + h;
        const T* xr = x + row * a.N;
        const int64_t n = a.N - t0;
        float v[3 * VE], dz[2 * VE], g[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) g[i] = 0.f;
        if (t0 >= len && !(t0 == 0 && dstate)) {      // behind the end
            if (dx) store8<IO, true>(dx + row * a.N + t0, n < VE ? (int)n : VE, g);
            continue;
        }
        before<IO>(xr, state ? state + row * (a.taps - 1) : nullptr, a.taps, t0, v);
        inside<IO>(xr, t0, a.N, len, v + VE);
        inside<IO>(dy + row * a.N, t0, a.N, len, dz);
        if (t0 + VE < len) {
            inside<IO>(xr, t0 + VE, a.N, len, v + 2 * VE);
            inside<IO>(dy + row * a.N, t0 + VE, a.N, len, dz + VE);
        } else {
#pragma unroll
            for (int i = 0; i < VE; ++i) v[2 * VE + i] = dz[VE + i] = 0.f;
        }
        if (a.act != LONGCONV_ACT_NONE) {
#pragma unroll
            for (int i = 0; i < VE + W - 1; ++i) {
                float z = bias;
#pragma unroll
                for (int j = 0; j < W; ++j)
                    if (j < a.taps) z = __builtin_fmaf(k[j], v[VE + i - j], z);
                dz[i] = t0 + i < len ? dz[i] * slope_by(a.act, z) : 0.f;
            }
        }
        if (t0 < len) {
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (j < a.taps) {
#pragma unroll
                    for (int i = 0; i < VE; ++i) {
                        g[i] = __builtin_fmaf(k[j], dz[i + j], g[i]);
                        sum[j] = __builtin_fmaf(dz[i], v[VE + i - j], sum[j]);
                    }
                }
#pragma unroll
            for (int i = 0; i < VE; ++i) sum_bias += dz[i];
        }
        const T* lr = dlast ? dlast + row * (a.taps - 1) : nullptr;
        if (lr)      // the last state's inputs are those of places len - taps + 1 .. len - 1
#pragma unroll
            for (int i = 0; i < VE; ++i) {
                const int64_t j = t0 + i - len + a.taps - 1;
                if (j >= 0 && t0 + i < len) g[i] += IO::ld(lr, j);
            }
        if (dx) store8<IO, true>(dx + row * a.N + t0, n < VE ? (int)n : VE, g);
        if (t0 == 0 && dstate)      // dstate[i] is the input i - (taps - 1) places behind the first
#pragma unroll
            for (int i = 0; i < W - 1; ++i)
                if (i < a.taps - 1) {
                    float s = 0.f;
#pragma unroll
                    for (int j = 1; j < W; ++j) {
                        const int t = i - (a.taps - 1) + j;
                        if (j < a.taps && t >= 0) {
#pragma unroll
                            for (int r = 0; r < W - 1; ++r)
                                if (r == t) s = __builtin_fmaf(k[j], dz[r], s);
                        }
                    }
                    if (lr && i >= len) s += IO::ld(lr, i - len);
                    IO::st(dstate + row * (a.taps - 1), i, s);
                }
    }
    // the workgroup's sums: across a wave, then across the four, always in the same order
    __shared__ float all[ST / 64][SUMS];
#pragma unroll
    for (int j = 0; j <= W; ++j) {
        float s = j < W ? sum[j < W ? j : 0] : sum_bias;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
        if (threadIdx.x % 64 == 0) all[threadIdx.x / 64][j] = s;
    }
    __syncthreads();
    if (threadIdx.x <= W) part[((size_t)h * parts + q) * SUMS + threadIdx.x] =
        (all[0][threadIdx.x] + all[1][threadIdx.x]) + (all[2][threadIdx.x] + all[3][threadIdx.x]);
}

// dk and dbias from the parts; W as in short_bwd_kernel, whose sum W is the bias's
__global__ void short_sums_kernel(const float* __restrict__ part, float* __restrict__ dk, float* __restrict__ dbias, int64_t H, int taps, int W,
                                  uint32_t parts)
{
    const uint32_t id = blockIdx.x * blockDim.x + threadIdx.x, h = id / (uint32_t)SUMS, j = id % (uint32_t)SUMS;
    if (h >= H || j > (uint32_t)taps) return;
    const uint32_t at = j < (uint32_t)taps ? j : (uint32_t)W;
    float s = 0.f;
    for (uint32_t q = 0; q < parts; ++q) s += part[((size_t)h * parts + q) * SUMS + at];
    if (j < (uint32_t)taps) {
        if (dk) dk[(size_t)h * taps + j] = s;
    } else if (dbias) dbias[h] = s;
}

template <class IO>
__global__ __launch_bounds__(ST) void short_step_kernel(ShortArgs a, const typename IO::T* __restrict__ x, typename IO::T* __restrict__ state,
                                                        typename IO::T* __restrict__ y)
{
    const int64_t id = (int64_t)blockIdx.x * ST + threadIdx.x;
    if (id >= a.B * a.H) return;
    const uint32_t h = (uint32_t)(id % a.H);
    typename IO::T* sr = state + (size_t)id * (a.taps - 1);
    typename IO::T w[SHORT_TAPS];
    w[0] = x[id];
#pragma unroll
    for (int j = 1; j < SHORT_TAPS; ++j)
        if (j < a.taps) w[j] = sr[a.taps - 1 - j];
    float z = a.bias ? a.bias[h] : 0.f;
#pragma unroll
    for (int j = 0; j < SHORT_TAPS; ++j)
        if (j < a.taps) z = __builtin_fmaf(a.k[(size_t)h * a.taps + j], IO::ld(w, j), z);
    IO::st(y, id, act_by(a.act, z));
#pragma unroll
    for (int j = 0; j < SHORT_TAPS - 1; ++j)
        if (j < a.taps - 1) sr[a.taps - 2 - j] = w[j];
}

// parts of a head in the backward pass: of four pieces a thread or more, and 2048 workgroups in all where there are that many pieces
uint32_t short_parts(int64_t B, int64_t H, int64_t N)
{
    const int64_t pieces = B * ((N + VE - 1) / VE);
    int64_t parts = (2048 + H - 1) / H;
    const int64_t most = (pieces + 4 * ST - 1) / (4 * ST);
    if (parts > most) parts = most;
    return (uint32_t)(parts < 1 ? 1 : parts);
}

template <class IO, int W>
hipError_t fwd(const ShortArgs& a, const void* x, const void* state, void* y, void* last, hipStream_t st)
{
    using T = typename IO::T;
    const int64_t P = (a.N + VE - 1) / VE, pieces = a.B * a.H * P;
    dim3 g;
    const hipError_t e = launch_grid((uint64_t)((pieces + ST - 1) / ST), ST, &g);
    if (e != hipSuccess) return e;
    if (pieces < (int64_t(1) << 31))
        hipLaunchKernelGGL((short_fwd_kernel<IO, W, uint32_t>), g, dim3(ST), 0, st, a, (const T*)x, (const T*)state, (T*)y, (T*)last, (uint32_t)pieces,
                           (uint32_t)P);
    else
        hipLaunchKernelGGL((short_fwd_kernel<IO, W, uint64_t>), g, dim3(ST), 0, st, a, (const T*)x, (const T*)state, (T*)y, (T*)last, (uint64_t)pieces,
                           (uint64_t)P);
    return hipGetLastError();
}
template <class IO, int W>
hipError_t bwd(const ShortArgs& a, const ShortGrads& d, void* ws, hipStream_t st)
{
    using T = typename IO::T;
    const int64_t P = (a.N + VE - 1) / VE;
    const uint32_t parts = short_parts(a.B, a.H, a.N);
    dim3 g;
    hipError_t e = launch_grid((uint64_t)a.H * parts, ST, &g);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((short_bwd_kernel<IO, W>), g, dim3(ST), 0, st, a, (const T*)d.dy, (const T*)d.x, (const T*)d.state, (const T*)d.dlast, (T*)d.dx,
                       (T*)d.dstate, (float*)ws, parts, (a.B * P + parts - 1) / parts, P);
    e = hipGetLastError();
    if (e != hipSuccess || (!d.dk && !d.dbias)) return e;
    hipLaunchKernelGGL(short_sums_kernel, dim3((unsigned)((a.H * SUMS + 255) / 256)), dim3(256), 0, st, (const float*)ws, d.dk, d.dbias, a.H, a.taps, W,
                       parts);
    return hipGetLastError();
}
template <class IO>
hipError_t step(const ShortArgs& a, const void* x, void* state, void* y, hipStream_t st)
{
    using T = typename IO::T;
    dim3 g;
    const hipError_t e = launch_grid((uint64_t)((a.B * a.H + ST - 1) / ST), ST, &g);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(short_step_kernel<IO>, g, dim3(ST), 0, st, a, (const T*)x, (T*)state, (T*)y);
    return hipGetLastError();
}

template <class F>
hipError_t by_io(int io, F&& f)
{
    if (io == LONGCONV_F32) return f(IoF32());
    return io == LONGCONV_F16 ? f(IoF16()) : f(IoBF16());
}

}  // namespace

size_t short_workspace_bytes(int64_t B, int64_t H, int64_t N) { return (size_t)H * short_parts(B, H, N) * SUMS * sizeof(float); }

hipError_t short_fwd(const ShortArgs& a, const void* x, const void* state, void* y, void* last, hipStream_t st)
{
    return by_io(a.io, [&](auto io) {
        using IO = decltype(io);
        return a.taps <= 4 ? fwd<IO, 4>(a, x, state, y, last, st) : fwd<IO, SHORT_TAPS>(a, x, state, y, last, st);
    });
}
hipError_t short_bwd(const ShortArgs& a, const ShortGrads& d, void* ws, hipStream_t st)
{
    return by_io(a.io, [&](auto io) {
        using IO = decltype(io);
        return a.taps <= 4 ? bwd<IO, 4>(a, d, ws, st) : bwd<IO, SHORT_TAPS>(a, d, ws, st);
    });
}
hipError_t short_step(const ShortArgs& a, const void* x, void* state, void* y, hipStream_t st)
{
    return by_io(a.io, [&](auto io) { return step<decltype(io)>(a, x, state, y, st); });
}

}  // namespace lc
