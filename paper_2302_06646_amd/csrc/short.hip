// Short causal convolution of each head with its own few taps, with bias and activation, in the convolution's layout [B,H,N]:
//     z[t] = bias + sum_{j < taps} k[j] x[t - j],      y = act(z)
// with the `taps - 1` inputs before a sequence's first as its state (zeros without one), its backward pass
//     dz = dy act'(z),   dx[t] = sum_j k[j] dz[t + j],   dk[j] = sum_{b,t} dz[t] x[t - j],   dbias = sum_{b,t} dz,
// z made again from x, and the form for one new input of each sequence.
//
// Memory and vector instructions side by side bound both passes.  16 x 1024 rows of 1024, bf16, silu, eight sets of tensors in turn: forward, which reads
// x and writes y, 16.5 us (4.1 TB/s; a copy of such a tensor 14.0, its vector instructions 12.5 by the counter); backward, which reads x and dy and
// writes dx, 27.8 us (3.6 TB/s; a sum of two such tensors 19.5, its vector instructions 20).  Results are not read again soon: with plain stores the
// forward pass took 20 us.  Places at and behind a sequence's end read as zeros, whatever lies there.
#include "act.hpp"
#include "vec8.hpp"

namespace lc {
namespace {

constexpr int ST = 256;                   // threads of a workgroup
constexpr int SUMS = SHORT_TAPS + 1;      // of dk and dbias

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

// A thread makes a piece of eight neighbouring outputs from its own piece and the neighbours' (which lie in the cache: their threads
// ask for them too), pieces of all rows one behind the other.  W: taps are at most W.  P: pieces of a row
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
    acts_by(a.act, z);
#pragma unroll
    for (int i = 0; i < VE; ++i) z[i] = t0 + i < len ? z[i] : 0.f;
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

// The gradients of eight places from dz of them and of the next W - 1, and the inputs v[8] .. v[15] there with those before
template <class IO, int W>
__device__ __forceinline__ void grads(const ShortArgs& a, const float (&k)[W], const float* dz, const float* v, int64_t t0, int64_t len, size_t row,
                                      const typename IO::T* dlast, typename IO::T* dx, typename IO::T* dstate, float (&sum)[W], float& sum_bias)
{
    using T = typename IO::T;
    float g[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) g[i] = 0.f;
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
    if (lr && t0 + VE + a.taps > len)      // the last state's inputs are those of places len - taps + 1 .. len - 1
#pragma unroll
        for (int i = 0; i < VE; ++i) {
            const int64_t j = t0 + i - len + a.taps - 1;
            if (j >= 0 && t0 + i < len) g[i] += IO::ld(lr, j);
        }
    const int64_t n = a.N - t0;
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

// A workgroup's sums of dk and dbias: across a wave, then across the four, always in the same order; to `part`, or where a head has one part
// to their place at once
template <int W>
__device__ __forceinline__ void put_sums(const ShortArgs& a, const float (&sum)[W], float sum_bias, uint32_t h, uint32_t q, uint32_t parts, float* part,
                                         float* dk, float* dbias)
{
    __shared__ float all[ST / 64][SUMS];
#pragma unroll
    for (int j = 0; j <= W; ++j) {
        float s = j < W ? sum[j < W ? j : 0] : sum_bias;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
        if (threadIdx.x % 64 == 0) all[threadIdx.x / 64][j] = s;
    }
    __syncthreads();
    const int j = threadIdx.x;
    if (j > W) return;
    const float s = (all[0][j] + all[1][j]) + (all[2][j] + all[3][j]);
    if (parts > 1) part[((size_t)h * parts + q) * SUMS + j] = s;
    else if (j == W) {
        if (dbias) dbias[h] = s;
    } else if (j < a.taps && dk) dk[(size_t)h * a.taps + j] = s;
}

template <class IO>
__device__ __forceinline__ void zeros8(typename IO::T* p, int n)
{
    const float z[VE] = {};
    store8<IO, true>(p, n, z);
}

// A workgroup takes part blockIdx.x % parts of head blockIdx.x / parts: `per` pieces of the B P of that head.
template <class IO, int W>
__global__ __launch_bounds__(ST) void short_bwd_kernel(ShortArgs a, const typename IO::T* __restrict__ dy, const typename IO::T* __restrict__ x,
                                                       const typename IO::T* __restrict__ state, const typename IO::T* __restrict__ dlast,
                                                       typename IO::T* __restrict__ dx, typename IO::T* __restrict__ dstate,
                                                       float* __restrict__ part, float* __restrict__ dk, float* __restrict__ dbias, uint32_t parts,
                                                       int64_t per, int64_t P)
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
        float v[3 * VE], dz[2 * VE];
        if (t0 >= len && !(t0 == 0 && dstate)) {      // behind the end
            if (dx) zeros8<IO>(dx + row * a.N + t0, n < VE ? (int)n : VE);
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
            float z[VE + W - 1];
#pragma unroll
            for (int i = 0; i < VE + W - 1; ++i) {
                z[i] = bias;
#pragma unroll
                for (int j = 0; j < W; ++j)
                    if (j < a.taps) z[i] = __builtin_fmaf(k[j], v[VE + i - j], z[i]);
            }
            slopes_by(a.act, z);
#pragma unroll
            for (int i = 0; i < VE + W - 1; ++i) dz[i] = t0 + i < len ? dz[i] * z[i] : 0.f;
        }
        grads<IO, W>(a, k, dz, v, t0, len, row, dlast, dx, dstate, sum, sum_bias);
    }
    put_sums(a, sum, sum_bias, h, q, parts, part, dk, dbias);
}

// ---- long rows, backward: a wave takes UNIT neighbouring pieces of one row, 64 at a time, so that head, taps and length are one for all its lanes ------
constexpr int CHUNKS = 2, UNIT = 64 * CHUNKS;

// v of the lane before, or behind; `edge` in the lane that has none
__device__ __forceinline__ float of_before(float edge, float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(edge), (int)__float_as_uint(v), 0x138, 0xf, 0xf, false));
}
__device__ __forceinline__ float of_behind(float edge, float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(edge), (int)__float_as_uint(v), 0x130, 0xf, 0xf, false));
}
__device__ __forceinline__ float of_lane(float v, int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane)); }

// eight elements of a row from place t0 on as they lie in memory, zero behind the row's N
template <class IO>
__device__ __forceinline__ void ask8(const typename IO::T* row, int64_t t0, int64_t N, Raw8<IO>& r)
{
    if (t0 + VE <= N) r.load(row + t0);
    else load_raw<IO>(row + t0, t0 < N ? (int)(N - t0) : 0, r);
}
// zero from place `len` on; `ends`: len is within the wave's places
template <class IO>
__device__ __forceinline__ void inside(const Raw8<IO>& r, int64_t t0, int64_t len, bool ends, float* v)
{
    float w[VE];
    r.get(w);
#pragma unroll
    for (int i = 0; i < VE; ++i) v[i] = w[i];
    if (ends) {
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = t0 + i < len ? v[i] : 0.f;
    }
}
// e[d - 1] <- the input d places before `base`
template <class IO, int W>
__device__ __forceinline__ void edge(const typename IO::T* row, const typename IO::T* state, int taps, int64_t base, float (&e)[W - 1])
{
#pragma unroll
    for (int d = 1; d < W; ++d) e[d - 1] = base > 0 ? IO::ld(row, base - d) : state && d < taps ? IO::ld(state, taps - 1 - d) : 0.f;
}
__device__ __forceinline__ int64_t quotient(int64_t n, int64_t d)      // both below 2^31 as a rule
{
    return (n | d) >> 32 ? n / d : (int64_t)((uint32_t)n / (uint32_t)d);
}

// A workgroup takes part blockIdx.x % parts of head blockIdx.x / parts: of the head's units every 4 parts'th by a wave, the next one asked for
// before this one is worked on, its 64 pieces from the last to the first, so that dz of the places behind is there.
template <class IO, int W>
__global__ __launch_bounds__(ST) void short_rows_bwd_kernel(ShortArgs a, const typename IO::T* __restrict__ dy, const typename IO::T* __restrict__ x,
                                                            const typename IO::T* __restrict__ state, const typename IO::T* __restrict__ dlast,
                                                            typename IO::T* __restrict__ dx, typename IO::T* __restrict__ dstate,
                                                            float* __restrict__ part, float* __restrict__ dk, float* __restrict__ dbias,
                                                            uint32_t parts, int64_t units, int64_t each)
{
    using T = typename IO::T;
    const uint32_t h = blockIdx.x / parts, q = blockIdx.x - h * parts;
    const int lane = threadIdx.x & 63;
    float k[W], sum[W], sum_bias = 0.f;
    const float bias = a.bias ? a.bias[h] : 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) {
        k[j] = j < a.taps ? a.k[(size_t)h * a.taps + j] : 0.f;
        sum[j] = 0.f;
    }
    struct Unit {
        int64_t base, len;
        size_t row;
        Raw8<IO> x[CHUNKS], dy[CHUNKS];
        float e[W - 1];
    };
    const auto ask = [&](int64_t u, Unit& r) {
        const int64_t b = quotient(u, each);
        r.base = (u - b * each) * (UNIT * VE);
        r.row = (size_t)b * a.H + h;
        r.len = length_of(a.lengths, b, a.N);
        const T *xr = x + r.row * a.N, *dr = dy + r.row * a.N;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) {
            ask8<IO>(xr, r.base + (64 * c + lane) * VE, a.N, r.x[c]);
            ask8<IO>(dr, r.base + (64 * c + lane) * VE, a.N, r.dy[c]);
        }
        edge<IO, W>(xr, state ? state + r.row * (a.taps - 1) : nullptr, a.taps, r.base, r.e);
    };
    const int64_t stride = 4 * (int64_t)parts;
    int64_t u = (int64_t)q * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Unit next;
    if (u < units) ask(u, next);
    for (; u < units; u += stride) {
        const Unit r = next;
        if (u + stride < units) ask(u + stride, next);
        float behind[W - 1];      // dz of the first places behind
#pragma unroll
        for (int i = 0; i < W - 1; ++i) behind[i] = 0.f;
        const int64_t end = r.base + UNIT * VE;
        if (end < r.len) {      // they are another unit's: a lane makes each
            const int64_t t = end + lane < r.len ? end + lane : r.len - 1;
            const T* xr = x + r.row * a.N;
            float z[1] = {bias};
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (j < a.taps) z[0] = __builtin_fmaf(k[j], IO::ld(xr, t - j), z[0]);
            slopes_by(a.act, z);
            const float dz = end + lane < r.len ? IO::ld(dy + r.row * a.N, t) * z[0] : 0.f;
#pragma unroll
            for (int i = 0; i < W - 1; ++i) behind[i] = of_lane(dz, i);
        }
#pragma unroll
        for (int c = CHUNKS - 1; c >= 0; --c) {
            const int64_t here = r.base + 64 * c * VE, t0 = here + lane * VE, n = a.N - t0;
            if (here >= a.N) continue;
            if (here >= r.len && !(here == 0 && dstate)) {      // behind the end
                if (dx) zeros8<IO>(dx + r.row * a.N + t0, n < VE ? (int)n : VE);
                continue;
            }
            const bool ends = here + 64 * VE > r.len;
            float v[2 * VE], dz[2 * VE];
            inside<IO>(r.x[c], t0, r.len, ends, v + VE);
            inside<IO>(r.dy[c], t0, r.len, ends, dz);
            float before[VE];
            if (c > 0) r.x[c > 0 ? c - 1 : 0].get(before);
#pragma unroll
            for (int d = 1; d < W; ++d) v[VE - d] = of_before(c > 0 ? of_lane(before[VE - d], 63) : r.e[d - 1], v[2 * VE - d]);
            if (a.act != LONGCONV_ACT_NONE) {
                float z[VE];
#pragma unroll
                for (int i = 0; i < VE; ++i) z[i] = bias;
#pragma unroll
                for (int j = 0; j < W; ++j)
                    if (j < a.taps) {
#pragma unroll
                        for (int i = 0; i < VE; ++i) z[i] = __builtin_fmaf(k[j], v[VE + i - j], z[i]);
                    }
                slopes_by(a.act, z);
#pragma unroll
                for (int i = 0; i < VE; ++i) dz[i] *= z[i];
                if (ends) {
#pragma unroll
                    for (int i = 0; i < VE; ++i) dz[i] = t0 + i < r.len ? dz[i] : 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < W - 1; ++i) {
                dz[VE + i] = of_behind(behind[i], dz[i]);
                behind[i] = of_lane(dz[i], 0);
            }
            grads<IO, W>(a, k, dz, v, t0, r.len, r.row, dlast, dx, dstate, sum, sum_bias);
        }
    }
    put_sums(a, sum, sum_bias, h, q, parts, part, dk, dbias);
}

// dk and dbias from the parts, a wave each; W as in short_bwd_kernel, whose sum W is the bias's
__global__ __launch_bounds__(ST) void short_sums_kernel(const float* __restrict__ part, float* __restrict__ dk, float* __restrict__ dbias, int64_t H,
                                                        int taps, int W, uint32_t parts)
{
    const int64_t id = (int64_t)blockIdx.x * (ST / 64) + (threadIdx.x >> 6), h = id / (taps + 1);
    if (h >= H) return;
    const int j = (int)(id - h * (taps + 1)), at = j < taps ? j : W;
    float s = 0.f;
    for (uint32_t q = threadIdx.x & 63; q < parts; q += 64) s += part[((size_t)h * parts + q) * SUMS + at];
#pragma unroll
    for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
    if (threadIdx.x & 63) return;
    if (j < taps) {
        if (dk) dk[h * taps + j] = s;
    } else if (dbias) dbias[h] = s;
}

// One new place of each sequence, a thread a head: 4 us with its launch for 64 x 1024 of them.
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

// Backward pass: rows of 64 pieces and more, the last 64 of them three quarters full and more, go by whole waves.  us, so and by pieces of all rows:
// 16 x 1024 rows of 1024, bf16, 28.8 and 37.5; 7 x 193 rows of 49 pieces, fp32, 10.9 and 9.9.  Forward the two took the same time.
bool long_rows(int64_t N)
{
    const int64_t P = (N + VE - 1) / VE, lanes = (P + 63) / 64 * 64;
    return P >= 64 && P * 4 >= lanes * 3;
}

// parts of a head in the backward pass: 1024 workgroups in all, if there are four units, or a thousand pieces, of that head for each
uint32_t short_parts(int64_t B, int64_t H, int64_t N)
{
    const int64_t P = (N + VE - 1) / VE, most = long_rows(N) ? (B * ((P + UNIT - 1) / UNIT) + 3) / 4 : (B * P + 4 * ST - 1) / (4 * ST);
    const int64_t parts = (1024 + H - 1) / H;
    return (uint32_t)(parts < most ? parts : most);
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
    const int64_t P = (a.N + VE - 1) / VE, each = (P + UNIT - 1) / UNIT;
    const uint32_t parts = short_parts(a.B, a.H, a.N);
    dim3 g;
    hipError_t e = launch_grid((uint64_t)a.H * parts, ST, &g);
    if (e != hipSuccess) return e;
    const T *dy = (const T*)d.dy, *x = (const T*)d.x, *state = (const T*)d.state, *dlast = (const T*)d.dlast;
    if (long_rows(a.N))
        hipLaunchKernelGGL((short_rows_bwd_kernel<IO, W>), g, dim3(ST), 0, st, a, dy, x, state, dlast, (T*)d.dx, (T*)d.dstate, (float*)ws, d.dk, d.dbias,
                           parts, a.B * each, each);
    else
        hipLaunchKernelGGL((short_bwd_kernel<IO, W>), g, dim3(ST), 0, st, a, dy, x, state, dlast, (T*)d.dx, (T*)d.dstate, (float*)ws, d.dk, d.dbias,
                           parts, (a.B * P + parts - 1) / parts, P);
    e = hipGetLastError();
    if (e != hipSuccess || parts == 1 || (!d.dk && !d.dbias)) return e;
    hipLaunchKernelGGL(short_sums_kernel, dim3((unsigned)((a.H * (a.taps + 1) + ST / 64 - 1) / (ST / 64))), dim3(ST), 0, st, (const float*)ws, d.dk,
                       d.dbias, a.H, a.taps, W, parts);
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
