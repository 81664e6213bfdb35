// Group norm with an activation, channels last: x [B,S,C], groups of C / G neighbouring channels over all S positions,
//     xhat = (x - mean) rstd,   z = gamma xhat + beta,   y = act(z)
// and its backward pass, with dz = dy act'(z) and m = S C / G:
//     dbeta = sum dz,   dgamma = sum dz xhat (over b and positions),   dx = rstd (gamma dz - (s1 + xhat s2) / m),
//     s1 = sum gamma dz,   s2 = sum gamma dz xhat over the group.
//
// Sums go by channel first: a thread keeps eight channels and walks over positions, so a group may be of any width, and dgamma, dbeta
// and the group's sums come from the same numbers.  Mean and variance are carried as (mean, sum of squared differences), merged
// pairwise, so a mean that is large against the deviation costs nothing.  All in fp32, in a fixed order.
//
// Forward and backward, 64 x 1024 x 256 in bf16, 32 groups, silu: 51 us (33 for the bytes), groups held by workgroups: kernels of 17 + 33
// + 5; in the backward one loads, vector issue (9.2 million instructions: 17 us at four cycles and 2.1 GHz) and stores follow each other
// in the one workgroup that a compute unit has registers for.
// 16 x 16384 x 256 in fp16, gelu: 216 us, in passes that read x twice and x, dy twice (1.07 GB, 210 us at a copy's rate): kernels of 30
// for the statistics, apply 52 (5.1 TB/s, issue takes 44: 24 million vector instructions), sums 63 (bound by issue, 30 million), dx 69
// (5.9 TB/s).
#pragma once
#include "act.hpp"
#include "vec8.hpp"

namespace lc {
namespace {

constexpr int GT = 512;              // threads
constexpr int SLAB = 64;             // pieces of eight channels of a workgroup, at most
constexpr int GROUPS_WANTED = 1024;  // workgroups of a pass over the tensor
constexpr int AHEAD = 4;             // pieces that a thread asks for before it uses the first

// (n, mean, m2) <- both sets together (the share to the last bit: means of channels differ by as much as the data do)
__device__ __forceinline__ void merge(float& n, float& mean, float& m2, float n2, float mean2, float m22)
{
    if (n2 == 0.f) return;
    const float all = n + n2, d = mean2 - mean, f = n2 / all;
    mean = __builtin_fmaf(d, f, mean);
    m2 += m22 + d * d * n * f;
    n = all;
}

// How a pass walks over a tensor: workgroup (b, part, slab) takes `slices` pieces of eight channels of `per` positions; its threads
// are `rows` positions by `slices`.
struct Walk {
    uint32_t P, slices, slabs, rows, parts;
    uint32_t half;      // the largest power of two below `rows`, 0 for one row
    int64_t per;
};
Walk walk(int64_t B, int64_t S, int64_t C)
{
    Walk w;
    w.P = (uint32_t)((C + VE - 1) / VE);
    w.slices = w.P < SLAB ? w.P : SLAB;
    w.slabs = (w.P + w.slices - 1) / w.slices;
    w.rows = GT / w.slices;
    for (w.half = w.rows > 1; 2 * w.half && 2 * w.half < w.rows; w.half *= 2) {}
    int64_t parts = GROUPS_WANTED / (B * w.slabs);
    const int64_t most = (S + 4 * w.rows - 1) / (4 * w.rows);      // four positions of a thread at least
    if (parts > most) parts = most;
    const int64_t least = (S * C >> 28) + 1;                       // of less than 2^28 elements each: byte offsets fit 31 bits
    if (parts < least) parts = least;
    w.per = (S + parts - 1) / parts;
    w.parts = (uint32_t)((S + w.per - 1) / w.per);
    return w;
}
// most rows (b, part) of partial results there can be: does not fall as B grows
size_t part_rows(int64_t B, int64_t S, int64_t C)
{
    const Walk w = walk(1, S, C);
    const int64_t most = (S + 4 * w.rows - 1) / (4 * w.rows), wanted = GROUPS_WANTED / w.slabs;
    const int64_t some = B > wanted ? B : wanted, least = B + (MAX_ELEMENTS >> 28);      // (parts of 2^28 elements: so many more than B at most)
    const int64_t rows = B * most < some ? B * most : some;
    return (size_t)(rows > least ? rows : least);
}

// the sum over a wave, in every lane: rows of sixteen lanes by permutations within the vector registers, then the four rows
__device__ __forceinline__ float wave_sum(float v)
{
    const auto moved = [](float x, auto control) {
        return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), decltype(control)::value, 0xf, 0xf, false));
    };
    v += moved(v, std::integral_constant<int, 0xB1>());       // neighbours within a pair
    v += moved(v, std::integral_constant<int, 0x4E>());       // pairs within four
    v += moved(v, std::integral_constant<int, 0x141>());      // fours within eight, mirrored
    v += moved(v, std::integral_constant<int, 0x140>());      // eights within sixteen, mirrored
    const auto row = [&](int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane)); };
    return (row(0) + row(16)) + (row(32) + row(48));
}

// How a thread's channels lie: of a row of fewer than eight (loaded by elements); anyhow; all eight in one group, and rows whole pieces,
// which is what C / G a multiple of eight gives and saves the group's numbers in eight copies.
constexpr int NARROW = 0, ANYHOW = 1, ONE = 2;
inline int mode_of(int64_t C, int64_t G) { return C < VE ? NARROW : C / G % VE == 0 ? ONE : ANYHOW; }

// A thread's eight channels.  The last piece of a row ends with the row: it begins `skip` channels early, which belong to the piece
// before, so that every load is whole and inside the tensor.
struct Piece {
    int c, skip, wide;           // first channel; channels of another thread; channels loaded
    bool on;
    uint32_t off, step, end;     // bytes from a part's first element to the thread's first piece; to its next one; to the last there may be
    template <class IO>
    __device__ __forceinline__ void from_row(uint32_t row, uint32_t rows, uint32_t positions, int64_t C)
    {
        const uint32_t size = sizeof(typename IO::T), bytes = (uint32_t)C * size;
        off = row * bytes + (uint32_t)c * size;
        step = rows * bytes;
        end = (positions - 1u) * bytes + (uint32_t)c * size;
    }
    __device__ __forceinline__ bool has(uint32_t o) const { return o <= end; }
    // where a piece is, or the last one of the part where it lies behind that
    template <class T>
    __device__ __forceinline__ T* at(T* base, uint32_t o) const
    {
        const uint32_t in = o < end ? o : end;
        typedef typename std::conditional<std::is_const<T>::value, const char, char>::type Byte;
        return reinterpret_cast<T*>(reinterpret_cast<Byte*>(base) + in);
    }
    __device__ __forceinline__ void set(int slot, bool there, int64_t C)
    {
        on = there && slot * VE < C;
        const int from = on ? slot * VE : 0, last = (int)C - VE;
        c = last < 0 ? 0 : from < last ? from : last;
        skip = from - c;
        wide = C < VE ? (int)C : VE;
    }
    __device__ __forceinline__ bool mine(int j) const { return on && j >= skip && j < wide; }
};
template <class IO, int MODE>
__device__ __forceinline__ void fetch(const typename IO::T* p, const Piece& q, Raw8<IO>& r)
{
    if constexpr (MODE == NARROW) load_raw<IO>(p, q.wide, r);
    else r.load(p);
}
template <class IO, int MODE>
__device__ __forceinline__ void put(typename IO::T* p, const Piece& q, const float (&v)[VE])
{
    if (MODE == ONE || (q.skip == 0 && q.wide == VE)) {
        store8<IO, true>(p, VE, v);
        return;
    }
#pragma unroll
    for (int j = 0; j < VE; ++j)
        if (q.mine(j)) IO::st(p, j, v[j]);
}
// a thread's numbers for its channels, those of others zero, at q[0 .. 7] in the order of the slots of its piece
__device__ __forceinline__ void to_slots(float* q, const Piece& p, const float (&v)[VE])
{
    if (p.skip == 0 && p.on && p.wide == VE) {
        reinterpret_cast<float4*>(q)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4*>(q)[1] = make_float4(v[4], v[5], v[6], v[7]);
        return;
    }
#pragma unroll
    for (int j = 0; j < VE; ++j) q[(j - p.skip) & (VE - 1)] = p.mine(j) ? v[j] : 0.f;
}
// eight parameters; p may be null
__device__ __forceinline__ void load_params(const float* p, const Piece& q, float or_else, float (&v)[VE])
{
#pragma unroll
    for (int j = 0; j < VE; ++j) v[j] = or_else;
    if (p) load8<IoF32>(p + q.c, q.wide, v);
}
// numbers of the eight channels' groups
template <int MODE>
struct Groups {
    float v[MODE == ONE ? 1 : VE];
    __device__ __forceinline__ float& operator[](int j) { return v[MODE == ONE ? 0 : j]; }
    __device__ __forceinline__ float operator[](int j) const { return v[MODE == ONE ? 0 : j]; }
};
// f(j, group of channel j), one division for the eight; channels beyond the last: the last group
template <int MODE, class F>
__device__ __forceinline__ void each_group(int c, uint32_t G, uint32_t D, F&& f)
{
    uint32_t g = (uint32_t)c / D, at = (uint32_t)c - g * D;
    if constexpr (MODE == ONE) f(0, g);
    else
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            f(j, g < G ? g : G - 1);
            if (++at == D) { at = 0; ++g; }
        }
}

// d = x - mean, z = (gamma rstd) d + beta and xhat = rstd d of a thread's channels.  The difference comes first, so that an entry that is
// the mean gives zero and beta: with x rstd - mean rstd, an instruction fewer, a group of one value would leave half a rounding of
// |mean| rstd, which is 316 |mean| where the variance is zero and eps 1e-5, and relu's slope would be chance.
template <int MODE>
struct Channels {
    Groups<MODE> mean, rstd;
    float scale[VE], beta[VE];           // scale: gamma, and gamma rstd after combine()
    float one;                           // 1, which the compiler is not to know: a multiply-add takes a half as it lies, a difference does not
    __device__ __forceinline__ void params(const Piece& p, const float* ga, const float* be)
    {
        load_params(ga, p, 1.f, scale);
        load_params(be, p, 0.f, beta);
    }
    __device__ __forceinline__ void set(int j, float m, float r)
    {
        mean[j] = m;
        rstd[j] = r;
    }
    __device__ __forceinline__ void combine()      // after params and set
    {
#pragma unroll
        for (int j = 0; j < VE; ++j) scale[j] *= rstd[j];
        one = 1.f;
        asm("" : "+v"(one));
    }
    __device__ __forceinline__ void load(const Piece& p, size_t b, const float* mn, const float* rs, const float* ga, const float* be, uint32_t G,
                                         uint32_t D)
    {
        params(p, ga, be);
        each_group<MODE>(p.c, G, D, [&](int j, uint32_t g) { set(j, mn[b * G + g], rs[b * G + g]); });
        combine();
    }
    __device__ __forceinline__ float d(int j, float x) const { return __builtin_fmaf(x, one, -mean[j]); }
    __device__ __forceinline__ float z(int j, float x) const { return __builtin_fmaf(d(j, x), scale[j], beta[j]); }
    // a and b: sums of dz and dz xhat, b until finish() of dz d
    __device__ __forceinline__ void add(int j, float x, float dz, float (&a)[VE], float (&b)[VE]) const
    {
        a[j] += dz;
        b[j] = __builtin_fmaf(dz, d(j, x), b[j]);
    }
    __device__ __forceinline__ void finish(float (&b)[VE]) const
    {
#pragma unroll
        for (int j = 0; j < VE; ++j) b[j] *= rstd[j];
    }
};
// dx = rstd (gamma dz - c1 - xhat c2), c1 and c2 the group's means of gamma dz and gamma dz xhat
template <int MODE>
struct Slope {
    Groups<MODE> c1, c2;                 // times -rstd
    __device__ __forceinline__ void set(int j, float a, float b, const Channels<MODE>& k)
    {
        c1[j] = -k.rstd[j] * a;
        c2[j] = -k.rstd[j] * b;
    }
    __device__ __forceinline__ float dx(int j, float x, float dz, const Channels<MODE>& k) const
    {
        return __builtin_fmaf(dz, k.scale[j], __builtin_fmaf(k.d(j, x) * k.rstd[j], c2[j], c1[j]));
    }
};

struct Place : Piece {
    uint32_t b, part, slab, r;
    int64_t from;      // the part's first position
    size_t base;       // and its first element
};
template <class IO>
__device__ __forceinline__ Place place(const Walk& w, int64_t S, int64_t C)
{
    Place p;
    p.slab = blockIdx.x % w.slabs;
    p.part = blockIdx.x / w.slabs % w.parts;
    p.b = blockIdx.x / w.slabs / w.parts;
    p.r = threadIdx.x / w.slices;
    p.from = p.part * w.per;
    p.base = ((size_t)p.b * S + p.from) * C;
    p.set((int)(p.slab * w.slices + threadIdx.x % w.slices), p.r < w.rows, C);
    p.template from_row<IO>(p.r, w.rows, (uint32_t)(S - p.from < w.per ? S - p.from : w.per), C);
    return p;
}

// mean and sum of squared differences of every channel over the part's positions -> part[(b, part)][2][C]
template <class IO, int MODE>
__global__ void __launch_bounds__(GT)
gnorm_stats_kernel(const typename IO::T* __restrict__ x, float* __restrict__ part, int64_t S, int64_t C, Walk w)
{
    __shared__ float sm[GT * VE], s2[GT * VE], sn[GT];
    const Place p = place<IO>(w, S, C);
    float mean[VE] = {}, m2[VE] = {}, n = 0.f;
    if (p.on)
        for (uint32_t o = p.off; p.has(o); o += AHEAD * p.step) {
            Raw8<IO> raw[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) fetch<IO, MODE>(p.at(x + p.base, o + u * p.step), p, raw[u]);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                if (!p.has(o + u * p.step)) break;
                float v[VE];
                raw[u].get(v);
                n += 1.f;
                const float g = __builtin_amdgcn_rcpf(n), f = __builtin_fmaf(g, __builtin_fmaf(-n, g, 1.f), g);      // 1 / n
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const float d = v[j] - mean[j];
                    mean[j] = __builtin_fmaf(d, f, mean[j]);
                    m2[j] = __builtin_fmaf(d, v[j] - mean[j], m2[j]);
                }
            }
        }
    // the rows' results together, half of them at a time
    for (uint32_t half = w.half; half; half >>= 1) {
        __syncthreads();
        if (p.r >= half && p.r < 2 * half && p.r < w.rows) {
            to_slots(sm + threadIdx.x * VE, p, mean);
            to_slots(s2 + threadIdx.x * VE, p, m2);
            sn[threadIdx.x] = n;
        }
        __syncthreads();
        if (p.r < half && p.r + half < w.rows) {
            const uint32_t other = threadIdx.x + half * w.slices;
            const float n2 = sn[other];
            if (n2 != 0.f) {
                const float all = n + n2, f = n2 / all, nf = n * f;
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const uint32_t slot = other * VE + ((j - p.skip) & (VE - 1));
                    const float d = sm[slot] - mean[j];
                    mean[j] = __builtin_fmaf(d, f, mean[j]);
                    m2[j] += __builtin_fmaf(d * d, nf, s2[slot]);
                }
                n = all;
            }
        }
    }
    if (p.r == 0 && p.on) {
        float* q = part + ((size_t)p.b * w.parts + p.part) * 2 * C + p.c;
#pragma unroll
        for (int j = 0; j < VE; ++j)
            if (p.mine(j)) {
                q[j] = mean[j];
                q[C + j] = m2[j];
            }
    }
}

// Entries first, first + T, ... of the parts' results of a group of D channels: f(row of part, channel of the group)
template <int T, class F>
__device__ __forceinline__ void each_entry(uint32_t first, uint32_t parts, uint32_t D, F&& f)
{
    const uint32_t dq = T / D, dc = T - dq * D;
    uint32_t q = first / D, c = first - q * D;
#pragma unroll 4
    while (q < parts) {
        f(q, c);
        q += dq;
        c += dc;
        if (c >= D) { c -= D; ++q; }
    }
}
constexpr int FEW = 1024;      // results of a group that one wave puts together; for more a workgroup of sixteen does

// T threads for each group: its channels' and parts' results together
template <int T>
__global__ void __launch_bounds__(T)
gnorm_group_kernel(const float* __restrict__ part, float* __restrict__ mean, float* __restrict__ rstd, int64_t S, int64_t C, uint32_t G,
                   uint32_t parts, int64_t per, float eps)
{
    __shared__ float sn[T / 64], sm[T / 64], s2[T / 64];
    const uint32_t b = blockIdx.x / G, g = blockIdx.x % G, D = (uint32_t)(C / G), lane = threadIdx.x % 64;
    float n = 0.f, m = 0.f, m2 = 0.f;
    const float* first = part + (size_t)b * parts * 2 * C + (size_t)g * D;
    each_entry<T>(threadIdx.x, parts, D, [&](uint32_t q, uint32_t c) {
        const float* row = first + (size_t)q * 2 * C + c;
        const int64_t here = S - q * per < per ? S - q * per : per;
        merge(n, m, m2, (float)here, row[0], row[C]);
    });
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        // the lower lane of a pair first, on both sides: every lane ends with the same numbers
        float n2 = __shfl_xor(n, s), a2 = __shfl_xor(m, s), b2 = __shfl_xor(m2, s);
        if (lane & s) {
            float t;
            t = n; n = n2; n2 = t;
            t = m; m = a2; a2 = t;
            t = m2; m2 = b2; b2 = t;
        }
        if (n == 0.f) { n = n2; m = a2; m2 = b2; }
        else merge(n, m, m2, n2, a2, b2);
    }
    if constexpr (T > 64) {
        if (lane == 0) {
            sn[threadIdx.x / 64] = n;
            sm[threadIdx.x / 64] = m;
            s2[threadIdx.x / 64] = m2;
        }
        __syncthreads();
        if (threadIdx.x == 0)
            for (int w = 1; w < T / 64; ++w) merge(n, m, m2, sn[w], sm[w], s2[w]);
    }
    if (threadIdx.x == 0) {
        mean[blockIdx.x] = m;
        rstd[blockIdx.x] = 1.f / sqrtf(m2 / n + eps);
    }
}

template <class IO, int ACT, int MODE>
__global__ void __launch_bounds__(GT)
gnorm_apply_kernel(const typename IO::T* __restrict__ x, typename IO::T* __restrict__ y, const float* __restrict__ mean,
                   const float* __restrict__ rstd, const float* __restrict__ gamma, const float* __restrict__ beta, int64_t S, int64_t C,
                   uint32_t G, Walk w)
{
    const Place p = place<IO>(w, S, C);
    if (!p.on) return;
    Channels<MODE> k;
    k.load(p, p.b, mean, rstd, gamma, beta, G, (uint32_t)(C / G));
    for (uint32_t o = p.off; p.has(o); o += AHEAD * p.step) {
        Raw8<IO> raw[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) fetch<IO, MODE>(p.at(x + p.base, o + u * p.step), p, raw[u]);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (!p.has(o + u * p.step)) break;
            float v[VE];
            raw[u].get(v);
#pragma unroll
            for (int j = 0; j < VE; ++j) v[j] = act_of<ACT>(k.z(j, v[j]));
            put<IO, MODE>(p.at(y + p.base, o + u * p.step), p, v);
        }
    }
}

// sums of dz and dz xhat of every channel over the part's positions -> part[(b, part)][2][C]
template <class IO, int ACT, int MODE>
__global__ void __launch_bounds__(GT)
gnorm_sums_kernel(const typename IO::T* __restrict__ dy, const typename IO::T* __restrict__ x, const float* __restrict__ mean,
                  const float* __restrict__ rstd, const float* __restrict__ gamma, const float* __restrict__ beta, float* __restrict__ part,
                  int64_t S, int64_t C, uint32_t G, Walk w)
{
    __shared__ float sa[GT * VE], sb[GT * VE];
    const Place p = place<IO>(w, S, C);
    float a[VE] = {}, b[VE] = {};
    if (p.on) {
        Channels<MODE> k;
        k.load(p, p.b, mean, rstd, gamma, beta, G, (uint32_t)(C / G));
        for (uint32_t o = p.off; p.has(o); o += AHEAD / 2 * p.step) {
            Raw8<IO> rx[AHEAD / 2], rg[AHEAD / 2];
#pragma unroll
            for (int u = 0; u < AHEAD / 2; ++u) {
                fetch<IO, MODE>(p.at(x + p.base, o + u * p.step), p, rx[u]);
                fetch<IO, MODE>(p.at(dy + p.base, o + u * p.step), p, rg[u]);
            }
#pragma unroll
            for (int u = 0; u < AHEAD / 2; ++u) {
                if (!p.has(o + u * p.step)) break;
                float v[VE], g[VE];
                rx[u].get(v);
                rg[u].get(g);
#pragma unroll
                for (int j = 0; j < VE; ++j) {
                    const float dz = g[j] * slope_of<ACT>(k.z(j, v[j]));
                    k.add(j, v[j], dz, a, b);
                }
            }
        }
        k.finish(b);
    }
    for (uint32_t half = w.half; half; half >>= 1) {
        __syncthreads();
        if (p.r >= half && p.r < 2 * half && p.r < w.rows) {
            to_slots(sa + threadIdx.x * VE, p, a);
            to_slots(sb + threadIdx.x * VE, p, b);
        }
        __syncthreads();
        if (p.r < half && p.r + half < w.rows) {
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const uint32_t slot = (threadIdx.x + half * w.slices) * VE + ((j - p.skip) & (VE - 1));
                a[j] += sa[slot];
                b[j] += sb[slot];
            }
        }
    }
    if (p.r == 0 && p.on) {
        float* q = part + ((size_t)p.b * w.parts + p.part) * 2 * C + p.c;
#pragma unroll
        for (int j = 0; j < VE; ++j)
            if (p.mine(j)) {
                q[j] = a[j];
                q[C + j] = b[j];
            }
    }
}

constexpr int RT = 1024, RC = 16;      // threads of a workgroup that sums channels, and channels of it

// workgroups 0 .. ceil(C / 16) - 1: dgamma and dbeta of sixteen channels, the rows of partial results spread over the threads; behind
// them s1 and s2, by a wave for every group where its results are few, else by a workgroup
__global__ void __launch_bounds__(RT)
gnorm_gather_kernel(const float* __restrict__ part, const float* __restrict__ gamma, float* __restrict__ s1, float* __restrict__ s2,
                    float* __restrict__ dgamma, float* __restrict__ dbeta, int64_t B, int64_t C, uint32_t G, uint32_t parts)
{
    __shared__ float sa[RT], sh[RT];
    const uint32_t D = (uint32_t)(C / G), blocks = (uint32_t)((C + RC - 1) / RC);
    float a = 0.f, h = 0.f;
    if (blockIdx.x >= blocks) {
        const bool few = (uint64_t)parts * D <= FEW;
        const uint32_t id = few ? (blockIdx.x - blocks) * (RT / 64) + threadIdx.x / 64 : blockIdx.x - blocks;
        if (id >= (uint32_t)B * G) return;
        const uint32_t b = id / G, g = id % G;
        const float* first = part + (size_t)b * parts * 2 * C + (size_t)g * D;
        const auto entry = [&](uint32_t q, uint32_t c) {
            const float* row = first + (size_t)q * 2 * C + c;
            const float ga = gamma ? gamma[g * D + c] : 1.f;
            a = __builtin_fmaf(ga, row[0], a);
            h = __builtin_fmaf(ga, row[C], h);
        };
        if (few) each_entry<64>(threadIdx.x % 64, parts, D, entry);
        else each_entry<RT>(threadIdx.x, parts, D, entry);
        a = wave_sum(a);
        h = wave_sum(h);
        if (!few) {
            if (threadIdx.x % 64 == 0) {
                sa[threadIdx.x / 64] = a;
                sh[threadIdx.x / 64] = h;
            }
            __syncthreads();
            if (threadIdx.x == 0)
                for (int w = 1; w < RT / 64; ++w) {
                    a += sa[w];
                    h += sh[w];
                }
        }
        if (threadIdx.x % (few ? 64 : RT) == 0) {
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

template <class IO, int ACT, int MODE>
__global__ void __launch_bounds__(GT)
gnorm_dx_kernel(const typename IO::T* __restrict__ dy, const typename IO::T* __restrict__ x, const float* __restrict__ mean,
                const float* __restrict__ rstd, const float* __restrict__ gamma, const float* __restrict__ beta, const float* __restrict__ s1,
                const float* __restrict__ s2, typename IO::T* __restrict__ dx, int64_t S, int64_t C, uint32_t G, float inv, Walk w)
{
    const Place p = place<IO>(w, S, C);
    if (!p.on) return;
    const uint32_t D = (uint32_t)(C / G);
    Channels<MODE> k;
    k.load(p, p.b, mean, rstd, gamma, beta, G, D);
    Slope<MODE> of_group;
    each_group<MODE>(p.c, G, D, [&](int j, uint32_t g) { of_group.set(j, s1[(size_t)p.b * G + g] * inv, s2[(size_t)p.b * G + g] * inv, k); });
    for (uint32_t o = p.off; p.has(o); o += AHEAD / 2 * p.step) {
        Raw8<IO> rx[AHEAD / 2], rg[AHEAD / 2];
#pragma unroll
        for (int u = 0; u < AHEAD / 2; ++u) {
            fetch<IO, MODE>(p.at(x + p.base, o + u * p.step), p, rx[u]);
            fetch<IO, MODE>(p.at(dy + p.base, o + u * p.step), p, rg[u]);
        }
#pragma unroll
        for (int u = 0; u < AHEAD / 2; ++u) {
            if (!p.has(o + u * p.step)) break;
            float v[VE], g[VE];
            rx[u].get(v);
            rg[u].get(g);
#pragma unroll
            for (int j = 0; j < VE; ++j) {
                const float dz = g[j] * slope_of<ACT>(k.z(j, v[j]));
                v[j] = of_group.dx(j, v[j], dz, k);
            }
            put<IO, MODE>(p.at(dx + p.base, o + u * p.step), p, v);
        }
    }
}

// ---- groups that fit a workgroup -------------------------------------------------------------------------------------
// A workgroup holds a slab of whole groups of one b in registers, as it came from memory: one read, one launch.  Its threads are `rows`
// positions by `slices` pieces; a thread has NP pieces, `rows` positions apart.  Whatever fits goes this way: 64 x 1024 x 256
// both ways 55 us of kernels against 69 in passes, 3 x 49 x 195 fp32 forward 8.7 against 14.1.  512 threads of eight pieces take 17 us forward
// where 1024 of four take 24 (what a thread does once).  A slab has segments of 64 bytes of a row, or fewer where those of 64 do not fit, down
// to its groups: from 2049 positions on forward and 1025 on backward (16-bit rows, C / G = 8).  What that costs, us of kernels held and in
// passes: 16 x 4096 x 256 forward (32 bytes) 40 and 30, backward (16 bytes) 83 and 41; 32 x 2048 x 256 backward (32 bytes) 54 and 41;
// 8 x 8192 x 256 forward (16 bytes) 76 and 33; 1 x 4096 x 256 14 and 16, 23 and 18: narrow segments pay in small forward passes alone.
constexpr int HT = 512, HSLAB = 128;      // threads, and pieces of a slab, at most

struct Hold {
    uint32_t P, slices, slabs, rows, np, blocks;      // blocks: rounded up to eight times a whole number; 0: does not fit
};
Hold hold(int64_t B, int64_t S, int64_t C, int64_t G, int bytes, uint32_t most)
{
    Hold h{};
    if (C < VE) return h;
    h.P = (uint32_t)((C + VE - 1) / VE);
    const uint32_t D = (uint32_t)(C / G);
    uint32_t unit = D;                                 // pieces of the smallest slab of whole groups and whole pieces
    while (unit % VE) unit += D;
    unit /= VE;
    if (unit > h.P) unit = h.P;
    // 64 bytes of a row and more, so that a line is asked for by two workgroups at most
    uint32_t slices = unit;
    while (slices < h.P && slices * VE * bytes < 64) slices += unit;
    if (slices > h.P) slices = h.P;
    while (slices > unit && (uint64_t)S * slices > (uint64_t)HT * most) slices -= slices == h.P && h.P % unit ? h.P % unit : unit;
    if (slices > HSLAB || (uint64_t)S * slices > (uint64_t)HT * most) return h;
    for (h.np = 1; (S + h.np - 1) / h.np * slices > HT; h.np *= 2) {}
    if (h.np > most) return h;
    h.slices = slices;
    h.slabs = (h.P + slices - 1) / slices;
    h.rows = (uint32_t)((S + h.np - 1) / h.np);
    h.blocks = (uint32_t)(((uint64_t)B * h.slabs + 7) / 8 * 8);
    return h;
}

struct Held : Piece {
    uint32_t b, s, r, W;       // W: channels of the slab's pieces
    int first;                 // the slab's first channel
    size_t base;               // the first element of b
    bool any;
    __device__ __forceinline__ uint32_t piece(int u) const { return off + u * step; }
};
// every XCD (workgroups go round them) takes neighbouring slabs, which share lines
template <class IO>
__device__ __forceinline__ Held held(const Hold& h, uint32_t B, int64_t S, int64_t C)
{
    Held p;
    const uint32_t id = (blockIdx.x & 7u) * (h.blocks / 8) + (blockIdx.x >> 3);
    p.any = id < B * h.slabs;
    p.b = id / h.slabs;
    p.s = threadIdx.x % h.slices;
    p.r = threadIdx.x / h.slices;
    p.W = h.slices * VE;
    p.first = (int)((id - p.b * h.slabs) * p.W);
    p.base = (size_t)p.b * S * C;
    p.set(p.first / VE + (int)p.s, p.r < h.rows, C);
    p.template from_row<IO>(p.r, h.rows, (uint32_t)S, C);
    return p;
}

// f(j, group of channel j counted from the slab's first); channels that belong to the slab before: 0, for nothing
template <int MODE, class F>
__device__ __forceinline__ void in_slab(const Held& p, uint32_t G, uint32_t D, F&& f)
{
    const uint32_t before = (uint32_t)p.first / D;
    each_group<MODE>(p.c, G, D, [&](int j, uint32_t g) { f(j, g > before ? g - before : 0u); });
}

// v[j]: a number of the thread for its channel j.  cols[k W + c]: its sums over the rows, in K shares (the return value).
__device__ __forceinline__ uint32_t sum_rows(const float (&v)[VE], float* all, float* cols, const Hold& h, const Held& p)
{
    const uint32_t T = blockDim.x;
    __syncthreads();
    if (p.r < h.rows) to_slots(all + p.r * p.W + p.s * VE, p, v);
    __syncthreads();
    uint32_t K = T / p.W;
    if (K < 1) K = 1;
    if (K > h.rows) K = h.rows;
    for (uint32_t i = threadIdx.x; i < K * p.W; i += T) {
        const uint32_t k = i / p.W;
        float t = 0.f;
#pragma unroll 8
        for (uint32_t r = k; r < h.rows; r += K) t += all[r * p.W + (i - k * p.W)];
        cols[i] = t;
    }
    __syncthreads();
    return K;
}
// group[g] = last(the sum of weight(c) cols over a group's channels and shares); a wave each
template <class F, class E>
__device__ __forceinline__ void sum_groups(const float* cols, float* group, uint32_t K, uint32_t D, uint32_t W, F&& weight, E&& last)
{
    for (uint32_t g = threadIdx.x / 64; g * D < W; g += blockDim.x / 64) {
        float t = 0.f;
        for (uint32_t i = threadIdx.x % 64; i < K * D; i += 64) {
            const uint32_t k = i / D, c = g * D + (i - k * D);
            if (c < W) t = __builtin_fmaf(weight(c), cols[k * W + c], t);      // (a group wider than the last slab's pieces ends with the channels)
        }
        t = wave_sum(t);
        if (threadIdx.x % 64 == 0) group[g] = last(t);
    }
    __syncthreads();
}

template <class IO, int ACT, int NP, int MODE>
__global__ void __launch_bounds__(HT)
gnorm_hold_fwd_kernel(const typename IO::T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ beta,
                      typename IO::T* __restrict__ y, float* __restrict__ mean, float* __restrict__ rstd, uint32_t B, int64_t S, int64_t C,
                      uint32_t G, float n, float eps, Hold h)
{
    __shared__ float all[HT * VE], cols[HSLAB * VE], group[HSLAB * VE];
    const Held p = held<IO>(h, B, S, C);
    if (!p.any) return;
    const uint32_t D = (uint32_t)(C / G);
    Raw8<IO> raw[NP];
#pragma unroll
    for (int u = 0; u < NP; ++u) raw[u].load(p.at(x + p.base, p.piece(u)));
    Channels<MODE> k;
    k.params(p, gamma, beta);
    const auto one = [](uint32_t) { return 1.f; };
    float t[VE] = {};
    Groups<MODE> mn, rs;
#pragma unroll
    for (int u = 0; u < NP; ++u) {
        if (!p.has(p.piece(u))) break;
        float v[VE];
        raw[u].get(v);
#pragma unroll
        for (int j = 0; j < VE; ++j) t[j] += v[j];
    }
    uint32_t K = sum_rows(t, all, cols, h, p);
    sum_groups(cols, group, K, D, p.W, one, [&](float s) { return s / n; });
    in_slab<MODE>(p, G, D, [&](int j, uint32_t g) { mn[j] = group[g]; });
#pragma unroll
    for (int j = 0; j < VE; ++j) t[j] = 0.f;
#pragma unroll
    for (int u = 0; u < NP; ++u) {
        if (!p.has(p.piece(u))) break;
        float v[VE];
        raw[u].get(v);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            const float d = v[j] - mn[j];
            t[j] = __builtin_fmaf(d, d, t[j]);
        }
    }
    K = sum_rows(t, all, cols, h, p);
    sum_groups(cols, group, K, D, p.W, one, [&](float s) { return 1.f / sqrtf(s / n + eps); });
    in_slab<MODE>(p, G, D, [&](int j, uint32_t g) { rs[j] = group[g]; });
#pragma unroll
    for (int j = 0; j < (MODE == ONE ? 1 : VE); ++j) k.set(j, mn[j], rs[j]);
    k.combine();
    if (p.r == 0) {      // the first channel of a group writes its numbers
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            const uint32_t c = (uint32_t)(p.c + j), g = c / D;
            if (p.mine(j) && g * D == c) {
                mean[(size_t)p.b * G + g] = mn[j];
                rstd[(size_t)p.b * G + g] = rs[j];
            }
        }
    }
#pragma unroll
    for (int u = 0; u < NP; ++u) {
        if (!p.has(p.piece(u)) || !p.on) break;
        float v[VE];
        raw[u].get(v);
#pragma unroll
        for (int j = 0; j < VE; ++j) v[j] = act_of<ACT>(k.z(j, v[j]));
        put<IO, MODE>(p.at(y + p.base, p.piece(u)), p, v);
    }
}

// part[b][2][C]: sums of dz and dz xhat over the positions
template <class IO, int ACT, int NP, int MODE>
__global__ void __launch_bounds__(HT)
gnorm_hold_bwd_kernel(const typename IO::T* __restrict__ dy, const typename IO::T* __restrict__ x, const float* __restrict__ mean,
                      const float* __restrict__ rstd, const float* __restrict__ gamma, const float* __restrict__ beta, float* __restrict__ part,
                      typename IO::T* __restrict__ dx, uint32_t B, int64_t S, int64_t C, uint32_t G, float inv, Hold h)
{
    __shared__ float all[HT * VE], ca[HSLAB * VE], ch[HSLAB * VE], g1[HSLAB * VE], g2[HSLAB * VE];
    const Held p = held<IO>(h, B, S, C);
    if (!p.any) return;
    const uint32_t D = (uint32_t)(C / G);
    Raw8<IO> rx[NP], rg[NP];
#pragma unroll
    for (int u = 0; u < NP; ++u) {
        rx[u].load(p.at(x + p.base, p.piece(u)));
        rg[u].load(p.at(dy + p.base, p.piece(u)));
    }
    Channels<MODE> k;
    k.load(p, p.b, mean, rstd, gamma, beta, G, D);
    float a[VE] = {}, b[VE] = {};
#pragma unroll
    for (int u = 0; u < NP; ++u) {
        if (!p.has(p.piece(u))) break;
        float v[VE], g[VE];
        rx[u].get(v);
        rg[u].get(g);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            const float dz = g[j] * slope_of<ACT>(k.z(j, v[j]));
            k.add(j, v[j], dz, a, b);
        }
    }
    k.finish(b);
    const uint32_t K = sum_rows(a, all, ca, h, p);
    sum_rows(b, all, ch, h, p);
    for (uint32_t i = threadIdx.x; i < p.W && p.first + (int)i < C; i += blockDim.x) {
        float ta = 0.f, tb = 0.f;
        for (uint32_t q = 0; q < K; ++q) {
            ta += ca[q * p.W + i];
            tb += ch[q * p.W + i];
        }
        float* q = part + (size_t)p.b * 2 * C + p.first + i;
        q[0] = ta;
        q[C] = tb;
    }
    if (!dx) return;
    const auto weight = [&](uint32_t c) { return gamma && p.first + (int)c < C ? gamma[p.first + c] : 1.f; };
    const auto mean_of = [&](float s) { return s * inv; };
    sum_groups(ca, g1, K, D, p.W, weight, mean_of);
    sum_groups(ch, g2, K, D, p.W, weight, mean_of);
    Slope<MODE> of_group;
    in_slab<MODE>(p, G, D, [&](int j, uint32_t g) { of_group.set(j, g1[g], g2[g], k); });
#pragma unroll
    for (int u = 0; u < NP; ++u) {
        if (!p.has(p.piece(u)) || !p.on) break;
        float v[VE], g[VE];
        rx[u].get(v);
        rg[u].get(g);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
            const float dz = g[j] * slope_of<ACT>(k.z(j, v[j]));
            v[j] = of_group.dx(j, v[j], dz, k);
        }
        put<IO, MODE>(p.at(dx + p.base, p.piece(u)), p, v);
    }
}

template <class F>
void by_mode(const GnormArgs& a, F&& f)
{
    switch (mode_of(a.C, a.G)) {
        case NARROW: f(std::integral_constant<int, NARROW>()); break;
        case ONE: f(std::integral_constant<int, ONE>()); break;
        default: f(std::integral_constant<int, ANYHOW>());
    }
}

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

template <class IO, int ACT>
hipError_t forward(const GnormArgs& a, const void* x, void* y, float* mean, float* rstd, float eps, void* ws, hipStream_t st)
{
    using T = typename IO::T;
    dim3 g, gg;
    const Hold h = hold(a.B, a.S, a.C, a.G, sizeof(T), 64 / Raw8<IO>::W);
    if (h.blocks) {
        const hipError_t e = launch_grid(h.blocks, HT, &g);
        if (e != hipSuccess) return e;
        const auto go = [&](auto np) {
            const auto kernel = mode_of(a.C, a.G) == ONE ? gnorm_hold_fwd_kernel<IO, ACT, decltype(np)::value, ONE>
                                                         : gnorm_hold_fwd_kernel<IO, ACT, decltype(np)::value, ANYHOW>;
            hipLaunchKernelGGL(kernel, g, dim3((h.slices * h.rows + 63) / 64 * 64), 0, st, (const T*)x,
                               a.gamma, a.beta, (T*)y, mean, rstd, (uint32_t)a.B, a.S, a.C, (uint32_t)a.G, (float)(a.S * (a.C / a.G)), eps, h);
        };
        if (h.np == 1) go(std::integral_constant<int, 1>());
        else if (h.np == 2) go(std::integral_constant<int, 2>());
        else if (h.np == 4) go(std::integral_constant<int, 4>());
        else if (h.np == 8) go(std::integral_constant<int, 8>());
        else if constexpr (Raw8<IO>::W == 4) go(std::integral_constant<int, 16>());
        return hipGetLastError();
    }
    const Walk w = walk(a.B, a.S, a.C);
    hipError_t e = launch_grid((uint64_t)a.B * w.parts * w.slabs, GT, &g);
    if (e == hipSuccess) e = launch_grid((uint64_t)a.B * a.G, 64, &gg);
    if (e != hipSuccess) return e;
    float* part = (float*)ws;
    if (a.C < VE) hipLaunchKernelGGL((gnorm_stats_kernel<IO, NARROW>), g, dim3(GT), 0, st, (const T*)x, part, a.S, a.C, w);
    else hipLaunchKernelGGL((gnorm_stats_kernel<IO, ANYHOW>), g, dim3(GT), 0, st, (const T*)x, part, a.S, a.C, w);
    if ((uint64_t)w.parts * (a.C / a.G) <= FEW)
        hipLaunchKernelGGL(gnorm_group_kernel<64>, gg, dim3(64), 0, st, (const float*)part, mean, rstd, a.S, a.C, (uint32_t)a.G, w.parts, w.per, eps);
    else
        hipLaunchKernelGGL(gnorm_group_kernel<1024>, gg, dim3(1024), 0, st, (const float*)part, mean, rstd, a.S, a.C, (uint32_t)a.G, w.parts, w.per, eps);
    by_mode(a, [&](auto mode) {
        hipLaunchKernelGGL((gnorm_apply_kernel<IO, ACT, decltype(mode)::value>), g, dim3(GT), 0, st, (const T*)x, (T*)y, (const float*)mean,
                           (const float*)rstd, a.gamma, a.beta, a.S, a.C, (uint32_t)a.G, w);
    });
    return hipGetLastError();
}

template <class IO, int ACT>
hipError_t backward(const GnormArgs& a, const void* dy, const void* x, const float* mean, const float* rstd, void* dx, float* dgamma,
                    float* dbeta, void* ws, hipStream_t st)
{
    using T = typename IO::T;
    dim3 g, gg;
    const float inv = (float)(1.0 / ((double)a.S * (a.C / a.G)));
    const Hold h = hold(a.B, a.S, a.C, a.G, sizeof(T), 32 / Raw8<IO>::W);
    if (h.blocks) {
        const hipError_t e = launch_grid(h.blocks, HT, &g);
        if (e != hipSuccess) return e;
        const auto go = [&](auto np) {
            const auto kernel = mode_of(a.C, a.G) == ONE ? gnorm_hold_bwd_kernel<IO, ACT, decltype(np)::value, ONE>
                                                         : gnorm_hold_bwd_kernel<IO, ACT, decltype(np)::value, ANYHOW>;
            hipLaunchKernelGGL(kernel, g, dim3((h.slices * h.rows + 63) / 64 * 64), 0, st,
                               (const T*)dy, (const T*)x, mean, rstd, a.gamma, a.beta, (float*)ws, (T*)dx, (uint32_t)a.B, a.S, a.C, (uint32_t)a.G,
                               inv, h);
        };
        if (h.np == 1) go(std::integral_constant<int, 1>());
        else if (h.np == 2) go(std::integral_constant<int, 2>());
        else if (h.np == 4) go(std::integral_constant<int, 4>());
        else if constexpr (Raw8<IO>::W == 4) go(std::integral_constant<int, 8>());
        if (dgamma || dbeta)
            hipLaunchKernelGGL(gnorm_gather_kernel, dim3((unsigned)((a.C + RC - 1) / RC)), dim3(RT), 0, st, (const float*)ws, a.gamma, (float*)nullptr,
                               (float*)nullptr, dgamma, dbeta, a.B, a.C, (uint32_t)a.G, 1u);
        return hipGetLastError();
    }
    const Walk w = walk(a.B, a.S, a.C);
    hipError_t e = launch_grid((uint64_t)a.B * w.parts * w.slabs, GT, &g);
    if (e == hipSuccess) e = launch_grid((uint64_t)(a.C + RC - 1) / RC + ((uint64_t)w.parts * (a.C / a.G) <= FEW ? ((uint64_t)a.B * a.G + RT / 64 - 1) / (RT / 64) : (uint64_t)a.B * a.G), RT, &gg);
    if (e != hipSuccess) return e;
    float* part = (float*)ws;
    float* s1 = (float*)((char*)ws + up256(part_rows(a.B, a.S, a.C) * 2 * a.C * sizeof(float)));
    float* s2 = s1 + a.B * a.G;
    by_mode(a, [&](auto mode) {
        constexpr int N = decltype(mode)::value;
        hipLaunchKernelGGL((gnorm_sums_kernel<IO, ACT, N>), g, dim3(GT), 0, st, (const T*)dy, (const T*)x, mean, rstd, a.gamma, a.beta, part, a.S,
                           a.C, (uint32_t)a.G, w);
        hipLaunchKernelGGL(gnorm_gather_kernel, gg, dim3(RT), 0, st, (const float*)part, a.gamma, s1, s2, dgamma, dbeta, a.B, a.C, (uint32_t)a.G,
                           w.parts);
        if (dx)
            hipLaunchKernelGGL((gnorm_dx_kernel<IO, ACT, N>), g, dim3(GT), 0, st, (const T*)dy, (const T*)x, mean, rstd, a.gamma, a.beta,
                               (const float*)s1, (const float*)s2, (T*)dx, a.S, a.C, (uint32_t)a.G, inv, w);
    });
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

template <class IO>
hipError_t gnorm_fwd_io(const GnormArgs& a, const void* x, void* y, float* mean, float* rstd, float eps, void* ws, hipStream_t st)
{
    return by_act<IO>(a.act, [&](auto act) { return forward<IO, decltype(act)::value>(a, x, y, mean, rstd, eps, ws, st); });
}

template <class IO>
hipError_t gnorm_bwd_io(const GnormArgs& a, const void* dy, const void* x, const float* mean, const float* rstd, void* dx, float* dgamma,
                        float* dbeta, void* ws, hipStream_t st)
{
    return by_act<IO>(a.act, [&](auto act) { return backward<IO, decltype(act)::value>(a, dy, x, mean, rstd, dx, dgamma, dbeta, ws, st); });
}

#define GNORM_IO(IO)                                                                                                                      \
    template hipError_t gnorm_fwd_io<IO>(const GnormArgs&, const void*, void*, float*, float*, float, void*, hipStream_t);                \
    template hipError_t gnorm_bwd_io<IO>(const GnormArgs&, const void*, const void*, const float*, const float*, void*, float*, float*,   \
                                         void*, hipStream_t)

}  // namespace lc
