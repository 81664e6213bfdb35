// Shared by the streaming operators around the convolution (dropout.hip, embed.hip, gnorm.hip, kreg.hip): eight elements of a
// tensor at a time as floats, at any element's address, and the counter-based generator behind every dropout mask.
#pragma once
#include <type_traits>

#include "mfma_util.hpp"
#include "operators.hpp"

namespace lc {

// Sixteen bytes at the address of any element: gfx950 loads and stores them in one instruction whatever the alignment.
typedef uint32_t At2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t At4 __attribute__((ext_vector_type(4), aligned(4)));
constexpr int VE = 8;      // elements of a piece

template <class IO>
__device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b)
{
    if constexpr (mu::IsBf<IO>::v) {
        a = __uint_as_float(w << 16);
        b = __uint_as_float(w & 0xffff0000u);
    } else {
        union { uint32_t u; mu::h2 h; } x;
        x.u = w;
        a = (float)x.h[0];
        b = (float)x.h[1];
    }
}

// a piece as it lies in memory: 4 words of two 16-bit elements, or 8 words of one float
template <class IO>
struct Raw8 {
    static constexpr int W = sizeof(typename IO::T) == 4 ? 8 : 4;
    typedef typename std::conditional<W == 8, At4, At2>::type V;
    uint32_t w[W];
    __device__ __forceinline__ void load(const typename IO::T* p)
    {
        const V* q = reinterpret_cast<const V*>(p);
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const V v = q[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[4 * i + j] = v[j];
        }
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void get(float (&v)[VE]) const
    {
        if constexpr (W == 8) {
#pragma unroll
            for (int i = 0; i < VE; ++i) v[i] = __uint_as_float(w[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) unpack2<IO>(w[i], v[2 * i], v[2 * i + 1]);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[VE])      // rounds to the nearest, the one rounding of a result
    {
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (W == 8) w[i] = __float_as_uint(v[i]);
            else w[i] = mu::IsBf<IO>::v ? mu::pack_bf2(v[2 * i], v[2 * i + 1]) : mu::pack_h2(v[2 * i], v[2 * i + 1]);
        }
    }
    // ONCE: with the hint that the line is not read again soon (put_once)
    template <bool ONCE = false>
    __device__ __forceinline__ void store(typename IO::T* p) const
    {
        V* q = reinterpret_cast<V*>(p);
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const V v = {w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
            if constexpr (ONCE) __builtin_nontemporal_store(v, q + i);
            else q[i] = v;
        }
    }
};

// a piece, or its first `n` elements (the others read as zero); n < 1: none
template <class IO>
__device__ __forceinline__ void load_raw(const typename IO::T* p, int n, Raw8<IO>& r)
{
    if (n >= VE) { r.load(p); return; }
    r.zero();
#pragma unroll
    for (int i = 0; i < VE; ++i)
        if (i < n) {
            if constexpr (Raw8<IO>::W == 8) r.w[i] = __float_as_uint(p[i]);
            else r.w[i / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(p + i) << (i % 2 * 16);
        }
}
// eight elements, or the first `n` of them (the others read as zero)
template <class IO>
__device__ __forceinline__ void load8(const typename IO::T* p, int n, float (&v)[VE])
{
    if (n >= VE) {
        Raw8<IO> r;
        r.load(p);
        r.get(v);
        return;
    }
#pragma unroll
    for (int i = 0; i < VE; ++i) v[i] = i < n ? IO::ld(p, i) : 0.f;
}
template <class IO, bool ONCE = false>
__device__ __forceinline__ void store8(typename IO::T* p, int n, const float (&v)[VE])
{
    if (n >= VE) {
        Raw8<IO> r;
        r.set(v);
        r.template store<ONCE>(p);
        return;
    }
#pragma unroll
    for (int i = 0; i < VE; ++i)
        if (i < n) IO::st(p, i, v[i]);
}

// ---------------------------------------------------------------------------------
// Dropout masks.  Philox4x32 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): a bijection of a
// 128-bit counter under a 64-bit key, so every piece of a mask is a function of its place alone and nothing is ever stored.  Seven
// rounds, the fewest that the authors report to pass BigCrush.  Sixteen bits decide an entry (p is therefore a multiple of 2^-16), so
// one counter serves the eight entries of a piece: entry e has half e mod 8 of counter (e / 8, call), low half of a word first.
// ---------------------------------------------------------------------------------
__device__ __forceinline__ uint64_t call_of(const Drop& d) { return d.step ? d.call + (uint64_t)*d.step : d.call; }

__device__ __forceinline__ uint4 philox(uint64_t block, uint64_t call, uint64_t seed)
{
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)call, c3 = (uint32_t)(call >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 7; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

// The kept entries of a block as masks of the halves of four words, as 16-bit data lie in memory: 0xffff kept, 0 dropped.
__device__ __forceinline__ uint4 kept_words(uint64_t block, const Drop& d, uint64_t call)
{
    typedef uint16_t us2 __attribute__((ext_vector_type(2)));
    if (d.threshold > 0xffffu) return make_uint4(0, 0, 0, 0);
    const uint4 r = philox(block, call, d.seed);
    const uint16_t t = (uint16_t)d.threshold;
    const us2 least = {t, t}, one = {1, 1};
    const auto mask = [&](uint32_t w) {      // what a half lacks of the threshold, as 0 or 1; less 1
        const us2 lacks = __builtin_elementwise_sub_sat(least, __builtin_bit_cast(us2, w));
        return __builtin_bit_cast(uint32_t, (us2)(__builtin_elementwise_min(lacks, one) - one));
    };
    return make_uint4(mask(r.x), mask(r.y), mask(r.z), mask(r.w));
}
// bit j: entry 8 block + j is kept
__device__ __forceinline__ uint32_t kept8(uint64_t block, const Drop& d, uint64_t call)
{
    const uint4 w = kept_words(block, d, call);
    return (w.x & 1u) | (w.x >> 16 & 2u) | (w.y & 4u) | (w.y >> 16 & 8u) | (w.z & 16u) | (w.z >> 16 & 32u) | (w.w & 64u) | (w.w >> 16 & 128u);
}
// bit j: entry e + j is kept
__device__ __forceinline__ uint32_t kept8_at(uint64_t e, const Drop& d, uint64_t call)
{
    const uint32_t at = (uint32_t)e & 7u;
    uint32_t m = kept8(e >> 3, d, call);
    if (at) m = (m | kept8((e >> 3) + 1, d, call) << 8) >> at;
    return m & 0xffu;
}

// the masks of entries e .. e + 7
__device__ __forceinline__ uint4 kept_words_at(uint64_t e, const Drop& d, uint64_t call)
{
    const uint32_t at = (uint32_t)e & 7u;
    uint4 a = kept_words(e >> 3, d, call);
    if (at) {
        const uint4 b = kept_words((e >> 3) + 1, d, call);
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        uint32_t v[5];
#pragma unroll
        for (int i = 0; i < 5; ++i) {      // words at / 2 ..
            v[i] = w[i];
#pragma unroll
            for (int k = 1; k < 4; ++k)
                if (at / 2 == (uint32_t)k && i + k < 8) v[i] = w[i + k];
        }
        const uint32_t by = at % 2 * 16;
        const auto pick = [&](int i) { return by ? v[i] >> 16 | v[i + 1] << 16 : v[i]; };
        a = make_uint4(pick(0), pick(1), pick(2), pick(3));
    }
    return a;
}

inline hipError_t launch_grid(uint64_t blocks, uint32_t threads, dim3* g)      // 1-D grid; a launch holds fewer than 2^32 threads
{
    if (blocks == 0 || blocks * threads > 0xffffffffull) return hipErrorInvalidValue;
    *g = dim3((unsigned)blocks);
    return hipSuccess;
}

}  // namespace lc
