// Dropout from a counter-based generator: y = r + m x with m = 0 or 65536 / (65536 - T), the mask a function of the entry's place,
// the call's number and the seed (vec8.hpp), never stored; its backward pass is the same kernel without r.  Entries may share a
// mask value in runs of `tie` (the rows of [B,H,N]: one value for a head's whole sequence).
//
// Bound by memory: a thread takes the eight entries of one generator block, sixteen bytes of each tensor (thirty-two in fp32), all asked
// for before the generator's hundred instructions.  64 x 1024 x 4096 in bf16: 263 us with the residual sum, 169 without, 6.1 and 6.4 TB/s;
// workgroups of 128, 512 and 1024 threads within 3 percent.  Stores without the nt hint take 273 and 168 there, and at 16 x 768 x 1024, tied,
// 15.3 and 11.7 for 12.4 and 9.7.
#include "vec8.hpp"

namespace lc {
namespace {

// bit j: entry e + j is kept, entries i sharing the value of number i / tie
template <class I>
__device__ __forceinline__ uint32_t kept8_tied(I e, I tie, const Drop& d, uint64_t call)
{
    uint32_t m = 0;
    I row = e / tie;
    int at = 0;
    while (at < VE) {
        const I left = (row + 1) * tie - e;      // entries from e to the row's end
        const int end = left < (I)VE ? (int)left : VE;
        if (kept8(row >> 3, d, call) >> (row & 7u) & 1u) m |= (1u << end) - (1u << at);
        at = end;
        ++row;
    }
    return m;
}

// I: unsigned type that holds n + 8 and the rows' numbers
template <class IO, class I, bool TIED>
__global__ void __launch_bounds__(256)
dropout_kernel(const typename IO::T* x, const typename IO::T* r, typename IO::T* y, I n, I tie, Drop d)
{
    const I e = ((I)blockIdx.x * 256 + threadIdx.x) * VE;
    if (e >= n) return;
    const int here = n - e < (I)VE ? (int)(n - e) : VE;
    const uint64_t call = call_of(d);
    Raw8<IO> rx, rr;
    rr.zero();
    if (here == VE) {
        rx.load(x + e);
        if (r) rr.load(r + e);
    } else {
        load_raw<IO>(x + e, here, rx);
        if (r) load_raw<IO>(r + e, here, rr);
    }
    uint4 m;
    if constexpr (TIED) {
        const uint32_t bits = kept8_tied<I>(e, tie, d, call);
        const auto word = [&](int i) { return (bits >> (2 * i) & 1u ? 0xffffu : 0u) | (bits >> (2 * i + 1) & 1u ? 0xffff0000u : 0u); };
        m = make_uint4(word(0), word(1), word(2), word(3));
    } else m = kept_words(e >> 3, d, call);
    const uint32_t mask[4] = {m.x, m.y, m.z, m.w};
    // (a dropped entry counts for nothing, whatever it holds: its bits become those of zero)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (Raw8<IO>::W == 4) rx.w[i] &= mask[i];
        else {
            rx.w[2 * i] &= (uint32_t)((int32_t)(mask[i] << 16) >> 16);
            rx.w[2 * i + 1] &= (uint32_t)((int32_t)mask[i] >> 16);
        }
    }
    float v[VE], s[VE];
    rx.get(v);
    rr.get(s);
#pragma unroll
    for (int i = 0; i < VE; ++i) v[i] = __builtin_fmaf(v[i], d.scale, s[i]);
    store8<IO, true>(y + e, here, v);
}

template <class IO>
hipError_t launch(const void* x, const void* r, void* y, int64_t n, int64_t tie, const Drop& d, hipStream_t st)
{
    using T = typename IO::T;
    dim3 g;
    const hipError_t e = launch_grid((uint64_t)((n + 256 * VE - 1) / (256 * VE)), 256, &g);
    if (e != hipSuccess) return e;
    const T *xt = (const T*)x, *rt = (const T*)r;
    const bool small = n < (int64_t(1) << 31);
    if (tie == 1 && small) hipLaunchKernelGGL((dropout_kernel<IO, uint32_t, false>), g, dim3(256), 0, st, xt, rt, (T*)y, (uint32_t)n, 1u, d);
    else if (tie == 1) hipLaunchKernelGGL((dropout_kernel<IO, uint64_t, false>), g, dim3(256), 0, st, xt, rt, (T*)y, (uint64_t)n, (uint64_t)1, d);
    else if (small) hipLaunchKernelGGL((dropout_kernel<IO, uint32_t, true>), g, dim3(256), 0, st, xt, rt, (T*)y, (uint32_t)n, (uint32_t)tie, d);
    else hipLaunchKernelGGL((dropout_kernel<IO, uint64_t, true>), g, dim3(256), 0, st, xt, rt, (T*)y, (uint64_t)n, (uint64_t)tie, d);
    return hipGetLastError();
}

}  // namespace

hipError_t dropout(const void* x, const void* residual, void* y, int64_t n, int64_t tie, int io, const Drop& d, hipStream_t st)
{
    if (io == LONGCONV_F32) return launch<IoF32>(x, residual, y, n, tie, d, st);
    return io == LONGCONV_F16 ? launch<IoF16>(x, residual, y, n, tie, d, st) : launch<IoBF16>(x, residual, y, n, tie, d, st);
}

}  // namespace lc
