// Shared by the selective scan's forward (scan.hip) and backward (scan_bwd.hip) kernels.
//
// One state s of one head is a recurrence along the sequence, h_t = a_t h_{t-1} + x_t, a_t = exp(dt_t A[h,s]).  A wave takes a chunk of
// 64 K neighbouring places, K of them in each lane: every lane runs through its places from zero, the lanes' results (decay of the lane,
// state behind it) are put together by a scan over the wave, and every lane runs through its places again from the state in front of it.
#pragma once
#include "vec8.hpp"

namespace lc {

// What the passes over segments leave: the state behind each segment of [B,H,segs], from zero (BACK: the gradient that it hands on to the
// segment before, from zero), and the sum of its dt
struct Segments {
    float *ends, *sums;
    int segs;
    int64_t len;      // places of a segment, a multiple of SPAN
};
// The passes of the backward call over segments (BACK); g: how the sequence is cut
hipError_t scan_back(const ScanArgs& a, const void* dy, void* ws, Segments* g, hipStream_t st);
size_t scan_segment_bytes(int64_t B, int64_t H, int64_t N, int S, int64_t G);
size_t scan_bwd_bytes(int64_t B, int64_t H, int64_t N, int S, int64_t G);      // of the backward call beyond those

namespace {

constexpr int SPAN = LONGCONV_SCAN_SPAN;      // places between two marks
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
// 1 / (1 + exp(-x))
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.f + exp2_of(-LOG2E * x)); }

// log(1 + exp(w)) to fp32's accuracy: log(1 + e) = log(f) e / (f - 1) with f = 1 + e rounded, whose rounding cancels (Goldberg, "What
// every computer scientist should know about floating-point arithmetic", ACM Computing Surveys 23 (1991), theorem 4)
__device__ __forceinline__ float softplus_of(float w)
{
    const float e = exp2_of(-LOG2E * fabsf(w)), f = 1.f + e, d = f - 1.f;
    const float l = d == 0.f ? e : 0.69314718055994531f * __builtin_amdgcn_logf(f) * (e * __builtin_amdgcn_rcpf(d));
    return w != w ? w : fmaxf(w, 0.f) + l;
}

__device__ __forceinline__ int64_t scan_length(const ScanArgs& a, int64_t b)
{
    if (!a.lengths) return a.N;
    const int64_t n = a.lengths[b];
    return n < 0 ? 0 : n > a.N ? a.N : n;
}

// x of another lane by the DPP control C, `otherwise` in lanes that have no such lane, or that the row mask leaves out
template <int C, int ROWS = 0xf>
__device__ __forceinline__ float dpp(float x, float otherwise)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp((int)__float_as_uint(otherwise), (int)__float_as_uint(x), C, ROWS, 0xf, false));
}
__device__ __forceinline__ float lane_of(float x, int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), lane)); }

// (decay p, state h) of each lane -> h behind all lanes up to it (p is used up)
__device__ __forceinline__ void scan_up(float& p, float& h)
{
    h = __builtin_fmaf(p, dpp<0x111>(h, 0.f), h); p *= dpp<0x111>(p, 1.f);                  // one lane down a row of sixteen
    h = __builtin_fmaf(p, dpp<0x112>(h, 0.f), h); p *= dpp<0x112>(p, 1.f);
    h = __builtin_fmaf(p, dpp<0x114>(h, 0.f), h); p *= dpp<0x114>(p, 1.f);
    h = __builtin_fmaf(p, dpp<0x118>(h, 0.f), h); p *= dpp<0x118>(p, 1.f);
    h = __builtin_fmaf(p, dpp<0x142, 0xa>(h, 0.f), h); p *= dpp<0x142, 0xa>(p, 1.f);        // a row's last lane to the next row
    h = __builtin_fmaf(p, dpp<0x143, 0xc>(h, 0.f), h);                                      // lane 31 to the upper half
}

// (decay p, value v) of each lane, towards lower lanes -> v in front of all lanes from it on (p is used up)
__device__ __forceinline__ void scan_down(float& p, float& v)
{
    v = __builtin_fmaf(p, dpp<0x101>(v, 0.f), v); p *= dpp<0x101>(p, 1.f);
    v = __builtin_fmaf(p, dpp<0x102>(v, 0.f), v); p *= dpp<0x102>(p, 1.f);
    v = __builtin_fmaf(p, dpp<0x104>(v, 0.f), v); p *= dpp<0x104>(p, 1.f);
    v = __builtin_fmaf(p, dpp<0x108>(v, 0.f), v); p *= dpp<0x108>(p, 1.f);
    // the rows' first lanes hold the rows' totals
    const int row = (int)(__lane_id() >> 4);
    const float v3 = lane_of(v, 48), v2 = __builtin_fmaf(lane_of(p, 32), v3, lane_of(v, 32)), v1 = __builtin_fmaf(lane_of(p, 16), v2, lane_of(v, 16));
    v = __builtin_fmaf(p, row == 0 ? v1 : row == 1 ? v2 : row == 2 ? v3 : 0.f, v);
}

__device__ __forceinline__ float sum_of_wave(float v)
{
    v += dpp<0xB1>(v, 0.f);
    v += dpp<0x4E>(v, 0.f);
    v += dpp<0x141>(v, 0.f);
    v += dpp<0x140>(v, 0.f);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}

// the value that comes into segment `seg` of a row from `from` and the segments before it (BACK: behind it)
template <bool BACKWARDS>
__device__ __forceinline__ float entering(const Segments& g, size_t row, int seg, int S, int s, float A2, float from)
{
    float h = from;
    if (BACKWARDS)
        for (int q = g.segs - 1; q > seg; --q)
            h = __builtin_fmaf(exp2_of(A2 * g.sums[row * g.segs + q]), h, g.ends[(row * g.segs + q) * S + s]);
    else
        for (int q = 0; q < seg; ++q) h = __builtin_fmaf(exp2_of(A2 * g.sums[row * g.segs + q]), h, g.ends[(row * g.segs + q) * S + s]);
    return h;
}

inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// four neighbouring elements of a row, zero outside 0 .. lim - 1; the row has N elements
typedef uint32_t At2x2 __attribute__((ext_vector_type(2), aligned(2)));
template <class IO>
__device__ __forceinline__ float4 load4(const typename IO::T* row, int64_t t, int64_t N, int64_t lim)
{
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (t < lim) {
        if (t + 4 <= N) {
            if constexpr (sizeof(typename IO::T) == 4) {
                const At4 q = *reinterpret_cast<const At4*>(row + t);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(q[i]);
            } else {
                const At2x2 q = *reinterpret_cast<const At2x2*>(row + t);
                unpack2<IO>(q[0], v[0], v[1]);
                unpack2<IO>(q[1], v[2], v[3]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = t + i < lim ? v[i] : 0.f;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (t + i < lim) v[i] = IO::ld(row, t + i);
        }
    }
    return make_float4(v[0], v[1], v[2], v[3]);
}

}  // namespace
}  // namespace lc
