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
__device__ __forceinline__ float softplus_of(float w, float* rate = nullptr)      // rate: its slope, 1 / (1 + exp(-w))
{
    const float e = exp2_of(-LOG2E * fabsf(w)), f = 1.f + e, d = f - 1.f;
    const float l = d == 0.f ? e : 0.69314718055994531f * __builtin_amdgcn_logf(f) * (e * __builtin_amdgcn_rcpf(d));
    if (rate) *rate = __builtin_amdgcn_rcpf(f) * (w < 0.f ? e : 1.f);
    return fmaxf(w, 0.f) + l;      // (NaN by way of l)
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
// (`lane` the same in all lanes)
__device__ __forceinline__ float lane_of(float x, int lane) { return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(x), lane)); }

// (decay p, state h) of each lane -> h behind all lanes up to it (p is used up), for two states at once.  A step adds, and multiplies by,
// a lower lane's value within the instruction (a lane that has no such lane keeps what it has), and the other state's two lie between an
// instruction and the next that permutes its result, which needs two.  In plain code the compiler spent three instructions on each.
#define LC_STEP(c, m)                                                                                                              \
    "v_fmac_f32_dpp %1, %1, %0 " c " row_mask:" m " bank_mask:0xf\n v_fmac_f32_dpp %3, %3, %2 " c " row_mask:" m " bank_mask:0xf\n" \
    "v_mul_f32_dpp %0, %0, %0 " c " row_mask:" m " bank_mask:0xf\n v_mul_f32_dpp %2, %2, %2 " c " row_mask:" m " bank_mask:0xf\n"
__device__ __forceinline__ void scan_up(float& p0, float& h0, float& p1, float& h1)
{
    asm("s_nop 1\n" LC_STEP("row_shr:1", "0xf") LC_STEP("row_shr:2", "0xf") LC_STEP("row_shr:4", "0xf") LC_STEP("row_shr:8", "0xf")
            LC_STEP("row_bcast:15", "0xa")      // a row's last lane to the next row
        "v_fmac_f32_dpp %1, %1, %0 row_bcast:31 row_mask:0xc bank_mask:0xf\n v_fmac_f32_dpp %3, %3, %2 row_bcast:31 row_mask:0xc bank_mask:0xf\n"
        "s_nop 1"
        : "+v"(p0), "+v"(h0), "+v"(p1), "+v"(h1));
}

__device__ __forceinline__ float scan_rows_down(float p, float v)      // the rows' first lanes hold the rows' totals
{
    const int row = (int)(__lane_id() >> 4);
    const float v3 = lane_of(v, 48), v2 = __builtin_fmaf(lane_of(p, 32), v3, lane_of(v, 32)), v1 = __builtin_fmaf(lane_of(p, 16), v2, lane_of(v, 16));
    return __builtin_fmaf(p, row == 0 ? v1 : row == 1 ? v2 : row == 2 ? v3 : 0.f, v);
}
// (decay p, value v) of each lane, towards lower lanes -> v in front of all lanes from it on (p is used up)
__device__ __forceinline__ void scan_down(float& p0, float& v0, float& p1, float& v1)
{
    asm("s_nop 1\n" LC_STEP("row_shl:1", "0xf") LC_STEP("row_shl:2", "0xf") LC_STEP("row_shl:4", "0xf") LC_STEP("row_shl:8", "0xf") "s_nop 1"
        : "+v"(p0), "+v"(v0), "+v"(p1), "+v"(v1));
    v0 = scan_rows_down(p0, v0);
    v1 = scan_rows_down(p1, v1);
}

// The same for one state: what an instruction permutes needs two more behind the one that made it.
#define LC_STEP1(c, m)                                                             \
    "v_fmac_f32_dpp %1, %1, %0 " c " row_mask:" m " bank_mask:0xf\n"              \
    "v_mul_f32_dpp %0, %0, %0 " c " row_mask:" m " bank_mask:0xf\n s_nop 0\n"
__device__ __forceinline__ void scan_up(float& p, float& h)
{
    asm("s_nop 1\n" LC_STEP1("row_shr:1", "0xf") "s_nop 0\n" LC_STEP1("row_shr:2", "0xf") "s_nop 0\n" LC_STEP1("row_shr:4", "0xf") "s_nop 0\n"
            LC_STEP1("row_shr:8", "0xf") "s_nop 0\n" LC_STEP1("row_bcast:15", "0xa") "s_nop 0\n"
        "v_fmac_f32_dpp %1, %1, %0 row_bcast:31 row_mask:0xc bank_mask:0xf\n s_nop 1"
        : "+v"(p), "+v"(h));
}
// (decay p, value v) of each lane, towards lower lanes -> v in front of all lanes from it on (p is used up)
__device__ __forceinline__ void scan_down(float& p, float& v)
{
    asm("s_nop 1\n" LC_STEP1("row_shl:1", "0xf") "s_nop 0\n" LC_STEP1("row_shl:2", "0xf") "s_nop 0\n" LC_STEP1("row_shl:4", "0xf") "s_nop 0\n"
            LC_STEP1("row_shl:8", "0xf") "s_nop 1"
        : "+v"(p), "+v"(v));
    v = scan_rows_down(p, v);
}
#undef LC_STEP1
#undef LC_STEP

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

// one element, rounded to the nearest by the instruction that does so
template <class IO>
__device__ __forceinline__ void put1(typename IO::T* p, uint32_t i, float v)
{
    if constexpr (mu::IsBf<IO>::v) p[i] = (uint16_t)mu::pack_bf2(v, v);
    else IO::st(p, i, v);
}

// Lane l has the wave's sum of v[l % 4]: two exchanges that halve what is to be added, then lanes of the same l % 4
__device__ __forceinline__ float sums_of_wave(float v0, float v1, float v2, float v3)
{
    const bool odd = __lane_id() & 1, high = __lane_id() & 2;
    const float a = (odd ? v1 : v0) + dpp<0xB1>(odd ? v0 : v1, 0.f), b = (odd ? v3 : v2) + dpp<0xB1>(odd ? v2 : v3, 0.f);
    float c = (high ? b : a) + dpp<0x4E>(high ? a : b, 0.f);
    c += dpp<0x124>(c, 0.f);
    c += dpp<0x128>(c, 0.f);
    const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(c), __float_as_uint(c), false, false);      // of the other row of a pair
    c = __uint_as_float(rows[0]) + __uint_as_float(rows[1]);
    const auto halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(c), __float_as_uint(c), false, false);
    return __uint_as_float(halves[0]) + __uint_as_float(halves[1]);
}

// x, with `v` in one lane
__device__ __forceinline__ float with_lane(float x, int lane, float v) { return (int)__lane_id() == lane ? v : x; }

// Of a chunk of a row: `row` points to its first place, the same for all lanes (so that a lane's address is one 32-bit offset), the row goes on
// for n places, and places from `lim` on count for nothing.

// eight neighbouring elements as they lie in memory, from place t on (`full`: a chunk's are all there, which all lanes know)
template <class IO>
__device__ __forceinline__ void ask8(const typename IO::T* row, int t, int n, int lim, Raw8<IO>& r, bool full)
{
    if (full) r.load(row + (uint32_t)t);
    else if (t < lim) load_raw<IO>(row + (uint32_t)t, n - t < VE ? n - t : VE, r);
    else r.zero();
}
// four of them
typedef uint32_t At2x2 __attribute__((ext_vector_type(2), aligned(2)));
template <class IO>
struct Raw4 {
    static constexpr int W = sizeof(typename IO::T) == 4 ? 4 : 2;
    uint32_t w[W];
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = 0;
    }
    __device__ __forceinline__ void ask(const typename IO::T* row, int t, int n, bool full)
    {
        if (full || t + 4 <= n) {
            typedef typename std::conditional<W == 4, At4, At2x2>::type V;
            const V q = *reinterpret_cast<const V*>(row + (uint32_t)t);
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = q[i];
            return;
        }
        zero();
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i < n) {
                if constexpr (W == 4) w[i] = __float_as_uint(row[t + i]);
                else w[i / 2] |= (uint32_t)*reinterpret_cast<const uint16_t*>(row + (uint32_t)(t + i)) << (i % 2 * 16);
            }
    }
    __device__ __forceinline__ float4 get(int t, int lim, bool full) const
    {
        float v[4];
        if constexpr (W == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
        } else {
            unpack2<IO>(w[0], v[0], v[1]);
            unpack2<IO>(w[1], v[2], v[3]);
        }
        if (!full) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = t + i < lim ? v[i] : 0.f;
        }
        return make_float4(v[0], v[1], v[2], v[3]);
    }
};

}  // namespace
}  // namespace lc
