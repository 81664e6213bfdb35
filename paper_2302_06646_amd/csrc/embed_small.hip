// Gradient of an embedding whose table has at most 256 rows (bytes), 16-bit rows in the convolution's layout [B,H,N]: a product with
// the tokens' one-hot matrix on the matrix cores,
//     dE[v,h] = f . sum over (b,t) of dy[b,h,t] [ids[b,t] = v],
// where dy's rows are the left operand as they lie in memory and the right one is made in registers from the tokens.  Its entries are 0
// and 2 (the sums are halved as they leave the registers), so the products are exact and the sums those of fp32; dy is read once, nothing
// is sorted and nothing transposed.  For a tile of tokens 16 j .. 16 j + 15 a lane needs [token = 16 j + lane mod 16] at eight places: a
// word of two halves that are 0x4000 (2.0 in both types) where the low four bits agree, once for all tiles, and a bit of the set of high
// four bits, moved under it: two plain instructions a word.  A wave keeps 32 channels by 256 tokens of dE (128 accumulators, two waves a
// SIMD), its workgroup's four waves share out a range of 32-place steps, and the ranges' sums are added in order by a second kernel.
// 8 x 16384 tokens x 256 in fp16: kernels of 44 us with dropout 0.1, 36 without (sorted, with it: 58).
// Bound by vector issue, 453 instructions a step with the generator's two blocks for every lane, 320 without, 32 of them matrix instructions,
// at two waves a SIMD.  About 12 us do not grow with the length (22 and 32 at half and whole length, without dropout): first loads, sums
// in LDS, the ranges' sums (17 MB out and in).  With rows asked for one to four steps ahead this kernel takes 38.9 to 40.5.
// What is not finite would reach every token of its channel (0 times infinity), and twice a sum may pass the range of bf16 and fp32 where
// the sum does not: a wave that finds such a sum takes its range's places one by one instead, so that it stays with its token.
// 228 us where every wave does so, 71 where one of them does, for 43.
#include "vec8.hpp"

namespace lc {
namespace {

constexpr int VT = 16, MT = 2, CH = 16 * MT, WAVES = 4, PAD = 4;      // tiles of 16 tokens; tiles of 16 channels; channels of a workgroup; its waves
constexpr int ROOM = SMALL_TABLE * (CH + PAD);                        // LDS floats of a workgroup's sums, [token][channel]
constexpr int AHEAD = 2;                                              // steps whose rows are asked for ahead
constexpr int PIECES = 512;                                           // workgroups wanted: two on each of 256 compute units

struct Steps {
    uint32_t of_row, all, each, ranges, blocks;      // steps of a sequence; of all; of a range; ranges; blocks of 32 channels
    uint32_t most;                                   // ranges there may be: does not fall as B grows
};
Steps steps(int64_t B, int64_t N, int64_t H)
{
    Steps s;
    s.of_row = (uint32_t)((N + 31) / 32);
    s.all = (uint32_t)B * s.of_row;
    s.blocks = (uint32_t)((H + CH - 1) / CH);
    const uint32_t wanted = PIECES / s.blocks > 1 ? PIECES / s.blocks : 1, worth = (s.all + 4 * WAVES - 1) / (4 * WAVES);      // four steps of a wave at least
    s.most = worth < wanted ? worth : wanted;
    s.each = (s.all + s.most - 1) / s.most;
    s.ranges = (s.all + s.each - 1) / s.each;
    return s;
}
__host__ __device__ inline size_t range_floats(const Steps& s) { return (size_t)SMALL_TABLE * s.blocks * CH; }

typedef uint16_t us2 __attribute__((ext_vector_type(2)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
union Frag {
    uint32_t w[4];
    mu::h8 h;
    b8 b;
};
template <class IO>
__device__ __forceinline__ mu::f4 product(const Frag& a, const Frag& b, mu::f4 c)
{
    if constexpr (mu::IsBf<IO>::v) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.b, b.b, c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(a.h, b.h, c, 0, 0, 0);
}

// A lane's eight places of a step are 8 (lane / 16) .. + 7 of it, or, at a sequence's end, the last eight, those of other lanes left
// out.  `element`: of the row's first place of the step and the lane's group, moved on by whole steps.
struct Cursor {
    uint32_t t;            // the step's first place
    int64_t element;
    __device__ __forceinline__ void next(uint32_t N, int64_t wrap)      // wrap: from behind a row's steps to the next row's first
    {
        t += 32;
        element += 32;
        if (t >= N) { t = 0; element += wrap; }
    }
    // how far the lane's eight places lie before those of its group (0 but at a sequence's end)
    __device__ __forceinline__ uint32_t early(uint32_t N, uint32_t in_step) const
    {
        const uint32_t want = t + in_step, last = N - VE;
        return want > last ? want - last : 0u;
    }
};

template <class ID>
struct Ids {
    typedef ID two __attribute__((ext_vector_type(16 / sizeof(ID)), aligned(sizeof(ID))));
    static constexpr int PER = 16 / sizeof(ID);
    two v[VE / PER];
    __device__ __forceinline__ void load(const ID* p)
    {
#pragma unroll
        for (int i = 0; i < VE / PER; ++i) v[i] = reinterpret_cast<const two*>(p)[i];
    }
    __device__ __forceinline__ ID operator[](int j) const { return v[j / PER][j % PER]; }
};
// bits 2 i, 2 i + 1 as masks of a word's halves
__device__ __forceinline__ uint32_t half_masks(uint32_t bits, int i)
{
    return (bits >> (2 * i) & 1u ? 0xffffu : 0u) | (bits >> (2 * i + 1) & 1u ? 0xffff0000u : 0u);
}
// two tokens in the halves of a word, any that is not in 0 .. 65535 as 65535
__device__ __forceinline__ uint32_t both(int32_t a, int32_t b)
{
    const uint32_t lo = (uint32_t)a < 0xffffu ? (uint32_t)a : 0xffffu, hi = (uint32_t)b < 0xffffu ? (uint32_t)b : 0xffffu;
    return lo | hi << 16;
}
__device__ __forceinline__ uint32_t both(int64_t a, int64_t b)
{
    const auto low = [](int64_t v) {      // the upper half not zero: 2^31 and more
        const uint32_t up = (uint32_t)((uint64_t)v >> 32);
        return (int32_t)((uint32_t)v | (up < 1u ? up : 1u) << 31);
    };
    return both(low(a), low(b));
}

template <class IO, class ID, bool DROP>
__global__ void __launch_bounds__(64 * WAVES, 2)
embed_small_kernel(const typename IO::T* __restrict__ dy, const ID* __restrict__ ids, float* __restrict__ part, uint32_t N, uint32_t H, uint32_t V,
                   Steps s, Drop d)
{
    __shared__ float sums[ROOM];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, group = lane >> 4;
    const uint32_t block = blockIdx.x % s.blocks, range = blockIdx.x / s.blocks, h0 = block * CH;
    const uint32_t begin = range * s.each, stop = begin + s.each < s.all ? begin + s.each : s.all, each = (stop - begin + WAVES - 1) / WAVES;
    const uint32_t from = begin + wave * each < stop ? begin + wave * each : stop, to = from + each < stop ? from + each : stop;
    const uint64_t call = DROP ? call_of(d) : 0;
    uint32_t h[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) h[m] = h0 + 16 * m + n < H ? h0 + 16 * m + n : H - 1;      // (channels there are not: nobody takes their sums)
    mu::f4 acc[MT][VT] = {};
    const uint32_t me = (uint32_t)n * 0x10001u;
    const us2 unit = {1, 1}, two = {0x4000, 0x4000}, top = {(uint16_t)(V - 1), (uint16_t)(V - 1)};
    const uint32_t row0 = from / s.of_row, in_step = (uint32_t)group * VE;
    const int64_t past = (int64_t)s.of_row * 32;
    // of the next step's tokens; of the rows asked for AHEAD steps before their use; of the step worked on
    Cursor tokens{(from - row0 * s.of_row) * 32, 0};
    tokens.element = (int64_t)row0 * N + tokens.t + in_step;
    Cursor rows = tokens, now = tokens;
    rows.element = now.element = ((int64_t)row0 * H + h[0]) * N + tokens.t + in_step;
    const int64_t wrap = (int64_t)H * N - past;
    int64_t apart[MT];      // from the first tile's row to the others'
#pragma unroll
    for (int m = 0; m < MT; ++m) apart[m] = (int64_t)(h[m] - h[0]) * N;
    Ids<ID> id;
    Raw8<IO> raw[AHEAD][MT];
    const auto ask_tokens = [&] {
        id.load(ids + tokens.element - tokens.early(N, in_step));
        tokens.next(N, (int64_t)N - past);
    };
    const auto ask_rows = [&](Raw8<IO>(&to_raw)[MT]) {
        const typename IO::T* p = dy + rows.element - rows.early(N, in_step);
#pragma unroll
        for (int m = 0; m < MT; ++m) to_raw[m].load(p + apart[m]);
        rows.next(N, wrap);
    };
    if (from < to) ask_tokens();
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        if (from + u < to) ask_rows(raw[u]);
    const auto work = [&](uint32_t step, Raw8<IO>(&mine)[MT]) {
        const uint32_t early = now.early(N, in_step);
        const int64_t element = now.element - early;
        now.next(N, wrap);
        Frag a[MT];
        uint32_t low[4], high[4], there[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t pair = both(id[2 * i], id[2 * i + 1]);
            const us2 over = __builtin_elementwise_min(__builtin_elementwise_sub_sat(__builtin_bit_cast(us2, pair), top), unit);
            there[i] = __builtin_bit_cast(uint32_t, (us2)(over - unit));      // a token of the table (what is not, multiplies zeros)
            low[i] = __builtin_bit_cast(uint32_t, (us2)(two << (__builtin_bit_cast(us2, pair ^ me) & (us2){15, 15}))) & 0x40004000u;
            high[i] = __builtin_bit_cast(uint32_t, (us2)(unit << (__builtin_bit_cast(us2, pair >> 4) & (us2){15, 15})));
        }
        if (step + 1 < to) ask_tokens();
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("" : "+v"(low[i]));      // (or the mask above is taken again for every tile, in slower instructions)
        if (__ballot(early)) {      // the first `early` of the eight are another lane's (all, where the group has none)
            const uint32_t valid = early < VE ? 0xffu << early & 0xffu : 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) there[i] &= half_masks(valid, i);
        }
        uint32_t keep[MT][4];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            uint4 k = make_uint4(~0u, ~0u, ~0u, ~0u);
            if constexpr (DROP) k = kept_words_at((uint64_t)(element + apart[m]), d, call);
            keep[m][0] = k.x; keep[m][1] = k.y; keep[m][2] = k.z; keep[m][3] = k.w;
        }
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) a[m].w[i] = mine[m].w[i] & there[i] & keep[m][i];
        if (step + AHEAD < to) ask_rows(mine);
#pragma unroll
        for (int j = 0; j < VT; ++j) {
            Frag b;
#pragma unroll
            for (int i = 0; i < 4; ++i) b.w[i] = (j <= 14 ? high[i] << (14 - j) : high[i] >> 1) & low[i];
#pragma unroll
            for (int m = 0; m < MT; ++m) acc[m][j] = product<IO>(a[m], b, acc[m][j]);
        }
    };
    for (uint32_t step = from; step < to; step += AHEAD) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (step + u < to) work(step + u, raw[u]);
    }
    float zero = 0.f;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < VT; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) zero = __builtin_fmaf(acc[m][j][r], 0.f, zero);
    const bool clean = __ballot(!(zero == 0.f)) == 0;
    for (int w = 0; w < WAVES; ++w) {      // (every wave comes here as often)
        if (w == wave) {
            if (clean) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int j = 0; j < VT; ++j) {
                        float4* q = reinterpret_cast<float4*>(sums + (16 * j + n) * (CH + PAD) + 16 * m + 4 * group);
                        const mu::f4 half = acc[m][j] * 0.5f;      // (exact: they are multiples of 2^-132, twice bf16's smallest number)
                        float4 t = make_float4(half[0], half[1], half[2], half[3]);
                        if (w) {
                            const float4 o = *q;
                            t = make_float4(o.x + t.x, o.y + t.y, o.z + t.z, o.w + t.w);
                        }
                        *q = t;
                    }
            } else {
                if (w == 0)
                    for (int i = lane; i < ROOM; i += 64) sums[i] = 0.f;
                // Tokens and rows of a step are asked for before the first is added; then a lane adds to its channel's column of the
                // table, place by place: LDS takes a wave's additions in order, and none waits for another.
                const bool there = lane < CH && h0 + lane < H;
                for (uint32_t step = from; step < to; ++step) {
                    const uint32_t b = step / s.of_row, t0 = (step - b * s.of_row) * 32, here = N - t0 < 32 ? N - t0 : 32;
                    const ID v = ids[(size_t)b * N + t0 + (lane & 31u) % here];
                    const uint32_t token = v >= 0 && v < (ID)V ? (uint32_t)v : V;
                    const size_t e = ((size_t)b * H + h0 + (there ? lane : 0)) * N + t0;
                    float x[32];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        Raw8<IO> r;
                        load_raw<IO>(dy + e + VE * q, (int)here - VE * q, r);
                        if constexpr (DROP) {
                            const uint4 k = kept_words_at(e + VE * q, d, call);
                            r.w[0] &= k.x; r.w[1] &= k.y; r.w[2] &= k.z; r.w[3] &= k.w;
                        }
                        float y[VE];
                        r.get(y);
#pragma unroll
                        for (int j = 0; j < VE; ++j) x[VE * q + j] = y[j];
                    }
#pragma unroll
                    for (uint32_t i = 0; i < 32; ++i) {
                        const uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)token, (int)i);
                        if (i < here && at < V && there)
                            __hip_atomic_fetch_add(sums + at * (CH + PAD) + lane, x[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
                    }
                }
            }
        }
        __syncthreads();
    }
    float* out = part + range * range_floats(s);
    for (uint32_t i = threadIdx.x; i < V * (CH / 4); i += 64 * WAVES) {
        const uint32_t v = i / (CH / 4), c = i % (CH / 4) * 4;
        *reinterpret_cast<float4*>(out + (size_t)v * s.blocks * CH + h0 + c) = *reinterpret_cast<const float4*>(sums + v * (CH + PAD) + c);
    }
}

constexpr int SUM_T = 256, SHARES = 4;

// dE = f times the ranges' sums, four shares of the ranges side by side and then in order
__global__ void __launch_bounds__(SUM_T)
embed_small_sum_kernel(const float* __restrict__ part, float* __restrict__ dE, uint32_t H, uint32_t V, float f, Steps s)
{
    __shared__ float4 sums[SHARES][64];
    const uint32_t share = threadIdx.x / 64, lane = threadIdx.x % 64, wide = s.blocks * CH / 4, i = blockIdx.x * 64 + lane;
    const uint32_t each = (s.ranges + SHARES - 1) / SHARES, from = share * each, to = from + each < s.ranges ? from + each : s.ranges;
    const size_t stride = (size_t)SMALL_TABLE * wide;
    const bool there = i < V * wide;
    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
    if (there) {
        const float4* p = reinterpret_cast<const float4*>(part) + i;
#pragma unroll 8
        for (uint32_t r = from; r < to; ++r) {
            const float4 v = p[r * stride];
            t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
        }
    }
    sums[share][lane] = t;
    __syncthreads();
    if (share || !there) return;
#pragma unroll
    for (int w = 1; w < SHARES; ++w) {
        const float4 v = sums[w][lane];
        t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
    }
    const float o[4] = {t.x * f, t.y * f, t.z * f, t.w * f};
    const uint32_t v = i / wide, c = (i - v * wide) * 4;
#pragma unroll
    for (uint32_t j = 0; j < 4; ++j)
        if (c + j < H) dE[(size_t)v * H + c + j] = o[j];
}

template <class IO, class ID>
hipError_t run(const EmbedArgs& a, const void* dy, float* dE, float* part, hipStream_t st)
{
    const Steps s = steps(a.B, a.N, a.H);
    dim3 g, gs;
    hipError_t e = launch_grid((uint64_t)s.ranges * s.blocks, 64 * WAVES, &g);
    if (e == hipSuccess) e = launch_grid(((uint64_t)a.V * s.blocks * (CH / 4) + 63) / 64, SUM_T, &gs);
    if (e != hipSuccess) return e;
    const auto kernel = a.drop.threshold ? embed_small_kernel<IO, ID, true> : embed_small_kernel<IO, ID, false>;
    hipLaunchKernelGGL(kernel, g, dim3(64 * WAVES), 0, st, (const typename IO::T*)dy, (const ID*)a.ids, part, (uint32_t)a.N, (uint32_t)a.H,
                       (uint32_t)a.V, s, a.drop);
    hipLaunchKernelGGL(embed_small_sum_kernel, gs, dim3(SUM_T), 0, st, (const float*)part, dE, (uint32_t)a.H, (uint32_t)a.V, a.scale * a.drop.scale, s);
    return hipGetLastError();
}

}  // namespace

size_t embed_small_workspace_bytes(int64_t B, int64_t N, int64_t H)
{
    const Steps s = steps(B, N, H);
    return s.most * range_floats(s) * sizeof(float);
}

hipError_t embed_small_bwd(const EmbedArgs& a, const void* dy, float* dE, void* ws, hipStream_t st)
{
    float* part = (float*)ws;
    if (a.io == LONGCONV_F16)
        return a.id_bytes == 8 ? run<IoF16, int64_t>(a, dy, dE, part, st) : run<IoF16, int32_t>(a, dy, dE, part, st);
    return a.id_bytes == 8 ? run<IoBF16, int64_t>(a, dy, dE, part, st) : run<IoBF16, int32_t>(a, dy, dE, part, st);
}

}  // namespace lc
