// Embedding: y = m . scale . E[id] with m a dropout mask (vec8.hpp), in the layout of dense layers [B,N,H] or in the convolution's
// [B,H,N], and the gradient dE[v] = scale . sum over the places with id = v of m . dy.
//
// The gradient adds up in a fixed order: the tokens' places are sorted by token (stable, so by place within a token), a thread
// takes eight columns of a chunk of consecutive sorted places and sums runs of one token in fp32; a run that crosses chunks leaves
// a partial sum in each, which are added in an order that the run's length gives.  Every row of dy is read once.
// 16384 tokens x 768 in bf16, V = 32768, dropout 0.1: 46 us, 25 for the bytes (126 MB, most of them zeros of dE): four sorting launches of
// 5 to 7, bound by their chains of loads, the sums 16 (scattered rows, and the generator), the joins 7.  Small tables of 16-bit rows in
// [B,H,N] go through the matrix cores instead (embed_small.hip).
#include <type_traits>

#include "vec8.hpp"

namespace lc {
namespace {

constexpr int RADIX = 512, SORT_T = 256, SORT_W = SORT_T / 64;                  // digits of at most nine bits; threads and waves of a tile
constexpr int TILE_MIN = 1024, TILES_MAX = 128, ROWS = TILE_MIN / SORT_T;        // tiles of a sorting pass; rows of 64 that a wave asks for at once
// Tokens that one workgroup sorts by itself, and its threads.  8192 (V = 32768, with 100 MB of zeros beside the sort): 20 us, four launches of
// tiles 30 and the gaps between them; 16384 do not fit its LDS, and took 53 us through memory (tiles 24).
constexpr int ALONE = 8192, ALONE_T = 1024;
constexpr int CHUNK_MIN = 8;                                                    // sorted places of a thread, at least (a whole number of AHEADs)
constexpr int AHEAD = 8;                                                        // rows of dy that a thread asks for before it adds the first
constexpr int JOIN_GROUPS = 256;                                                // workgroups that join a run's partial sums
constexpr int JOIN_T = 1024;                                                    // and their threads

// a token's row, or V for one that names none
template <class ID>
__device__ __forceinline__ uint32_t row_of(const ID* ids, int64_t i, uint32_t V)
{
    const ID v = ids[i];
    return v >= 0 && (uint64_t)v < V ? (uint32_t)v : V;
}

// ---- forward ---------------------------------------------------------------------------------------------------------

// [B,N,H]: a thread writes eight consecutive elements, of one row or of the end of one and the beginning of the next ones.  Bound by
// memory: 16384 tokens x 768, fp32 table to bf16, V = 32768: 10.8 us back to back, 43 MB at 4.0 TB/s.  Two and four pieces a thread, asked
// for at once, were no faster (kernel 12.4 and 10.8 against 9.7 to 11.6 us).
template <class IO, class W, class ID, class I>
__global__ void __launch_bounds__(256)
embed_rows_kernel(const ID* __restrict__ ids, const typename W::T* __restrict__ E, typename IO::T* __restrict__ y, I n, uint32_t H, uint32_t V,
                  float scale, Drop d)
{
    const I e = ((I)blockIdx.x * 256 + threadIdx.x) * VE;
    if (e >= n) return;
    const I row = e / H;
    const uint32_t c = (uint32_t)(e - row * H), r = row_of(ids, (int64_t)row, V);
    const bool whole = c + VE <= H;
    Raw8<W> raw;
    if (H < VE) raw.zero();
    else raw.load(E + (size_t)(r < V ? r : 0) * H + (whole ? c : 0));
    const int here = n - e < (I)VE ? (int)(n - e) : VE;
    float v[VE];
    raw.get(v);
    if (!whole) {
        I rw = row;
        uint32_t cc = c;
        for (int i = 0; i < here; ++i) {
            const uint32_t q = row_of(ids, (int64_t)rw, V);
            const float t = q < V ? W::ld(E, (size_t)q * H + cc) : 0.f;
#pragma unroll
            for (int j = 0; j < VE; ++j)
                if (j == i) v[j] = t;
            if (++cc == H) { cc = 0; ++rw; }
        }
    }
    const uint32_t m = whole && r >= V ? 0u : d.threshold ? kept8(e >> 3, d, call_of(d)) : 0xffu;
    const float f = scale * d.scale;
#pragma unroll
    for (int i = 0; i < VE; ++i) v[i] = m >> i & 1u ? v[i] * f : 0.f;
    store8<IO, true>(y + e, here, v);
}

constexpr int TT = 64, TH = 64;      // tokens and channels of a tile

// [B,H,N]: a workgroup takes a tile of 64 tokens and 64 channels through LDS: rows of the table in, rows of the sequences out.  Bound by
// the writes: 8 x 16384 tokens x 256 to fp16, V = 256: 13.4 us, 68 MB at 5.1 TB/s.
template <class IO, class W, class ID>
__global__ void __launch_bounds__(256)
embed_columns_kernel(const ID* __restrict__ ids, const typename W::T* __restrict__ E, typename IO::T* __restrict__ y, uint32_t N, uint32_t H,
                     uint32_t V, uint32_t tiles_t, uint32_t tiles_h, float scale, Drop d)
{
    __shared__ float tile[TH][TT + 1];
    const uint32_t tt = blockIdx.x % tiles_t, th = blockIdx.x / tiles_t % tiles_h, b = blockIdx.x / tiles_t / tiles_h;
    const uint32_t t0 = tt * TT, h0 = th * TH, tid = threadIdx.x, s = tid % 8;
#pragma unroll
    for (uint32_t k = 0; k < TT / 32; ++k) {
        const uint32_t t = tid / 8 + 32 * k, h = h0 + VE * s;
        const uint32_t r = t0 + t < N ? row_of(ids, (int64_t)b * N + t0 + t, V) : V;
        float v[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = 0.f;
        if (r < V && h < H) load8<W>(E + (size_t)r * H + h, (int)(H - h), v);
#pragma unroll
        for (int i = 0; i < VE; ++i) tile[VE * s + i][t] = v[i];
    }
    __syncthreads();
    const uint64_t call = call_of(d);
    const float f = scale * d.scale;
#pragma unroll
    for (uint32_t k = 0; k < TH / 32; ++k) {
        const uint32_t h = h0 + tid / 8 + 32 * k, t = t0 + VE * s;
        if (h >= H || t >= N) continue;
        const size_t e = ((size_t)b * H + h) * N + t;
        const uint32_t m = d.threshold ? kept8_at(e, d, call) : 0xffu;
        float v[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = m >> i & 1u ? tile[h - h0][VE * s + i] * f : 0.f;
        store8<IO, true>(y + e, (int)(N - t), v);
    }
}

// ---- gradient --------------------------------------------------------------------------------------------------------

// dE <- 0, by the workgroups of a sorting launch that have nothing to sort: the sort takes its time and hardly any of the memory's
struct Fill {
    float* p;
    int64_t n;
    Fill share(int i, int of) const      // piece i of so many, whole sixteen bytes each
    {
        const int64_t each = (n / 4 + of - 1) / of * 4, from = each * i < n ? each * i : n, to = i + 1 < of && from + each < n ? from + each : n;
        return {p + from, to - from};
    }
    unsigned groups(int threads) const      // four pieces of sixteen bytes a thread, and 1024 workgroups at most
    {
        const int64_t want = (n + threads * 16 - 1) / (threads * 16);
        return (unsigned)(want < 1024 ? want : 1024);
    }
};
__device__ __forceinline__ void fill_zero(const Fill& f, int64_t group, int64_t groups)
{
    const int64_t stride = groups * blockDim.x * 4;
    for (int64_t i = (group * blockDim.x + threadIdx.x) * 4; i < f.n; i += stride) {
        if (i + 4 <= f.n) put_once(reinterpret_cast<float4*>(f.p + i), make_float4(0.f, 0.f, 0.f, 0.f));
        else
            for (int64_t j = i; j < f.n; ++j) f.p[j] = 0.f;
    }
}

// [B,H,N] -> rows of `stride` channels, dropped entries zero (the factor of the kept ones comes in with `scale`, so nothing is rounded),
// in tiles of 64 x 64: by a kernel, or behind a sort's launches as the zeros are.
struct Transpose {
    const void* dy;
    void* out;
    uint32_t N, H, stride, tiles_t, tiles_h;
    Drop d;
    uint32_t from, tiles;      // this launch's share of the tiles
    Transpose share(int i, int of) const
    {
        Transpose t = *this;
        const uint32_t each = (tiles + of - 1) / of, at = each * i < tiles ? each * i : tiles;
        t.from = from + at;
        t.tiles = tiles - at < each ? tiles - at : each;
        return t;
    }
};
typedef float TransposeTile[TT][TH + 1];
template <class IO>
__device__ __forceinline__ void transpose_tile(const Transpose& a, uint32_t number, TransposeTile& tile)
{
    typedef typename IO::T T;
    const uint32_t id = a.from + number, tt = id % a.tiles_t, th = id / a.tiles_t % a.tiles_h, b = id / a.tiles_t / a.tiles_h;
    const uint32_t t0 = tt * TT, h0 = th * TH, tid = threadIdx.x, s = tid % 8;
    const uint64_t call = call_of(a.d);
#pragma unroll
    for (uint32_t k = 0; k < TH / 32; ++k) {
        const uint32_t hh = tid / 8 + 32 * k, h = h0 + hh, t = t0 + VE * s;
        float v[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = 0.f;
        if (h < a.H && t < a.N) {
            const size_t e = ((size_t)b * a.H + h) * a.N + t;
            load8<IO>((const T*)a.dy + e, (int)(a.N - t), v);
            const uint32_t m = a.d.threshold ? kept8_at(e, a.d, call) : 0xffu;
#pragma unroll
            for (int i = 0; i < VE; ++i) v[i] = m >> i & 1u ? v[i] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < VE; ++i) tile[VE * s + i][hh] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (uint32_t k = 0; k < TT / 32; ++k) {
        const uint32_t t = tid / 8 + 32 * k, h = h0 + VE * s;
        if (t0 + t >= a.N || h >= a.stride) continue;      // (stride is a multiple of eight)
        float v[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = tile[t][VE * s + i];
        store8<IO>((T*)a.out + ((size_t)b * a.N + t0 + t) * a.stride + h, VE, v);
    }
}
template <class IO>
__global__ void __launch_bounds__(256) embed_transpose_kernel(Transpose a)
{
    __shared__ TransposeTile tile;
    transpose_tile<IO>(a, blockIdx.x, tile);
}

// One pass of the stable sort by token: `shift` and `bits` name the digit.  ID: the pass reads the tokens themselves, whose places are
// their numbers; without (void) it reads the pairs that the pass before left.
template <class ID>
struct Tokens {
    const ID* ids;
    const uint32_t *key, *pos;
    uint32_t V;
    __device__ __forceinline__ uint32_t k(int64_t i) const
    {
        if constexpr (std::is_void<ID>::value) return key[i];
        else return row_of(ids, i, V);
    }
    __device__ __forceinline__ uint32_t p(int64_t i) const
    {
        if constexpr (std::is_void<ID>::value) return pos[i];
        else return (uint32_t)i;
    }
};

// The place of a lane's token among those of its wave's share with the digit: behind those of earlier rows (next[digit], which the
// first lane with the digit moves on by their number) and of earlier lanes.
__device__ __forceinline__ uint32_t place_of(uint32_t digit, bool there, int bits, uint32_t* next)
{
    const int lane = threadIdx.x & 63;
    uint64_t same = __ballot(there);
    for (int b = 0; b < bits; ++b) {
        const uint64_t ones = __ballot(digit >> b & 1u), want = (uint64_t)0 - (digit >> b & 1u);
        same &= ~(ones ^ want);
    }
    const int leader = there ? __ffsll((unsigned long long)same) - 1 : lane;
    uint32_t first = 0;
    if (there && lane == leader) first = atomicAdd(&next[digit], (uint32_t)__popcll(same));
    first = (uint32_t)__shfl((int)first, leader);
    return first + (uint32_t)__popcll(same & ((1ull << lane) - 1ull));
}

// Sum of the numbers of the threads before, for threads 0 .. 255 of a workgroup (all of it has to call).
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t (&waves)[SORT_W])
{
    const int tid = threadIdx.x, lane = tid & 63;
    uint32_t s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t t = (uint32_t)__shfl_up((int)s, d);
        if (lane >= d) s += t;
    }
    if (tid < SORT_T && lane == 63) waves[tid >> 6] = s;
    __syncthreads();
    s -= v;
#pragma unroll
    for (int w = 0; w < SORT_W; ++w)
        if (w < (tid >> 6)) s += waves[w];
    return s;
}

// What the workgroups behind a sorting launch's tiles do meanwhile: zeros, then tiles of the transposition (IO void: there is none).
struct Beside {
    Fill fill;
    uint32_t fills;
    Transpose t;
};
template <class IO>
union SortRoom {
    uint32_t at[SORT_W][RADIX];
    TransposeTile tile;
};
template <>
union SortRoom<void> {
    uint32_t at[SORT_W][RADIX];
};
template <class IO>
__device__ __forceinline__ void beside_the_sort(const Beside& a, uint32_t group, SortRoom<IO>& room)
{
    if (group < a.fills) fill_zero(a.fill, group, a.fills);
    else if constexpr (!std::is_void<IO>::value) transpose_tile<IO>(a.t, group - a.fills, room.tile);
}

// Counts of a tile's tokens by digit: hist[tile][digit], and by waves behind those of all tiles: hist[tiles + 4 tile + wave][digit].
template <class ID, class IO>
__global__ void __launch_bounds__(SORT_T)
sort_count_kernel(Tokens<ID> in, uint32_t* __restrict__ hist, uint32_t* __restrict__ joins, int64_t M, int64_t tile, uint32_t tiles, int shift,
                  int bits, Beside beside)
{
    __shared__ SortRoom<IO> room;
    if (blockIdx.x >= tiles) {
        beside_the_sort<IO>(beside, blockIdx.x - tiles, room);
        return;
    }
    uint32_t(&n)[SORT_W][RADIX] = room.at;
    if (blockIdx.x == 0 && threadIdx.x == 0) *joins = 0;
    const int tid = threadIdx.x, wave = tid >> 6, digits = 1 << bits;
    const uint32_t mask = (uint32_t)digits - 1u;
    const int64_t share = tile / SORT_W, from = blockIdx.x * tile + wave * share + (tid & 63);
    for (int i = tid; i < digits; i += SORT_T)
#pragma unroll
        for (int w = 0; w < SORT_W; ++w) n[w][i] = 0;
    __syncthreads();
    for (int64_t r = 0; r < share; r += 64 * ROWS) {
        uint32_t k[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) k[u] = in.k(from + r + 64 * u < M ? from + r + 64 * u : M - 1);
#pragma unroll
        for (int u = 0; u < ROWS; ++u)
            if (from + r + 64 * u < M) atomicAdd(&n[wave][k[u] >> shift & mask], 1u);
    }
    __syncthreads();
    for (int i = tid; i < digits; i += SORT_T) {
        uint32_t all = 0;
#pragma unroll
        for (int w = 0; w < SORT_W; ++w) {
            hist[((size_t)tiles + blockIdx.x * SORT_W + w) * RADIX + i] = n[w][i];
            all += n[w][i];
        }
        hist[(size_t)blockIdx.x * RADIX + i] = all;
    }
}

// Puts a tile's tokens where they belong: behind all of smaller digits, those of the same digit in earlier tiles, in earlier waves'
// shares of the tile, in earlier rows of 64, and in earlier lanes.
template <class ID, class IO>
__global__ void __launch_bounds__(SORT_T)
sort_place_kernel(Tokens<ID> in, const uint32_t* __restrict__ hist, uint32_t* __restrict__ key, uint32_t* __restrict__ pos, int64_t M,
                  int64_t tile, uint32_t tiles, int shift, int bits, Beside beside)
{
    __shared__ SortRoom<IO> room;
    __shared__ uint32_t waves[SORT_W];
    if (blockIdx.x >= tiles) {
        beside_the_sort<IO>(beside, blockIdx.x - tiles, room);
        return;
    }
    uint32_t(&at)[SORT_W][RADIX] = room.at;      // next place of a wave's tokens with a digit
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, digits = 1 << bits;
    const uint32_t mask = (uint32_t)digits - 1u;
    const int64_t share = tile / SORT_W, from = blockIdx.x * tile + wave * share;
    uint32_t k[ROWS], p[ROWS];
    const auto ask = [&](int64_t r) {
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int64_t i = from + r + 64 * u + lane < M ? from + r + 64 * u + lane : M - 1;
            k[u] = in.k(i);
            p[u] = in.p(i);
        }
    };
    ask(0);
    uint2 all = make_uint2(0, 0), before = make_uint2(0, 0), own[SORT_W];      // digits 2 tid, 2 tid + 1
    if (2 * tid < digits) {
        const auto counts = [&](uint32_t row) { return *reinterpret_cast<const uint2*>(hist + (size_t)row * RADIX + 2 * tid); };
#pragma unroll
        for (int w = 0; w < SORT_W; ++w) own[w] = counts(tiles + blockIdx.x * SORT_W + w);
#pragma unroll 16
        for (uint32_t t = 0; t < tiles; ++t) {
            const uint2 c = counts(t);
            all.x += c.x;
            all.y += c.y;
            if (t < blockIdx.x) { before.x += c.x; before.y += c.y; }
        }
    }
    const uint32_t start = sum_before(all.x + all.y, waves);
    if (2 * tid < digits) {
        uint2 next = make_uint2(start + before.x, start + all.x + before.y);
#pragma unroll
        for (int w = 0; w < SORT_W; ++w) {
            *reinterpret_cast<uint2*>(&at[w][2 * tid]) = next;
            next.x += own[w].x;
            next.y += own[w].y;
        }
    }
    __syncthreads();
    for (int64_t r = 0; r < share && from + r < M; r += 64 * ROWS) {      // (the same for every lane of a wave)
        if (r) ask(r);
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const bool there = from + r + 64 * u + lane < M;
            const uint32_t to = place_of(k[u] >> shift & mask, there, bits, at[wave]);
            if (there) {
                key[to] = k[u];
                pos[to] = p[u];
            }
        }
    }
}

// All passes by one workgroup (the first of the launch), for few tokens: they stay in LDS, and each wave's share in its registers.
template <class ID>
__global__ void __launch_bounds__(ALONE_T)
sort_alone_kernel(Tokens<ID> in, uint32_t* __restrict__ key, uint32_t* __restrict__ pos, uint32_t* __restrict__ joins, int M, int passes, int bits,
                  Fill fill)
{
    constexpr int WAVES = ALONE_T / 64, R = ALONE / ALONE_T;
    __shared__ uint32_t at[WAVES][RADIX], lk[ALONE], lp[ALONE], waves[SORT_W];
    if (blockIdx.x > 0) {
        fill_zero(fill, blockIdx.x - 1, gridDim.x - 1);
        return;
    }
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, digits = 1 << bits;
    if (tid == 0) *joins = 0;
    const uint32_t mask = (uint32_t)digits - 1u;
    const int rows = (M + ALONE_T - 1) / ALONE_T, from = wave * rows * 64;      // rows of 64 of a wave, in order
    uint32_t k[R], p[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = from + 64 * r + lane < M ? from + 64 * r + lane : M - 1;
        k[r] = in.k(i);
        p[r] = (uint32_t)i;
    }
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * bits;
        for (int i = lane; i < digits; i += 64) at[wave][i] = 0;
        if (pass) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int i = from + 64 * r + lane < M ? from + 64 * r + lane : M - 1;
                k[r] = lk[i];
                p[r] = lp[i];
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < rows && from + 64 * r + lane < M) atomicAdd(&at[wave][k[r] >> shift & mask], 1u);
        __syncthreads();
        uint2 mine = make_uint2(0, 0);
        if (2 * tid < digits)
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                mine.x += at[w][2 * tid];
                mine.y += at[w][2 * tid + 1];
            }
        const uint32_t start = sum_before(mine.x + mine.y, waves);
        if (2 * tid < digits) {
            uint2 next = make_uint2(start, start + mine.x);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                uint2* a = reinterpret_cast<uint2*>(&at[w][2 * tid]);
                const uint2 c = *a;
                *a = next;
                next.x += c.x;
                next.y += c.y;
            }
        }
        __syncthreads();
        const bool out = pass == passes - 1;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r >= rows || from + 64 * r >= M) break;      // (the same for every lane of a wave)
            const bool there = from + 64 * r + lane < M;
            const uint32_t to = place_of(k[r] >> shift & mask, there, bits, at[wave]);
            if (there) {
                (out ? key : lk)[to] = k[r];
                (out ? pos : lp)[to] = p[r];
            }
        }
        __syncthreads();      // (what a pass has written, the next one reads)
    }
}

// Sums of runs.  Partial sums lie at part[2 chunk + w]: w = 0 of a run that came in from the chunk before, 1 of one that began here
// and goes on, which is noted down in `joins` (how many, from the third word on their chunks and tokens; in any order, they have nothing to do with each other).
// A thread's columns are eight from c on; where the row's end is not a multiple of eight the last thread begins `skip` columns early
// (NARROW: rows of fewer than eight).  key, pos: readable up to a whole chunk.
template <class IO, bool DROP, bool NARROW>
__global__ void __launch_bounds__(256)
embed_sum_kernel(const typename IO::T* __restrict__ dy, const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos,
                 float* __restrict__ dE, float* __restrict__ part, uint32_t* __restrict__ joins, uint32_t M, uint32_t H, uint32_t stride, uint32_t P,
                 uint32_t V, uint32_t chunk_size, uint32_t chunks, float scale, Drop d)
{
    const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    const uint32_t chunk = (uint32_t)(id / P), slice = (uint32_t)(id - (uint64_t)chunk * P);
    if (chunk >= chunks) return;
    const uint32_t from = chunk * chunk_size, to = from + chunk_size < M ? from + chunk_size : M;
    const uint32_t last = H > VE ? H - VE : 0, c = slice * VE < last ? slice * VE : last, skip = slice * VE - c;
    const int wide = NARROW ? (int)H : VE;
    const uint64_t call = DROP ? call_of(d) : 0;
    const float f = scale * d.scale;
    uint32_t cur = key[from];
    bool came_in = from > 0 && key[from - 1] == cur;
    float acc[VE] = {};
    const auto keep = [&](int w) {
        float4* q = reinterpret_cast<float4*>(part + (((size_t)chunk * 2 + w) * P + slice) * VE);
        q[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
        q[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
    };
    const auto finish = [&] {
        if (cur >= V) return;
        if (came_in) { keep(0); return; }
        float v[VE];
#pragma unroll
        for (int i = 0; i < VE; ++i) v[i] = acc[i] * f;
        float* row = dE + (size_t)cur * H + c;
        if (skip == 0 && wide == VE) store8<IoF32>(row, VE, v);
        else
#pragma unroll
            for (int i = 0; i < VE; ++i)
                if (i >= (int)skip && i < wide) row[i] = v[i];
    };
    for (uint32_t i = from; i < to; i += AHEAD) {
        uint32_t k[AHEAD], p[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; u += 4) {
            const uint4 a = *reinterpret_cast<const uint4*>(key + i + u), b = *reinterpret_cast<const uint4*>(pos + i + u);
            k[u] = a.x; k[u + 1] = a.y; k[u + 2] = a.z; k[u + 3] = a.w;
            p[u] = b.x; p[u + 1] = b.y; p[u + 2] = b.z; p[u + 3] = b.w;
        }
        Raw8<IO> raw[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (i + u >= to) k[u] = V;
            if (k[u] >= V) p[u] = 0;      // (a row that is there, and goes nowhere)
            const typename IO::T* row = dy + (size_t)p[u] * stride + c;
            if constexpr (NARROW) load_raw<IO>(row, wide, raw[u]);
            else raw[u].load(row);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (k[u] != cur) {
                finish();
                cur = k[u];
                came_in = false;
#pragma unroll
                for (int j = 0; j < VE; ++j) acc[j] = 0.f;
            }
            float v[VE];
            raw[u].get(v);
            const uint32_t m = DROP ? kept8_at((size_t)p[u] * H + c, d, call) : 0xffu;
#pragma unroll
            for (int j = 0; j < VE; ++j) acc[j] += !DROP || (m >> j & 1u) ? v[j] : 0.f;
        }
        if (k[AHEAD - 1] >= V) break;      // the tokens that name no row sort last
    }
    if (cur >= V) return;
    if (to < M && key[to] == cur) {
        keep(came_in ? 0 : 1);
        if (!came_in && slice == 0) reinterpret_cast<uint2*>(joins + 2)[atomicAdd(joins, 1u)] = make_uint2(chunk, cur);
    } else finish();
}

// Runs over several chunks: their partial sums, four columns a lane and, where a row has fewer than 256, several chunks side by side in
// a wave; in an order that the run's length alone gives.  Most runs are of two or three chunks: a wave takes one (of 256 columns).
// Those that would take it more than LONG_RUN steps (common tokens) it leaves to its whole workgroup, whose waves take the chunks in
// turn and whose sums are then added in order.  All that are long go that way: the workgroup's list is emptied before it can overflow.
constexpr uint32_t LONG_RUN = 8;
__global__ void __launch_bounds__(JOIN_T)
embed_join_kernel(const uint32_t* __restrict__ key, const float* __restrict__ part, const uint32_t* __restrict__ joins, float* __restrict__ dE,
                  uint32_t M, uint32_t H, uint32_t P, uint32_t chunk_size, uint32_t wide, float f)
{
    constexpr uint32_t WAVES = JOIN_T / 64, LIST = 256;
    __shared__ float4 sums[WAVES][64];
    __shared__ uint32_t longs[LIST], count;
    const uint32_t blocks = (P * 2 + wide - 1) / wide, items = joins[0] * blocks, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    const uint32_t side = 64 / wide, mine = lane / wide;      // chunks of a wave at once; the lane's among them
    // the last chunk of a run, the last that begins with its token: the lanes look at the next 64, and, if all do, at 64 places of what is
    // left at a time
    const auto last_chunk = [&](uint2 run) {
        const auto begins = [&](uint32_t q, uint32_t end) { return (uint32_t)__popcll(__ballot(q < end && key[(size_t)q * chunk_size] == run.y)); };
        uint32_t end = (M + chunk_size - 1) / chunk_size, last = run.x + begins(run.x + 1 + lane, end);
        if (last < run.x + 64) return last;
        while (last + 1 < end) {
            const uint32_t step = (end - last - 1 + 63) / 64;
            last += step * begins(last + step * (lane + 1), end);
            if (last + step < end) end = last + step;
        }
        return last;
    };
    const auto add = [&](float4& s, uint32_t chunk, uint32_t& q, uint32_t last, uint32_t by, uint32_t col) {
        if (col >= P * 2) return;
#pragma unroll 4
        for (; q <= last; q += by) {
            const float4 v = *reinterpret_cast<const float4*>(part + ((size_t)q * 2 + (q == chunk)) * (P * VE) + col * 4);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    };
    const auto side_by_side = [&](float4& s) {
        for (uint32_t m = wide; m < 64; m <<= 1) {
            s.x += __shfl_xor(s.x, (int)m);
            s.y += __shfl_xor(s.y, (int)m);
            s.z += __shfl_xor(s.z, (int)m);
            s.w += __shfl_xor(s.w, (int)m);
        }
    };
    const auto write = [&](const float4& s, uint32_t k, uint32_t col) {
        if (mine || col >= P * 2) return;
        const float v[4] = {s.x * f, s.y * f, s.z * f, s.w * f};
        const uint32_t slice = col / 2, from = slice * VE, at = H > VE ? (from < H - VE ? from : H - VE) : 0;
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {      // (column at + i; those before `from` are the slice's before)
            const uint32_t i = col % 2 * 4 + j;
            if (at + i >= from && at + i < H) dE[(size_t)k * H + at + i] = v[j];
        }
    };
    const uint2* runs = reinterpret_cast<const uint2*>(joins + 2);
    const uint32_t round = gridDim.x * LIST;      // items of all workgroups in a round: LIST of each, so that its list holds all that are long
    for (uint32_t begin = 0; begin < items; begin += round) {
        const uint32_t end = items - begin < round ? items : begin + round;
        if (threadIdx.x == 0) count = 0;
        __syncthreads();
        for (uint32_t item = begin + wave * gridDim.x + blockIdx.x; item < end; item += gridDim.x * WAVES) {      // (a run's columns to several workgroups)
            const uint2 run = runs[item / blocks];
            const uint32_t chunk = run.x, col = item % blocks * wide + lane % wide;
            uint32_t q = chunk + mine;
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
            add(s, chunk, q, chunk + 1, side, col);      // (the two there always are, asked for beside the search)
            const uint32_t last = last_chunk(run);
            if (last - chunk > LONG_RUN * side) {
                if (lane == 0) longs[atomicAdd(&count, 1u)] = item;
                continue;
            }
            add(s, chunk, q, last, side, col);
            side_by_side(s);
            write(s, run.y, col);
        }
        __syncthreads();
        const uint32_t n = count;
        for (uint32_t i = 0; i < n; ++i) {
            const uint32_t item = longs[i], col = item % blocks * wide + lane % wide;
            const uint2 run = runs[item / blocks];
            const uint32_t chunk = run.x, last = last_chunk(run);
            uint32_t q = chunk + wave * side + mine;
            float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
            add(s, chunk, q, last, WAVES * side, col);
            side_by_side(s);
            sums[wave][lane] = s;
            __syncthreads();
            if (wave == 0) {
                for (uint32_t w = 1; w < WAVES; ++w) {
                    const float4 v = sums[w][lane];
                    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
                }
                write(s, run.y, col);
            }
            __syncthreads();
        }
        __syncthreads();      // (the list is read before the next round's begins)
    }
}

size_t up256(size_t x) { return (x + 255) & ~size_t(255); }

struct Layout {      // of the workspace
    size_t hist, key[2], pos[2], part, joins, rows, total;
    int64_t M, tile, tiles, chunk, chunks;
    uint32_t P;
    int passes, bits, sorted;      // which of the two pairs the last pass leaves
};

Layout lay_out(int64_t B, int64_t N, int64_t V, int64_t H, int io, int layout)
{
    Layout l;
    l.M = B * N;
    // a pass reads the counts of every tile in every tile: no more than 128 of them, however many tokens there are
    l.tile = TILE_MIN * ((l.M + (int64_t)TILE_MIN * TILES_MAX - 1) / ((int64_t)TILE_MIN * TILES_MAX));
    l.tiles = (l.M + l.tile - 1) / l.tile;
    l.P = (uint32_t)((H + VE - 1) / VE);
    // long chunks leave few partial sums, short ones make enough threads: at least 2^16 where there are so many.  Sums and joins, us:
    // 16384 tokens x 768 16 + 7 in chunks of 16 (98304 threads), 16 + 9 of 8; 2695 x 193 7.8 + 5.7 of 16, 5.8 + 6.8 of 8
    l.chunk = 32;
    while (l.chunk > CHUNK_MIN && l.M / l.chunk * l.P < (1 << 16)) l.chunk /= 2;
    l.chunks = (l.M + l.chunk - 1) / l.chunk;
    int need = 0;
    while (V >> need) ++need;                       // bits of V, the number of no token
    l.passes = (need + 8) / 9;
    l.bits = (need + l.passes - 1) / l.passes;
    l.sorted = (l.passes - 1) & 1;
    size_t off = 0;
    const auto take = [&](size_t bytes) { const size_t at = off; off += up256(bytes); return at; };
    l.hist = take((size_t)(l.M < (int64_t)TILE_MIN * TILES_MAX ? (l.M + TILE_MIN - 1) / TILE_MIN : TILES_MAX) * (1 + SORT_W) * RADIX * sizeof(uint32_t));
    for (int i = 0; i < 2; ++i) {
        l.key[i] = take((size_t)(l.M + 32) * sizeof(uint32_t));
        l.pos[i] = take((size_t)(l.M + 32) * sizeof(uint32_t));
    }
    // (room for a number of chunks that grows with M: those of 32 places, or shorter ones, that are fewer than 2^17 threads)
    static_assert(CHUNK_MIN % AHEAD == 0, "a chunk that is not the last has no places left over");
    const int64_t most = (l.M + CHUNK_MIN - 1) / CHUNK_MIN, some = (l.M + 31) / 32 + ((1 << 17) + l.P - 1) / l.P + 1;
    l.part = take((size_t)(most < some ? most : some) * 2 * l.P * VE * sizeof(float));
    l.joins = take((size_t)((most < some ? most : some) + 1) * 2 * sizeof(uint32_t));
    l.rows = take(layout == LONGCONV_CHANNELS_FIRST ? (size_t)l.M * l.P * VE * (io == LONGCONV_F32 ? 4 : 2) : 0);
    l.total = off;
    return l;
}

template <class IO, class ID>
hipError_t sort_pass(const Tokens<ID>& in, char* ws, const Layout& l, int pass, int to, const Fill& fill, const Transpose* t, hipStream_t st)
{
    uint32_t* hist = (uint32_t*)(ws + l.hist);
    const unsigned tiles = (unsigned)l.tiles;
    Beside part[2] = {};
    dim3 g[2];
    for (int i = 0; i < 2; ++i) {
        part[i].fill = fill.share(2 * pass + i, 2 * l.passes);
        part[i].fills = part[i].fill.groups(SORT_T);
        if (t) part[i].t = t->share(2 * pass + i, 2 * l.passes);
        const hipError_t e = launch_grid((uint64_t)tiles + part[i].fills + part[i].t.tiles, SORT_T, &g[i]);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((sort_count_kernel<ID, IO>), g[0], dim3(SORT_T), 0, st, in, hist, (uint32_t*)(ws + l.joins), l.M, l.tile, tiles, pass * l.bits,
                       l.bits, part[0]);
    hipLaunchKernelGGL((sort_place_kernel<ID, IO>), g[1], dim3(SORT_T), 0, st, in, (const uint32_t*)hist, (uint32_t*)(ws + l.key[to]),
                       (uint32_t*)(ws + l.pos[to]), l.M, l.tile, tiles, pass * l.bits, l.bits, part[1]);
    return hipGetLastError();
}

// -> key[], pos[] of Layout::sorted; and the zeros and the transposition (if any)
template <class IO, class ID>
hipError_t sort_tokens(const ID* ids, int64_t V, char* ws, const Layout& l, const Fill& fill, const Transpose* t, hipStream_t st)
{
    const Tokens<ID> in{ids, nullptr, nullptr, (uint32_t)V};
    if (l.M <= ALONE) {
        hipLaunchKernelGGL((sort_alone_kernel<ID>), dim3(1 + fill.groups(ALONE_T)), dim3(ALONE_T), 0, st, in, (uint32_t*)(ws + l.key[l.sorted]),
                           (uint32_t*)(ws + l.pos[l.sorted]), (uint32_t*)(ws + l.joins), (int)l.M, l.passes, l.bits, fill);
        if constexpr (!std::is_void<IO>::value) hipLaunchKernelGGL(embed_transpose_kernel<IO>, dim3(t->tiles), dim3(256), 0, st, *t);
        return hipGetLastError();
    }
    hipError_t e = sort_pass<IO, ID>(in, ws, l, 0, 0, fill, t, st);
    for (int pass = 1; pass < l.passes && e == hipSuccess; ++pass) {
        const int from = (pass - 1) & 1;
        const Tokens<void> pairs{nullptr, (const uint32_t*)(ws + l.key[from]), (const uint32_t*)(ws + l.pos[from]), (uint32_t)V};
        e = sort_pass<IO, void>(pairs, ws, l, pass, pass & 1, fill, t, st);
    }
    return e;
}

template <class IO, class W, class ID>
hipError_t forward(const EmbedArgs& a, const void* E, void* y, hipStream_t st)
{
    using T = typename IO::T;
    dim3 g;
    const ID* ids = (const ID*)a.ids;
    const typename W::T* table = (const typename W::T*)E;
    if (a.layout == LONGCONV_CHANNELS_FIRST) {
        const uint64_t tt = (a.N + TT - 1) / TT, th = (a.H + TH - 1) / TH;
        const hipError_t e = launch_grid(a.B * tt * th, 256, &g);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((embed_columns_kernel<IO, W, ID>), g, dim3(256), 0, st, ids, table, (T*)y, (uint32_t)a.N, (uint32_t)a.H,
                           (uint32_t)a.V, (uint32_t)tt, (uint32_t)th, a.scale, a.drop);
        return hipGetLastError();
    }
    const int64_t n = a.B * a.N * a.H;
    const hipError_t e = launch_grid((uint64_t)((n + 256 * VE - 1) / (256 * VE)), 256, &g);
    if (e != hipSuccess) return e;
    if (n < (int64_t(1) << 31))
        hipLaunchKernelGGL((embed_rows_kernel<IO, W, ID, uint32_t>), g, dim3(256), 0, st, ids, table, (T*)y, (uint32_t)n, (uint32_t)a.H,
                           (uint32_t)a.V, a.scale, a.drop);
    else
        hipLaunchKernelGGL((embed_rows_kernel<IO, W, ID, uint64_t>), g, dim3(256), 0, st, ids, table, (T*)y, (uint64_t)n, (uint32_t)a.H,
                           (uint32_t)a.V, a.scale, a.drop);
    return hipGetLastError();
}

// lanes of a wave for a row's columns, four each: as many as it takes, in powers of two, and 64 at most
uint32_t join_width(const Layout& l)
{
    uint32_t w = 64;
    while (w / 2 >= l.P * 2) w /= 2;
    return w;
}
// a wave for every 256 columns of every run that there may be, up to JOIN_GROUPS workgroups
unsigned join_groups(const Layout& l)
{
    const uint64_t waves = (uint64_t)l.chunks * ((l.P * 2 + 63) / 64), groups = (waves + JOIN_T / 64 - 1) / (JOIN_T / 64);
    return (unsigned)(groups < JOIN_GROUPS ? groups : JOIN_GROUPS);
}

template <class IO>
hipError_t backward(const EmbedArgs& a, const void* dy, float* dE, char* ws, hipStream_t st)
{
    using T = typename IO::T;
    const Layout l = lay_out(a.B, a.N, a.V, a.H, a.io, a.layout);
    dim3 g;
    const Fill fill{dE, a.V * a.H};
    const T* rows = (const T*)dy;
    uint32_t stride = (uint32_t)a.H;
    hipError_t e;
    if (a.layout == LONGCONV_CHANNELS_FIRST) {
        const uint32_t tt = (uint32_t)((a.N + TT - 1) / TT), th = (uint32_t)((a.H + TH - 1) / TH);
        rows = (const T*)(ws + l.rows);
        stride = l.P * VE;
        const Transpose t{dy, ws + l.rows, (uint32_t)a.N, (uint32_t)a.H, stride, tt, th, a.drop, 0, (uint32_t)a.B * tt * th};
        e = a.id_bytes == 8 ? sort_tokens<IO>((const int64_t*)a.ids, a.V, ws, l, fill, &t, st)
                            : sort_tokens<IO>((const int32_t*)a.ids, a.V, ws, l, fill, &t, st);
    } else {
        e = a.id_bytes == 8 ? sort_tokens<void>((const int64_t*)a.ids, a.V, ws, l, fill, nullptr, st)
                            : sort_tokens<void>((const int32_t*)a.ids, a.V, ws, l, fill, nullptr, st);
    }
    if (e != hipSuccess) return e;
    const uint32_t *key = (const uint32_t*)(ws + l.key[l.sorted]), *pos = (const uint32_t*)(ws + l.pos[l.sorted]);
    float* part = (float*)(ws + l.part);
    uint32_t* joins = (uint32_t*)(ws + l.joins);
    if ((e = launch_grid(((uint64_t)l.chunks * l.P + 255) / 256, 256, &g)) != hipSuccess) return e;
    const auto sum = [&](auto drop, auto narrow) {
        hipLaunchKernelGGL((embed_sum_kernel<IO, decltype(drop)::value, decltype(narrow)::value>), g, dim3(256), 0, st, rows, key, pos, dE, part, joins,
                           (uint32_t)l.M, (uint32_t)a.H, stride, l.P, (uint32_t)a.V, (uint32_t)l.chunk, (uint32_t)l.chunks, a.scale, a.drop);
    };
    const bool drop = a.drop.threshold && a.layout == LONGCONV_CHANNELS_LAST;
    if (a.H < VE) drop ? sum(std::true_type(), std::true_type()) : sum(std::false_type(), std::true_type());
    else drop ? sum(std::true_type(), std::false_type()) : sum(std::false_type(), std::false_type());
    if (l.chunks > 1)
        hipLaunchKernelGGL(embed_join_kernel, dim3(join_groups(l)), dim3(JOIN_T), 0, st, key, (const float*)part, (const uint32_t*)joins, dE, (uint32_t)l.M,
                           (uint32_t)a.H, l.P, (uint32_t)l.chunk, join_width(l), a.scale * a.drop.scale);
    return hipGetLastError();
}

template <class IO, class W>
hipError_t forward_ids(const EmbedArgs& a, const void* E, void* y, hipStream_t st)
{
    return a.id_bytes == 8 ? forward<IO, W, int64_t>(a, E, y, st) : forward<IO, W, int32_t>(a, E, y, st);
}

}  // namespace

hipError_t embed_fwd(const EmbedArgs& a, const void* E, int table, void* y, hipStream_t st)
{
    if (a.io == LONGCONV_F32) return forward_ids<IoF32, IoF32>(a, E, y, st);
    if (a.io == LONGCONV_F16)
        return table == LONGCONV_F32 ? forward_ids<IoF16, IoF32>(a, E, y, st) : forward_ids<IoF16, IoF16>(a, E, y, st);
    return table == LONGCONV_F32 ? forward_ids<IoBF16, IoF32>(a, E, y, st) : forward_ids<IoBF16, IoBF16>(a, E, y, st);
}

size_t embed_workspace_bytes(int64_t B, int64_t N, int64_t V, int64_t H, int io, int layout)
{
    return embed_is_small(N, V, io, layout) ? embed_small_workspace_bytes(B, N, H) : lay_out(B, N, V, H, io, layout).total;
}

hipError_t embed_bwd(const EmbedArgs& a, const void* dy, float* dE, void* ws, hipStream_t st)
{
    if (embed_is_small(a.N, a.V, a.io, a.layout)) return embed_small_bwd(a, dy, dE, ws, st);
    if (a.io == LONGCONV_F32) return backward<IoF32>(a, dy, dE, (char*)ws, st);
    return a.io == LONGCONV_F16 ? backward<IoF16>(a, dy, dE, (char*)ws, st) : backward<IoBF16>(a, dy, dE, (char*)ws, st);
}

}  // namespace lc
