// Dense product between layers, y = act(x W^T + bias) + residual, x and y each as [B,N,.] or [B,.,N], and its backward pass
//     dz = dy act'(z),   dx = dz W,   dW = dz^T x,   dbias = sum over places of dz,      z made again by the same product.
// Behind an activation dz is rounded to the I/O type in front of dx and dW, as the matrix instructions' operands are that wide: a second rounding of
// the size of dy's own (fp16, 131072 x 256 -> 1024 with gelu: errors of the gradients 2.9e-4 instead of 2.1e-4).
//
// All four products are one kernel: out[s][f] = sum_k F(f,k) S(s,k), f the index that is neighbouring in the result's memory.  Either operand
// may have k neighbouring in its memory (its tile then lies in LDS as rows along k) or its own index (rows along that).
#pragma once
#include "act.hpp"
#include "vec8.hpp"

namespace lc {
namespace {

constexpr int LT = 256;               // threads: four waves, two by two
constexpr int TF = 128, TS = 128;     // tile of the result (there are smaller and larger ones)

// One operand: element (i, k) of batch b and segment q of the sum lies at p + b batch + q seg + i ld + k, or + k ld + i
struct Side {
    const void* p;
    int64_t n, ld, batch, seg;        // n: values of i
};
// What becomes of the result: `rows` of n_f values, ld apart
struct Product {
    Side F, S;
    int64_t K, segs, batches;         // the sum goes over `segs` segments of K
    int64_t splits, per;              // shares of the sum, of `per` steps each
    bool wide;                        // tiles of 256 by 256
    // EPI_OUT, EPI_DZ
    void* out;
    int64_t ld, batch;                // of out, residual, dy
    const float* bias;
    bool bias_f;                      // bias goes by f, not by s
    int act;
    const void* residual;             // EPI_OUT
    const void* dy;                   // EPI_DZ: out = dy act'(z)
    float* sums;                      // EPI_DZ: [batches tiles 2][n of the bias], sums of dz over a tile's places, before dz is rounded
    // EPI_SUM: [batches][splits][n_s][n_f]
    float* part;
};
enum { EPI_OUT, EPI_DZ, EPI_SUM };

typedef __bf16 b8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ mu::f4 mfma(IoF16, const uint4& a, const uint4& b, const mu::f4& c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(mu::h8, a), __builtin_bit_cast(mu::h8, b), c, 0, 0, 0);
}
__device__ __forceinline__ mu::f4 mfma(IoBF16, const uint4& a, const uint4& b, const mu::f4& c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
}
__device__ __forceinline__ mu::f4 mfma(IoF32, const float4& a, const float4& b, const mu::f4& c)      // sixteen k: four of each of four lanes
{
    mu::f4 d = __builtin_amdgcn_mfma_f32_16x16x4f32(a.x, b.x, c, 0, 0, 0);
    d = __builtin_amdgcn_mfma_f32_16x16x4f32(a.y, b.y, d, 0, 0, 0);
    d = __builtin_amdgcn_mfma_f32_16x16x4f32(a.z, b.z, d, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a.w, b.w, d, 0, 0, 0);
}

// A tile of BT values of i by BK values of k in LDS, KF: rows along k, else rows along i
template <class IO, bool KF, int BT = 128>
struct Tile {
    using T = typename IO::T;
    static constexpr int E = sizeof(T), BK = E == 4 ? 32 : 64, STEP = E == 4 ? 16 : 32;      // k of a step of the loop, of a matrix instruction
    static constexpr int ROW = KF ? BK + 16 / E : BT + 32 / E, ROWS = KF ? BT : BK;        // elements from row to row
    static constexpr int BYTES = ROW * ROWS * E;
    static constexpr int PER_ROW = (KF ? BK : BT) / VE, PIECES = BT * BK / VE / LT;
    using Frag = typename std::conditional<E == 4, float4, uint4>::type;

    static __device__ __forceinline__ void load(const Side& d, int64_t off, int64_t i0, int64_t k0, int64_t K, Raw8<IO> (&r)[PIECES])
    {
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int id = threadIdx.x + j * LT, line = id / PER_ROW, at = id % PER_ROW * VE;
            const int64_t slow = (KF ? i0 : k0) + line, fast = (KF ? k0 : i0) + at, n_slow = KF ? d.n : K, n_fast = KF ? K : d.n;
            if (slow < n_slow && fast < n_fast) {
                const int64_t n = n_fast - fast;
                load_raw<IO>((const T*)d.p + off + slow * d.ld + fast, n < VE ? (int)n : VE, r[j]);
            } else r[j].zero();
        }
    }
    static __device__ __forceinline__ void put(T* lds, const Raw8<IO> (&r)[PIECES])
    {
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            const int id = threadIdx.x + j * LT, line = id / PER_ROW, at = id % PER_ROW * VE;
            uint4* const to = reinterpret_cast<uint4*>(lds + line * ROW + at);
#pragma unroll
            for (int q = 0; q < Raw8<IO>::W / 4; ++q) to[q] = make_uint4(r[j].w[4 * q], r[j].w[4 * q + 1], r[j].w[4 * q + 2], r[j].w[4 * q + 3]);
        }
    }
    // a lane's k of matrix step `m` for i = i0 + lane % 16: eight from 8 (lane / 16) on, fp32 four from 4 (lane / 16) on
    static __device__ __forceinline__ Frag frag(const T* lds, int i0, int m)
    {
        const int i = threadIdx.x & 15, g = threadIdx.x >> 4 & 3;
        if constexpr (KF) {
            return *reinterpret_cast<const Frag*>(lds + (i0 + i) * ROW + m * STEP + g * (E == 4 ? 4 : 8));
        } else if constexpr (E == 4) {
            const T* p = lds + (m * STEP + 4 * g) * ROW + i0 + i;
            return make_float4(p[0], p[ROW], p[2 * ROW], p[3 * ROW]);
        } else {
            // lane i of 16 gives the address of numbers 4 (i % 4) .. + 3 of row i / 4 and receives column i of the four rows
            typedef __fp16 t4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) t4 lds_t4;
            const T* p = lds + (m * STEP + 8 * g + i / 4) * ROW + i0 + i % 4 * 4;
            const t4 a = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_t4*)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_t4*)(p + 4 * ROW));
            const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
            return make_uint4(x.x, x.y, y.x, y.y);
        }
    }
};

template <class IO>
__device__ __forceinline__ void store4(typename IO::T* p, int n, const float (&v)[4])
{
    if constexpr (sizeof(typename IO::T) == 4) {
        if (n >= 4) {
            const At4 w = {__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
            *reinterpret_cast<At4*>(p) = w;
            return;
        }
    } else if (n >= 4) {
        typedef uint32_t A2 __attribute__((ext_vector_type(2), aligned(2)));
        const A2 w = mu::IsBf<IO>::v ? A2{mu::pack_bf2(v[0], v[1]), mu::pack_bf2(v[2], v[3])} : A2{mu::pack_h2(v[0], v[1]), mu::pack_h2(v[2], v[3])};
        *reinterpret_cast<A2*>(p) = w;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < n) IO::st(p, i, v[i]);
}
template <class IO>
__device__ __forceinline__ void load4(const typename IO::T* p, int n, float (&v)[4])
{
    if (n >= 4) {
        if constexpr (sizeof(typename IO::T) == 4) {
            const At4 w = *reinterpret_cast<const At4*>(p);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
        } else {
            typedef uint32_t A2 __attribute__((ext_vector_type(2), aligned(2)));
            const A2 w = *reinterpret_cast<const A2*>(p);
            unpack2<IO>(w[0], v[0], v[1]);
            unpack2<IO>(w[1], v[2], v[3]);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? IO::ld(p, i) : 0.f;
}

// Workgroup: one tile, of one batch and one share of the sum.  A wave has a quarter of it, in tiles of 16 by 16.  Operands are asked for into
// registers two steps ahead, at any alignment.  fp32: the matrix instructions bound it, 7 x 385 places, 193 -> 1009, 25 us, of which those of the
// units that get four of the 784 workgroups are 12; 512 -> 1024 for 8192 places 80 us, 107 of the 153 TFLOP/s that a large product reaches.
template <class IO, bool FK, bool SK, int EPI, int BT>
__global__ __launch_bounds__(LT, 2) void product_kernel(Product a, uint32_t tiles_f, uint32_t tiles_s)
{
    using T = typename IO::T;
    using TileF = Tile<IO, FK, BT>;
    using TileS = Tile<IO, SK, BT>;
    constexpr int BK = TileF::BK, STEP = TileF::STEP, NT = BT / 32;
    __shared__ __align__(16) unsigned char lds[TileF::BYTES + TileS::BYTES];
    T *const lf = reinterpret_cast<T*>(lds), *const ls = reinterpret_cast<T*>(lds + TileF::BYTES);
    uint32_t w = blockIdx.x;
    const uint32_t tf = w % tiles_f;
    w /= tiles_f;
    const uint32_t ts = w % tiles_s;
    w /= tiles_s;
    const uint32_t split = w % (uint32_t)a.splits, batch = w / (uint32_t)a.splits;
    const int64_t f0 = (int64_t)tf * BT, s0 = (int64_t)ts * BT, steps = (a.K + BK - 1) / BK;
    const int64_t first = (int64_t)split * a.per, end = first + a.per < steps * a.segs ? first + a.per : steps * a.segs;
    const int wave = threadIdx.x >> 6, wf = (wave & 1) * (BT / 2), ws = (wave >> 1) * (BT / 2);
    mu::f4 acc[NT][NT];
#pragma unroll
    for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) acc[i][j] = mu::f4{0.f, 0.f, 0.f, 0.f};
    Raw8<IO> rf[2][TileF::PIECES], rs[2][TileS::PIECES];
    int64_t seg = first / steps, k0 = (first - seg * steps) * BK, asked = first;      // of the step to be asked for next
    const auto ask = [&](int u) {
        if (asked >= end) return;
        TileF::load(a.F, batch * a.F.batch + seg * a.F.seg, f0, k0, a.K, rf[u]);
        TileS::load(a.S, batch * a.S.batch + seg * a.S.seg, s0, k0, a.K, rs[u]);
        ++asked;
        k0 += BK;
        if (k0 >= a.K) {
            k0 = 0;
            ++seg;
        }
    };
    ask(0);
    ask(1);
    for (int64_t at = first; at < end; at += 2) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if (at + u >= end) break;
            __syncthreads();
            TileF::put(lf, rf[u]);
            TileS::put(ls, rs[u]);
            __syncthreads();
            ask(u);
#pragma unroll
            for (int m = 0; m < BK / STEP; ++m) {
                typename TileF::Frag x[NT], y[NT];
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    x[i] = TileF::frag(lf, wf + 16 * i, m);
                    y[i] = TileS::frag(ls, ws + 16 * i, m);
                }
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int j = 0; j < NT; ++j) acc[i][j] = mfma(IO(), x[i], y[j], acc[i][j]);
            }
        }
    }
    // a lane has f = 4 (lane / 16) .. + 3 and s = lane % 16 of each tile of 16 by 16
    const int col = threadIdx.x & 15, g = threadIdx.x >> 4 & 3;
    if constexpr (EPI == EPI_SUM) {
        float* const to = a.part + (size_t)(batch * a.splits + split) * a.S.n * a.F.n;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int64_t s = s0 + ws + 16 * j + col;
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const int64_t f = f0 + wf + 16 * i + 4 * g, n = a.F.n - f;
                const float v[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                if (s < a.S.n && n > 0) store4<IoF32>(to + s * a.F.n + f, n < 4 ? (int)n : 4, v);
            }
        }
        return;
    }
    float by_f[NT][4] = {}, by_s[NT] = {};
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int64_t f = f0 + wf + 16 * i + 4 * g, n_f = a.F.n - f;
        const int n = n_f < 4 ? (int)n_f : 4;
        float bf[4] = {0.f, 0.f, 0.f, 0.f};
        if (a.bias && a.bias_f && n > 0) load4<IoF32>(a.bias + f, n, bf);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int64_t s = s0 + ws + 16 * j + col;
            if (s >= a.S.n || n <= 0) continue;
            const size_t at = (size_t)batch * a.batch + s * a.ld + f;
            const float bs = a.bias && !a.bias_f ? a.bias[s] : 0.f;
            float v[4], r[4] = {0.f, 0.f, 0.f, 0.f};
            if (EPI == EPI_DZ) load4<IO>((const T*)a.dy + at, n, r);
            else if (a.residual) load4<IO>((const T*)a.residual + at, n, r);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float z = acc[i][j][q] + bf[q] + bs;
                if (EPI == EPI_DZ) {
                    v[q] = q < n ? r[q] * slope_by(a.act, z) : 0.f;
                    by_f[i][q] += v[q];
                    by_s[j] += v[q];
                } else v[q] = act_by(a.act, z) + r[q];
            }
            store4<IO>((T*)a.out + at, n, v);
        }
    }
    if constexpr (EPI == EPI_DZ) {
        if (!a.sums) return;
        if (a.bias_f) {      // places are s: over the lanes of a row of sixteen
            float* const to = a.sums + ((size_t)(batch * tiles_s + ts) * 2 + (wave >> 1)) * a.F.n;
#pragma unroll
            for (int i = 0; i < NT; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float v = by_f[i][q];
#pragma unroll
                    for (int d = 1; d < 16; d *= 2) v += __shfl_xor(v, d);
                    const int64_t f = f0 + wf + 16 * i + 4 * g + q;
                    if (col == 0 && f < a.F.n) to[f] = v;
                }
        } else {             // places are f: over the four rows of lanes
            float* const to = a.sums + ((size_t)(batch * tiles_f + tf) * 2 + (wave & 1)) * a.S.n;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                float v = by_s[j];
                v += __shfl_xor(v, 16);
                v += __shfl_xor(v, 32);
                const int64_t s = s0 + ws + 16 * j + col;
                if (g == 0 && s < a.S.n) to[s] = v;
            }
        }
    }
}

// ---- 16-bit operands whose rows are whole pieces of 16 bytes ---------------------------------------------------------------
// The tile of an operand is brought into LDS by the memory instructions themselves, 1 KB of it a wave instruction, the next step's while
// this one's is worked on.  They write LDS in the order of lanes, so where a piece of 16 bytes comes to lie is chosen by which piece a lane
// asks for: rows along k (128 bytes) exchange their eight pieces by the row's number / 2, rows along i their pairs of pieces by bits 0, 1 and
// 3 of it, so that sixteen lanes' reads of a fragment fall on all banks.  What lies beyond the operand reads as zero (the buffer's range).
// (Written out, because the compiler takes every read of LDS for one of what such an instruction writes and waits for all of them first.)
typedef uint32_t range_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ range_t make_range(const void* p, uint32_t bytes)
{
    const uint64_t a = reinterpret_cast<uint64_t>(p);
    return range_t{(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)a), (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32)),
                   (uint32_t)__builtin_amdgcn_readfirstlane((int)bytes), 0x00027000u};
}
constexpr uint32_t BEYOND = 0x80000000u;
// 16 bytes of each lane from byte `off` on to LDS byte `to` + 16 lane; they are there when vmcnt says so.  (m0 is named, so that no value that the
// compiler puts there for an instruction of its own is taken to last across this.)
__device__ __forceinline__ void bring16(const range_t& r, uint32_t off, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off), "s"(r), "s"(to) : "memory", "m0");
}

// rows (k fast) or columns (k slow) i0 .. i0 + BI - 1 of an operand, 64 values of k a step, by NW waves
template <bool KF, int BI, int NW>
struct Fast {
    static constexpr int BK = 64, BYTES = BI * BK * 2, LOADS = BYTES / 1024 / NW;
    static constexpr int SLOTS = KF ? 8 : BI / 8, LINES = 64 / SLOTS;      // pieces of a row in LDS, rows of a wave instruction
    const char* base;
    uint32_t off[LOADS], at_k;      // of this lane's pieces; the first one's k (KF)
    int64_t ld;
    int cols;

    __device__ __forceinline__ void init(const Side& d, int64_t offset, int64_t i0)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int64_t left = d.n - i0;
        cols = (int)(left < BI ? left : BI);
        ld = d.ld;
        base = reinterpret_cast<const char*>(d.p) + (offset + (KF ? i0 * ld : i0)) * 2;
        const int slot = lane % SLOTS;
        at_k = 0;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int row = (j * NW + wave) * LINES + lane / SLOTS;
            if (KF) {
                const int c = slot ^ (row >> 1 & 7);
                at_k = (uint32_t)c * 8;      // (the same for all j: NW LINES is a multiple of sixteen)
                off[j] = row < cols ? (uint32_t)(row * ld * 2) + c * 16 : BEYOND;
            } else {
                const int c = ((slot >> 1) ^ ((row & 3) | (row >> 1 & 4))) * 2 + (slot & 1);
                off[j] = c * 8 < cols ? (uint32_t)(row * ld * 2) + c * 16 : BEYOND;
            }
        }
    }
    // step: k0 .. k0 + 63 of a segment of K, whose elements begin `seg` elements behind the operand's
    __device__ __forceinline__ void load(int64_t seg, int64_t k0, int64_t K, uint32_t lds) const
    {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const int64_t left = K - k0;
        const uint32_t here = (uint32_t)(left < BK ? left : BK);
        if (KF) {
            const range_t r = make_range(base + (seg + k0) * 2, (uint32_t)((cols - 1) * ld + here) * 2);
            const bool is = at_k < here;
#pragma unroll
            for (int j = 0; j < LOADS; ++j) bring16(r, is ? off[j] : BEYOND, lds + (j * NW + wave) * 1024);
        } else {
            const range_t r = make_range(base + (seg + k0 * ld) * 2, (uint32_t)((here - 1) * ld + cols) * 2);
#pragma unroll
            for (int j = 0; j < LOADS; ++j) bring16(r, off[j], lds + (j * NW + wave) * 1024);
        }
    }
    // a lane's eight k, from 32 m + 8 (lane / 16) on, for i = i0 + lane % 16
    static __device__ __forceinline__ uint4 frag(const char* lds, int i0, int m)
    {
        const int i = threadIdx.x & 15, g = threadIdx.x >> 4 & 3;
        if constexpr (KF) {
            return *reinterpret_cast<const uint4*>(lds + (i0 + i) * 128 + (((m * 4 + g) ^ (i >> 1)) << 4));
        } else {
            typedef __fp16 t4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) t4 lds_t4;
            const char* p = lds + (m * 32 + 8 * g + (i >> 2)) * (BI * 2) + (((i0 >> 4) ^ ((i >> 2) | (g & 1) << 2)) << 5) + (i & 3) * 8;
            const t4 a = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_t4*)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4f16((lds_t4*)(p + 4 * BI * 2));
            const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
            return make_uint4(x.x, x.y, y.x, y.y);
        }
    }
};

// Workgroup: a tile of BF by BS, WF by WS waves, NB tiles of each operand in LDS at once.  The result goes through LDS, each wave's part by itself, so that memory sees rows of f.
template <class IO, bool FK, bool SK, int EPI, int BF, int BS, int WF, int WS, int NB>
__global__ __launch_bounds__(64 * WF * WS, NB == 1 ? 4 : 2) void fast_product_kernel(Product a, uint32_t tiles_f, uint32_t tiles_s)
{
    using T = typename IO::T;
    constexpr int NW = WF * WS, NF = BF / WF / 16, NS = BS / WS / 16;      // tiles of 16 of a wave
    using SideF = Fast<FK, BF, NW>;
    using SideS = Fast<SK, BS, NW>;
    constexpr int STAGE = SideF::BYTES + SideS::BYTES;
    __shared__ __align__(1024) char lds[NB * STAGE];
    uint32_t w = blockIdx.x;
    {   // workgroups go round the eight dies: each die gets a run of neighbouring tiles, which share operands in its cache
        const uint32_t n = gridDim.x, each = n / 8, rest = n % 8, die = w % 8, at = w / 8;
        w = die * each + (die < rest ? die : rest) + at;
    }
    const uint32_t tf = w % tiles_f;
    w /= tiles_f;
    const uint32_t ts = w % tiles_s;
    w /= tiles_s;
    const uint32_t split = w % (uint32_t)a.splits, batch = w / (uint32_t)a.splits;
    const int64_t f0 = (int64_t)tf * BF, s0 = (int64_t)ts * BS, steps = (a.K + 63) / 64;
    const int64_t first = (int64_t)split * a.per, end = first + a.per < steps * a.segs ? first + a.per : steps * a.segs;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wf = wave % WF * (BF / WF), ws = wave / WF * (BS / WS);
    SideF sf;
    SideS ss;
    sf.init(a.F, batch * a.F.batch, f0);
    ss.init(a.S, batch * a.S.batch, s0);
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds);
    int64_t seg = first / steps, k0 = (first - seg * steps) * 64;      // of the step to be asked for next
    const auto ask = [&](int buf) {
        sf.load(seg * a.F.seg, k0, a.K, lds0 + buf * STAGE);
        ss.load(seg * a.S.seg, k0, a.K, lds0 + buf * STAGE + SideF::BYTES);
        k0 += 64;
        if (k0 >= a.K) {
            k0 = 0;
            ++seg;
        }
    };
    mu::f4 acc[NF][NS], ones[NS];
#pragma unroll
    for (int j = 0; j < NS; ++j) {
        ones[j] = mu::f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NF; ++i) acc[i][j] = ones[j];
    }
    const bool sums = EPI == EPI_SUM && a.sums && f0 == 0 && wf == 0;
    const uint32_t one = mu::IsBf<IO>::v ? 0x3f803f80u : 0x3c003c00u;
    const uint4 all_ones = make_uint4(one, one, one, one);
    if (NB == 2 && first < end) ask(0);
    int buf = 0;
    for (int64_t at = first; at < end; ++at, buf ^= NB - 1) {
        if (NB == 1) {
            __syncthreads();      // (the step before is read)
            ask(0);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");      // this step's tiles are here, the last one's are read
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (NB == 2 && at + 1 < end) ask(buf ^ 1);
        const char *const lf = lds + buf * STAGE, *const ls = lf + SideF::BYTES;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            uint4 x[NF], y[NS];
#pragma unroll
            for (int i = 0; i < NF; ++i) x[i] = SideF::frag(lf, wf + 16 * i, m);
#pragma unroll
            for (int j = 0; j < NS; ++j) y[j] = SideS::frag(ls, ws + 16 * j, m);
#pragma unroll
            for (int i = 0; i < NF; ++i)
#pragma unroll
                for (int j = 0; j < NS; ++j) acc[i][j] = mfma(IO(), x[i], y[j], acc[i][j]);
            if (EPI == EPI_SUM && sums) {
#pragma unroll
                for (int j = 0; j < NS; ++j) ones[j] = mfma(IO(), all_ones, y[j], ones[j]);
            }
        }
    }
    __syncthreads();
    const int col = lane & 15, g = lane >> 4;
    if constexpr (EPI == EPI_SUM) {
        if (sums && g == 0) {
#pragma unroll
            for (int j = 0; j < NS; ++j) {
                const int64_t s = s0 + ws + 16 * j + col;
                if (s < a.S.n) a.sums[(size_t)split * a.S.n + s] = ones[j][0];      // (dW: one batch)
            }
        }
    }
    // 64 values of f by SP of s at a time in this wave's share of LDS, fp32, the sixteen pieces of a row exchanged by s
    constexpr int MINE = NB * STAGE / NW, FP = NF * 16 < 64 ? NF * 16 : 64, FIT = MINE / (FP * 4) < NS * 16 ? MINE / (FP * 4) : NS * 16;
    constexpr int SP = NB == 1 && EPI == EPI_DZ ? 16 : FIT;      // (fewer registers)
    constexpr int LANES = FP / 8, ROWS = 64 / LANES;      // lanes of a row of f, rows of a wave instruction
    static_assert(FP % 64 == 0 && SP % 16 == 0 && SP % ROWS == 0, "whole tiles");
    float* const mine = reinterpret_cast<float*>(lds + wave * MINE);
    const int q = lane % LANES, r0 = lane / LANES;
    constexpr int ITS = SP / ROWS;
    static_assert(NS * 16 % SP == 0, "whole passes");
    const bool whole = f0 + BF <= a.F.n && s0 + BS <= a.S.n;
    const T* const from = EPI == EPI_DZ ? (const T*)a.dy : EPI == EPI_OUT ? (const T*)a.residual : nullptr;
#pragma unroll
    for (int fp = 0; fp < NF * 16 / FP; ++fp) {
        const int64_t f = f0 + wf + fp * FP + 8 * q;
        const int n = whole || a.F.n - f >= 8 ? 8 : (int)(a.F.n - f);
        float bf[8] = {}, by_f[8] = {};
        if (EPI != EPI_SUM && a.bias && a.bias_f && n > 0) load8<IoF32>(a.bias + f, n, bf);
#pragma unroll
        for (int sp = 0; sp < NS * 16 / SP; ++sp) {
            const int64_t sr = s0 + ws + sp * SP + r0;      // this lane's rows: sr, sr + ROWS, ...
            Raw8<IO> other[EPI == EPI_SUM ? 1 : ITS];
            float bs[EPI == EPI_SUM ? 1 : ITS];
            if constexpr (EPI != EPI_SUM) {
                const T* const at = from ? from + (size_t)batch * a.batch + sr * a.ld + f : nullptr;
#pragma unroll
                for (int it = 0; it < ITS; ++it) {
                    const bool is = whole || (sr + it * ROWS < a.S.n && n > 0);
                    bs[it] = 0.f;
                    if (a.bias && !a.bias_f && is) bs[it] = a.bias[sr + it * ROWS];
                    if (!from) continue;
                    if (whole) other[it].load(at + it * ROWS * a.ld);
                    else if (is) load_raw<IO>(at + it * ROWS * a.ld, n, other[it]);
                    else other[it].zero();
                }
            }
#pragma unroll
            for (int j = 0; j < SP / 16; ++j)
#pragma unroll
                for (int i = 0; i < FP / 16; ++i) {
                    const int s = 16 * j + col;
                    const mu::f4 v = acc[fp * (FP / 16) + i][sp * (SP / 16) + j];
                    *reinterpret_cast<float4*>(mine + s * FP + (((4 * i + g) ^ (s & 15)) << 2)) = make_float4(v[0], v[1], v[2], v[3]);
                }
            mu::wave_lds_fence();
#pragma unroll
            for (int it = 0; it < ITS; ++it) {
                const int r = it * ROWS + r0;
                const int64_t s = sr + it * ROWS;
                const float4 u = *reinterpret_cast<const float4*>(mine + r * FP + (((2 * q) ^ (r & 15)) << 2));
                const float4 t = *reinterpret_cast<const float4*>(mine + r * FP + (((2 * q + 1) ^ (r & 15)) << 2));
                float v[8] = {u.x, u.y, u.z, u.w, t.x, t.y, t.z, t.w};
                const bool is = whole || (s < a.S.n && n > 0);
                if constexpr (EPI == EPI_SUM) {
                    if (is) store8<IoF32>(a.part + (size_t)(batch * a.splits + split) * a.S.n * a.F.n + s * a.F.n + f, n, v);
                } else {
                    float o[8] = {}, by_s = 0.f;
                    if (from) other[it].get(o);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] += bf[e] + bs[it];
                    if constexpr (EPI == EPI_DZ) slopes_by(a.act, v);
                    else acts_by(a.act, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (EPI == EPI_DZ) {
                            v[e] = is ? o[e] * v[e] : 0.f;
                            if (!whole && e >= n) v[e] = 0.f;
                            by_f[e] += v[e];
                            by_s += v[e];
                        } else v[e] += o[e];
                    }
                    if (is) store8<IO>((T*)a.out + (size_t)batch * a.batch + s * a.ld + f, n, v);
                    if (EPI == EPI_DZ && a.sums && !a.bias_f) {      // places are f: over the lanes of a row
#pragma unroll
                        for (int d = 1; d < LANES; d *= 2) by_s += __shfl_xor(by_s, d);
                        float* const at = a.sums + ((size_t)(batch * tiles_f + tf) * (BF / 64) + (wf / 64 + fp)) * a.S.n;
                        if (q == 0 && s < a.S.n) at[s] = by_s;
                    }
                }
            }
            mu::wave_lds_fence();
        }
        if constexpr (EPI == EPI_DZ) {
            if (a.sums && a.bias_f) {      // places are s: over the lanes that have the same f
                float* const at = a.sums + ((size_t)(batch * tiles_s + ts) * WS + wave / WF) * a.F.n;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float v = by_f[e];
#pragma unroll
                    for (int d = LANES; d < 64; d *= 2) v += __shfl_xor(v, d);
                    if (r0 == 0 && e < n) at[f + e] = v;
                }
            }
        }
    }
}

// dbias without dW: the sums that the products of dW make beside them, by the same instructions in the same order, so that the bits do not depend on
// which results are asked for.  Workgroup: 128 columns of dz, one share of the places.  Memory bounds it: 16 x 1024 places, 2048 columns, bf16 19 us with the
// join of the shares (67 MB).
template <class IO, bool SK>
__global__ __launch_bounds__(LT, 2) void ones_kernel(Product a, uint32_t tiles_s)
{
    using SideS = Fast<SK, 128, 4>;
    __shared__ __align__(1024) char lds[2 * SideS::BYTES];
    const uint32_t ts = blockIdx.x % tiles_s, split = blockIdx.x / tiles_s;
    const int64_t s0 = (int64_t)ts * 128, steps = (a.K + 63) / 64;
    const int64_t first = (int64_t)split * a.per, end = first + a.per < steps * a.segs ? first + a.per : steps * a.segs;
    const int lane = threadIdx.x & 63, ws = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 32;
    SideS ss;
    ss.init(a.S, 0, s0);
    const uint32_t lds0 = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char*)lds);
    int64_t seg = first / steps, k0 = (first - seg * steps) * 64;      // of the step to be asked for next
    const auto ask = [&](int buf) {
        ss.load(seg * a.S.seg, k0, a.K, lds0 + buf * SideS::BYTES);
        k0 += 64;
        if (k0 >= a.K) {
            k0 = 0;
            ++seg;
        }
    };
    const uint32_t one = mu::IsBf<IO>::v ? 0x3f803f80u : 0x3c003c00u;
    const uint4 all_ones = make_uint4(one, one, one, one);
    mu::f4 ones[2] = {mu::f4{0.f, 0.f, 0.f, 0.f}, mu::f4{0.f, 0.f, 0.f, 0.f}};
    if (first < end) ask(0);
    int buf = 0;
    for (int64_t at = first; at < end; ++at, buf ^= 1) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");      // this step's tile is here, the last one's is read
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (at + 1 < end) ask(buf ^ 1);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int j = 0; j < 2; ++j) ones[j] = mfma(IO(), all_ones, SideS::frag(lds + buf * SideS::BYTES, ws + 16 * j, m), ones[j]);
    }
    if (lane >= 16) return;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int64_t s = s0 + ws + 16 * j + lane;
        if (s < a.S.n) a.sums[(size_t)split * a.S.n + s] = ones[j][0];
    }
}

// out[i] = sum over the shares, in their order
template <class IO>
__global__ __launch_bounds__(256) void linear_join_kernel(const float* __restrict__ part, typename IO::T* __restrict__ out, int64_t n, int64_t shares)
{
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= n) return;
    const int here = n - at < 4 ? (int)(n - at) : 4;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int64_t q = 0; q < shares; ++q) {
        float w[4];
        load4<IoF32>(part + q * n + at, here, w);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += w[i];
    }
    store4<IO>(out + at, here, v);
}

// What EPI_OUT and EPI_DZ do, of the shares of a sum.  Workgroup: 256 values of f, four a lane, by FINISH rows of s, every fourth a wave's; EPI_DZ's sums
// over its places.
constexpr int FINISH = 16;
template <class IO, int EPI>
__global__ __launch_bounds__(256) void linear_finish_kernel(Product a, uint32_t blocks_f, uint32_t blocks_s)
{
    using T = typename IO::T;
    __shared__ float4 lds[3][64];
    uint32_t w = blockIdx.x;
    const uint32_t bf = w % blocks_f;
    w /= blocks_f;
    const uint32_t bs = w % blocks_s;
    const int64_t batch = w / blocks_s;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t f = (int64_t)bf * 256 + 4 * lane, left = a.F.n - f, each = a.S.n * a.F.n;
    const int n = left < 4 ? (int)left : 4;
    float bias[4] = {0.f, 0.f, 0.f, 0.f}, by_f[4] = {0.f, 0.f, 0.f, 0.f};
    if (a.bias && a.bias_f && n > 0) load4<IoF32>(a.bias + f, n, bias);
#pragma unroll
    for (int k = 0; k < FINISH / 4; ++k) {
        const int64_t s = (int64_t)bs * FINISH + 4 * k + wave;
        float by_s = 0.f;
        if (s < a.S.n && n > 0) {
            const float* const from = a.part + batch * a.splits * each + s * a.F.n + f;
            const size_t at = (size_t)batch * a.batch + s * a.ld + f;
            const float of_s = a.bias && !a.bias_f ? a.bias[s] : 0.f;
            float v[4], r[4] = {0.f, 0.f, 0.f, 0.f};
            if (EPI == EPI_DZ) load4<IO>((const T*)a.dy + at, n, r);
            else if (a.residual) load4<IO>((const T*)a.residual + at, n, r);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = bias[i] + of_s;
#pragma unroll 4
            for (int64_t q = 0; q < a.splits; ++q) {
                float u[4];
                load4<IoF32>(from + q * each, n, u);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += u[i];
            }
            if (EPI == EPI_DZ) slopes_by(a.act, v);
            else acts_by(a.act, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (EPI == EPI_DZ) {
                    v[i] = i < n ? r[i] * v[i] : 0.f;
                    by_f[i] += v[i];
                    by_s += v[i];
                } else v[i] += r[i];
            }
            store4<IO>((T*)a.out + at, n, v);
        }
        if (EPI == EPI_DZ && a.sums && !a.bias_f) {      // places are f
#pragma unroll
            for (int d = 1; d < 64; d *= 2) by_s += __shfl_xor(by_s, d);
            if (lane == 0 && s < a.S.n) a.sums[(size_t)(batch * blocks_f + bf) * a.S.n + s] = by_s;
        }
    }
    if (EPI == EPI_DZ && a.sums && a.bias_f) {      // places are s
        if (wave) lds[wave - 1][lane] = make_float4(by_f[0], by_f[1], by_f[2], by_f[3]);
        __syncthreads();
        if (wave || n <= 0) return;
#pragma unroll
        for (int r = 0; r < 3; ++r) {
            const float4 u = lds[r][lane];
            by_f[0] += u.x;
            by_f[1] += u.y;
            by_f[2] += u.z;
            by_f[3] += u.w;
        }
        store4<IoF32>(a.sums + (size_t)(batch * blocks_s + bs) * a.F.n + f, n, by_f);
    }
}

constexpr int COLUMN_ROWS = 256;      // places that a workgroup adds up

// part[share][M] <- sums of dy over places: of [T,M], shares of COLUMN_ROWS places
template <class IO>
__global__ __launch_bounds__(256) void columns_last_kernel(const typename IO::T* __restrict__ dy, float* __restrict__ part, int64_t T, int64_t M,
                                                           uint32_t wide)
{
    const uint32_t share = blockIdx.x / wide;
    const int64_t m = (int64_t)(blockIdx.x - share * wide) * 256 + threadIdx.x, first = (int64_t)share * COLUMN_ROWS;
    if (m >= M) return;
    const int64_t end = first + COLUMN_ROWS < T ? first + COLUMN_ROWS : T;
    float v = 0.f;
    for (int64_t t = first; t < end; ++t) v += IO::ld(dy, t * M + m);
    part[(size_t)share * M + m] = v;
}
// of [B,M,N]: a share for each sequence
template <class IO>
__global__ __launch_bounds__(256) void columns_first_kernel(const typename IO::T* __restrict__ dy, float* __restrict__ part, int64_t rows, int64_t N)
{
    for (int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); row < rows; row += (int64_t)gridDim.x * 4) {
        float v = 0.f;
        for (int64_t t = threadIdx.x & 63; t < N; t += 64) v += IO::ld(dy, row * N + t);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
        if ((threadIdx.x & 63) == 0) part[row] = v;
    }
}
// dbias[m] = the sum of shares, a workgroup of 32 rows of 32 columns
__global__ __launch_bounds__(1024) void columns_join_kernel(const float* __restrict__ part, float* __restrict__ dbias, int64_t M, int64_t shares)
{
    __shared__ float lds[32][33];
    const int c = threadIdx.x & 31, r = threadIdx.x >> 5;
    const int64_t m = (int64_t)blockIdx.x * 32 + c;
    float v = 0.f;
    if (m < M) {
#pragma unroll 8
        for (int64_t q = r; q < shares; q += 32) v += part[q * M + m];
    }
    lds[r][c] = v;
    __syncthreads();
    v = lds[c][r];      // row c's sum of column r: each half wave adds up one column
#pragma unroll
    for (int d = 1; d < 32; d *= 2) v += __shfl_xor(v, d);
    const int64_t to = (int64_t)blockIdx.x * 32 + r;
    if (c == 0 && to < M) dbias[to] = v;
}

// ---- few places ------------------------------------------------------------------------------------------------------------
// y = act(x W^T + bias) + residual for up to 16 NT rows of x: W is what is read, each piece of it once, straight into the matrix instructions'
// operands.  Workgroup: 16 columns m; its eight waves take the sum's steps in turn and add up through LDS.  us, so and by tiles: bf16, 768 -> 2048,
// 16 places 3.7 and 13.6, 64 places 6.3 and 14.1; 4096 -> 4096, 64 places, 21 and 67; fp32, 768 -> 2048, 64 places, 11.9 and 26.7.
constexpr int FEW = 64;      // places
template <class IO, int NT>
__global__ __launch_bounds__(512) void few_kernel(Product a)
{
    using T = typename IO::T;
    constexpr bool F4 = sizeof(T) == 4;
    constexpr int PER = F4 ? 4 : 8, STEP = 4 * PER, NW = 8;      // k of a lane, of a step
    using Frag = typename std::conditional<F4, float4, uint4>::type;
    __shared__ float lds[NW][NT][16][17];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, g = lane >> 4;
    const int64_t m0 = (int64_t)blockIdx.x * 16;
    const auto frag = [&](const Side& d, int64_t row, int64_t k) {
        Frag r;
        const T* const p = (const T*)d.p + row * d.ld + k;
        const int64_t n = row < d.n ? a.K - k : 0;
        if constexpr (F4) {
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            if (n > 0) load4<IoF32>(p, n < 4 ? (int)n : 4, v);
            r = make_float4(v[0], v[1], v[2], v[3]);
        } else {
            Raw8<IO> q;
            load_raw<IO>(p, n < 8 ? (int)n : 8, q);
            r = make_uint4(q.w[0], q.w[1], q.w[2], q.w[3]);
        }
        return r;
    };
    mu::f4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = mu::f4{0.f, 0.f, 0.f, 0.f};
    constexpr int AHEAD = NT == 1 ? 4 : 2;      // steps whose operands are asked for at once
    for (int64_t k0 = (int64_t)wave * STEP; k0 < a.K; k0 += (int64_t)AHEAD * NW * STEP) {
        Frag w[AHEAD], x[AHEAD][NT];
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            const int64_t k = k0 + (int64_t)s * NW * STEP + g * PER;
            w[s] = frag(a.F, m0 + i, k);
#pragma unroll
            for (int t = 0; t < NT; ++t) x[s][t] = frag(a.S, 16 * t + i, k);
        }
#pragma unroll
        for (int s = 0; s < AHEAD; ++s)
#pragma unroll
            for (int t = 0; t < NT; ++t) acc[t] = mfma(IO(), w[s], x[s][t], acc[t]);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) lds[wave][t][i][4 * g + r] = acc[t][r];
    __syncthreads();
    for (int id = threadIdx.x; id < NT * 256; id += 512) {
        const int t = id >> 8, row = id >> 4 & 15, c = id & 15;
        const int64_t s = 16 * t + row, m = m0 + c;
        if (s >= a.S.n || m >= a.F.n) continue;
        float z = a.bias ? a.bias[m] : 0.f;
#pragma unroll
        for (int r = 0; r < NW; ++r) z += lds[r][t][row][c];
        z = act_by(a.act, z);
        if (a.residual) z += IO::ld((const T*)a.residual, s * a.ld + m);
        IO::st((T*)a.out, s * a.ld + m, z);
    }
}
template <class IO>
hipError_t launch_few(const Product& p, hipStream_t st)
{
    const dim3 g((unsigned)((p.F.n + 15) / 16));
    if (p.S.n <= 16) hipLaunchKernelGGL((few_kernel<IO, 1>), g, dim3(512), 0, st, p);
    else if (p.S.n <= 32) hipLaunchKernelGGL((few_kernel<IO, 2>), g, dim3(512), 0, st, p);
    else hipLaunchKernelGGL((few_kernel<IO, 4>), g, dim3(512), 0, st, p);
    return hipGetLastError();
}

// Whether an operand's rows are whole pieces of 16 bytes, wherever a tile begins, and a tile's 256 rows lie within 2 GB (BEYOND is beyond)
inline bool whole_pieces(const Side& d, bool kf, int64_t K) { return d.ld % 8 == 0 && (kf ? K : d.n) % 8 == 0 && d.batch % 8 == 0 && d.seg % 8 == 0 && d.ld < (1 << 22); }

template <class IO, int EPI, bool FK, bool SK, int BF, int BS, int WF, int WS, int NB>
hipError_t launch_fast(const Product& p, int64_t* shares, hipStream_t st)
{
    const uint32_t tf = (uint32_t)((p.F.n + BF - 1) / BF), ts = (uint32_t)((p.S.n + BS - 1) / BS);
    dim3 g;
    const hipError_t e = launch_grid((uint64_t)tf * ts * (uint64_t)p.splits * (uint64_t)p.batches, 64 * WF * WS, &g);
    if (e != hipSuccess) return e;
    if (shares) *shares = EPI == EPI_SUM ? p.splits : p.batches * (p.bias_f ? (int64_t)ts * WS : (int64_t)tf * (BF / 64));
    hipLaunchKernelGGL((fast_product_kernel<IO, FK, SK, EPI, BF, BS, WF, WS, NB>), g, dim3(64 * WF * WS), 0, st, p, tf, ts);
    return hipGetLastError();
}
// Products over K with an epilogue.  Tiles of 256 by 256, two of each operand in LDS (one workgroup a compute unit, half the operand traffic), where
// the sum is long, and where they are full to three quarters and more, and so is the last round of 256 units.  Else tiles of 128 by 128, one of
// each operand (four workgroups a unit, whose loads, products and epilogues lie side by side).  us, 256 and 128, bf16: 16384 x K -> 2048: K = 768
// 61 and 60, 1024 76 and 71 (in other layouts 78 to 81 and 78 to 85), 1536 101 and 108, 2048 121 and 129, 4096 217 and 241; 8192^3 957 and 1300;
// 131072 x 256 -> 1024 with gelu, fp16, 220 and 187.  Two operands of 128 each in LDS, two workgroups a unit: K = 768 69, the last 234.  (Back to back on
// one set of tensors; under the profiler and on two sets in turn K = 768 takes 69, of tiles of 128.)
inline bool wide_tiles(int64_t f, int64_t s, int64_t batches, int64_t K)
{
    const int64_t tiles = ((f + 255) / 256) * ((s + 255) / 256) * batches, rounds = (tiles + 255) / 256;
    return K >= 1024 && tiles > rounds * 192 && f * s * batches >= tiles * (256 * 192);
}

template <class IO, int EPI, bool FK, bool SK>
hipError_t launch_sides(Product p, int64_t* shares, hipStream_t st)
{
    dim3 g;
    if constexpr (sizeof(typename IO::T) == 2) {
        if (whole_pieces(p.F, FK, p.K) && whole_pieces(p.S, SK, p.K)) {
            if (p.wide) return launch_fast<IO, EPI, FK, SK, 256, 256, 2, 4, 2>(p, shares, st);
            return launch_fast<IO, EPI, FK, SK, 128, 128, 2, 2, EPI == EPI_SUM ? 2 : 1>(p, shares, st);
        }
    }
    // Tiles of 64 where those of 128 are fewer than two a unit.  us, 64 and 128: fp32 2695 x 193 -> 1009 22 and 28, 4096 x 512 -> 1024 51 and 51, 8192 x
    // 512 -> 1024 (512 tiles of 128) 95 and 80; bf16 2048 x 511 -> 1000 12 and 20, 8192 x 511 -> 1000 35 and 29.
    const auto tiles = [&](int64_t n, int64_t t) { return (uint64_t)((n + t - 1) / t); };
    const bool small = tiles(p.F.n, 128) * tiles(p.S.n, 128) * (uint64_t)p.splits * (uint64_t)p.batches < 512;
    const int64_t t = small ? 64 : 128;
    const uint32_t tf = (uint32_t)tiles(p.F.n, t), ts = (uint32_t)tiles(p.S.n, t);
    const hipError_t e = launch_grid((uint64_t)tf * ts * (uint64_t)p.splits * (uint64_t)p.batches, LT, &g);
    if (e != hipSuccess) return e;
    if (shares) *shares = EPI == EPI_SUM ? 0 : p.batches * 2 * (p.bias_f ? ts : tf);
    if (small) hipLaunchKernelGGL((product_kernel<IO, FK, SK, EPI, 64>), g, dim3(LT), 0, st, p, tf, ts);
    else hipLaunchKernelGGL((product_kernel<IO, FK, SK, EPI, 128>), g, dim3(LT), 0, st, p, tf, ts);
    return hipGetLastError();
}
// shares: how many sums of dz's columns it leaves at p.sums (0: none)
template <class IO, int EPI>
hipError_t launch_product(const Product& p, bool fk, bool sk, int64_t* shares, hipStream_t st)
{
    if (fk && sk) return launch_sides<IO, EPI, true, true>(p, shares, st);
    if (fk) return launch_sides<IO, EPI, true, false>(p, shares, st);
    if (sk) return launch_sides<IO, EPI, false, true>(p, shares, st);
    return launch_sides<IO, EPI, false, false>(p, shares, st);
}

// p: dW's product.  Where its sums of columns come beside it, they alone
template <class IO>
hipError_t launch_ones(const Product& p, bool fk, bool sk, int64_t* shares, hipStream_t st)
{
    *shares = 0;
    if constexpr (sizeof(typename IO::T) == 2) {
        if (!whole_pieces(p.F, fk, p.K) || !whole_pieces(p.S, sk, p.K)) return hipSuccess;
        const uint32_t ts = (uint32_t)((p.S.n + 127) / 128);
        dim3 g;
        const hipError_t e = launch_grid((uint64_t)ts * (uint64_t)p.splits, LT, &g);
        if (e != hipSuccess) return e;
        *shares = p.splits;
        if (sk) hipLaunchKernelGGL((ones_kernel<IO, true>), g, dim3(LT), 0, st, p, ts);
        else hipLaunchKernelGGL((ones_kernel<IO, false>), g, dim3(LT), 0, st, p, ts);
    }
    return hipGetLastError();
}

inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// How the places are cut: [B,.,N] by sequences, [B,N,.] not at all; rows of one place are both
struct Cut {
    bool x_first, y_first;
    int64_t batches, places;      // of the products that have the places as an index
    Cut(const LinearArgs& a)
    {
        x_first = a.x_first && a.N > 1;
        y_first = a.y_first && a.N > 1;
        batches = x_first || y_first ? a.B : 1;
        places = x_first || y_first ? a.N : a.B * a.N;
    }
};
// rows [place][c] or [c][place] of a batch
inline Side rows_of(const void* p, bool first, const Cut& c, int64_t width)
{
    return Side{p, c.places, first ? c.places : width, c.places * width, 0};
}

// Shares of a long sum of few tiles: as many as make 256 workgroups of 128 by 128 (fp32: 512 of 64 by 64), of four steps at least.  us, cut and whole:
// bf16, 128 x 4096 -> 4096 26 and 68, 512 x 2048 -> 2048 25 and 37, 300 x 2051 -> 777 21 and 25, 1024 x 1024 -> 1024 24 and 17.5 (not taken); fp32, 128
// x 4096 -> 4096 60 and 126, 512 x 1024 -> 1024 26 and 35, 300 x 515 -> 777 17 and 20.  Two shares: bf16, 1408 x 2048 -> 1408 26 and 37;
// fp32, five shapes of 172 to 256 tiles, K = 640 (20 steps) 25 to 27 and 23.5 (not taken), 768 27 to 28.5 and 27.2 (not taken), 896 (28 steps) 30 to 31 and
// 31, 1024 33 and 34.6, 1280 38 and 42, 2048 55 and 64.
template <class IO>
struct Cuts {
    static constexpr bool F4 = sizeof(typename IO::T) == 4;
    static constexpr int64_t SIDE = F4 ? 64 : 128, BK = Tile<IO, true>::BK, WANT = F4 ? 512 : 256, LONG = F4 ? 512 : 2048;
    static int64_t steps(int64_t K) { return (K + BK - 1) / BK; }
    static int64_t of(int64_t f, int64_t s, int64_t batches, int64_t K, int64_t* per)
    {
        const int64_t tiles = ((f + SIDE - 1) / SIDE) * ((s + SIDE - 1) / SIDE) * batches;
        if (K < LONG) return 1;
        const int64_t want = WANT / tiles, most = steps(K) / 4, n = want < most ? want : most;
        if (n < 2 || (n == 2 && steps(K) < 28)) return 1;
        *per = (steps(K) + n - 1) / n;
        return (steps(K) + *per - 1) / *per;
    }
    // bytes for them of T places to M columns, and of any fewer places: WANT tiles are the most
    static size_t bytes(int64_t T, int64_t K, int64_t M)
    {
        if (K < LONG) return 0;
        const size_t all = (size_t)(steps(K) / 4) * T * M * sizeof(float), most = (size_t)WANT * SIDE * SIDE * sizeof(float);
        return up256(all < most ? all : most);
    }
};
// y, dz or dx by p, whose result's shares have room at `part`
template <class IO, int EPI>
hipError_t product(Product p, bool fk, bool sk, void* part, int64_t* shares, hipStream_t st)
{
    p.splits = Cuts<IO>::of(p.F.n, p.S.n, p.batches, p.K, &p.per);
    if (p.splits == 1) {
        p.per = INT64_MAX / 4;
        p.wide = wide_tiles(p.F.n, p.S.n, p.batches, p.K);
        return launch_product<IO, EPI>(p, fk, sk, shares, st);
    }
    p.wide = false;
    p.part = (float*)part;
    float* const sums = p.sums;
    p.sums = nullptr;
    int64_t none = 0;
    hipError_t e = launch_product<IO, EPI_SUM>(p, fk, sk, &none, st);
    p.sums = sums;
    const uint32_t bf = (uint32_t)((p.F.n + 255) / 256), bs = (uint32_t)((p.S.n + FINISH - 1) / FINISH);
    dim3 g;
    if (e == hipSuccess) e = launch_grid((uint64_t)p.batches * bf * bs, 256, &g);
    if (e != hipSuccess) return e;
    if (shares) *shares = p.batches * (p.bias_f ? bs : bf);
    hipLaunchKernelGGL((linear_finish_kernel<IO, EPI>), g, dim3(256), 0, st, p, bf, bs);
    return hipGetLastError();
}

// z = x W^T + bias and what follows it
template <class IO, int EPI>
hipError_t forward(const LinearArgs& a, const void* x, Product p, void* part, int64_t* shares, hipStream_t st)
{
    const Cut c(a);
    const Side X = rows_of(x, c.x_first, c, a.K), W{a.W, a.M, a.K, 0, 0};
    p.K = a.K;
    p.segs = 1;
    p.batches = c.batches;
    p.bias = a.bias;
    p.act = a.act;
    p.batch = c.places * a.M;
    p.ld = c.y_first ? c.places : a.M;
    p.bias_f = !c.y_first;
    p.F = c.y_first ? X : W;
    p.S = c.y_first ? W : X;
    if (EPI == EPI_OUT && !c.x_first && !c.y_first && c.places <= FEW) return launch_few<IO>(p, st);
    return product<IO, EPI>(p, c.y_first ? !c.x_first : true, c.y_first ? true : !c.x_first, part, shares, st);
}

// Shares of the sum over places of dW, of four steps at least: as many as make 256 workgroups of 256 by 256 where there are 16 such tiles and
// more (fewer: more shares, and with them more sums to write and join), else 512 of 128 by 128.  us, the two: 768 x 2048 (24 tiles) 65 + 11 and
// 98 + 8, 256 x 1024 (4 tiles) 133 and 104.
struct Shares {
    int64_t shares, per;
    bool wide;
};
inline int64_t shares_wanted(int64_t K, int64_t M, bool f32, bool* wide)
{
    const int64_t t = f32 ? 64 : 128;      // (fp32: four workgroups a unit, of 64 by 64)
    const int64_t large = ((K + 255) / 256) * ((M + 255) / 256), tiles = ((K + t - 1) / t) * ((M + t - 1) / t);
    *wide = !f32 && large >= 16;
    return *wide ? (large >= 256 ? 1 : 256 / large) : (512 + tiles - 1) / tiles;
}
template <class IO>
Shares shares_of(int64_t B, int64_t N, int64_t K, int64_t M, bool by_batch)
{
    constexpr int BK = Tile<IO, true>::BK;
    Shares r;
    int64_t want = shares_wanted(K, M, sizeof(typename IO::T) == 4, &r.wide);
    const int64_t steps = by_batch ? B * ((N + BK - 1) / BK) : (B * N + BK - 1) / BK;
    if (want > (steps + 3) / 4) want = (steps + 3) / 4;
    r.per = (steps + want - 1) / want;
    r.shares = (steps + r.per - 1) / r.per;
    return r;
}

template <class IO>
hipError_t linear_fwd_io(const LinearArgs& a, const void* x, const void* residual, void* y, void* ws, hipStream_t st)
{
    Product p = {};
    p.out = y;
    p.residual = residual;
    return forward<IO, EPI_OUT>(a, x, p, ws, nullptr, st);
}

// the most shares that sums of dbias come in: two for each 64 places (a tile's halves; a tile of 256 makes four, but is full to three quarters, so of
// 192 places and more), or as many as dW's sums; one for each FINISH places where a sum is cut, which are at most 128 tiles of 128 (256 of 64)
inline int64_t bias_shares(int64_t B, int64_t N)
{
    const int64_t tiles = B * 2 * ((N + 63) / 64), cut = B * ((N + FINISH - 1) / FINISH), most = 128 * 128 / FINISH, few = cut < most ? cut : most;
    return tiles > few ? tiles : few;
}
inline size_t most_of(size_t a, size_t b, size_t c) { return a > b ? (a > c ? a : c) : b > c ? b : c; }
template <class IO>
size_t linear_workspace_io(int64_t B, int64_t N, int64_t K, int64_t M, int backward)
{
    const size_t cuts = Cuts<IO>::bytes(B * N, K, M), back = Cuts<IO>::bytes(B * N, M, K);
    if (!backward) return cuts + 256;
    if (N == 1) {      // in either layout the places of one sequence (Cut); of longer ones the layouts that cut most are counted
        N = B;
        B = 1;
    }
    bool wide;
    const int64_t want = shares_wanted(K, M, sizeof(typename IO::T) == 4, &wide), steps = (B * ((N + 15) / 16) + 3) / 4;      // (never more shares than either)
    const int64_t shares = want < steps ? want : steps, bias = bias_shares(B, N);
    return up256((size_t)B * N * M * sizeof(typename IO::T)) + most_of(up256((size_t)shares * K * M * sizeof(float)), cuts, back) +
           up256((size_t)(bias > shares ? bias : shares) * M * sizeof(float));
}

template <class IO>
hipError_t linear_bwd_io(const LinearArgs& a, const LinearGrads& d, void* ws, hipStream_t st)
{
    using T = typename IO::T;
    const Cut c(a);
    char* at = (char*)ws;
    void* const dz_room = at;
    at += up256((size_t)a.B * a.N * a.M * sizeof(T));
    const bool by_batch = c.x_first || c.y_first;
    const Shares sh = shares_of<IO>(a.B, a.N, a.K, a.M, by_batch);
    float* const part = (float*)at;      // of dz, dW and dx in turn
    at += most_of(up256((size_t)sh.shares * a.K * a.M * sizeof(float)), Cuts<IO>::bytes(a.B * a.N, a.K, a.M), Cuts<IO>::bytes(a.B * a.N, a.M, a.K));
    float* const sums = (float*)at;
    const void* dz = d.dy;
    hipError_t e = hipSuccess;
    int64_t shares = 0;      // sums of dz's columns that wait at `sums`
    if (a.act != LONGCONV_ACT_NONE) {
        Product p = {};
        p.out = dz_room;
        p.dy = d.dy;
        p.sums = d.dbias ? sums : nullptr;
        e = forward<IO, EPI_DZ>(a, d.x, p, part, &shares, st);
        if (e != hipSuccess) return e;
        dz = dz_room;
    }
    if (d.dW || (d.dbias && !shares)) {      // dW[m][k] = sum over places of dz[place][m] x[place][k]
        Product p = {};
        p.F = rows_of(d.x, c.x_first, c, a.K);
        p.F.seg = p.F.batch;
        p.F.n = a.K;
        p.S = rows_of(dz, c.y_first, c, a.M);
        p.S.seg = p.S.batch;
        p.S.n = a.M;
        p.K = c.places;
        p.segs = c.batches;
        p.batches = 1;
        p.splits = sh.shares;
        p.per = sh.per;
        p.wide = sh.wide;
        p.part = sh.shares == 1 && d.dW_f32 ? (float*)d.dW : part;
        p.sums = d.dbias && !shares ? sums : nullptr;
        int64_t left = 0;
        e = d.dW ? launch_product<IO, EPI_SUM>(p, c.x_first, c.y_first, &left, st) : launch_ones<IO>(p, c.x_first, c.y_first, &left, st);
        if (e != hipSuccess) return e;
        if (p.sums) shares = left;
        if (d.dW && p.part != d.dW) {
            const int64_t n = a.K * a.M;
            const dim3 g((unsigned)((n + 1023) / 1024));
            if (d.dW_f32) hipLaunchKernelGGL(linear_join_kernel<IoF32>, g, dim3(256), 0, st, part, (float*)d.dW, n, sh.shares);
            else hipLaunchKernelGGL(linear_join_kernel<IO>, g, dim3(256), 0, st, part, (T*)d.dW, n, sh.shares);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    if (d.dbias && !shares) {
        if (c.y_first) {
            shares = a.B;
            const int64_t groups = (a.B * a.M + 3) / 4;
            hipLaunchKernelGGL(columns_first_kernel<IO>, dim3((unsigned)(groups < 1 << 20 ? groups : 1 << 20)), dim3(256), 0, st, (const T*)dz, sums, a.B * a.M, a.N);
        } else {
            shares = (a.B * a.N + COLUMN_ROWS - 1) / COLUMN_ROWS;
            const uint32_t wide = (uint32_t)((a.M + 255) / 256);
            hipLaunchKernelGGL(columns_last_kernel<IO>, dim3((unsigned)(shares * wide)), dim3(256), 0, st, (const T*)dz, sums, a.B * a.N, a.M, wide);
        }
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (d.dbias) {
        hipLaunchKernelGGL(columns_join_kernel, dim3((unsigned)((a.M + 31) / 32)), dim3(1024), 0, st, sums, d.dbias, a.M, shares);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!d.dx) return hipSuccess;
    // dx[place][k] = sum_m dz[place][m] W[m][k]
    Product p = {};
    const Side Z = rows_of(dz, c.y_first, c, a.M), W{a.W, a.K, a.K, 0, 0};
    p.K = a.M;
    p.segs = 1;
    p.batches = c.batches;
    p.act = LONGCONV_ACT_NONE;
    p.out = d.dx;
    p.batch = c.places * a.K;
    p.ld = c.x_first ? c.places : a.K;
    p.F = c.x_first ? Z : W;
    p.S = c.x_first ? W : Z;
    return product<IO, EPI_OUT>(p, c.x_first ? !c.y_first : false, c.x_first ? false : !c.y_first, part, nullptr, st);
}

}  // namespace

template <class IO>
size_t linear_workspace_of(int64_t B, int64_t N, int64_t K, int64_t M, int backward)
{
    return linear_workspace_io<IO>(B, N, K, M, backward);
}
template <class IO>
hipError_t linear_fwd_of(const LinearArgs& a, const void* x, const void* residual, void* y, void* ws, hipStream_t st)
{
    return linear_fwd_io<IO>(a, x, residual, y, ws, st);
}
template <class IO>
hipError_t linear_bwd_of(const LinearArgs& a, const LinearGrads& d, void* ws, hipStream_t st)
{
    return linear_bwd_io<IO>(a, d, ws, st);
}

}  // namespace lc
