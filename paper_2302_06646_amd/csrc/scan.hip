// Selective state space scan, in the convolution's layout [B,H,N], with S states of each head and B, C of each of G groups of heads:
//     dt = softplus(delta + bias[h]) (or delta + bias[h]),   h_t[s] = exp(dt_t A[h,s]) h_{t-1}[s] + dt_t B_t[s] u_t,
//     y_t = (sum_s C_t[s] h_t[s] + D[h] u_t) silu(z_t),
// from a given state or zero, for whole sequences and for one new place of each.  The backward pass is in scan_bwd.hip.
#include "scan.hpp"

namespace lc {
namespace {

constexpr int FW = 8, FT = FW * 64;      // waves and threads of a workgroup
constexpr int FC = 2;                    // heads of a wave
constexpr int FB = 2;                    // states whose B and C are brought in at a time

enum Mode { WHOLE, STATES, BACK };

// Workgroup: 16 heads of one group, one segment.  B and C of two states at a time are laid out in fp32 for all of them.
// WHOLE: y, marks and the last state.  STATES: what Segments holds of segments 0 .. segs - 2.  BACK: the same for the gradient of the state,
// g_t = C_t dy_t + a_{t+1} g_{t+1}, as v_t = a_t (C_t dy_t + v_{t+1}) in reversed time, of segments 1 .. segs - 1.
template <class IO, int K, int MODE>
__global__ __launch_bounds__(FT) void scan_kernel(ScanArgs a, const typename IO::T* __restrict__ dy, const float* state, typename IO::T* __restrict__ y,
                                                  float* last, float* __restrict__ marks, Segments g, int blocks)
{
    using T = typename IO::T;
    constexpr int CH = 64 * K;
    __shared__ float4 lds[2][FB][2][CH / 4];           // [buffer][state][B or C][K / 4][lane]
    __shared__ float carry[FW][FC][SCAN_STATES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int run_segs = MODE == WHOLE ? g.segs : g.segs - 1;
    int64_t w = blockIdx.x;
    const int seg = (int)(w % run_segs) + (MODE == BACK);
    w /= run_segs;
    const int blk = (int)(w % blocks);
    w /= blocks;
    const int64_t grp = w % a.G, b = w / a.G, heads = a.H / a.G;
    const int64_t len = scan_length(a, b), N = a.N;
    const int64_t begin = seg * g.len, stop = begin + g.len < N ? begin + g.len : N, end = stop < len ? stop : len;
    const int S = a.S, phases = (S + FB - 1) / FB;
    const T* Bm = (const T*)a.Bm + (size_t)(b * a.G + grp) * S * N;
    const T* Cm = (const T*)a.Cm + (size_t)(b * a.G + grp) * S * N;
    int64_t head[FC];
    bool mine[FC];
    size_t row[FC];
    float bias[FC], D[FC], total[FC];
#pragma unroll
    for (int c = 0; c < FC; ++c) {
        const int64_t i = (int64_t)blk * FW * FC + wave * FC + c;
        mine[c] = i < heads;
        head[c] = grp * heads + (mine[c] ? i : 0);
        row[c] = (size_t)b * a.H + head[c];
        bias[c] = a.bias ? a.bias[head[c]] : 0.f;
        D[c] = a.D ? a.D[head[c]] : 0.f;
        total[c] = 0.f;
        if (lane < S) {
            // (the given state is read here alone where one workgroup has the whole row: `last`, which it writes, may be `state`.  Where
            // several have it the pass over STATES puts it in the place that no segment uses.)
            const float given = MODE == BACK || !state ? 0.f : state[row[c] * S + lane];
            float* const kept = g.ends + (row[c] * g.segs + g.segs - 1) * S + lane;
            if (MODE == STATES && seg == 0 && mine[c]) *kept = given;
            carry[wave][c][lane] =
                MODE == WHOLE ? entering<false>(g, row[c], seg, S, lane, LOG2E * a.A[head[c] * S + lane], g.segs > 1 ? *kept : given) : 0.f;
        }
    }
    // the four places 4 q .. of a chunk as they lie in `lds`: lane 4 q / K, group (4 q % K) / 4 (BACK: in reversed order)
    const auto bring = [&](int64_t t0, int ph, int i, float4& v) {      // piece i of this thread
        const int id = threadIdx.x + i * FT, q = id % (CH / 4), which = id / (CH / 4) % 2, s = ph * FB + id / (CH / 2);
        v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (id >= FB * CH / 2 || s >= S || (MODE == STATES && which == 1) || (MODE == BACK && which == 0)) return;
        const int64_t t = t0 + (MODE == BACK ? CH - 4 - 4 * q : 4 * q);
        v = load4<IO>((which ? Cm : Bm) + (size_t)s * N, t, N, end);
        if (MODE == BACK) v = make_float4(v.w, v.z, v.y, v.x);
    };
    const auto put = [&](int buf, int i, const float4& v) {
        const int id = threadIdx.x + i * FT, q = id % (CH / 4), which = id / (CH / 4) % 2, st = id / (CH / 2);
        if (st < FB) lds[buf][st][which][q % (K / 4) * 64 + q / (K / 4)] = v;
    };
    constexpr int PIECES = (FB * CH / 2 + FT - 1) / FT;
    int64_t t0 = begin;
    if (MODE == BACK) t0 = end <= begin ? begin - CH : begin + (end - 1 - begin) / CH * CH;
    for (; MODE == BACK ? t0 >= begin : t0 < end; t0 += MODE == BACK ? -CH : CH) {
        float dt[FC][K], x[FC][K], out[FC][K], sum[FC];
        const int64_t at = t0 + (MODE == BACK ? 63 - lane : lane) * K;      // this lane's places
#pragma unroll
        for (int c = 0; c < FC; ++c) {
            sum[c] = 0.f;
            if (!mine[c]) continue;
#pragma unroll
            for (int j = 0; j < K; j += 4) {
                const float4 d4 = load4<IO>((const T*)a.delta + row[c] * N, at + j, N, end);
                const float4 u4 = MODE == BACK ? load4<IO>(dy + row[c] * N, at + j, N, end) : load4<IO>((const T*)a.u + row[c] * N, at + j, N, end);
                const float d[4] = {d4.x, d4.y, d4.z, d4.w}, u[4] = {u4.x, u4.y, u4.z, u4.w};
                float z[4] = {0.f, 0.f, 0.f, 0.f};
                if (MODE == BACK && a.z) {
                    const float4 z4 = load4<IO>((const T*)a.z + row[c] * N, at + j, N, end);
                    z[0] = z4.x; z[1] = z4.y; z[2] = z4.z; z[3] = z4.w;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float wv = d[i] + bias[c];
                    const float v = at + j + i < end ? a.softplus ? softplus_of(wv) : wv : 0.f;
                    const int to = MODE == BACK ? K - 1 - j - i : j + i;
                    dt[c][to] = v;
                    sum[c] += v;
                    if (MODE == BACK) x[c][to] = a.z ? u[i] * z[i] * logistic(z[i]) : u[i];
                    else x[c][to] = v * u[i];
                    out[c][to] = D[c] * u[i];
                }
            }
        }
        __syncthreads();      // (the buffers of the chunk before are read, the carries written)
        float4 next[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            bring(t0, 0, i, next[i]);
            put(0, i, next[i]);
        }
        __syncthreads();
        for (int ph = 0; ph < phases; ++ph) {
            const int buf = ph & 1;
            if (ph + 1 < phases)
#pragma unroll
                for (int i = 0; i < PIECES; ++i) bring(t0, ph + 1, i, next[i]);
#pragma unroll
            for (int st = 0; st < FB; ++st) {
                const int s = ph * FB + st;
                if (s >= S) continue;
                float Bv[K], Cv[K];
#pragma unroll
                for (int j = 0; j < K / 4; ++j) {
                    if (MODE != BACK) {
                        const float4 q = lds[buf][st][0][j * 64 + lane];
                        Bv[4 * j] = q.x; Bv[4 * j + 1] = q.y; Bv[4 * j + 2] = q.z; Bv[4 * j + 3] = q.w;
                    }
                    if (MODE != STATES) {
                        const float4 q = lds[buf][st][1][j * 64 + lane];
                        Cv[4 * j] = q.x; Cv[4 * j + 1] = q.y; Cv[4 * j + 2] = q.z; Cv[4 * j + 3] = q.w;
                    }
                }
#pragma unroll
                for (int c = 0; c < FC; ++c) {
                    if (!mine[c]) continue;
                    const float A2 = LOG2E * a.A[head[c] * S + s];
                    const float in = carry[wave][c][s];
                    float d[K], h = lane == 0 ? in : 0.f;
#pragma unroll
                    for (int i = 0; i < K; ++i) {
                        d[i] = exp2_of(A2 * dt[c][i]);
                        if (MODE == BACK) h = d[i] * __builtin_fmaf(x[c][i], Cv[i], h);
                        else h = __builtin_fmaf(d[i], h, x[c][i] * Bv[i]);
                    }
                    float p = exp2_of(A2 * sum[c]);
                    scan_up(p, h);
                    if (MODE == WHOLE) {
                        if (marks && t0 % SPAN == 0 && lane == 0) marks[(row[c] * ((N + SPAN - 1) / SPAN) + t0 / SPAN) * S + s] = in;
                        float v = dpp<0x138>(h, in);      // of the lane before
#pragma unroll
                        for (int i = 0; i < K; ++i) {
                            v = __builtin_fmaf(d[i], v, x[c][i] * Bv[i]);
                            out[c][i] = __builtin_fmaf(Cv[i], v, out[c][i]);
                        }
                    }
                    if (lane == 63) carry[wave][c][s] = h;
                }
            }
            if (ph + 1 < phases)
#pragma unroll
                for (int i = 0; i < PIECES; ++i) put(buf ^ 1, i, next[i]);
            __syncthreads();
        }
#pragma unroll
        for (int c = 0; c < FC; ++c) {
            if (!mine[c]) continue;
            if (MODE != WHOLE) {
                total[c] += sum_of_wave(sum[c]);
                continue;
            }
            if (a.z) {
#pragma unroll
                for (int j = 0; j < K; j += 4) {
                    const float4 z4 = load4<IO>((const T*)a.z + row[c] * N, at + j, N, end);
                    const float z[4] = {z4.x, z4.y, z4.z, z4.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) out[c][j + i] *= z[i] * logistic(z[i]);
                }
            }
            T* to = y + row[c] * N;
#pragma unroll
            for (int i = 0; i < K; ++i) out[c][i] = at + i < end ? out[c][i] : 0.f;
            if constexpr (K >= VE) {
#pragma unroll
                for (int j = 0; j < K; j += VE) {
                    const int64_t n = N - at - j;
                    if (n > 0) store8<IO, true>(to + at + j, n < VE ? (int)n : VE, reinterpret_cast<float(&)[VE]>(out[c][j]));
                }
            } else {
#pragma unroll
                for (int i = 0; i < K; ++i)
                    if (at + i < N) IO::st(to, at + i, out[c][i]);
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < FC; ++c) {
        if (!mine[c]) continue;
        if (MODE == WHOLE) {
            // behind the sequence's end: zeros from the first place that no chunk wrote
            const int64_t zero = end > begin ? begin + (end - begin + CH - 1) / CH * CH : begin;
            for (int64_t t = zero + lane; t < stop; t += 64) IO::st(y + row[c] * N, t, 0.f);
            if (last && seg == g.segs - 1 && lane < S) last[row[c] * S + lane] = carry[wave][c][lane];
        } else {
            if (lane < S) g.ends[(row[c] * g.segs + seg) * S + lane] = carry[wave][c][lane];
            if (lane == 0) g.sums[row[c] * g.segs + seg] = total[c];
        }
    }
}

// One new place of each sequence: four states of a head in a thread, `lanes` neighbouring threads for a head
template <class IO>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanArgs a, float* __restrict__ state, typename IO::T* __restrict__ y, int log_lanes)
{
    using T = typename IO::T;
    const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, at = id >> log_lanes;
    const int s0 = 4 * (int)(id & ((1 << log_lanes) - 1)), S = a.S;
    if (at >= a.B * a.H) return;      // (whole heads: their lanes leave together)
    const int64_t b = at / a.H, h = at - b * a.H, grp = h / (a.H / a.G);
    const T *Bm = (const T*)a.Bm + (size_t)(b * a.G + grp) * S, *Cm = (const T*)a.Cm + (size_t)(b * a.G + grp) * S;
    const float u = IO::ld((const T*)a.u, at), w = IO::ld((const T*)a.delta, at) + (a.bias ? a.bias[h] : 0.f);
    const float dt = a.softplus ? softplus_of(w) : w;
    float* sr = state + (size_t)at * S;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int s = s0 + i;
        if (s < S) {
            const float v = __builtin_fmaf(exp2_of(LOG2E * a.A[h * S + s] * dt), sr[s], dt * u * IO::ld(Bm, s));
            sr[s] = v;
            sum = __builtin_fmaf(IO::ld(Cm, s), v, sum);
        }
    }
    for (int d = 1; d < 1 << log_lanes; d *= 2) sum += __shfl_xor(sum, d);
    if (s0 == 0) {
        float out = a.D ? __builtin_fmaf(a.D[h], u, sum) : sum;
        if (a.z) {
            const float z = IO::ld((const T*)a.z, at);
            out *= z * logistic(z);
        }
        IO::st(y, at, out);
    }
}

int64_t row_blocks(const ScanArgs& a) { return (a.H / a.G + FW * FC - 1) / (FW * FC); }

// Segments: none where the heads alone are 256 workgroups; else as many as make 512, of 1024 places at least.
int segments(int64_t B, int64_t H, int64_t N, int64_t G)
{
    const int64_t groups = B * G * ((H / G + FW * FC - 1) / (FW * FC)), most = (N + 1023) / 1024;
    if (groups >= 256) return 1;
    const int64_t want = (512 + groups - 1) / groups;
    return (int)(want < most ? want : most);
}

template <class IO, int K, int MODE>
hipError_t launch(const ScanArgs& a, const void* dy, const float* state, void* y, float* last, float* marks, const Segments& g, hipStream_t st)
{
    using T = typename IO::T;
    const int64_t blocks = row_blocks(a);
    dim3 grid;
    const hipError_t e = launch_grid((uint64_t)(a.B * a.G * blocks * (MODE == WHOLE ? g.segs : g.segs - 1)), FT, &grid);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((scan_kernel<IO, K, MODE>), grid, dim3(FT), 0, st, a, (const T*)dy, state, (T*)y, last, marks, g, (int)blocks);
    return hipGetLastError();
}
Segments segments_of(const ScanArgs& a, void* ws)
{
    Segments g;
    g.segs = segments(a.B, a.H, a.N, a.G);
    g.len = ((a.N + g.segs - 1) / g.segs + SPAN - 1) / SPAN * SPAN;
    g.segs = (int)((a.N + g.len - 1) / g.len);
    g.ends = (float*)ws;
    g.sums = g.ends + (size_t)a.B * a.H * g.segs * a.S;
    return g;
}

template <class IO>
hipError_t fwd(const ScanArgs& a, const float* state, void* y, float* last, float* marks, void* ws, hipStream_t st)
{
    const Segments g = segments_of(a, ws);
    if (g.segs > 1) {
        const hipError_t e = launch<IO, 8, STATES>(a, nullptr, state, nullptr, nullptr, nullptr, g, st);
        if (e != hipSuccess) return e;
    }
    return a.N <= 256 ? launch<IO, 4, WHOLE>(a, nullptr, state, y, last, marks, g, st) : launch<IO, 8, WHOLE>(a, nullptr, state, y, last, marks, g, st);
}

template <class F>
hipError_t by_io(int io, F&& f)
{
    if (io == LONGCONV_F32) return f(IoF32());
    return io == LONGCONV_F16 ? f(IoF16()) : f(IoBF16());
}

}  // namespace

size_t scan_segment_bytes(int64_t B, int64_t H, int64_t N, int S, int64_t G)
{
    // rows times segments of any batch up to B: at most one segment for each 1024 places, and where there are several at most 512 /
    // (workgroups of a sequence) + B, with B < 256
    const int64_t blocks = G * ((H / G + FW * FC - 1) / (FW * FC)), all = B * ((N + 1023) / 1024), some = 512 / blocks + 1 + (B < 256 ? B : 256);
    return up256((size_t)(all < some ? all : some) * H * (S + 1) * sizeof(float));
}
size_t scan_workspace_bytes(int64_t B, int64_t H, int64_t N, int S, int64_t G, int backward)
{
    return scan_segment_bytes(B, H, N, S, G) + (backward ? scan_bwd_bytes(B, H, N, S, G) : 0);
}

hipError_t scan_fwd(const ScanArgs& a, const float* state, void* y, float* last, float* marks, void* ws, hipStream_t st)
{
    return by_io(a.io, [&](auto io) { return fwd<decltype(io)>(a, state, y, last, marks, ws, st); });
}

hipError_t scan_back(const ScanArgs& a, const void* dy, void* ws, Segments* g, hipStream_t st)
{
    *g = segments_of(a, ws);
    if (g->segs == 1) return hipSuccess;
    return by_io(a.io, [&](auto io) { return launch<decltype(io), 8, BACK>(a, dy, nullptr, nullptr, nullptr, nullptr, *g, st); });
}

hipError_t scan_step(const ScanArgs& a, float* state, void* y, hipStream_t st)
{
    int log_lanes = 0;
    while (4 << log_lanes < a.S) ++log_lanes;
    dim3 g;
    const hipError_t e = launch_grid((uint64_t)(((a.B * a.H << log_lanes) + 255) / 256), 256, &g);
    if (e != hipSuccess) return e;
    return by_io(a.io, [&](auto io) {
        using IO = decltype(io);
        hipLaunchKernelGGL(scan_step_kernel<IO>, g, dim3(256), 0, st, a, state, (typename IO::T*)y, log_lanes);
        return hipGetLastError();
    });
}

}  // namespace lc
