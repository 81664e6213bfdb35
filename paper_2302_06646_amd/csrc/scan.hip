// Selective state space scan, in the convolution's layout [B,H,N], with S states of each head and B, C of each of G groups of heads:
//     dt = softplus(delta + bias[h]) (or delta + bias[h]),   h_t[s] = exp(dt_t A[h,s]) h_{t-1}[s] + dt_t B_t[s] u_t,
//     y_t = (sum_s C_t[s] h_t[s] + D[h] u_t) silu(z_t),
// from a given state or zero, for whole sequences and for one new place of each.  The backward pass is in scan_bwd.hip.
#include "scan.hpp"

namespace lc {
namespace {

constexpr int FW = 8, FT = FW * 64;      // waves of a workgroup, each with a head of its own; threads
constexpr int FB = 8;                    // states whose B and C are brought in at a time, while those before are worked on

enum Mode { WHOLE, STATES, BACK };

// Workgroup: eight heads of one group, one segment.  B and C of FB states at a time are laid out in fp32 for all of them; a wave has two
// states at a time.
// What bounds it is the vector instructions: for each state eight places of a lane take 72 of them, eight exponentials (8 cycles each) and five
// multiplications or multiply-adds a place among them (2.7).  16 x 1024 x 1024, 16 states, gated, bf16: 132 us, 100 of them vector
// instructions by the counter (54 M, at 2.4 GHz); 8 x 256 x 16384, fp16, uneven lengths, 266 and 128 (70 M), at two waves a SIMD.
// WHOLE: y, marks and the last state.  STATES: what Segments holds of segments 0 .. segs - 2.  BACK: the same for the gradient of the state,
// g_t = C_t dy_t + a_{t+1} g_{t+1}, as v_t = a_t (C_t dy_t + v_{t+1}) in reversed time, of segments 1 .. segs - 1.
// A and the states between chunks are kept one in a lane, lane s for state s.
template <class IO, int K, int MODE>
__global__ __launch_bounds__(FT, 4) void scan_kernel(ScanArgs a, const typename IO::T* __restrict__ dy, const float* state, typename IO::T* __restrict__ y,
                                                  float* last, float* __restrict__ marks, Segments g, int blocks)
{
    using T = typename IO::T;
    constexpr int CH = 64 * K;
    __shared__ float4 lds[2][FB][2][CH / 4];           // [buffer][state][B or C][K / 4][lane]
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
    const int S = a.S;
    const T* Bm = (const T*)a.Bm + (size_t)(b * a.G + grp) * S * N;
    const T* Cm = (const T*)a.Cm + (size_t)(b * a.G + grp) * S * N;
    // (a wave that has no head left runs along with the group's first one and writes nothing)
    const int64_t mine_of = (int64_t)blk * FW + wave;
    const bool mine = mine_of < heads;
    const int64_t head = grp * heads + (mine ? mine_of : 0);
    const size_t row = (size_t)b * a.H + head;
    const T* const delta = (const T*)a.delta + row * N;
    const T* const in = (MODE == BACK ? dy : (const T*)a.u) + row * N;
    const T* const zr = a.z ? (const T*)a.z + row * N : nullptr;
    const float bias = a.bias ? a.bias[head] : 0.f, D = a.D ? a.D[head] : 0.f;
    float total = 0.f, A2 = 0.f, carry = 0.f;
    if (lane < S) {
        A2 = LOG2E * a.A[head * S + lane];
        // (the given state is read here alone where one workgroup has the whole row: `last`, which it writes, may be `state`.  Where
        // several have it the pass over STATES puts it in the place that no segment uses.)
        const float given = MODE == BACK || !state ? 0.f : state[row * S + lane];
        float* const kept = g.ends + (row * g.segs + g.segs - 1) * S + lane;
        if (MODE == STATES && seg == 0 && mine) *kept = given;
        if (MODE == WHOLE) carry = entering<false>(g, row, seg, S, lane, A2, g.segs > 1 ? *kept : given);
    }
    // Pieces of four places of B and C: piece 4 q .. of a chunk lies in `lds` at lane 4 q / K, group (4 q % K) / 4 (BACK: in reversed order)
    constexpr int PER = CH / 4, PIECES = FB * 2 * PER / FT;
    static_assert(FB * 2 * PER % FT == 0 && FT % PER == 0, "whole rows of pieces a thread");
    const int q4 = threadIdx.x % PER, line = threadIdx.x / PER;      // its rows of pieces: line, line + FT / PER, ...
    Raw4<IO> raw[PIECES];
    const int t4 = MODE == BACK ? CH - 4 - 4 * q4 : 4 * q4, tl = (MODE == BACK ? 63 - lane : lane) * K;      // places of a piece, of the lane
    const auto left = [&](int64_t t0, int64_t to) { return (int)(to - t0 < CH ? to - t0 : CH); };
    const auto whole = [&](int64_t t0) { return t0 + CH + VE <= N && t0 + CH <= end; };      // (a piece of eight may reach past a chunk of 256)
    const auto bring = [&](int64_t t0, int s0) {
        const int n = N - t0 < CH ? (int)(N - t0) : CH, lim = left(t0, end);
        const bool full = whole(t0) && s0 + FB <= S;
        const T *const Bt = Bm + t0, *const Ct = Cm + t0;
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int r = line + i * (FT / PER), s = s0 + r / 2, which = r % 2;      // B or C of a state
            if ((MODE == STATES && which == 1) || (MODE == BACK && which == 0)) raw[i].zero();
            else if (full || (s < S && t4 < lim)) raw[i].ask((which ? Ct : Bt) + (size_t)s * N, t4, n, full);
            else raw[i].zero();
        }
    };
    const auto put = [&](int buf, int64_t t0) {
        const int lim = left(t0, end);
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int r = line + i * (FT / PER);
            const float4 v = raw[i].get(t4, lim, lim == CH);
            lds[buf][r / 2][r % 2][q4 % (K / 4) * 64 + q4 / (K / 4)] = MODE == BACK ? make_float4(v.w, v.z, v.y, v.x) : v;
        }
    };
    Raw8<IO> rd, ru, rz;      // a piece of eight of this chunk, asked for during the one before
    const auto ask = [&](const T* from, int64_t t0, Raw8<IO>& r) {
        int lim = left(t0, end);
        if (K < VE && tl + K < lim) lim = tl + K;
        ask8<IO>(from + t0, tl, N - t0 < CH + VE ? (int)(N - t0) : CH + VE, lim, r, whole(t0));
    };
    const auto ask_all = [&](int64_t t0) {
        ask(delta, t0, rd);
        ask(in, t0, ru);
        if (MODE == BACK && zr) ask(zr, t0, rz);
    };
    int64_t t0 = begin;
    if (MODE == BACK) t0 = end <= begin ? begin - CH : begin + (end - 1 - begin) / CH * CH;
    const auto going = [&](int64_t t) { return MODE == BACK ? t >= begin : t < end; };
    int buf = 0;
    if (going(t0)) {
        ask_all(t0);
        bring(t0, 0);
    }
    for (; going(t0); t0 += MODE == BACK ? -CH : CH) {
        float dt[K], x[K], out[K], sum = 0.f;
        const int lim = left(t0, end);
        {
            float d[VE], u[VE], z[VE];
            rd.get(d);
            ru.get(u);
            if (MODE == BACK && zr) rz.get(z);
#pragma unroll
            for (int i = 0; i < K; ++i) d[i] += bias;
            if (a.softplus) {
#pragma unroll
                for (int i = 0; i < K; ++i) d[i] = softplus_of(d[i]);
            }
            if (MODE == BACK && zr) {
#pragma unroll
                for (int i = 0; i < K; ++i) u[i] *= z[i] * logistic(z[i]);
            }
            if (lim < CH) {
#pragma unroll
                for (int i = 0; i < K; ++i) {
                    d[i] = tl + i < lim ? d[i] : 0.f;
                    u[i] = tl + i < lim ? u[i] : 0.f;
                }
            }
#pragma unroll
            for (int i = 0; i < K; ++i) {
                const int to = MODE == BACK ? K - 1 - i : i;
                dt[to] = d[i];
                sum += d[i];
                x[to] = MODE == BACK ? u[i] : d[i] * u[i];
                out[to] = D * u[i];
            }
        }
        const int64_t t_next = t0 + (MODE == BACK ? -CH : CH);
        if (going(t_next)) ask_all(t_next);
        if (MODE == WHOLE && zr) ask(zr, t0, rz);
        if (MODE == WHOLE && marks && t0 % SPAN == 0 && mine && lane < S) marks[(row * ((N + SPAN - 1) / SPAN) + t0 / SPAN) * S + lane] = carry;
        for (int s0 = 0; s0 < S; s0 += FB, buf ^= 1) {
            put(buf, t0);
            __syncthreads();      // (the other buffer's readers are past it too: it is filled behind the next one of these)
            if (s0 + FB < S) bring(t0, s0 + FB);
            else if (going(t_next)) bring(t_next, 0);
            const int here = S - s0 < FB ? S - s0 : FB;
            for (int s1 = 0; s1 < here; s1 += 2) {      // (a state that is not there: B and C zero)
                float Bv[2][K], Cv[2][K], d[2][K], h[2], p[2], was[2];
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    const int s = s0 + s1 + st;
#pragma unroll
                    for (int j = 0; j < K / 4; ++j) {
                        if (MODE != BACK) {
                            const float4 q = lds[buf][s1 + st][0][j * 64 + lane];
                            Bv[st][4 * j] = q.x; Bv[st][4 * j + 1] = q.y; Bv[st][4 * j + 2] = q.z; Bv[st][4 * j + 3] = q.w;
                        }
                        if (MODE != STATES) {
                            const float4 q = lds[buf][s1 + st][1][j * 64 + lane];
                            Cv[st][4 * j] = q.x; Cv[st][4 * j + 1] = q.y; Cv[st][4 * j + 2] = q.z; Cv[st][4 * j + 3] = q.w;
                        }
                    }
                    const float A_s = lane_of(A2, s);
                    was[st] = lane_of(carry, s);
                    h[st] = lane == 0 ? was[st] : 0.f;
#pragma unroll
                    for (int i = 0; i < K; ++i) {
                        d[st][i] = exp2_of(A_s * dt[i]);
                        if (MODE == BACK) h[st] = d[st][i] * __builtin_fmaf(x[i], Cv[st][i], h[st]);
                        else h[st] = __builtin_fmaf(d[st][i], h[st], x[i] * Bv[st][i]);
                    }
                    p[st] = exp2_of(A_s * sum);
                }
                scan_up(p[0], h[0], p[1], h[1]);
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    carry = with_lane(carry, s0 + s1 + st, lane_of(h[st], 63));
                    if (MODE == WHOLE) {
                        float v = dpp<0x138>(h[st], was[st]);      // of the lane before
#pragma unroll
                        for (int i = 0; i < K; ++i) {
                            v = __builtin_fmaf(d[st][i], v, x[i] * Bv[st][i]);
                            out[i] = __builtin_fmaf(Cv[st][i], v, out[i]);
                        }
                    }
                }
            }
        }
        if (MODE != WHOLE) {
            total += sum_of_wave(sum);
            continue;
        }
        if (!mine) continue;
        T* const to = y + (row * N + t0) + (uint32_t)tl;
        const int n = left(t0, N) - tl;
        if (zr) {
            float z[VE];
            rz.get(z);
#pragma unroll
            for (int i = 0; i < K; ++i) out[i] *= z[i] * logistic(z[i]);
        }
        if (lim < CH) {
#pragma unroll
            for (int i = 0; i < K; ++i) out[i] = tl + i < lim ? out[i] : 0.f;
        }
        if constexpr (K == VE) {
            if (lim == CH) store8<IO, true>(to, VE, out);
            else if (n > 0) store8<IO, true>(to, n < VE ? n : VE, out);
        } else {
#pragma unroll
            for (int i = 0; i < K; ++i)
                if (i < n) IO::st(to, i, out[i]);
        }
    }
    if (!mine) return;
    if (MODE == WHOLE) {
        // behind the sequence's end: zeros from the first place that no chunk wrote
        const int64_t zero = end > begin ? begin + (end - begin + CH - 1) / CH * CH : begin;
        for (int64_t t = zero + lane; t < stop; t += 64) IO::st(y + row * N, t, 0.f);
        if (last && seg == g.segs - 1 && lane < S) last[row * S + lane] = carry;
    } else {
        if (lane < S) g.ends[(row * g.segs + seg) * S + lane] = carry;
        if (lane == 0) g.sums[row * g.segs + seg] = total;
    }
}

// One new place of each sequence: four states of a head in a thread, 1 << log_lanes neighbouring threads for a head.  The launch bounds it: 64 x 1024
// heads of 16 states 6.1 us, for 8.4 MB of states.
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

int64_t row_blocks(const ScanArgs& a) { return (a.H / a.G + FW - 1) / FW; }

// Segments: none where the heads alone are 256 workgroups; else as many as make 512, of 1024 places at least.  us at B x 256 heads x 16384, 16 states,
// B = 1: 16 segments 61, 8 68, 4 123, one 250; B = 4: 4 198, 8 194, one 269; B = 8 (256 workgroups): one 275, 2 316.
int segments(int64_t B, int64_t H, int64_t N, int64_t G)
{
    const int64_t groups = B * G * ((H / G + FW - 1) / FW), most = (N + 1023) / 1024;
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
    // (us, four places a lane and eight: 64 x 256 rows of 128, 16 states, 42 and 59, of 250 48 and 68)
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
    const int64_t blocks = G * ((H / G + FW - 1) / FW), all = B * ((N + 1023) / 1024), some = 512 / blocks + 1 + (B < 256 ? B : 256);
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
