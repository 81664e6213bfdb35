// Backward pass of the selective scan (formulas of the forward pass: scan.hip).  With g_t the gradient of the state h_t, q_t = g_t a_t h_{t-1}:
//     dy' = dy silu(z),   dz = dy (C h + D u) silu'(z),   g_t = C_t dy'_t + a_{t+1} g_{t+1}   (behind the last place: dlast),
//     du = dt sum_s g B + D dy',   ddt = sum_s A q + u sum_s g B,   ddelta = ddt (1 - exp(-dt) with softplus),
//     dA = sum_{b,t} dt q,   dB = sum over the group's heads of g dt u,   dC = ... of dy' h,   dD = sum dy' u,   dbias = sum ddelta.
//
// Chunks of SPAN places, from the last to the first.  A wave has NS states and walks over a block of heads: the sums over heads, dB and dC,
// stay in its registers for the chunk; the sums over states, of every head, go through LDS between the NW waves.  h runs again from the
// forward pass's marks, one for each chunk.
// 16 x 1024 x 1024, 16 states, gated, bf16: 359 us under the profiler, the call with its joining launch 356 back to back.  A wave spends some 550 vector
// instructions on a head's chunk, 15 for each of its 16 places and states and the rest on the two scans, sums and a head's beginning and end; by the
// counter they are 245 us at 2.4 GHz, at two waves a SIMD (217 registers).
// States a wave: with four of them and four waves, and with one and sixteen, registers spill (1395 and 815 us at 16 states).  More than 16 states go
// in groups of 16 for each chunk, the sums over states kept in memory between them.
#include "scan.hpp"

namespace lc {
namespace {

constexpr int K = SPAN / 64;      // places of a lane
constexpr int GROUP = 16;         // states that a workgroup's waves hold at once

// where place t of a chunk lies in LDS: a wave's reads of four places a lane are one run of memory
__device__ __forceinline__ int place(int t) { return (t % K / 4 * 64 + t / K) * 4 + t % 4; }

// to LDS, without waiting for what is there (one lane adds to a place, so the order is its program's)
__device__ __forceinline__ void add(float* to, float v) { __hip_atomic_fetch_add(to, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }

// v is made by here: the compiler otherwise puts off what is only needed later, and keeps what it is made of for as long
__device__ __forceinline__ void made(float& v) { asm volatile("" : "+v"(v)); }

struct Parts {
    float *dB, *dC;      // [blocks][B,G,S,N], or null: dB and dC are written themselves
    float *dA;           // [B segs][H,S]
    float *dDb;          // [B segs][H,2]: of D and of the bias
    float *more;         // [B,H,segs][3][SPAN]: a chunk's sums over the states so far, where there are more than a workgroup's waves hold
};

// MANY: more states than NS NW, which go one group behind the other for each chunk.
template <class IO, int NS, int NW, bool GATED, bool MANY>
__global__ __launch_bounds__(64 * NW, 2) void scan_bwd_kernel(ScanArgs a, ScanGrads d, Segments g, Parts parts, int blocks, int CB)
{
    using T = typename IO::T;
    constexpr int TH = 64 * NW, SP = NS * NW, TPT = SPAN / TH;      // threads, states with those that are not there, places of a thread
    extern __shared__ __align__(16) float lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tid = threadIdx.x;
    const int S = a.S, row_of = MANY ? (S + SP - 1) / SP * SP : SP;      // states of a head in LDS
    float* const stages = lds;                       // [2][3][SPAN]: dt, dt u, dy' of a head, and of the next one
    float* const sums = stages + 2 * 3 * SPAN;       // [2][NW][3][SPAN]: sums over a wave's states of g B, A q, C h, and of the head before
    float* const gcar = sums + 2 * NW * 3 * SPAN;    // [CB][row_of]: what the chunk behind hands on
    float* const dAsum = gcar + CB * row_of;         // [CB][row_of]
    float* const small = dAsum + CB * row_of;        // [NW][CB][2]: of dD and dbias
    int64_t w = blockIdx.x;
    const int seg = (int)(w % g.segs);
    w /= g.segs;
    const int blk = (int)(w % blocks);
    w /= blocks;
    const int64_t grp = w % a.G, b = w / a.G, in_group = a.H / a.G;
    const int64_t N = a.N, len = scan_length(a, b);
    const int64_t begin = seg * g.len, stop = begin + g.len < N ? begin + g.len : N, end = stop < len ? stop : len;
    const int64_t head0 = grp * in_group + (int64_t)blk * CB;
    const int heads = (int)(in_group - (int64_t)blk * CB < CB ? in_group - (int64_t)blk * CB : CB);
    const int64_t n_marks = (N + SPAN - 1) / SPAN;
    const size_t bg = (size_t)(b * a.G + grp) * S;      // rows of B, C
    for (int i = tid; i < heads * row_of; i += TH) {
        const int c = i / row_of, s = i % row_of;
        const size_t row = (size_t)b * a.H + head0 + c;
        float from = 0.f;
        if (s < S) from = entering<true>(g, row, seg, S, s, LOG2E * a.A[(head0 + c) * S + s], d.dlast ? d.dlast[row * S + s] : 0.f);
        gcar[c * row_of + s] = from;
        dAsum[c * row_of + s] = 0.f;
    }
    for (int i = tid; i < NW * CB * 2; i += TH) small[i] = 0.f;

    const int64_t top = end > begin ? begin + (end - 1 - begin) / SPAN * SPAN : begin - SPAN;
    for (int64_t t0 = top; t0 >= begin; t0 -= SPAN)
    for (int s0 = 0; s0 < (MANY ? S : 1); s0 += SP) {
        const bool final = !MANY || s0 + SP >= S;      // of the groups of states
        float dBv[NS][K], dCv[NS][K];
        float Bv[NS][K], Cv[NS][K];      // for all heads
        const int lim = (int)(end - t0 < SPAN ? end - t0 : SPAN), left = (int)(N - t0 < SPAN ? N - t0 : SPAN);
        const auto bring = [&](int n, float (&Bq)[K], float (&Cq)[K]) {
            const int s = s0 + wave * NS + n;
            Raw8<IO> rB, rC;
            ask8<IO>((const T*)a.Bm + ((bg + s) * N + t0), lane * K, left, s < S ? lim : 0, rB, lim == SPAN && s < S);
            ask8<IO>((const T*)a.Cm + ((bg + s) * N + t0), lane * K, left, s < S ? lim : 0, rC, lim == SPAN && s < S);
            rB.get(Bq);
            rC.get(Cq);
            if (lim < SPAN) {
#pragma unroll
                for (int i = 0; i < K; ++i) {
                    Bq[i] = lane * K + i < lim ? Bq[i] : 0.f;
                    Cq[i] = lane * K + i < lim ? Cq[i] : 0.f;
                }
            }
        };
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            bring(n, Bv[n], Cv[n]);
#pragma unroll
            for (int i = 0; i < K; ++i) dBv[n][i] = dCv[n][i] = 0.f;
        }
        const auto one_of = [&](int c) { return c < heads ? c : heads - 1; };      // (the last head once more: nobody reads it)
        // Of this thread's places and of the wave's states (lane n for state wave NS + n), of head c, asked for during the one before.  Nothing is
        // asked for under a condition, and nothing converted: either would wait for it at once.  What is not there is asked for elsewhere and
        // made zero in lay().
        T nd[TPT], nu[TPT], ny[TPT], nz[TPT];
        float nA, nm, nD, nbias;
        const int s_mine = s0 + wave * NS + (lane < NS ? lane : 0), s_there = s_mine < S ? s_mine : 0;
        const float *const Dr = a.D ? a.D : a.A, *const br = a.bias ? a.bias : a.A;
        const auto ask = [&](int c) {
            const size_t row = (size_t)b * a.H + head0 + c, at0 = row * N + t0;
#pragma unroll
            for (int i = 0; i < TPT; ++i) {
                const uint32_t t = (uint32_t)(tid * TPT + i < lim ? tid * TPT + i : lim - 1);
                nd[i] = ((const T*)a.delta + at0)[t];
                nu[i] = ((const T*)a.u + at0)[t];
                ny[i] = ((const T*)d.dy + at0)[t];
                nz[i] = GATED ? ((const T*)a.z + at0)[t] : T();
            }
            nD = Dr[head0 + c];
            nbias = br[head0 + c];
            nA = a.A[(head0 + c) * S + s_there];
            nm = d.marks[(row * n_marks + t0 / SPAN) * S + s_there];
        };
        // this thread's places: for all waves, and what it needs of them itself
        struct Own {
            float dt[TPT], u[TPT], dyg[TPT], dyz[TPT], rate[TPT], A, mark, D;
        };
        const auto lay = [&](int c) {
            Own o;
            o.A = s_mine < S ? nA : 0.f;
            o.mark = s_mine < S ? nm : 0.f;
            made(o.A);
            made(o.mark);
            o.D = a.D ? nD : 0.f;
            const float bias = a.bias ? nbias : 0.f;
            float* const stage = stages + (c & 1) * 3 * SPAN;
#pragma unroll
            for (int i = 0; i < TPT; ++i) {
                const bool is = tid * TPT + i < lim;
                const float x = IO::ld(nd, i) + bias, u = is ? IO::ld(nu, i) : 0.f, dy = is ? IO::ld(ny, i) : 0.f, z = is ? IO::ld(nz, i) : 0.f, q = GATED ? logistic(z) : 1.f;
                float rate;
                const float sp = softplus_of(x, &rate), y = a.softplus ? sp : x;
                o.dt[i] = is ? y : 0.f;
                o.rate[i] = a.softplus ? rate : 1.f;
                o.u[i] = u;
                o.dyg[i] = GATED ? dy * (z * q) : dy;
                o.dyz[i] = dy * (q * (1.f + z * (1.f - q)));
                const int to = place(tid * TPT + i);
                stage[to] = o.dt[i];
                stage[SPAN + to] = o.dt[i] * o.u[i];
                stage[2 * SPAN + to] = o.dyg[i];
            }
            return o;
        };
        __syncthreads();      // (the chunk before is done with `stages`)
        ask(0);
        Own own = lay(0);
        ask(one_of(1));
        __syncthreads();
        float e[K], x[K], f[K], cl;      // dt, dt u, dy' of the lane's places; lane n: what the chunk behind hands on to state wave NS + n
        const auto take = [&](int c) {
            const float* const stage = stages + (c & 1) * 3 * SPAN;
#pragma unroll
            for (int j = 0; j < K / 4; ++j) {
                const float4 q = reinterpret_cast<const float4*>(stage)[j * 64 + lane];
                const float4 r = reinterpret_cast<const float4*>(stage + SPAN)[j * 64 + lane];
                const float4 v = reinterpret_cast<const float4*>(stage + 2 * SPAN)[j * 64 + lane];
                e[4 * j] = q.x; e[4 * j + 1] = q.y; e[4 * j + 2] = q.z; e[4 * j + 3] = q.w;
                x[4 * j] = r.x; x[4 * j + 1] = r.y; x[4 * j + 2] = r.z; x[4 * j + 3] = r.w;
                f[4 * j] = v.x; f[4 * j + 1] = v.y; f[4 * j + 2] = v.z; f[4 * j + 3] = v.w;
            }
            cl = gcar[one_of(c) * row_of + s_mine];
        };
        take(0);
        for (int c = 0; c < heads; ++c) {
            const size_t at0 = ((size_t)b * a.H + head0 + c) * N + t0;
            const int here = (int)(stop - t0 < SPAN ? stop - t0 : SPAN);
            const float Al = own.A, ml = own.mark;
            float* const part = sums + (c & 1) * NW * 3 * SPAN;
            float gB[K], Aq[K], Ch[K], sum = 0.f;
#pragma unroll
            for (int i = 0; i < K; ++i) sum += e[i];
            float dA[NS < 2 ? 2 : NS];
            dA[1] = 0.f;
            // both states at once (a state that is not there: A, B, C and all that comes of them zero)
            constexpr int P = NS < 2 ? 1 : 2;
#pragma unroll
            for (int n = 0; n < NS; n += P) {
                float dec[P][K], q[P][K], v[P], p[P], all[P], A[P], in[P], back[P];
#pragma unroll
                for (int r = 0; r < P; ++r) {
                    const float(&B)[K] = Bv[n + r];
                    A[r] = lane_of(Al, n + r);
                    in[r] = lane_of(ml, n + r);
                    back[r] = lane_of(cl, n + r);
                    const float A2 = LOG2E * A[r];
                    v[r] = lane == 0 ? in[r] : 0.f;
#pragma unroll
                    for (int i = 0; i < K; ++i) {
                        dec[r][i] = exp2_of(A2 * e[i]);
                        v[r] = __builtin_fmaf(dec[r][i], v[r], x[i] * B[i]);
                    }
                    p[r] = all[r] = exp2_of(A2 * sum);
                }
                if constexpr (P == 2) scan_up(p[0], v[0], p[1], v[1]);
                else scan_up(p[0], v[0]);
#pragma unroll
                for (int r = 0; r < P; ++r) {
                    const float(&B)[K] = Bv[n + r];
                    const float(&C)[K] = Cv[n + r];
                    float w = dpp<0x138>(v[r], in[r]);      // the state in front of the lane
#pragma unroll
                    for (int i = 0; i < K; ++i) {
                        q[r][i] = dec[r][i] * w;
                        w = __builtin_fmaf(x[i], B[i], q[r][i]);
                        dCv[n + r][i] = __builtin_fmaf(f[i], w, dCv[n + r][i]);
                        if (GATED) Ch[i] = n + r ? __builtin_fmaf(C[i], w, Ch[i]) : C[i] * w;
                    }
                    v[r] = lane == 63 ? back[r] : 0.f;
#pragma unroll
                    for (int i = K - 1; i >= 0; --i) v[r] = dec[r][i] * __builtin_fmaf(C[i], f[i], v[r]);
                    p[r] = all[r];
                }
                if constexpr (P == 2) scan_down(p[0], v[0], p[1], v[1]);
                else scan_down(p[0], v[0]);
#pragma unroll
                for (int r = 0; r < P; ++r) {
                    const float(&B)[K] = Bv[n + r];
                    const float(&C)[K] = Cv[n + r];
                    float w = dpp<0x130>(v[r], back[r]);      // what the lane behind hands on
                    float s = 0.f;
#pragma unroll
                    for (int i = K - 1; i >= 0; --i) {
                        const float gt = __builtin_fmaf(C[i], f[i], w), qt = gt * q[r][i];
                        dBv[n + r][i] = __builtin_fmaf(gt, x[i], dBv[n + r][i]);
                        gB[i] = n + r ? __builtin_fmaf(gt, B[i], gB[i]) : gt * B[i];
                        Aq[i] = n + r ? __builtin_fmaf(A[r], qt, Aq[i]) : A[r] * qt;
                        s = __builtin_fmaf(e[i], qt, s);
                        w = dec[r][i] * gt;
                    }
                    dA[n + r] = s;
                    cl = with_lane(cl, n + r, lane_of(w, 0));
                }
            }
            if (lane < NS) gcar[c * row_of + s0 + wave * NS + lane] = cl;
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int i = 0; i < K; ++i) {
                    made(dBv[n][i]);
                    made(dCv[n][i]);
                }
            float4* const to = reinterpret_cast<float4*>(part + wave * 3 * SPAN);
#pragma unroll
            for (int j = 0; j < K / 4; ++j) {
                to[j * 64 + lane] = make_float4(gB[4 * j], gB[4 * j + 1], gB[4 * j + 2], gB[4 * j + 3]);
                to[SPAN / 4 + j * 64 + lane] = make_float4(Aq[4 * j], Aq[4 * j + 1], Aq[4 * j + 2], Aq[4 * j + 3]);
                if (GATED) to[SPAN / 2 + j * 64 + lane] = make_float4(Ch[4 * j], Ch[4 * j + 1], Ch[4 * j + 2], Ch[4 * j + 3]);
            }
            const Own next = lay(c + 1);
            ask(one_of(c + 2));
            __syncthreads();
            take(c + 1);      // (on its way while this head's end is made)
            float sD = 0.f, sb = 0.f;
#pragma unroll
            for (int i = 0; i < TPT; ++i) {
                const int at = place(tid * TPT + i);
                float wB = 0.f, wA = 0.f, wC = 0.f;
#pragma unroll
                for (int r = 0; r < NW; ++r) {
                    wB += part[r * 3 * SPAN + at];
                    wA += part[r * 3 * SPAN + SPAN + at];
                    if (GATED) wC += part[r * 3 * SPAN + 2 * SPAN + at];
                }
                const uint32_t t = (uint32_t)(tid * TPT + i);
                if (MANY) {      // (a thread reads here what it wrote itself)
                    float* const m = parts.more + (((size_t)b * a.H + head0 + c) * g.segs + seg) * (3 * SPAN) + t;
                    if (s0 > 0) {
                        wB += m[0];
                        wA += m[SPAN];
                        if (GATED) wC += m[2 * SPAN];
                    }
                    if (!final) {
                        m[0] = wB;
                        m[SPAN] = wA;
                        if (GATED) m[2 * SPAN] = wC;
                    }
                }
                const float dw = __builtin_fmaf(wB, own.u[i], wA) * own.rate[i];
                if ((int)t < here && final) {
                    const bool is = (int)t < lim;
                    if (d.du) put1<IO>((T*)d.du + at0, t, is ? __builtin_fmaf(own.dt[i], wB, own.D * own.dyg[i]) : 0.f);
                    if (d.ddelta) put1<IO>((T*)d.ddelta + at0, t, is ? dw : 0.f);
                    if (GATED && d.dz) put1<IO>((T*)d.dz + at0, t, is ? __builtin_fmaf(own.D, own.u[i], wC) * own.dyz[i] : 0.f);
                    if (is) {
                        sD = __builtin_fmaf(own.dyg[i], own.u[i], sD);
                        sb += dw;
                    }
                }
            }
            // lanes 0, 1: dA of the first two states; 2, 3: the shares of dD and dbias
            const float t = sums_of_wave(dA[0], dA[1], sD, sb);
            if (lane < 2 && lane < NS) add(&dAsum[c * row_of + s0 + wave * NS + lane], t);
            if (lane == 2 || lane == 3) add(&small[(wave * CB + c) * 2 + lane - 2], t);
            own = next;
        }
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            const int s = s0 + wave * NS + n;
            if (s >= S) continue;
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                float(&v)[K] = which ? dCv[n] : dBv[n];
                const int64_t t = t0 + lane * K;
                const int64_t n_here = stop - t;
#pragma unroll
                for (int i = 0; i < K; ++i) v[i] = t + i < end ? v[i] : 0.f;
                float* const f32 = which ? parts.dC : parts.dB;
                T* const io = (T*)(which ? d.dC : d.dB);
                if (f32) {
                    if (n_here > 0) store8<IoF32>(f32 + ((size_t)blk * a.B * a.G * S + bg + s) * N + t, n_here < VE ? (int)n_here : VE, v);
                } else if (io && n_here > 0) store8<IO, true>(io + (bg + s) * N + t, n_here < VE ? (int)n_here : VE, v);
            }
        }
    }
    // behind the sequence's end, from the first place that no chunk wrote
    const int64_t zero = top + SPAN > begin ? top + SPAN : begin;
    for (int c = 0; c < heads; ++c) {
        const size_t row = (size_t)b * a.H + head0 + c;
        for (int64_t t = zero + tid; t < stop; t += TH) {
            if (d.du) IO::st((T*)d.du + row * N, t, 0.f);
            if (d.ddelta) IO::st((T*)d.ddelta + row * N, t, 0.f);
            if (d.dz) IO::st((T*)d.dz + row * N, t, 0.f);
        }
    }
    if (!parts.dB)
        for (int s = 0; s < S; ++s)
            for (int64_t t = zero + tid; t < stop; t += TH) {
                if (d.dB) IO::st((T*)d.dB + (bg + s) * N, t, 0.f);
                if (d.dC) IO::st((T*)d.dC + (bg + s) * N, t, 0.f);
            }
    __syncthreads();
    for (int i = tid; i < heads * S; i += TH) {
        const int c = i / S, s = i % S;
        const size_t h = head0 + c, row = (size_t)b * a.H + h;
        parts.dA[((size_t)(b * g.segs + seg) * a.H + h) * S + s] = dAsum[c * row_of + s];
        if (d.dstate && seg == 0) d.dstate[row * S + s] = gcar[c * row_of + s];
    }
    for (int i = tid; i < heads * 2; i += TH) {
        float s = 0.f;
        for (int r = 0; r < NW; ++r) s += small[r * CB * 2 + i];
        parts.dDb[((size_t)(b * g.segs + seg) * a.H + head0) * 2 + i] = s;
    }
}

// What the workgroups left, added up.  Workgroups 0 .. joiners - 1: dB and dC from the sums of blocks of heads, 64 pieces of four places, each by four
// threads that take every fourth block; of `joins` such sets every joiners'th, as a launch holds fewer than 2^32 threads and B and C 2^33 elements.
// The others: dA, dD, dbias from the sums of sequences and segments.  (One launch: each of the two spends most of its time on the way to what other
// dies wrote.)
constexpr int64_t MOST_JOINERS = 1 << 20;
template <class IO>
__global__ __launch_bounds__(256) void scan_join_kernel(ScanArgs a, ScanGrads d, Parts parts, int blocks, int64_t joins, int64_t joiners, int64_t shares)
{
    using T = typename IO::T;
    if ((int64_t)blockIdx.x < joiners) {
        __shared__ float4 lds[3][64];
        const int64_t P = (a.N + 3) / 4, rows = a.B * a.G * a.S;
        const int lane = threadIdx.x & 63, quarter = threadIdx.x >> 6;
        for (int64_t set = blockIdx.x; set < joins; set += joiners) {
            int64_t id = set * 64 + lane;
            const bool is = id < 2 * rows * P, second = id >= rows * P;
            if (second) id -= rows * P;
            if (!is) id = 0;
            const int64_t row = id / P, t = (id - row * P) * 4, len = scan_length(a, row / (a.G * a.S));
            const float* from = (second ? parts.dC : parts.dB) + row * a.N + t;
            const int n = a.N - t < 4 ? (int)(a.N - t) : 4;
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            if (t < len && n == 4) {
#pragma unroll 8
                for (int q = quarter; q < blocks; q += 4) {
                    const At4 w = *reinterpret_cast<const At4*>(from + (size_t)q * rows * a.N);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] += __uint_as_float(w[i]);
                }
            } else if (t < len)
                for (int q = quarter; q < blocks; q += 4)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i < n) v[i] += from[(size_t)q * rows * a.N + i];
            if (set != blockIdx.x) __syncthreads();      // (the set before is read)
            if (quarter) lds[quarter - 1][lane] = make_float4(v[0], v[1], v[2], v[3]);
            __syncthreads();
            T* const to = (T*)(second ? d.dC : d.dB);
            if (quarter || !is || !to) continue;
#pragma unroll
            for (int r = 0; r < 3; ++r) {
                const float4 w = lds[r][lane];
                v[0] += w.x;
                v[1] += w.y;
                v[2] += w.z;
                v[3] += w.w;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (i < n) put1<IO>(to + row * a.N + t, i, t + i < len ? v[i] : 0.f);
        }
        return;
    }
    const int64_t id = ((int64_t)blockIdx.x - joiners) * 256 + threadIdx.x, in_A = a.H * a.S;
    if (id >= in_A + 2 * a.H) return;
    const int64_t i = id - in_A, each = id < in_A ? in_A : 2 * a.H;
    const float* const from = id < in_A ? parts.dA + id : parts.dDb + i;
    float* const to = id < in_A ? d.dA : i & 1 ? d.dbias : d.dD;
    if (!to) return;
    float s = 0.f;
#pragma unroll 8
    for (int64_t q = 0; q < shares; ++q) s += from[q * each];
    to[id < in_A ? id : i >> 1] = s;
}

// Heads of a workgroup: as many as leave 256 workgroups, counting the segments that a sequence is cut into, 32 at most.  us with 8, 16, 32 at 16 states,
// gated, bf16: 16 x 1024 x 1024 480, 392, 357 (taken); 4 x 1024 x 1024 117, 103 (taken), 175; 4 x 1024 x 4096 470, 388 (taken), 675; 1 x 1024 x 16384 in four
// segments 548, 474 (taken), 762; 2 x 256 x 2048 in two 75 (taken), 112, 189; 2 x 1024 x 8192 466 (taken), 725, 1323; 8 x 256 x 16384 955 (taken), 1453, 2634.
int block_heads(int64_t B, int64_t H, int64_t G, int segs)
{
    int CB = 32;
    while (CB > 8 && B * G * ((H / G + CB - 1) / CB) * segs < 256) CB /= 2;
    return CB;
}

template <class IO, int NS, int NW, bool GATED, bool MANY>
hipError_t launch_of(const ScanArgs& a, const ScanGrads& d, const Segments& g, const Parts& parts, int blocks, int CB, hipStream_t st)
{
    dim3 grid;
    hipError_t e = launch_grid((uint64_t)(a.B * a.G * blocks * g.segs), 64 * NW, &grid);
    if (e != hipSuccess) return e;
    const size_t row_of = MANY ? (a.S + NS * NW - 1) / (NS * NW) * (NS * NW) : NS * NW;
    const size_t bytes = (2 * (3 + 3 * NW) * SPAN + 2 * CB * row_of + 2 * NW * CB) * sizeof(float);
    if (bytes > 65536) {
        e = hipFuncSetAttribute(reinterpret_cast<const void*>(&scan_bwd_kernel<IO, NS, NW, GATED, MANY>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((scan_bwd_kernel<IO, NS, NW, GATED, MANY>), grid, dim3(64 * NW), bytes, st, a, d, g, parts, blocks, CB);
    return hipGetLastError();
}

template <class IO, int NS, int NW, bool MANY = false>
hipError_t launch(const ScanArgs& a, const ScanGrads& d, const Segments& g, const Parts& parts, int blocks, int CB, hipStream_t st)
{
    return a.z ? launch_of<IO, NS, NW, true, MANY>(a, d, g, parts, blocks, CB, st) : launch_of<IO, NS, NW, false, MANY>(a, d, g, parts, blocks, CB, st);
}

template <class IO>
hipError_t run(const ScanArgs& a, const ScanGrads& d, void* ws, hipStream_t st)
{
    Segments g;
    hipError_t e = scan_back(a, d.dy, ws, &g, st);
    if (e != hipSuccess) return e;
    const int CB = block_heads(a.B, a.H, a.G, g.segs), blocks = (int)((a.H / a.G + CB - 1) / CB);
    const size_t rows = (size_t)a.B * a.G * a.S;
    Parts parts;
    char* p = (char*)ws + scan_segment_bytes(a.B, a.H, a.N, a.S, a.G);
    parts.dA = (float*)p;
    p += up256((size_t)a.B * g.segs * a.H * a.S * sizeof(float));
    parts.dDb = (float*)p;
    p += up256((size_t)a.B * g.segs * a.H * 2 * sizeof(float));
    parts.more = (float*)p;
    if (a.S > GROUP) p += up256((size_t)a.B * g.segs * a.H * 3 * SPAN * sizeof(float));
    parts.dB = parts.dC = nullptr;
    if (blocks > 1) {
        parts.dB = (float*)p;
        parts.dC = parts.dB + blocks * rows * a.N;
    }
    if (a.S <= 4) e = launch<IO, 1, 4>(a, d, g, parts, blocks, CB, st);
    else if (a.S <= 8) e = launch<IO, 2, 4>(a, d, g, parts, blocks, CB, st);
    else if (a.S <= 16) e = launch<IO, 2, 8>(a, d, g, parts, blocks, CB, st);
    else e = launch<IO, 2, 8, true>(a, d, g, parts, blocks, CB, st);
    if (e != hipSuccess) return e;
    const int64_t joins = blocks > 1 && (d.dB || d.dC) ? (int64_t)(2 * rows * ((a.N + 3) / 4) + 63) / 64 : 0;
    const int64_t joiners = joins < MOST_JOINERS ? joins : MOST_JOINERS, others = d.dA || d.dD || d.dbias ? (a.H * (a.S + 2) + 255) / 256 : 0;
    if (joiners + others == 0) return hipSuccess;
    dim3 grid;
    e = launch_grid((uint64_t)(joiners + others), 256, &grid);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(scan_join_kernel<IO>, grid, dim3(256), 0, st, a, d, parts, blocks, joins, joiners, (int64_t)a.B * g.segs);
    return hipGetLastError();
}

}  // namespace

size_t scan_bwd_bytes(int64_t B, int64_t H, int64_t N, int S, int64_t G)
{
    // the most of any batch up to B.  Sequences times segments: as scan_segment_bytes says, with 512 workgroups at most where there are
    // several segments.  Blocks: of 32 heads, or of 8 as long as those of twice as many are fewer than 256 workgroups.
    const int64_t all = B * ((N + 1023) / 1024), some = 513 + (B < 256 ? B : 256), shares = all < some || B > some ? (all < some ? all : B) : some;
    const int64_t in_group = H / G, narrow = B * G * ((in_group + 7) / 8), wide = B * G * ((in_group + 31) / 32);
    const int64_t blocks = narrow < 512 ? narrow : wide < 512 ? 512 : wide;
    return up256((size_t)shares * H * S * sizeof(float)) + (S > GROUP ? up256((size_t)shares * H * 3 * SPAN * sizeof(float)) : 0) + up256((size_t)shares * H * 2 * sizeof(float)) +
           (in_group > 8 ? up256((size_t)blocks * S * N * 2 * sizeof(float)) : 0);
}

hipError_t scan_bwd(const ScanArgs& a, const ScanGrads& d, void* ws, hipStream_t st)
{
    if (a.io == LONGCONV_F32) return run<IoF32>(a, d, ws, st);
    return a.io == LONGCONV_F16 ? run<IoF16>(a, d, ws, st) : run<IoBF16>(a, d, ws, st);
}

}  // namespace lc
