// Launch interfaces of the operators around the convolution: dropout (dropout.hip, kreg.hip), embedding (embed.hip), group norm
// (gnorm.hip), and beside it: short convolution (short.hip), selective scan (scan.hip), dense product (linear.hip).  Arguments are checked by the C-ABI layer.
#pragma once
#include "engines.hpp"

namespace lc {

constexpr int64_t MAX_ELEMENTS = int64_t(1) << 34;      // of one tensor: what one launch covers

// A dropout mask that is never stored (generator: vec8.hpp)
struct Drop {
    uint32_t threshold;      // an entry is kept if its 16 bits are at least this; 0: all are kept, 65536: none
    float scale;             // of the kept entries: 65536 / (65536 - threshold), 0 if none are
    uint64_t seed, call;
    const int64_t* step;     // added to `call` on the device (graphs that replay with another mask each time); may be null
};

// 0 <= p <= 1, checked by the caller
inline Drop make_drop(float p, uint64_t seed, uint64_t call, const int64_t* step)
{
    Drop d;
    d.threshold = (uint32_t)((double)p * 65536.0 + 0.5);
    d.scale = d.threshold >= 65536u ? 0.f : (float)(65536.0 / (double)(65536u - d.threshold));
    d.seed = seed;
    d.call = call;
    d.step = step;
    return d;
}

hipError_t dropout(const void* x, const void* residual, void* y, int64_t n, int64_t tie, int io, const Drop& d, hipStream_t st);
hipError_t kreg_fwd_seeded(const float* k, float* kbar, int64_t H, int64_t N, int p, float lam, const Drop& drop, hipStream_t st);
hipError_t kreg_bwd_seeded(const float* k, const float* dkbar, float* dk, int64_t H, int64_t N, int p, float lam, const Drop& drop,
                           hipStream_t st);

struct EmbedArgs {
    const void* ids;
    int id_bytes;            // 4 or 8
    int64_t B, N, V, H;
    int io, layout;          // longconv_dtype_t of y and dy; longconv_layout_t
    float scale;
    Drop drop;
};
hipError_t embed_fwd(const EmbedArgs& a, const void* E, int table, void* y, hipStream_t st);
size_t embed_workspace_bytes(int64_t B, int64_t N, int64_t V, int64_t H, int io, int layout);
hipError_t embed_bwd(const EmbedArgs& a, const void* dy, float* dE, void* ws, hipStream_t st);
// The gradient of a table of few rows on the matrix cores (embed_small.hip), whatever their number: us of kernels, and of those of the
// sorted way, dropout 0.1: 8 x 16384 x 256 with V = 256 44 and 58, 64 43 and 58, 5 42 and 69; 1024 tokens x 64, V = 256 17 and 19; 128 x 64
// 11 and 14.  (A step takes eight places at a time: N >= 8.)
constexpr int SMALL_TABLE = 256;
inline bool embed_is_small(int64_t N, int64_t V, int io, int layout)
{
    return V <= SMALL_TABLE && N >= 8 && io != LONGCONV_F32 && layout == LONGCONV_CHANNELS_FIRST;
}
size_t embed_small_workspace_bytes(int64_t B, int64_t N, int64_t H);
hipError_t embed_small_bwd(const EmbedArgs& a, const void* dy, float* dE, void* ws, hipStream_t st);

struct GnormArgs {
    const float *gamma, *beta;      // may be null: ones, zeros
    int64_t B, S, C, G;
    int io, act;                    // longconv_dtype_t, longconv_act_t
};
size_t gnorm_workspace_bytes(int64_t B, int64_t S, int64_t C, int64_t G, int io, int backward);
hipError_t gnorm_fwd(const GnormArgs& a, const void* x, void* y, float* mean, float* rstd, float eps, void* ws, hipStream_t st);
hipError_t gnorm_bwd(const GnormArgs& a, const void* dy, const void* x, const float* mean, const float* rstd, void* dx, float* dgamma,
                     float* dbeta, void* ws, hipStream_t st);

// ---- operators beside the convolution ----------------------------------------------------------------------------------

// Short causal convolution (short.hip)
constexpr int SHORT_TAPS = 8;      // at most
struct ShortArgs {
    const float *k, *bias;          // [H,taps], [H] or null
    const int64_t* lengths;         // [B] on the device, or null: all N
    int64_t B, H, N;
    int taps, act, io;
};
struct ShortGrads {                 // state, dlast may be null, and so may any result
    const void *dy, *x, *state, *dlast;
    void *dx, *dstate;
    float *dk, *dbias;
};
size_t short_workspace_bytes(int64_t B, int64_t H, int64_t N);
hipError_t short_fwd(const ShortArgs& a, const void* x, const void* state, void* y, void* last, hipStream_t st);
hipError_t short_bwd(const ShortArgs& a, const ShortGrads& d, void* ws, hipStream_t st);
hipError_t short_step(const ShortArgs& a, const void* x, void* state, void* y, hipStream_t st);

// Selective state space scan (scan.hip, scan_bwd.hip)
constexpr int SCAN_STATES = 64;      // at most
struct ScanArgs {
    const void *u, *delta, *Bm, *Cm, *z;      // z may be null
    const float *A, *D, *bias;                // [H,S], [H] or null, [H] or null
    const int64_t* lengths;                   // [B] on the device, or null: all N
    int64_t B, H, N, G;
    int S, softplus, io;
};
struct ScanGrads {                            // dlast may be null, and so may any result
    const void* dy;
    const float *marks, *dlast;
    void *du, *ddelta, *dB, *dC, *dz;
    float *dA, *dD, *dbias, *dstate;
};
size_t scan_workspace_bytes(int64_t B, int64_t H, int64_t N, int S, int64_t G, int backward);
hipError_t scan_fwd(const ScanArgs& a, const float* state, void* y, float* last, float* marks, void* ws, hipStream_t st);
hipError_t scan_bwd(const ScanArgs& a, const ScanGrads& d, void* ws, hipStream_t st);
hipError_t scan_step(const ScanArgs& a, float* state, void* y, hipStream_t st);

// Dense product (linear.hip, linear.hpp)
struct LinearArgs {
    const void* W;                            // [M,K] in the I/O type
    const float* bias;                        // [M] or null
    int64_t B, N, K, M;
    int act, io;
    bool x_first, y_first;                    // [B,.,N], else [B,N,.]
};
struct LinearGrads {                          // any result may be null
    const void *dy, *x;
    void *dx, *dW;
    float* dbias;
    bool dW_f32;                              // dW is float32, not the I/O type
};
size_t linear_workspace_bytes(int64_t B, int64_t N, int64_t K, int64_t M, int io, int backward);
hipError_t linear_fwd(const LinearArgs& a, const void* x, const void* residual, void* y, void* ws, hipStream_t st);
hipError_t linear_bwd(const LinearArgs& a, const LinearGrads& d, void* ws, hipStream_t st);

}  // namespace lc
