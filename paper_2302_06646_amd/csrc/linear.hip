// The dense product: the C-ABI layer's entry points, and the kernels (linear.hpp) of fp32 rows.  Those of fp16 and bf16 rows are compiled
// beside it, in files of their own.
#include "linear.hpp"

namespace lc {

extern template size_t linear_workspace_of<IoF16>(int64_t, int64_t, int64_t, int64_t, int);
extern template size_t linear_workspace_of<IoBF16>(int64_t, int64_t, int64_t, int64_t, int);
extern template hipError_t linear_fwd_of<IoF16>(const LinearArgs&, const void*, const void*, void*, void*, hipStream_t);
extern template hipError_t linear_fwd_of<IoBF16>(const LinearArgs&, const void*, const void*, void*, void*, hipStream_t);
extern template hipError_t linear_bwd_of<IoF16>(const LinearArgs&, const LinearGrads&, void*, hipStream_t);
extern template hipError_t linear_bwd_of<IoBF16>(const LinearArgs&, const LinearGrads&, void*, hipStream_t);

size_t linear_workspace_bytes(int64_t B, int64_t N, int64_t K, int64_t M, int io, int backward)
{
    if (io == LONGCONV_F32) return linear_workspace_of<IoF32>(B, N, K, M, backward);
    return io == LONGCONV_F16 ? linear_workspace_of<IoF16>(B, N, K, M, backward) : linear_workspace_of<IoBF16>(B, N, K, M, backward);
}
hipError_t linear_fwd(const LinearArgs& a, const void* x, const void* residual, void* y, void* ws, hipStream_t st)
{
    if (a.io == LONGCONV_F32) return linear_fwd_of<IoF32>(a, x, residual, y, ws, st);
    return a.io == LONGCONV_F16 ? linear_fwd_of<IoF16>(a, x, residual, y, ws, st) : linear_fwd_of<IoBF16>(a, x, residual, y, ws, st);
}
hipError_t linear_bwd(const LinearArgs& a, const LinearGrads& d, void* ws, hipStream_t st)
{
    if (a.io == LONGCONV_F32) return linear_bwd_of<IoF32>(a, d, ws, st);
    return a.io == LONGCONV_F16 ? linear_bwd_of<IoF16>(a, d, ws, st) : linear_bwd_of<IoBF16>(a, d, ws, st);
}

}  // namespace lc
