// Group norm: the C-ABI layer's entry points, and the kernels (gnorm.hpp) of fp32 rows.  Those of fp16 and bf16 rows are compiled beside
// it, in files of their own.
#include "gnorm.hpp"

namespace lc {

extern template hipError_t gnorm_fwd_io<IoF16>(const GnormArgs&, const void*, void*, float*, float*, float, void*, hipStream_t);
extern template hipError_t gnorm_fwd_io<IoBF16>(const GnormArgs&, const void*, void*, float*, float*, float, void*, hipStream_t);
extern template hipError_t gnorm_bwd_io<IoF16>(const GnormArgs&, const void*, const void*, const float*, const float*, void*, float*, float*, void*,
                                               hipStream_t);
extern template hipError_t gnorm_bwd_io<IoBF16>(const GnormArgs&, const void*, const void*, const float*, const float*, void*, float*, float*, void*,
                                                hipStream_t);

size_t gnorm_workspace_bytes(int64_t B, int64_t S, int64_t C, int64_t G, int io, int backward)
{
    return up256(part_rows(B, S, C) * 2 * C * sizeof(float)) + (backward ? up256((size_t)B * G * 2 * sizeof(float)) : 0);
}

hipError_t gnorm_fwd(const GnormArgs& a, const void* x, void* y, float* mean, float* rstd, float eps, void* ws, hipStream_t st)
{
    if (a.io == LONGCONV_F32) return gnorm_fwd_io<IoF32>(a, x, y, mean, rstd, eps, ws, st);
    return a.io == LONGCONV_F16 ? gnorm_fwd_io<IoF16>(a, x, y, mean, rstd, eps, ws, st)
                                : gnorm_fwd_io<IoBF16>(a, x, y, mean, rstd, eps, ws, st);
}

hipError_t gnorm_bwd(const GnormArgs& a, const void* dy, const void* x, const float* mean, const float* rstd, void* dx, float* dgamma,
                     float* dbeta, void* ws, hipStream_t st)
{
    if (a.io == LONGCONV_F32) return gnorm_bwd_io<IoF32>(a, dy, x, mean, rstd, dx, dgamma, dbeta, ws, st);
    return a.io == LONGCONV_F16 ? gnorm_bwd_io<IoF16>(a, dy, x, mean, rstd, dx, dgamma, dbeta, ws, st)
                                : gnorm_bwd_io<IoBF16>(a, dy, x, mean, rstd, dx, dgamma, dbeta, ws, st);
}

}  // namespace lc
