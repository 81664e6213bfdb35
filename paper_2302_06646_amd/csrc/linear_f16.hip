#include "linear.hpp"

namespace lc {
template size_t linear_workspace_of<IoF16>(int64_t, int64_t, int64_t, int64_t, int);
template hipError_t linear_fwd_of<IoF16>(const LinearArgs&, const void*, const void*, void*, void*, hipStream_t);
template hipError_t linear_bwd_of<IoF16>(const LinearArgs&, const LinearGrads&, void*, hipStream_t);
}  // namespace lc
