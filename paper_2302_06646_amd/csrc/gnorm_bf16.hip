// Group norm of bf16 rows (gnorm.hpp)
#include "gnorm.hpp"

namespace lc {
GNORM_IO(IoBF16);
}  // namespace lc
