// Group norm of fp16 rows (gnorm.hpp)
#include "gnorm.hpp"

namespace lc {
GNORM_IO(IoF16);
}  // namespace lc
