#include "st_entropy_impl.h"

namespace st {
ST_ENTROPY(double)
}  // namespace st
