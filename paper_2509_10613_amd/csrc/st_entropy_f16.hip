#include "st_entropy_impl.h"

namespace st {
ST_ENTROPY(f16)
}  // namespace st
