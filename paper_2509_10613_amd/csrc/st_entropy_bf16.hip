#include "st_entropy_impl.h"

namespace st {
ST_ENTROPY(bf16)
}  // namespace st
