// The message behind sigkernel_last_error(), for entry points outside sk_api.hip.
#pragma once

namespace sk {

// Keeps `message` for sigkernel_last_error() on this thread and returns `code`.
int set_error(int code, const char* message);

}  // namespace sk
