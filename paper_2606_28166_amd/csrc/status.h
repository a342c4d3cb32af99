// Error reporting shared by the C entry points (internal to libtandem).
#pragma once

#include "tandem.h"

namespace tandem {

// Records msg as this thread's last handle-less failure and returns s.
tandem_status report(tandem_status s, const char* msg) noexcept;

}  // namespace tandem
