// The library's error state: hvd_last_error() returns the last message.
#pragma once

#include <string>

#include "../../include/hvd.h"

namespace hvd {

// Records the message for this thread and returns s.
hvd_status set_err(hvd_status s, const std::string& m);

}  // namespace hvd
