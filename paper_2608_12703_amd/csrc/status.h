// Errors of the C-ABI, shared by the files that define entry points.
#pragma once

#include <string>

#include "../../include/ad.h"

namespace ad {

// Records the text that ad_last_error() returns on this thread, and returns s.
ad_status fail(ad_status s, const std::string& msg);
// AD_EHIP with the runtime's text when a launch since the last check failed.
ad_status check_hip(const char* where);

}  // namespace ad
