// Error reporting shared by the C entry points (lionmuon_last_error).
#pragma once

#include <string>

#include "lionmuon.h"

namespace lm {

lm_status set_error(lm_status st, const std::string& msg);
// Compute units of the current device (a full MI355X when there is none).
int current_cus();

}  // namespace lm
