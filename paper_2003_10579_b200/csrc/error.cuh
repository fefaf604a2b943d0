// Message of the last failure of a call without a simulation handle on this thread (sim_last_error(NULL)).
#pragma once
#include "../../include/straggler_sim.h"

namespace ssim {

// Never throws: a message that cannot be stored is dropped.  Returns `st`.
sim_status record_error(sim_status st, const char* msg) noexcept;

}  // namespace ssim
