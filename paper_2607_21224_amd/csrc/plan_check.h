// Whether a multi-tensor plan's handle may be used for a call: filled by
// cpdp_plan_build or cpdp_plan_build_static and unchanged since (a cpdp_status).
#pragma once

#include "cpdp.h"

namespace cpdp {

int check_plan_handle(const cpdp_plan* plan);

}  // namespace cpdp
