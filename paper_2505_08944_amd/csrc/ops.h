// Host side of the routing rule, shared by the calls with and without queues.
#pragma once

#include "aep.h"
#include "aep_internal.h"

namespace aep {

// AEP_OK, or why the router is refused.
aep_status check_router(const aep_router* r);
RouterArgs router_args(const aep_router& r);

}  // namespace aep
