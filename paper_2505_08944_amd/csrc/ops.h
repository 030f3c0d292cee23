// Host side of the calls that need no context: what they share, and the routing rule,
// which the calls with queues share too.
#pragma once

#include "aep.h"
#include "aep_internal.h"

namespace aep {

// AEP_OK, or why the router is refused.
aep_status check_router(const aep_router* r);
RouterArgs router_args(const aep_router& r);

// What the kernels of a dense product take; of w, its alignment and type count here.
LinearArgs linear_args(const aep_linear_desc& l, const void* x, const void* w, const void* scale, const void* bias,
                       const void* residual, void* y);

// One workgroup per CU of the current device, a multiple of the 8 XCDs.
int persistent_workgroups();
// Whether p is not a multiple of a (a power of two).
inline bool off(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

}  // namespace aep
