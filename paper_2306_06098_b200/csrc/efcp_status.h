// The device's sticky status of the calls without a handle: EFCP_ETIMEOUT once a wait inside one of their kernels
// has run out.
#pragma once

namespace efcp {

// Its address on the current device, null when there is none.
int* device_status();

}  // namespace efcp
