// Status words of several blocks, or of several launches of a call, as one.
#pragma once

#ifdef __CUDACC__
#define VPP_HOST_DEVICE __host__ __device__
#else
#define VPP_HOST_DEVICE
#endif

namespace vpp {
// Of two status words (VPP_DEV_*) the one that says more about the results: after a timeout (3) they are undefined, with a bad page (2) those that
// read it, and bad lengths (1) are seen by every block, so that no other word stands beside them.
VPP_HOST_DEVICE inline int worse_status(int a, int b) { return a > b ? a : b; }
}  // namespace vpp
