// api.h -- what the C ABI's translation units share: error reporting and the
// device query.
#pragma once
#include <hip/hip_runtime.h>

#include <string>

namespace dash {
namespace api {

// sets dash_last_error and returns code
int fail(int code, const std::string& msg);
int hip_fail(hipError_t e, const char* what);

struct DeviceInfo {
  int device = -1;
  int cus = 0;
  int occ64 = 0, occ128 = 0, occ256 = 0;
  bool probed = false;  // nxcd is known (the probe allocates, so it runs only when XCD placement is asked for)
  int nxcd = 0;  // XCDs, when workgroup i runs on XCD i % nxcd (0: not usable for XCD-local placement)
};
// The current device's properties (queried once per device).  With xcd, also
// whether XCD-local placement is usable: that probe runs a kernel on a small
// buffer it allocates, so only calls that ask for XCD placement run it.
int device_info(DeviceInfo* out, bool xcd = false);

// One lane stores 0 into the words that are not null, on `stream`.
int clear_flags(int* flag, int* status, void* stream);

}  // namespace api
}  // namespace dash
