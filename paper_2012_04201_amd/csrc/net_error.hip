// The message of a thread's last failed call.
#include <stdio.h>

#include "net_common.h"

static thread_local char message[256];

int net_fail(int code, const char* msg) {
  snprintf(message, sizeof message, "%s", msg);
  return code;
}
int net_launched(void) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? (int)BBO_OK : net_fail(BBO_DEVICE_ERROR, hipGetErrorString(e));
}
void net_begin(void) { message[0] = 0; }

extern "C" const char* bbo_net_last_error(void) { return message; }
