// Host build of the library (lock-step emulation): csrc/policy.hip.
#define TT_HOST_EMULATION 1
#include "policy.hip"
