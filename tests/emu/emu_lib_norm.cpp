// Host build of the library (lock-step emulation): csrc/norm.hip.
#define TT_HOST_EMULATION 1
#include "norm.hip"
