// Host build of the library (lock-step emulation): csrc/rows8.hip.
#define TT_HOST_EMULATION 1
#include "rows8.hip"
