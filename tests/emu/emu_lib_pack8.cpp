// Host build of the library (lock-step emulation): csrc/pack8.hip.
#define TT_HOST_EMULATION 1
#include "pack8.hip"
