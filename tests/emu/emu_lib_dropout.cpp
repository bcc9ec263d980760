// Host build of the library (lock-step emulation): csrc/dropout.hip.
#define TT_HOST_EMULATION 1
#include "dropout.hip"
