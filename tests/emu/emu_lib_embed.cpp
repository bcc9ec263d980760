// Host build of the library (lock-step emulation): csrc/embed.hip.
#define TT_HOST_EMULATION 1
#include "embed.hip"
