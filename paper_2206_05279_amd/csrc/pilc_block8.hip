// libpilc, third part: what lies between a network's last states and its logits, in 8 bits: matrices under scales and the norm that
// answers in them.  Kernels and entry points are in the two headers below.
#include <hip/hip_runtime.h>

#include "pilc_block8_host.hpp"

#include "pilc_block8.hpp"
#include "pilc_rms.hpp"
