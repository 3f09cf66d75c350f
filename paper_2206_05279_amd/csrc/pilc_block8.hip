// libpilc, third part: what lies between a network's last states and its logits, in 8 bits.  Kernels and entry points are in the
// three headers below.
#include <hip/hip_runtime.h>

#include "pilc_block8_device.hpp"
#include "pilc_fit_host.hpp"

#include "pilc_block8.hpp"
#include "pilc_rms.hpp"
#include "pilc_product.hpp"
