// libpilc, fourth part: the product of matrices in 8 bits.
#include <hip/hip_runtime.h>

#include "pilc_block8_host.hpp"

#include "pilc_product.hpp"
