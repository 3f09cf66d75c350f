// libpilc, second part: the operators of a program that learns the laws the coder works under.  Their
// kernels and entry points are in the three headers below.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "pilc_fit_device.hpp"
#include "pilc_host.hpp"
#include "pilc_row_rules.hpp"

#include "pilc_logprobs.hpp"
#include "pilc_norm.hpp"
#include "pilc_adamw.hpp"
