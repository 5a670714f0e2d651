// What train_kernel_stubs.cpp keeps of the last launches.
#pragma once

#include "pf_internal.h"

namespace pf {
extern GatedBwdArgs g_gated;
extern ActBwdArgs g_dbias;
extern NormArgs g_norm;
extern int g_launches, g_sums;
}  // namespace pf
