// What block_kernel_stubs.cpp keeps of the last launch.
#pragma once

#include "pf_internal.h"

namespace pf {
extern ActBwdArgs g_act;
extern int g_act_launches, g_dbias_launches;
}  // namespace pf
