// What the operators of include/razer_step.h share on the host side (internal to the library).
#pragma once
#include "razer_kernels.hpp"
#include "../../include/razer_step.h"

namespace razer {

razer_status check_cfg(const razer_config& c, SvConfig& out);     // razer_api.hip

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

}  // namespace razer
