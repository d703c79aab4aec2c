// What the operators on weights with group scales share on the host.  Internal to the library.
#pragma once

#include "dsq_launch.h"

// longest row of codes (a row of 2^20 bf16 activations is 2 MB)
constexpr int64_t DSQ_GROUPS_MAX_K = 1 << 20;

// bits, shape and group of codes with group scales: DSQ_OK or the status of the call
DSQ_HIDDEN int dsq_check_groups(int64_t N, int64_t K, int bits, int64_t group);
