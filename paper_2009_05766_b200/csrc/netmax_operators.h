// What a context's round takes from the operators on real weights (netmax_operators.cu).
#pragma once
#include <cstdint>

#include "../../include/netmax.h"

namespace netmax {
// Both record the message that netmax_last_error(NULL) returns.
int check_step(const netmax_step& step);
// On the current device.  peers and weights: entry draw_stride * i is worker i's.  error: the word that a wait which runs out raises
// (NULL: the workspace's); launches: counted up.
int enqueue_step(const netmax_step& step, int draw_stride, unsigned int* error, int64_t* launches);
}  // namespace netmax
