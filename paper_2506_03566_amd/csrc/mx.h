// Microscaled 4-bit weights: the packed form and its launches (mx.hip), shared by the entry points.
#pragma once
#include "common.h"

namespace poss {

// Packed weights as the kernels see them (the layout stands in mx.hip).
struct MxPacked { const u32x4 *codes; const uint32_t *scales; const int32_t *ref; int ksteps, kgroups, tiles; };
MxPacked mx_packed_at(const void *packed, int N, int K);

// Leaves the message that poss_last_error(NULL) returns; the code is handed through.
int set_error(int code, const char *fmt, ...);

}  // namespace poss
