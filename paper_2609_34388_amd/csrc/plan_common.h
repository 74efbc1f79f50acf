// Host helpers shared by the API files: argument checks and planning rules
// (defined in api.cpp).
#pragma once

#include <cstdint>

#include "recguide.h"
#include "rg_internal.h"

namespace rg {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int64_t round_up(int64_t x, int64_t m) { return (x + m - 1) / m * m; }

// Whether a grid of this many work groups, rounded up to 8, is one launch.
inline bool fits_launch(int64_t groups, int threads) { return round_up(groups, 8) * threads <= kMaxLaunchThreads; }

rg_status validate_layout(const rg_attn_layout* L);
rg_status validate_branches(const rg_attn_layout* L, const rg_branch_layout* B);
bool pack_branches(const rg_branch_layout* B, int r, int32_t (&w)[3], int32_t& rep);

int device_cus();

}  // namespace rg
