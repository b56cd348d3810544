// Which bit of mf_ctx::kernels_configured says that a kernel's limit of dynamic LDS has been raised.  The bits of all kernels stand here, so that no
// two share one.
#pragma once

constexpr unsigned long long lds_bit(int number) { return 1ull << number; }

// score.hip, pair_mlp_kernel: 0 .. 15
constexpr unsigned long long lds_bit_pair(int H, bool sm, bool slowdown, bool split) { return lds_bit((H == 128 ? 8 : 0) + (sm ? 4 : 0) + (slowdown ? 2 : 0) + (split ? 1 : 0)); }
// small.hip, small_kernel, of 1, 2, 4 or 8 columns a lane: 16 .. 19
constexpr unsigned long long lds_bit_small(int columns) { return lds_bit(16 + (columns == 1 ? 0 : columns == 2 ? 1 : columns == 4 ? 2 : 3)); }
// fit_wide.hip, wide_kernel: 20 .. 23
constexpr unsigned long long lds_bit_wide(int H, bool grad) { return lds_bit(20 + (H == 128 ? 2 : 0) + (grad ? 1 : 0)); }
// fit.hip, fit_kernel, of 1 .. 4 tiles of columns: 32 .. 63
constexpr unsigned long long lds_bit_fit(int H, int tiles, bool grad, bool extra) { return lds_bit(32 + (H == 128 ? 16 : 0) + (grad ? 8 : 0) + (extra ? 4 : 0) + tiles - 1); }
