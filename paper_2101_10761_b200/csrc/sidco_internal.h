// Shared by the translation units of the library; not part of the C ABI.
#pragma once

#include <cuda.h>
#include <stdint.h>

namespace sidco_internal {

// Count one kernel launch towards sidco_launch_count().
void note_launch();

// Tensor map over `rows` rows of `width` bytes, `pitch` bytes apart; boxes of box_width bytes (with or without the 128-byte
// swizzle) x box_rows rows, zeros outside.  False if the driver has no such call or refuses the arguments.
bool byte_map(CUtensorMap* map, const void* base, int64_t width, int64_t rows, int64_t pitch, int box_width, int box_rows,
              bool swizzle);

// Tensor map for stores into a matrix of SIDCO_T_* elements: boxes of 128 bytes x box_rows rows with the 128-byte swizzle.
bool out_map(CUtensorMap* map, void* base, int type, int64_t width, int64_t rows, int64_t pitch, int box_width, int box_rows);

// How many CTAs of the product kernels gave up a bounded wait on the current device (synchronises it).
int orthogonalize_timeouts(int* count);
int mx4_matmul_timeouts(int* count);

}  // namespace sidco_internal
