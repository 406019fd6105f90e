// Shared by the translation units of the library; not part of the C ABI.
#pragma once

namespace sidco_internal {

// Count one kernel launch towards sidco_launch_count().
void note_launch();

// How many CTAs of the product kernels gave up a bounded wait on the current device (synchronises it).
int orthogonalize_timeouts(int* count);
int mx4_matmul_timeouts(int* count);

}  // namespace sidco_internal
