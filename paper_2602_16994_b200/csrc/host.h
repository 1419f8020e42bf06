// What the host sides of the library share.
#pragma once

namespace specv {

// a kernel has been enqueued (spec_kernel_launches)
__attribute__((visibility("hidden"))) void count_launch();

// spec_test_hooks for step.cu's kernels (each source has its own copy of the constants), on the current device
__attribute__((visibility("hidden"))) int set_step_hooks(long long cycles, int hold);

}  // namespace specv
