// What the host sides of the library share.
#pragma once

namespace specv {

// a kernel has been enqueued (spec_kernel_launches)
__attribute__((visibility("hidden"))) void count_launch();

// spec_test_hooks for the other sources' kernels (each source has its own copy of the constants), on the current device
__attribute__((visibility("hidden"))) int set_step_hooks(long long cycles, int hold);
__attribute__((visibility("hidden"))) int set_serve_hooks(long long cycles, int hold);
__attribute__((visibility("hidden"))) int set_prefix_hooks(long long cycles, int hold);

}  // namespace specv
