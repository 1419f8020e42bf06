// What the host sides of the library share.
#pragma once

namespace specv {

// a kernel has been enqueued (spec_kernel_launches)
__attribute__((visibility("hidden"))) void count_launch();

// the limit of the waits in step.cu's kernels (each source has its own copy of the constant), on the current device
__attribute__((visibility("hidden"))) int set_step_wait(long long cycles);

}  // namespace specv
