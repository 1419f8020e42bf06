// What the host sides of the library share.
#pragma once

namespace specv {

// a kernel has been enqueued (spec_kernel_launches)
__attribute__((visibility("hidden"))) void count_launch();

}  // namespace specv
