// Test infrastructure: record_launches.cpp with the limits that the HIP runtime has for a launch.  Where one is passed the launch is refused, as the runtime would.
#define hipLaunchKernel record_launch
#include "record_launches.cpp"
#undef hipLaunchKernel

extern "C" {

static uint64_t refused = 0;

int hipLaunchKernel(const void* host, Size grid, Size block, void** args, size_t shared, void* stream)
{
    const uint64_t threads = (uint64_t)grid.x * block.x;
    if (threads == 0 || threads >= ((uint64_t)1 << 32) || grid.y == 0 || grid.y > 65535 || grid.z != 1 || block.y != 1 || block.z != 1 || block.x > 1024) {
        ++refused;
        return 9;  // hipErrorInvalidConfiguration
    }
    return record_launch(host, grid, block, args, shared, stream);
}

uint64_t recorded_refused(void) { return refused; }
uint64_t recorded_last_threads_in_all(void) { return (uint64_t)last_grid.x * last_grid.y * last_block.x; }

}  // extern "C"
