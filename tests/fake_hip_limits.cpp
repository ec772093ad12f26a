// The runtime of fake_hip.cpp with what the real one says of launches: a grid dimension of more than 2^32 - 1 threads is refused.  It can also be
// told to refuse one launch, and it counts those asked for and those taken.
#define hipLaunchKernel hipLaunchKernel_of_any_size
#include "fake_hip.cpp"
#undef hipLaunchKernel

namespace {
int asked = 0, taken = 0, refuse = -1;
}

extern "C" {
hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** a, size_t lds, hipStream_t s) {
    const unsigned long long most = 0xffffffffull;
    if (asked++ == refuse || (unsigned long long)grid.x * block.x > most || (unsigned long long)grid.y * block.y > most ||
        (unsigned long long)grid.z * block.z > most)
        return last_error = hipErrorInvalidConfiguration;
    ++taken;
    return hipLaunchKernel_of_any_size(f, grid, block, a, lds, s);
}
// The launch number n from here on is refused (-1: none); both counts start again.
void fake_refuse(int n) { asked = taken = 0; refuse = n; }
int fake_asked() { return asked; }
int fake_taken() { return taken; }
}
