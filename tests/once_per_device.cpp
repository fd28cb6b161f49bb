// csrc/once_per_device.h by itself
#include "../paper_2006_11735_amd/csrc/once_per_device.h"

// Of `count` pairs of a kernel and a device: whether the call was made for each; it returns `fails` the first `fails` times
extern "C" void once_per_device(const long long *kernel, const int *device, int count, int fails, int *made)
{
    static_assert(sizeof(long long) == sizeof(void *), "numbers for addresses");
    icnn::OncePerDevice once;
    for (int i = 0; i < count; ++i) {
        made[i] = 0;
        once((const void *)kernel[i], device[i], [&] {
            made[i] = 1;
            return fails > 0 ? fails-- : 0;
        });
    }
}
