// What has to be done once for a kernel on each device.  Host code alone, so that it can be tested without a GPU.
#pragma once
#include <mutex>

namespace icnn {

class OncePerDevice {
public:
    // fn(), unless it has returned 0 for them before
    template <class F>
    int operator()(const void *kernel, int device, F &&fn)
    {
        std::lock_guard<std::mutex> g(lock_);
        for (int i = 0; i < n_; ++i)
            if (done_[i].kernel == kernel && done_[i].device == device) return 0;
        const int e = fn();
        if (e == 0 && n_ < kMost) done_[n_++] = {kernel, device};
        return e;
    }

private:
    static constexpr int kMost = 1024;                     // (beyond, fn is called anew)
    struct Done {
        const void *kernel;
        int device;
    };
    std::mutex lock_;
    Done done_[kMost];
    int n_ = 0;
};

}  // namespace icnn
