// What has to be done once on every device, callers being on several host threads.
#pragma once
#include <mutex>

namespace mq {

class PerDevice {
    std::mutex mutex;
    bool done[16] = {};

  public:
    // f(), unless it has succeeded (returned 0) on `device` before: a failure is not kept, and is f's value.
    template <class F>
    int operator()(int device, F f) {
        std::lock_guard<std::mutex> lock(mutex);
        const bool counted = device >= 0 && device < 16;
        if (counted && done[device]) return 0;
        const int rc = f();
        if (counted) done[device] = rc == 0;
        return rc;
    }
};

}  // namespace mq
