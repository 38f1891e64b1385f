// A number that is asked for once per device, on the host.
#pragma once

#include <atomic>

namespace cmpq {

// What ask() answers for `device`, asked once: a number above 0, or 0 where there is none or it could not be had (ask() has then
// left no error behind), which is kept too.  Devices past the last entry are asked every time.
struct AskedOnce {
    std::atomic<int> kept[64] = {};  // 0: not asked yet, below 0: there is none

    template <class Ask>
    int get(int device, Ask ask) {
        std::atomic<int>* slot = device >= 0 && device < 64 ? &kept[device] : nullptr;
        if (slot)
            if (const int n = slot->load(std::memory_order_relaxed)) return n > 0 ? n : 0;
        const int n = ask();
        if (slot) slot->store(n > 0 ? n : -1, std::memory_order_relaxed);
        return n > 0 ? n : 0;
    }
};

}  // namespace cmpq
