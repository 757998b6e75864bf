// What is asked once on every device of a process, at its first use there.
#pragma once

#include <atomic>
#include <cstdint>

namespace adpsgd_impl {

// ask() where it has not succeeded on `device` yet, else `good`.  `done` has a bit for each device; from 64 on they are asked every time.
template <class E, class F>
E once_a_device(std::atomic<uint64_t>& done, int device, E good, const F& ask) {
    const uint64_t bit = device >= 0 && device < 64 ? uint64_t(1) << device : 0;
    if (done.load(std::memory_order_relaxed) & bit) return good;
    const E e = ask();
    if (e == good) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

}  // namespace adpsgd_impl
