// Host check of csrc/per_device.hpp: every device is asked, once where the answer was good, again where it was not.
#include <cstdio>

#include "per_device.hpp"

int main() {
    std::atomic<uint64_t> done{0}, other{0};
    int asked = 0, answer = 0;
    auto ask = [&] { ++asked; return answer; };
    auto on = [&](int device) { return adpsgd_impl::once_a_device(done, device, 0, ask); };
    if (on(0) != 0 || on(0) != 0 || asked != 1) return 1;
    if (on(1) != 0 || on(1) != 0 || on(0) != 0 || asked != 2) return 2;      // a second device is asked too
    answer = 7;
    if (on(2) != 7 || on(2) != 7 || asked != 4) return 3;                     // a refusal comes back, and is no answer for good
    answer = 0;
    if (on(2) != 0 || on(2) != 0 || asked != 5) return 4;
    if (on(63) != 0 || on(63) != 0 || asked != 6) return 5;
    if (on(64) != 0 || on(64) != 0 || asked != 8) return 6;
    if (adpsgd_impl::once_a_device(other, 0, 0, ask) != 0 || asked != 9) return 7;      // another kernel is asked for itself
    std::puts("ok");
    return 0;
}
