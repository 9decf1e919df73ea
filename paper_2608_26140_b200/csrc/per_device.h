// What has to be found out or set once for every device of a process (a kernel's attributes, how many of its clusters run at a
// time), from whichever thread comes first.
#pragma once
#include <array>
#include <mutex>

namespace acache {

template <class T, int DEVICES = 64>
class PerDevice {
public:
    // The device's value; `fill(value)` makes it at the first call for that device, which the others wait for.
    template <class Fill>
    T of(int device, Fill&& fill) {
        if (device < 0 || device >= DEVICES) {       // nowhere to keep it
            T value{};
            fill(value);
            return value;
        }
        std::call_once(once_[device], [&] { fill(values_[device]); });
        return values_[device];
    }

private:
    std::array<std::once_flag, DEVICES> once_;
    std::array<T, DEVICES> values_{};
};

}  // namespace acache
