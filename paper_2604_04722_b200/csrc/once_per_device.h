// Values of a device that are asked for once per process and only read from then on.
#pragma once
#include <atomic>
#include <new>

namespace kvq {

template <class T>
class OncePerDevice {
  public:
    static constexpr int kDevices = 64;
    // Makes the value of `device` if there is none yet; fill(T&) returns zero for success.  Threads that come here together
    // each fill a value of their own, and the first that is complete stays: nobody ever sees one that is being filled, and
    // none changes once it can be seen.  Nothing waits and nothing throws.  Devices out of range have no value.
    template <class Fill>
    auto make(int device, Fill fill) -> decltype(fill(*static_cast<T*>(nullptr))) {
        using Error = decltype(fill(*static_cast<T*>(nullptr)));
        if (device < 0 || device >= kDevices || of(device)) return Error{};
        T* const mine = new (std::nothrow) T();
        if (!mine) return Error{};
        const Error e = fill(*mine);
        const T* none = nullptr;
        if (e != Error{} || !value_[device].compare_exchange_strong(none, mine, std::memory_order_acq_rel)) delete mine;
        return e;
    }
    // The value of `device`, or nullptr.
    const T* of(int device) const {
        return device >= 0 && device < kDevices ? value_[device].load(std::memory_order_acquire) : nullptr;
    }

  private:
    std::atomic<const T*> value_[kDevices] = {};       // (kept until the process ends: launches of any handle read them)
};

}  // namespace kvq
