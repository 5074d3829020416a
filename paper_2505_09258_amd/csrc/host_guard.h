// What every entry point of the C ABI runs behind.
#pragma once

#include <exception>
#include <new>

#include "legend.h"

namespace legend {

// records the message of the calling thread's last failure and returns `code`; never allocates
int fail(int code, const char* fmt, ...) noexcept;

// Every entry point runs its body through this: no C++ exception (the containers of the host runtime
// can throw std::bad_alloc) leaves the library through the C ABI.
template <class F>
int guarded(const char* what, F&& body) noexcept {
    try {
        return body();
    } catch (const std::bad_alloc&) {
        return fail(LEGEND_E_NOMEM, "%s: out of host memory", what);
    } catch (const std::exception& e) {
        return fail(LEGEND_E_STATE, "%s: unexpected failure in the host runtime: %s", what, e.what());
    } catch (...) {
        return fail(LEGEND_E_STATE, "%s: unexpected failure in the host runtime", what);
    }
}

}  // namespace legend
