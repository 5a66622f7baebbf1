// Status helpers shared by the library's translation units.
#pragma once

#include <exception>

#include "aug.h"

namespace aug {

// Record a printf-style message for aug_last_error() and return `s`.
aug_status fail(aug_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

// f(), with what it throws as a status: the containers of the host code throw where
// memory runs out, and no exception may leave the C interface.
template <typename F>
aug_status without_exceptions(const char* who, F&& f) {
  try {
    return f();
  } catch (const std::exception& e) {
    return fail(AUG_ERR_NO_SPACE, "%s: out of host memory (%s)", who, e.what());
  }
}

}  // namespace aug
