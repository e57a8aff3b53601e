// Errors of the C entry points: a failing check throws Fail, run_guarded turns
// it (and anything else thrown) into a status and the thread's error text, so
// that no exception leaves a C function.
#pragma once

#include <hip/hip_runtime.h>

#include <functional>
#include <new>
#include <string>

#include "phyai.h"

namespace phyai {

struct Fail {
  int code;
  std::string msg;
};

inline std::string& last_error() {
  static thread_local std::string text;
  return text;
}

[[noreturn]] inline void fail(int code, const std::string& msg) { throw Fail{code, msg}; }

inline void hip_check(hipError_t e, const char* what) {
  if (e != hipSuccess) fail(PHYAI_EHIP, std::string(what) + ": " + hipGetErrorString(e));
}
#define HIPC(x) ::phyai::hip_check((x), #x)

inline int run_guarded(const std::function<void()>& f) {
  std::string& text = last_error();
  try {
    f();
    text.clear();
    return PHYAI_OK;
  } catch (const Fail& x) {
    text = x.msg;
    return x.code;
  } catch (const std::bad_alloc&) {
    text = "host allocation failed";
    return PHYAI_ENOMEM;
  } catch (const std::exception& x) {
    text = x.what();
    return PHYAI_EINVAL;
  } catch (...) {
    text = "unknown failure";
    return PHYAI_EINVAL;
  }
}

}  // namespace phyai
