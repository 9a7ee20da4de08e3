// What the source files of the C ABI share.
#pragma once
#include <new>
#include <string>

#include "axon.h"

namespace axon {

// sets the calling thread's axon_last_error() and returns ``code``
int fail(int code, const std::string& msg);
void clear_error();
// AXON_OK, or the last launch's error
int check_launch(const char* what);

// the checks that a loss's two calls, on logits and on a model, share
int check_preference(int32_t pairs, float beta, float label_smoothing);
int check_policy(float clip_low, float clip_high, float kl_coef, int32_t per_sequence);

// runs an entry point's body; no exception leaves it
template <typename F>
int entry(F&& body) {
  try {
    clear_error();
    return body();
  } catch (const std::bad_alloc&) {
    return fail(AXON_E_OOM, "out of memory");  // (short enough to need none)
  } catch (...) {
    return fail(AXON_E_INVALID, "host failure");
  }
}

}  // namespace axon
