// What the entry points of the fitting operators check alike.
#pragma once

#include <climits>
#include <exception>
#include <string>

#include "train.h"

namespace dpa4c {

namespace {

int invalid(const std::string& msg) {
  set_error(msg);
  return DPA4C_ERR_INVALID_ARG;
}

int check_work(const char* who, const void* work, int64_t have, int64_t need) {
  if (need > 0 && (!work || have < need || reinterpret_cast<uintptr_t>(work) % 256))
    return invalid(std::string(who) + ": needs " + std::to_string(need) +
                   " bytes of 256-byte aligned scratch");
  return 0;
}

int check_rows(const char* who, int64_t n, int n_groups, int most) {
  if (n < 0 || n > INT32_MAX) return invalid(std::string(who) + ": n must be 0 .. 2^31 - 1");
  if (n_groups < 1) return invalid(std::string(who) + ": n_groups must be positive");
  if (n_groups > most) {
    set_error(std::string(who) + ": at most " + std::to_string(most) + " groups");
    return DPA4C_ERR_UNSUPPORTED;
  }
  return 0;
}

// no C++ exception leaves an entry point
template <class Fn>
int guarded(Fn&& fn) {
  try {
    return fn();
  } catch (const std::exception& e) {
    return invalid(e.what());
  }
}

}  // namespace

}  // namespace dpa4c
