// Host helpers shared by the entry points of the operators around the decode step: the reason in words.
#pragma once
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "amk.h"

namespace amk {

struct Reason {
  char* msg;
  size_t n;
  const char* call;
  Reason(char* m, size_t bytes, const char* c) : msg(m), n(bytes), call(c) {
    if (msg && n) msg[0] = 0;
  }
  // writes "call: text" and hands the status on
  __attribute__((format(printf, 3, 4))) amk_status operator()(amk_status s, const char* fmt, ...) const {
    if (msg && n) {
      const int k = snprintf(msg, n, "%s: ", call);
      if (k >= 0 && (size_t)k < n) {
        va_list ap;
        va_start(ap, fmt);
        vsnprintf(msg + k, n - (size_t)k, fmt, ap);
        va_end(ap);
      }
    }
    return s;
  }
};

inline bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

}  // namespace amk
