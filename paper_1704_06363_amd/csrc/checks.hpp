// checks.hpp -- argument checks shared by the entry points: each returns HMOE_OK or an error code with
// its message set.
#pragma once
#include "host.hpp"

namespace hmoe {

// Sets the thread's error message and returns `code`.
template <typename... Args>
int fail(int code, const char* fmt, Args... args) {
  set_error(fmt, args...);
  return code;
}

inline int check_dtype(hmoe_dtype_t dt) {
  if (dt != HMOE_F32 && dt != HMOE_BF16) return fail(HMOE_EDTYPE, "unknown dtype %d", (int)dt);
  return HMOE_OK;
}

inline int check_width(const char* name, int64_t w) {
  if (w <= 0 || w % 8 != 0) return fail(HMOE_ESHAPE, "%s = %lld must be a positive multiple of 8", name, (long long)w);
  return HMOE_OK;
}

inline int check_ptr(const char* name, const void* p, bool need_align = true) {
  if (!p) return fail(HMOE_EINVAL, "%s is NULL", name);
  if (need_align && !aligned16(p)) return fail(HMOE_ESHAPE, "%s is not 16-byte aligned", name);
  return HMOE_OK;
}

inline int check_k(int32_t K) {
  if (K < 1 || K > 4096) return fail(HMOE_EINVAL, "K = %d outside [1, 4096]", K);
  return HMOE_OK;
}

inline int check_n(int64_t n) {
  if (n < 0 || n >= (int64_t(1) << 31)) return fail(HMOE_EINVAL, "n = %lld outside [0, 2^31)", (long long)n);
  return HMOE_OK;
}

inline int check_ws(size_t need, size_t have, const void* ws) {
  if (need > 0 && (have < need || ws == nullptr))
    return fail(HMOE_EWORKSPACE, "workspace of %zu bytes given, %zu needed", have, need);
  return HMOE_OK;
}

}  // namespace hmoe
