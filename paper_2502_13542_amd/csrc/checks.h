// Host-side argument checks shared by the entry points.
#pragma once

#include <stdint.h>

#include "launch.h"

namespace actqkv {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

int check_shape(const actqkv_shape* sh);
int check_batch(int batch);

}  // namespace actqkv

#define ACTQKV_REQUIRE_PTR(p)                                                       \
  do {                                                                              \
    if ((p) == nullptr) return set_error(ACTQKV_EINVAL, #p " is NULL");             \
    if (!aligned16(p)) return set_error(ACTQKV_EALIGN, #p " is not 16-byte aligned"); \
  } while (0)
#define ACTQKV_REQUIRE_SMALL(p, a)                                                          \
  do {                                                                                      \
    if ((p) == nullptr) return set_error(ACTQKV_EINVAL, #p " is NULL");                     \
    if ((reinterpret_cast<uintptr_t>(p) & ((a)-1)) != 0)                                    \
      return set_error(ACTQKV_EALIGN, #p " is not %d-byte aligned", int(a));                \
  } while (0)
#define ACTQKV_OPTIONAL_SMALL(p, a)                                                         \
  do {                                                                                      \
    if ((p) != nullptr && (reinterpret_cast<uintptr_t>(p) & ((a)-1)) != 0)                  \
      return set_error(ACTQKV_EALIGN, #p " is not %d-byte aligned", int(a));                \
  } while (0)
#define ACTQKV_OPTIONAL_PTR(p)                                                                   \
  do {                                                                                           \
    if ((p) != nullptr && !aligned16(p)) return set_error(ACTQKV_EALIGN, #p " is not 16-byte aligned"); \
  } while (0)
#define ACTQKV_TRY(expr)      \
  do {                        \
    int rc_ = (expr);         \
    if (rc_ != ACTQKV_OK) return rc_; \
  } while (0)
