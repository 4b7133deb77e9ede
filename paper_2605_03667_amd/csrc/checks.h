// Argument checks that the ABI layers of the training operators share.
#pragma once

#include <math.h>

#include "../../include/elas.h"
#include "internal.h"

namespace elas {

inline int check_scale(double v, const char* name) {
  if (!isfinite(v)) return fail(ELAS_ERR_SHAPE, "%s must be finite", name);
  return ELAS_OK;
}

// Alignment of a pointer that only needs its element's; NULL is an error.
inline int check_elem_ptr(const void* p, size_t size, const char* name) {
  if (p == nullptr) return fail(ELAS_ERR_NULL, "%s is NULL", name);
  if ((uintptr_t)p % size) return fail(ELAS_ERR_ALIGN, "%s is not %zu-byte aligned", name, size);
  return ELAS_OK;
}

inline int check_optional_ptr(const void* p, size_t size, const char* name) {
  return p == nullptr ? ELAS_OK : check_elem_ptr(p, size, name);
}

inline int check_absent(const void* p, const char* name, const char* needs) {
  if (p != nullptr) return fail(ELAS_ERR_FLAGS, "%s is given without %s", name, needs);
  return ELAS_OK;
}

inline int check_workspace(const void* ws, size_t have, size_t need) {
  if (have < need) return fail(ELAS_ERR_WORKSPACE, "workspace %zu bytes, %zu needed", have, need);
  return need ? check_ptr(ws, "workspace") : ELAS_OK;
}

}  // namespace elas
