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

// The memory of a call's operands and results: rows of `width` bytes, `pitch` bytes apart (one row: a buffer).  A result that
// overlaps anything else of its call would be written by one thread while another reads it.
class Memory {
 public:
  const char* name = nullptr;
  Memory() = default;
  Memory(const void* p, int64_t bytes, const char* of) : Memory(p, 1, bytes, bytes, of) {}
  // (nothing, where p is NULL or there are no bytes; an end beyond the address space is the address space's)
  Memory(const void* p, int64_t rows, int64_t width, int64_t pitch, const char* of)
      : name(of), at_((uintptr_t)p), width_((uint64_t)width), pitch_(rows > 1 ? (uint64_t)pitch : 0) {
    uint64_t size = 0;
    if (!p || rows <= 0 || width <= 0) return;
    if (__builtin_mul_overflow((uint64_t)(rows - 1), pitch_, &size) || __builtin_add_overflow(size, width_, &size) ||
        __builtin_add_overflow(size, at_, &end_))
      end_ = UINT64_MAX;
  }
  uint64_t begin() const { return at_; }
  uint64_t end() const { return end_; }
  bool overlaps(const Memory& o) const {
    if (!(at_ < o.end_ && o.at_ < end_)) return false;
    // rows of one pitch beside each other, or a buffer behind the values of one row, are apart
    const uint64_t pitch = pitch_ ? pitch_ : o.pitch_;
    if (!pitch || (pitch_ && o.pitch_ && pitch_ != o.pitch_)) return true;
    const uint64_t off = o.at_ >= at_ ? (o.at_ - at_) % pitch : (pitch - (at_ - o.at_) % pitch) % pitch;
    return !(width_ <= off && o.width_ <= pitch - off);
  }

 private:
  uint64_t at_ = 0, width_ = 0, pitch_ = 0, end_ = 0;      // (an end of 0: nothing overlaps it)
};

// The first `results` of n are written; the others may overlap one another.
inline int check_apart(const Memory* m, int results, int n) {
  for (int i = 0; i < results; ++i)
    for (int k = i + 1; k < n; ++k)
      if (m[i].overlaps(m[k])) return fail(ELAS_ERR_OVERLAP, "%s overlaps %s", m[i].name, m[k].name);
  return ELAS_OK;
}
template <int N>
int check_apart(const Memory (&m)[N], int results) {
  return check_apart(m, results, N);
}

}  // namespace elas
