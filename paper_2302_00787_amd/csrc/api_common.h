// Argument checks and sizes that the C entry points share.
#pragma once
#include "../../include/favorsharp.h"

#include <stddef.h>
#include <stdint.h>

#include "fs_common.h"

namespace fs {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }
inline int ceil_div(int a, int b) { return (a + b - 1) / b; }

inline bool tensor_ok(const fs_tensor* t, int d, bool need_ptr = true) {
  if (t == nullptr) return false;
  if (need_ptr && t->ptr == nullptr) return false;
  if (t->dtype != FS_F32 && t->dtype != FS_BF16) return false;
  if (t->stride_l < d) return false;
  const int q = t->dtype == FS_BF16 ? 8 : 4;
  if (t->stride_l % q || t->stride_b % q || t->stride_h % q) return false;
  if (((uintptr_t)t->ptr) % 16) return false;
  return true;
}

inline TensorDev dev(const fs_tensor* t) { return TensorDev{t->ptr, t->dtype, t->stride_b, t->stride_h, t->stride_l}; }

// B*H is a grid dimension of most kernels (at most 65535 workgroups there)
constexpr long long kMaxSequences = 65535;
inline bool sequences_ok(int B, int H) { return (long long)B * H <= kMaxSequences; }

inline bool groups_ok(int g, int B, int H) { return g == 1 || g == H || g == B * H; }

}  // namespace fs
