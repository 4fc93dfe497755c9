// The buffers of one call, and whether what it writes shares bytes with what else it
// reads or writes (host only).
#pragma once

#include <cstddef>
#include <cstdint>
#include <initializer_list>

namespace dcp {

// `rows` pieces of `width` bytes, `stride` bytes apart (contiguous: one piece).  kActs: a
// bf16 matrix of the call's activations, whose elements the kernels read and write in one
// lane, reads first, so that an output may be an input's very buffer.
struct Buffer {
  enum Kind { kRead, kWritten, kActsRead, kActsWritten };
  const void* p;
  Kind kind;
  size_t width;
  int64_t rows = 1;
  size_t stride = 0;
  bool written() const { return kind == kWritten || kind == kActsWritten; }
  bool empty() const { return !p || rows == 0 || width == 0; }
};

inline bool share_bytes(const Buffer& a, const Buffer& b) {
  const uintptr_t pa = reinterpret_cast<uintptr_t>(a.p), pb = reinterpret_cast<uintptr_t>(b.p);
  if (pa > pb) return share_bytes(b, a);
  const size_t d = pb - pa;
  if (a.rows == 1) return d < a.width;
  // the last piece of a that starts at or before b, and the one behind it
  const size_t at = d / a.stride, in = d % a.stride;
  if (at < size_t(a.rows) && in < a.width) return true;
  if (at + 1 >= size_t(a.rows)) return false;
  const size_t gap = a.stride - in;
  // (two matrices of one call have one stride: what holds for b's first piece holds for all)
  return gap < (b.rows == 1 || b.stride == a.stride ? b.width : b.stride * size_t(b.rows - 1) + b.width);
}

// The first output that shares bytes with another buffer of the call, unless both are
// activations in the same place and one of them is only read; null if there is none.
inline const Buffer* clash(std::initializer_list<Buffer> all) {
  for (const Buffer* a = all.begin(); a != all.end(); ++a) {
    if (a->empty()) continue;
    for (const Buffer* b = a + 1; b != all.end(); ++b) {
      if (b->empty() || !(a->written() || b->written()) || !share_bytes(*a, *b)) continue;
      const bool acts = a->kind >= Buffer::kActsRead && b->kind >= Buffer::kActsRead;
      if (acts && a->p == b->p && a->width == b->width && !(a->written() && b->written())) continue;
      return a->written() ? a : b;
    }
  }
  return nullptr;
}

}  // namespace dcp
