// qsl_memory.h -- host side: where the arrays of a call lie, and whether two of them share memory.  Not a public header.
#pragma once

#include <stdint.h>

#include <initializer_list>

namespace {

uint64_t align_up(uint64_t x, uint64_t a) { return (x + a - 1) / a * a; }
bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// rows of `width` elements that do not overlap and whose offsets, in elements, stay below 2^48
bool stride_ok(uint64_t rows, uint64_t width, uint64_t stride) {
  return stride >= width && stride < 1ull << 48 && (rows <= 1 || stride <= (1ull << 48) / rows);
}

// `rows` pieces of `bytes` each, `step` from one to the next, up to `end` (0: none)
struct Memory { uintptr_t at, end; uint64_t bytes, step, rows; };
Memory array(const void* p, uint64_t bytes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return Memory{at, p && bytes ? at + bytes : 0, bytes, bytes, 1};
}
// rows > 0; width and stride in elements of `size` bytes
Memory rows_at(const void* p, uint64_t rows, uint64_t width, uint64_t stride, uint64_t size) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return Memory{at, p ? at + ((rows - 1) * stride + width) * size : 0, width * size, stride * size, rows};
}
bool meet(const Memory& a, const Memory& b) {
  if (a.end <= b.at || b.end <= a.at) return false;
  if (a.rows > 1 && b.rows == 1) return meet(b, a);
  if (b.rows == 1) return true;
  if (a.rows > 1) {      // of the same step: pieces in turn, the later ones in the gaps of the others; of another they are taken to meet
    const Memory& f = a.at <= b.at ? a : b;
    const uint64_t x = (b.at + a.at - 2 * f.at) % f.step;
    return a.step != b.step || x < f.bytes || x + (&f == &a ? b : a).bytes > f.step;
  }
  // one piece among many: where it begins, or the next piece behind that
  const uint64_t x = a.at > b.at ? a.at - b.at : 0, k = x / b.step;
  return x < k * b.step + b.bytes || (k + 1 < b.rows && a.end - b.at > (k + 1) * b.step);
}
// no output shares memory with another or with an input
bool apart(std::initializer_list<Memory> out, std::initializer_list<Memory> in) {
  for (const Memory* o = out.begin(); o != out.end(); ++o) {
    for (const Memory* p = out.begin(); p != o; ++p) if (meet(*o, *p)) return false;
    for (const Memory& i : in) if (meet(*o, i)) return false;
  }
  return true;
}

}  // namespace
