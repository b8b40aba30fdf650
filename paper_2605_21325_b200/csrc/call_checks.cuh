// Checks of a call's buffers on the host: alignment, overlaps.
#pragma once
#include "common.cuh"

namespace tri_inv {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
template <class... P>
bool all_aligned(P... p) { return (aligned16(p) && ...); }
// whether pointers to values of the storage type are aligned to that type
template <class... P>
bool on_type(int dtype, P... p) { return (((reinterpret_cast<uintptr_t>(p) & (dtype == TRI_INV_F32 ? 3u : 1u)) == 0) && ...); }

// A buffer of a call, and whether one that is written meets another (one that is absent or empty meets nothing)
struct Span { const void* p; __int128 bytes; };   // (a descriptor's products may pass 64 bits)
inline bool meets(Span a, Span b) {
  const __int128 x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && a.bytes > 0 && b.bytes > 0 && x < y + b.bytes && y < x + a.bytes;
}
template <class... S>
bool meets_any(Span a, S... b) { return (meets(a, b) || ...); }

// The same of tensors of `rows` rows of `width` bytes, `ld` bytes from one to the next: those of equal ld may lie beside each other in the rows of one buffer.
struct Rows { const void* p; __int128 rows, width, ld; };
inline Span span_of(Rows a) { return Span{a.p, a.rows > 0 && a.width > 0 ? (a.rows - 1) * a.ld + a.width : 0}; }
inline bool meets(Rows a, Rows b) {
  if (!meets(span_of(a), span_of(b))) return false;
  if (a.ld != b.ld || a.rows == 1 || b.rows == 1) return true;
  __int128 gap = ((__int128)reinterpret_cast<uintptr_t>(b.p) - (__int128)reinterpret_cast<uintptr_t>(a.p)) % a.ld;
  if (gap < 0) gap += a.ld;
  return gap < a.width || gap + b.width > a.ld;
}
inline bool same(Rows a, Rows b) { return a.p == b.p && (a.ld == b.ld || a.rows <= 1); }

}  // namespace tri_inv
