// Do strided boxes of bytes meet?  Host arithmetic for the checks of the layer operators' arguments: a result may not lie over an input (other
// than exactly, where a call works in place) or over another result.
#pragma once

#include <algorithm>
#include <cstdint>

namespace muon {

// n[0] * n[1] * n[2] runs of n[3] consecutive bytes; s: bytes between neighbours of the first three dimensions (not negative).
struct Box {
  uintptr_t base;
  int64_t n[4];
  int64_t s[3];
  __int128 end;                        // one past the last byte; the base where there is none, so that an empty box meets nothing
  Box(const void* p, int64_t n0, int64_t n1, int64_t n2, int64_t bytes, int64_t s0, int64_t s1, int64_t s2)
      : base(reinterpret_cast<uintptr_t>(p)), n{n0, n1, n2, bytes}, s{s0, s1, s2}, end(base) {
    if (p && n0 > 0 && n1 > 0 && n2 > 0 && bytes > 0) end += bytes + __int128(s0) * (n0 - 1) + __int128(s1) * (n1 - 1) + __int128(s2) * (n2 - 1);
  }
  bool empty() const { return end == __int128(base); }
};
inline Box run_of(const void* p, int64_t bytes) { return Box(p, 1, 1, 1, bytes, 0, 0, 0); }

// Whether sum stride_k d_k = delta has a solution with lo_k <= d_k <= hi_k.  Largest stride first: what the smaller ones can still reach leaves one or
// two values to try where the strides nest, as those of tensors do.
class StrideSum {
  struct Term {
    int64_t stride, lo, hi;
  };
  Term term_[8];
  __int128 least_[9], most_[9];
  int count_ = 0, steps_ = 0;
  static constexpr int kSteps = 1 << 20;     // beyond it the answer is yes: a layout that nobody can tell apart is not one to write to

  bool reaches(int k, __int128 delta) {
    if (delta < least_[k] || delta > most_[k]) return false;
    if (k == count_) return delta == 0;
    if (++steps_ > kSteps) return true;
    const Term& t = term_[k];
    auto floor_div = [](__int128 a, int64_t b) { return a >= 0 ? a / b : -((-a + b - 1) / b); };
    __int128 d = std::max<__int128>(t.lo, -floor_div(-(delta - most_[k + 1]), t.stride));
    const __int128 end = std::min<__int128>(t.hi, floor_div(delta - least_[k + 1], t.stride));
    for (; d <= end; ++d)
      if (reaches(k + 1, delta - d * t.stride)) return true;
    return false;
  }

 public:
  void add(int64_t stride, int64_t lo, int64_t hi) {
    if (stride == 0 || (lo == 0 && hi == 0)) return;
    for (int k = 0; k < count_; ++k)
      if (term_[k].stride == stride) {
        term_[k].lo += lo;
        term_[k].hi += hi;
        return;
      }
    term_[count_++] = {stride, lo, hi};
  }
  bool reaches(__int128 delta) {
    std::sort(term_, term_ + count_, [](const Term& a, const Term& b) { return a.stride > b.stride; });
    least_[count_] = most_[count_] = 0;
    for (int k = count_ - 1; k >= 0; --k) {
      least_[k] = least_[k + 1] + __int128(term_[k].stride) * term_[k].lo;
      most_[k] = most_[k + 1] + __int128(term_[k].stride) * term_[k].hi;
    }
    return reaches(0, delta);
  }
};

inline bool same_box(const Box& a, const Box& b) {
  if (a.base != b.base || a.n[3] != b.n[3]) return false;
  for (int k = 0; k < 3; ++k)
    if (a.n[k] != b.n[k] || (a.n[k] > 1 && a.s[k] != b.s[k])) return false;
  return true;
}

inline bool boxes_meet(const Box& a, const Box& b) {
  if (a.end <= __int128(b.base) || b.end <= __int128(a.base) || a.empty() || b.empty()) return false;
  const __int128 delta = __int128(b.base) - __int128(a.base);
  StrideSum sum;                       // place in a minus place in b
  for (int k = 0; k < 4; ++k) {
    sum.add(k < 3 ? a.s[k] : 1, 0, a.n[k] - 1);
    sum.add(k < 3 ? b.s[k] : 1, -(b.n[k] - 1), 0);
  }
  return sum.reaches(delta);
}

// Whether two runs of the box meet.
inline bool box_meets_itself(const Box& a) {
  if (a.empty()) return false;
  for (int first = 0; first < 3; ++first) {          // the first dimension in which the two places differ
    if (a.n[first] <= 1) continue;
    if (a.s[first] == 0) return true;
    StrideSum sum;
    sum.add(a.s[first], 1, a.n[first] - 1);
    __int128 rest = a.n[3];
    for (int k = first + 1; k < 3; ++k) rest += __int128(a.s[k]) * (a.n[k] - 1);
    if (a.s[first] >= rest) continue;                // it steps over all that the others span
    for (int k = first + 1; k < 4; ++k) sum.add(k < 3 ? a.s[k] : 1, -(a.n[k] - 1), a.n[k] - 1);
    if (sum.reaches(0)) return true;
  }
  return false;
}

}  // namespace muon
