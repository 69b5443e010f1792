// Aligned words over rows that begin anywhere.  Internal to the library; plain C++ too, so that its reads can be checked on the host.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define MUON_BOTH __host__ __device__ __forceinline__
#else
#define MUON_BOTH inline
#endif

namespace muon {

// The word at `word`, on a border of 4 bytes.  Of a row's elements E, which lie in [first, last), those in the word are read, all at once where they fill
// it; nothing else is, and counts as zeros.  load(const T*) reads a T.
template <typename E, typename Load>
MUON_BOTH uint32_t word_within(const char* word, const char* first, const char* last, Load load) {
  if (word >= first && word + 4 <= last) return load(reinterpret_cast<const uint32_t*>(word));
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < 4; k += int(sizeof(E)))
    if (word + k >= first && word + k < last) w |= uint32_t(load(reinterpret_cast<const E*>(word + k))) << (8 * k);
  return w;
}

// N elements E from `p` on, which begin anywhere in a row's [first, last) and end in it: the N sizeof(E) / 4 words and one that hold them, and by how many
// bytes they have to be shifted.
template <typename E, int N, typename Load>
MUON_BOTH uint32_t words_of_run(const char* p, const char* first, const char* last, uint32_t (&w)[N * sizeof(E) / 4 + 1], Load load) {
  constexpr int kWords = N * int(sizeof(E)) / 4;
  const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(p)) & 3u;
  const char* q = p - off;
  w[0] = word_within<E>(q, first, last, load);
#pragma unroll
  for (int i = 1; i < kWords; ++i) w[i] = load(reinterpret_cast<const uint32_t*>(q) + i);
  w[kWords] = off ? word_within<E>(q + 4 * kWords, first, last, load) : 0u;
  return off;
}

}  // namespace muon
