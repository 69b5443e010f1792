"""What the kernels for rows that begin anywhere read: `csrc/words.h`, compiled for the host, with every read written down."""
import os
import re
import shutil
import subprocess

import pytest

from test_layer_sources import CSRC

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include <vector>
#include "words.h"

// Every run of N elements of every row of up to 40 elements at every offset in a word: nothing outside of the row is read, and the run comes out.
template <typename E, int N>
int check() {
  constexpr int kBytes = N * int(sizeof(E));
  alignas(8) static char memory[256];
  for (int i = 0; i < 256; ++i) memory[i] = char(7 * i + 3);
  int bad = 0;
  for (int offset = 0; offset < 4; offset += int(sizeof(E)))
    for (int cols = N; cols <= 40; ++cols)
      for (int col = 0; col + N <= cols; ++col) {
        const char *first = memory + 16 + offset, *last = first + cols * int(sizeof(E)), *p = first + col * int(sizeof(E));
        auto load = [&](const auto* q) {
          const char* at = reinterpret_cast<const char*>(q);
          bad += at < first || at + sizeof(*q) > last || reinterpret_cast<uintptr_t>(at) % sizeof(*q) != 0;
          auto v = *q;
          memcpy(&v, at, sizeof(v));
          return v;
        };
        uint32_t w[kBytes / 4 + 1];
        const uint32_t off = muon::words_of_run<E, N>(p, first, last, w, load);
        for (int i = 0; i < kBytes / 4; ++i) {
          const uint32_t got = off ? w[i] >> (8 * off) | w[i + 1] << (32 - 8 * off) : w[i];
          bad += memcmp(&got, p + 4 * i, 4) != 0;
        }
      }
  return bad;
}
int main() {
  const int bad = check<uint16_t, 16>() + check<uint8_t, 8>() + check<uint8_t, 4>() + check<uint16_t, 2>();
  printf("%d\n", bad);
  return bad != 0;
}
"""


def test_nothing_outside_of_the_row_is_read(tmp_path):
    compiler = shutil.which(os.environ.get("CXX", "g++"))
    if compiler is None:
        pytest.skip("no C++ compiler")
    (tmp_path / "words.cpp").write_text(PROGRAM)
    subprocess.check_call([compiler, "-std=c++17", "-O1", "-Wno-unknown-pragmas", "-I" + CSRC, str(tmp_path / "words.cpp"), "-o", str(tmp_path / "words")])
    assert subprocess.run([str(tmp_path / "words")], capture_output=True, text=True).stdout.strip() == "0"


def test_the_kernels_form_words_there_alone():
    """Rows of any alignment: no kernel reads whole words of them by itself."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "pack8.cu")).read())
    assert text.count("words_of_run<") == 3 and "reinterpret_cast<const uint32_t*>(p" not in text and "reinterpret_cast<const uint32_t*>(base" not in text
