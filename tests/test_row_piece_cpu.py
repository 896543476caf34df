"""Host check of the addresses that the 4-bit experts' rows are loaded from: the kernels' own header compiled with g++.  Every 16-byte piece lies within its row, at a multiple
of 16 bytes, and is the lane's own where the row reaches that far: rows shorter than a chunk of 128, rows that end within one, long ones."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1904_08368_amd", "csrc")
SRC = r'''
#include <cstdio>
#include "row_piece.hpp"
int main() {
  const int odd[] = {1008, 1408, 2000, 4096, 4112, 7168, 65536, 0x7fffff00 / 16 / 16 * 16};
  for (int i = 1; i <= 64 + 8; ++i) {
    const int k = i <= 64 ? 16 * i : odd[i - 65], chunks = (k + 127) / 128;
    for (int chunk = 0; chunk < chunks; ++chunk)
      for (int col = 0; col < 16; ++col) {
        const int at = relay::row_piece(chunk, col, k), own = chunk * 128 + col * 8;
        if (at < 0 || at + 8 > k || at % 8 || (own + 8 <= k && at != own)) { std::printf("k=%d chunk=%d lane=%d: %d\n", k, chunk, col, at); return 1; }
      }
  }
  return 0;
}
'''


def test_pieces_lie_within_their_row(tmp_path):
    src, exe = tmp_path / "piece.cpp", tmp_path / "piece"
    src.write_text(SRC)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout[-400:]


def test_rows_are_loaded_by_it():
    """The one place that loads x and h for the rows adds this offset, and no other, to the start of a row."""
    text = open(os.path.join(CSRC, "experts_w4.hip")).read()
    body = text[text.index("void load_x("):]
    body = body[:body.index("\n  }\n")]
    assert "row_piece(chunk, lane & 15, k)" in body and re.search(r"w\.row\[i\] \+ at\)", body)
    starts = re.findall(r"where\.row\[i\] = (.*?);", text)
    assert len(starts) == 2 and not any("lane" in s for s in starts), starts
