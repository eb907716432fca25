"""How the attention shares heads out over lanes, on the CPU (csrc/attention_rule.h)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <stdio.h>
#include "attention_rule.h"
using namespace isp_dev;
#define CHECK(...) do { if (!(__VA_ARGS__)) { printf("%s\n", #__VA_ARGS__); return 1; } } while (0)
int main() {
  for (int w = 4; w <= 8; w += 4)
    for (int dh = 1; dh <= 256; ++dh) {
      const int l = att_lanes_per_head(dh, w);
      CHECK(l * w >= dh && (l == 1 || l / 2 * w < dh) && (l & (l - 1)) == 0 && l <= 64);
    }
  for (int group = 1; group <= 64; ++group)
    for (int most = 2; most <= 4; most += 2) {
      const int q = att_share(group, most);
      CHECK((q == 1 || q == 2 || q == 4) && q <= most && group % q == 0 && (q == most || group % (2 * q)));
    }
  CHECK(att_wide(2, 1, 8, 8, 1600, 100) && !att_wide(2, 1, 8, 8, 1599, 100) && !att_wide(4, 1, 8, 8, 1600, 100) && !att_wide(2, 2, 8, 8, 1600, 100));
  CHECK(!att_wide(2, 1, 8, 7, 1600, 100) && !att_wide(2, 1, 4, 8, 1600, 100) && !att_wide(2, 1, 2, 16, 1600, 100) && att_wide(2, 1, 3, 20, 1600, 100));
  CHECK(att_wide(2, 1, 1, 64, 1600, 100) && !att_wide(2, 1, 1, 32, 1600, 100));
  for (int64_t x = 2; x <= 4096; x += 2) {
    const int64_t p = att_packed_pitch(x);
    CHECK(p % 128 == 0 && p >= 2 * x && p < 2 * x + 128);
    CHECK(!att_packs(x, false, 0, 1000) && !att_packs(x, false, 1000, 1000) && !att_packs(x, true, 4 * 1000 * 1000, 1000 * 1000));
    if (x % 128 == 0) CHECK(!att_packs(x, true, int64_t(1) << 31, 1000));  // (nothing is saved)
  }
  CHECK(att_packs(120, false, 40000003, 232965) && !att_packs(120, false, 2404585, 169343) && !att_packs(64, true, 16851165, 1048576));
  CHECK(att_packs(100, false, 6000000, 60000) && att_packs(64, true, 16851165, 300000));
  return 0;
}
"""


def test_lanes(tmp_path):
    src, exe = tmp_path / "rule.cpp", tmp_path / "rule"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-I" + os.path.join(ROOT, "paper_2403_14853_amd", "csrc"), str(src), "-o", str(exe)])
    res = subprocess.run([str(exe)], stdout=subprocess.PIPE, text=True)
    assert res.returncode == 0, res.stdout
