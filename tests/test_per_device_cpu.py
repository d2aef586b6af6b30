"""What is set once per device (csrc/per_device.h), with a fake device: compiled with the host compiler, no GPU."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2308_13137_gb300 import build

MAIN = r"""
#include "per_device.h"
#include <cstdio>
#include <vector>
int main() {
  std::atomic<uint64_t> done{0};
  std::vector<int> set;
  bool work = true;
  auto call = [&](int dev) { return omq_once_per_device(done, dev, [&] { if (work) set.push_back(dev); return work; }); };
  // a second device is set too, each once, in any order of calls
  for (int dev : {0, 0, 3, 0, 3, 63, 63, 1, 0}) if (!call(dev)) return 1;
  if (set != std::vector<int>{0, 3, 63, 1}) return 2;
  // a failure is reported and tried again
  work = false;
  if (call(5) || !call(0)) return 3;
  work = true;
  if (!call(5) || set.back() != 5 || set.size() != 5) return 4;
  // beyond the flag's devices: at every call
  for (int i = 0; i < 2; ++i) if (!call(64) || !call(-1)) return 5;
  if (set.size() != 9) return 6;
  static std::atomic<int> known[64];
  int asked = 0;
  auto value = [&](int dev) { return omq_value_per_device(known, dev, [&] { ++asked; return 100 + dev; }); };
  for (int dev : {0, 7, 0, 7, 63}) if (value(dev) != 100 + dev) return 7;
  if (asked != 3 || value(70) != 170 || asked != 4) return 8;
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_each_device_is_set_once(tmp_path):
    src, exe = tmp_path / "main.cpp", tmp_path / "main"
    src.write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0


def test_the_serving_kernels_use_it():
    """No flag of the process for an attribute of the current device."""
    for f in sorted(os.listdir(build.CSRC)):
        if f.startswith("serve_"):
            with open(os.path.join(build.CSRC, f)) as s:
                text = s.read()
            assert "cudaFuncSetAttribute" not in text and not re.search(r"static bool \w+ = false", text), f
