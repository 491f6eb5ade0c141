"""Launch set-up is kept for each device and safe among host threads (csrc/per_device.h)."""
import glob
import os
import re
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_28511_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <thread>
#include <vector>

#include "per_device.h"

#define CHECK(x) if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; }

int main() {
  static moe::PerDevice p;
  int calls[3] = {}, v = -1;
  auto setup = [&](int dev, int st) {
    return p.get(dev, 0, &v, [&](int* out) { ++calls[dev]; *out = 10 * dev; return st; });
  };
  CHECK(setup(0, 0) == 0 && v == 0 && calls[0] == 1);   // a value of 0 counts as known
  CHECK(setup(0, 7) == 0 && v == 0 && calls[0] == 1);
  CHECK(setup(1, 7) == 7 && calls[1] == 1);             // another device; a failure is tried again
  CHECK(setup(1, 0) == 0 && v == 10 && calls[1] == 2);
  CHECK(setup(1, 7) == 0 && v == 10 && calls[1] == 2);
  CHECK(setup(2, 0) == 0 && v == 20 && calls[2] == 1);
  CHECK(setup(0, 7) == 0 && v == 0 && calls[0] == 1);

  static moe::PerDevice q;
  std::vector<std::thread> th;
  std::atomic<int> wrong{0};
  for (int t = 0; t < 8; ++t)
    th.emplace_back([&] {
      for (int d = 0; d < moe::kMaxDevices; ++d) {
        int w = -1;
        if (q.get(d, 0, &w, [&](int* out) { *out = d + 5; return 0; }) != 0 || w != d + 5) ++wrong;
      }
    });
  for (auto& t : th) t.join();
  CHECK(wrong == 0);
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ is needed")
@pytest.mark.parametrize("flags", [[], ["-fsanitize=thread"]])
def test_per_device(tmp_path, flags):
    src, exe = tmp_path / "t.cc", tmp_path / "t"
    src.write_text(PROGRAM)
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", *flags, "-I", CSRC, str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    if r.returncode and flags:
        pytest.skip("no thread sanitizer here")
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    if flags and "FATAL: ThreadSanitizer" in r.stderr:
        pytest.skip("the thread sanitizer does not start here")
    assert r.returncode == 0, r.stdout + r.stderr


def test_no_kernel_is_set_up_once_for_all_devices():
    """Where a source sets a kernel's attributes, no flag or number beside it is a plain static."""
    for path in glob.glob(os.path.join(CSRC, "*.cu")):
        text = open(path).read()
        if "cudaFuncSetAttribute" in text:
            found = re.findall(r"^\s+static (?:bool|int|size_t)\b.*$", text, re.M)
            assert not found, (os.path.basename(path), found)
