"""What the library keeps per device is looked up for the device that is current: compiled on its own against a cudaGetDevice that
answers as told."""
import os
import shutil
import subprocess

import pytest

from paper_2605_01255_b200 import build as acx_build

PROGRAM = r"""
#include "acx_device.h"
static int device = 0;
static cudaError_t answer = cudaSuccess;
extern "C" cudaError_t cudaGetDevice(int* d) { *d = device; return answer; }
int main() {
  static acx::DeviceNumbers<3> numbers;
  static acx::DeviceOnce once;
  for (device = 0; device < 64; ++device) {
    if (numbers.here()[1].load() != 0 || !once.needed()) return 1;   // nothing of another device's
    numbers.here()[1].store(100 + device);
    once.done();
  }
  for (device = 0; device < 64; ++device)
    if (numbers.here()[0].load() != 0 || numbers.here()[1].load() != 100 + device || numbers.here()[2].load() != 0 || once.needed()) return 2;
  if (numbers.here() != nullptr) return 3;                           // a 65th device
  device = 0;
  answer = cudaErrorNoDevice;
  return numbers.here() == nullptr ? 0 : 4;
}
"""


@pytest.mark.skipif(not shutil.which("g++"), reason="no g++")
def test_numbers_and_set_up_are_kept_per_device(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    cuda = os.path.dirname(os.path.dirname(acx_build._nvcc()))
    subprocess.run(["g++", "-std=c++17", "-I", acx_build.CSRC, "-I", os.path.join(cuda, "include"), str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0
