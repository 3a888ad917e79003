"""Settings that belong to a device (the kernels' shared-memory limits) are made on every device that
calls come from, and a setting that failed is tried again: the host runtime's own header, compiled with
the host compiler."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2607_14898_gb300", "csrc")
PROGRAM = r"""
#include "fd_once.h"
#include <cstdio>
enum Status { kOk = 0, kFailed = 7 };
int main() {
  static fd::OncePerDevice once;
  int calls[3] = {};
  bool broken = true;
  auto on = [&](int device) {
    return once.run(device, [&] {
      ++calls[device];
      return device == 1 && broken ? kFailed : kOk;
    });
  };
  bool good = on(0) == kOk && on(0) == kOk && on(1) == kFailed && on(2) == kOk;
  good = good && calls[0] == 1 && calls[1] == 1 && calls[2] == 1;
  good = good && on(1) == kFailed && calls[1] == 2;  // not kept
  broken = false;
  good = good && on(1) == kOk && on(1) == kOk && on(0) == kOk && calls[1] == 3 && calls[0] == 1;
  int past = 0;  // devices that it has no place for: every time
  for (int i = 0; i < 2; ++i) good = good && once.run(1000, [&] { ++past; return kOk; }) == kOk;
  for (int i = 0; i < 2; ++i) good = good && once.run(-1, [&] { ++past; return kOk; }) == kOk;
  good = good && past == 4;
  std::puts(good ? "good" : "bad");
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs a host compiler")
def test_each_device_once_and_failures_again(tmp_path):
    source, binary = tmp_path / "once.cpp", tmp_path / "once"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, str(source), "-o",
                    str(binary)], check=True)
    assert subprocess.run([str(binary)], capture_output=True, text=True).stdout.strip() == "good"


def test_the_bounded_cache_launchers_use_it():
    """No result of a device's call is kept in a static of the whole process."""
    for name in ("fd_cache_attn.cu", "fd_cache_chunk.cu", "fd_cache_evict.cu", "fd_rotary.cu"):
        text = open(os.path.join(CSRC, name)).read()
        assert "static const cudaError_t" not in text, name
        assert text.count("cudaFuncSetAttribute(") == 0 or "OncePerDevice" in text, name
