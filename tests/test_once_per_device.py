"""Set-up once per device: nobody goes on before it has succeeded, and what failed is tried again."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2601_19404_b200", "csrc")

PROGRAM = r"""
#include "once_per_device.h"
#include <chrono>
#include <cstdio>
#include <initializer_list>
#include <thread>

static std::atomic<int> begun{0}, finished{0}, early{0};

int main() {
  static rpo::OncePerDevice once;
  auto slow = [] { ++begun; std::this_thread::sleep_for(std::chrono::milliseconds(300)); ++finished; return 0; };
  std::thread first([&] { once.run(2, slow); });
  while (begun.load() == 0) std::this_thread::yield();                 // the first thread is inside its set-up
  std::thread second([&] { once.run(2, slow); if (finished.load() == 0) ++early; });
  first.join();
  second.join();
  if (early.load()) return std::printf("a second thread went on before the set-up was done\n"), 1;
  const int n = begun.load();
  if (once.run(2, slow) != 0 || begun.load() != n) return std::printf("done twice\n"), 1;
  int calls = 0;
  auto fails = [&] { ++calls; return calls == 1 ? 7 : 0; };
  if (once.run(3, fails) != 7 || once.run(3, fails) != 0 || once.run(3, fails) != 0 || calls != 2) return std::printf("a failure was not tried again\n"), 1;
  calls = 0;
  auto counts = [&] { ++calls; return 0; };
  for (int d : {-1, 64, 1000}) { once.run(d, counts); once.run(d, counts); }
  if (calls != 6) return std::printf("devices out of range\n"), 1;
  return 0;
}
"""


def test_once_per_device(tmp_path):
    src, exe = tmp_path / "once.cpp", tmp_path / "once"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
