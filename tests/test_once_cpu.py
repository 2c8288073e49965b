"""The once-per-device rule of the launchers (csrc/ptenc_once.h), compiled alone and driven from several host threads."""
import os
import shutil
import subprocess

import pytest

import paper_2602_16839_b200 as pt

PROGRAM = r"""
#include <chrono>
#include <cstdio>
#include <initializer_list>
#include <thread>

#include "ptenc_once.h"

#define CHECK(x) do { if (!(x)) { std::printf("failed: %s\n", #x); return 1; } } while (0)

static PtencOnce a, b, c, d;

int main() {
  // one thread is still at it when a second one comes: the second must not come back before the attribute is set
  std::atomic<int> inside{0}, set{0};
  std::atomic<bool> go{false};
  std::thread slow([&] {
    ptenc_first_use(a, 0, [&] { ++inside; while (!go) std::this_thread::yield(); ++set; return 0; });
  });
  while (inside == 0) std::this_thread::yield();
  int seen = -1;
  std::thread late([&] { ptenc_first_use(a, 0, [&] { ++set; return 0; }); seen = set; });
  std::this_thread::sleep_for(std::chrono::milliseconds(50));
  const bool early = seen == 0;
  go = true;
  slow.join();
  late.join();
  CHECK(!early && seen > 0);
  // done once: not again on that device, but on another one
  int calls = 0;
  auto count = [&] { ++calls; return 0; };
  CHECK(ptenc_first_use(b, 3, count) == 0 && ptenc_first_use(b, 3, count) == 0 && calls == 1);
  CHECK(ptenc_first_use(b, 4, count) == 0 && calls == 2);
  // a failure is reported and tried again
  int e = 7;
  auto fails = [&] { ++calls; return e; };
  calls = 0;
  CHECK(ptenc_first_use(c, 0, fails) == 7 && ptenc_first_use(c, 0, fails) == 7 && calls == 2);
  e = 0;
  CHECK(ptenc_first_use(c, 0, fails) == 0 && ptenc_first_use(c, 0, fails) == 0 && calls == 3);
  // ordinals out of the table: every time
  calls = 0;
  for (int dev : {-1, PTENC_MAX_DEVICES}) CHECK(ptenc_first_use(d, dev, count) == 0 && ptenc_first_use(d, dev, count) == 0);
  CHECK(calls == 4);
  std::printf("fine\n");
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_nobody_launches_ahead_of_the_attributes(tmp_path):
    (tmp_path / "once.cpp").write_text(PROGRAM)
    csrc = os.path.join(os.path.dirname(pt.__file__), "csrc")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-pthread", "-I", csrc, str(tmp_path / "once.cpp"), "-o", str(tmp_path / "once")])
    r = subprocess.run([str(tmp_path / "once")], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.strip() == "fine", r.stdout
