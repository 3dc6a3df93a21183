"""The host side of the cache in 4 bits under calls from several threads at once, without a GPU."""
import os
import re
import subprocess
import sys

import pytest

from paper_2512_16483_b200 import build

PROGRAM = """
#include <stdio.h>
#include <thread>
#include <vector>
#include "per_device.h"
int stored[fvar::kMaxDevices + 1], runs[fvar::kMaxDevices + 1];        // plain: what orders them is what is tested
int main() {
  static fvar::PerDevice set_up;
  std::vector<std::thread> threads;
  for (int t = 0; t < 8; ++t)
    threads.emplace_back([] {
      for (int k = 0; k < 2000; ++k) {
        const int dev = k % 5 == 4 ? fvar::kMaxDevices : k % 5;        // devices 0 - 3, and one that is not remembered
        const cudaError_t e = set_up.once(dev, [dev] { ++runs[dev]; if (runs[dev] == 1) return cudaErrorUnknown; stored[dev] = 7 + dev; return cudaSuccess; });
        if (e == cudaSuccess && dev < fvar::kMaxDevices && stored[dev] != 7 + dev) { printf("not stored\\n"); return; }
      }
    });
  for (auto &t : threads) t.join();
  printf("%d %d %d %d %d\\n", runs[0], runs[1], runs[2], runs[3], runs[fvar::kMaxDevices]);
}
"""


def test_a_device_is_set_up_once_whoever_comes_first(tmp_path):
    """Under the thread sanitizer, which ends the program with an error at a race.  The first attempt of each device fails and is repeated."""
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    cuda = os.path.dirname(os.path.dirname(build._nvcc()))
    p = subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=thread", "-I" + build.CSRC, "-I" + os.path.join(cuda, "include"), str(src), "-o", str(exe), "-pthread"],
                       capture_output=True, text=True)
    if p.returncode != 0 and "tsan" in p.stderr:
        pytest.skip("no thread sanitizer here")
    assert p.returncode == 0, p.stderr
    p = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert p.returncode == 0 and p.stdout == "2 2 2 2 3200\n", (p.stdout, p.stderr[-2000:])


def test_nothing_else_is_kept_between_the_calls():
    """What the attention's host side remembers stands behind that lock."""
    for name in ("attention_kv4.cu", "attention_kv4_many.cu", "kv4.cu"):
        with open(os.path.join(build.CSRC, name)) as f:
            kept = re.findall(r"^\s+static (?!constexpr|_*assert)([^(;]*);", f.read(), re.M)
        assert all(re.match(r"PerDevice \w+$|int resident\[kMaxDevices\]", k) for k in kept), (name, kept)


ERRORS = """
import threading
from paper_2512_16483_b200 import binding as fv
import ctypes as ct
lib, P = fv.load_library(), 4096
cache = ct.byref(fv._Kv4(P, P, P, P, 2, 4, 64, 40, 0))
calls = {b"kv4: rows outside the cache": lambda: lib.fvar_kv4_read(cache, 3, 39, None, None, P, P, None),
         b"attention_kv4: bad arguments": lambda: lib.fvar_attention_kv4(P, 512, cache, 8, 0, 40, None, P, None, 0, None),
         b"kv4_write: K and V must be 16-byte aligned": lambda: lib.fvar_kv4_write(cache, P + 8, P, 256, 3, 0, None, None, None),
         b"kv4: NULL cache or array": lambda: lib.fvar_kv4_read(None, 3, 39, None, None, P, P, None)}
wrong, gate = [], threading.Barrier(len(calls))
def work(text, call):
    gate.wait()
    for _ in range(20000):
        if call() != fv.EINVAL or lib.fvar_last_error(None) != text:
            wrong.append(text)
threads = [threading.Thread(target=work, args=x) for x in calls.items()]
[t.start() for t in threads], [t.join() for t in threads]
print(len(wrong))
"""


def test_each_thread_has_the_error_of_its_own_call():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    p = subprocess.run([sys.executable, "-c", ERRORS], cwd=root, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and p.stdout == "0\n", (p.returncode, p.stdout, p.stderr[-2000:])
