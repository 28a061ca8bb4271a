"""What launchers keep between calls (csrc/per_device.h, compiled for the host): a device's set-up and numbers are its
own, a failure is tried again, and a number belongs to the key that it was found for whatever threads call."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_34866_gb300", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <thread>
#include <vector>
#include "per_device.h"
using namespace jab;
static SetUp ready;
static Found found;
int main() {
  int calls = 0;
  for (int round = 0; round < 3; ++round)
    for (int dev = 0; dev < 4; ++dev)
      if (ready.once(dev, [&] { ++calls; return 0; }) != 0) return printf("status\n"), 1;
  if (calls != 4) return printf("set up %d times\n", calls), 1;
  // a device whose set-up fails twice; one that is not among those kept
  int tries = 0, status[4];
  for (int i = 0; i < 4; ++i) status[i] = ready.once(9, [&] { return tries++ < 2 ? 7 : 0; });
  if (tries != 3 || status[0] != 7 || status[1] != 7 || status[2] != 0 || status[3] != 0) return printf("retry\n"), 1;
  for (int i = 0; i < 3; ++i) ready.once(kDevices, [&] { ++tries; return 0; });
  if (tries != 6) return printf("far device\n"), 1;
  // numbers: by device and key, two keys in turn found once each, a failed search not kept
  int searches = 0;
  for (int i = 0; i < 5; ++i)
    for (int dev = 0; dev < 2; ++dev)
      for (uint32_t key : {64u, 1u, 0u})
        if (found.get(dev, key, [&] { ++searches; return (int)(100 * (dev + 1) + key); }) != (int)(100 * (dev + 1) + key)) return printf("number\n"), 1;
  if (searches != 2 + 2 * (5 + 5)) return printf("%d searches\n", searches), 1;  // (64 and 0 have one place)
  if (found.get(5, 3, [] { return 0; }) != 0 || found.get(5, 3, [] { return 8; }) != 8) return printf("failed search\n"), 1;
  // many threads, keys that share places: what comes back is the key's
  std::vector<std::thread> t;
  std::atomic<int> wrong{0};
  for (int k = 0; k < 8; ++k)
    t.emplace_back([&, k] {
      for (int i = 0; i < 200000; ++i) {
        const uint32_t key = (uint32_t)(i * 7 + k) % 40;
        if (found.get(11, key, [&] { return (int)key + 1000; }) != (int)key + 1000) ++wrong;
      }
    });
  for (auto& x : t) x.join();
  if (wrong) return printf("%d wrong\n", wrong.load()), 1;
  printf("ok\n");
}
"""


def test_state_by_device_and_key(tmp_path):
    src, exe = tmp_path / "state.cpp", tmp_path / "state"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O2", "-pthread", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.stdout


def test_launchers_of_the_serving_kernels_keep_nothing_else():
    """Their static state is of these two kinds (or the driver's entry point, which is the process's)."""
    for name in ("qlinear.cu", "kv_attn.cu", "kv_attn_tile.cu", "kv_cache.cu", "serve_api.cu"):
        with open(os.path.join(CSRC, name)) as f:
            kept = [line.strip() for line in f if line.strip().startswith("static ") and "constexpr" not in line and "__device__" not in line
                    and "static_assert" not in line]
        for line in kept:
            assert line.startswith(("static SetUp ", "static Found ", "static PFN_cuTensorMapEncodeTiled")), (name, line)
