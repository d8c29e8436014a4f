"""CPU: the table of kernels' shared-memory limits (csrc/smem_table.h) between threads, with a stand-in for the attribute."""
import os
import subprocess

import pytest

from paper_2503_20354_b200 import build as lib_build

PROGRAM = r"""
#include <chrono>
#include <cstdio>
#include <thread>
#include <vector>
#include "smem_table.h"
using surgeon::SmemTable;
static SmemTable table;
static int fails = 0;
#define CHECK(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); ++fails; } } while (0)

// One thread sets the larger size and is held up before it can note it down; another asks for the smaller one meanwhile.
static void larger_is_noted_late() {
  static int kernel;
  std::atomic<int> attribute{0}, calls{0};
  std::thread a([&] {
    CHECK(table.allow(&kernel, 0, 200, [&](int n) {
      attribute = n;
      ++calls;
      for (int i = 0; i < 200 && calls < 2; ++i) std::this_thread::sleep_for(std::chrono::milliseconds(1));
      return 0;
    }) == 0);
  });
  while (calls == 0) std::this_thread::yield();
  std::thread b([&] { CHECK(table.allow(&kernel, 0, 100, [&](int n) { attribute = n; ++calls; return 0; }) == 0); });
  a.join();
  b.join();
  CHECK(attribute == 200);                          // what both were promised
  CHECK(table.allow(&kernel, 0, 200, [&](int n) { attribute = n; return 0; }) == 0);
  CHECK(attribute == 200);
}

// Many threads, kernels and sizes: an attribute is never below a size that was allowed before.
static void never_lowered() {
  constexpr int kKernels = 24;
  static char kernels[kKernels];
  static std::atomic<int> attribute[2][kKernels];
  std::atomic<int> bad{0};
  std::vector<std::thread> threads;
  for (int t = 0; t < 8; ++t)
    threads.emplace_back([&, t] {
      unsigned x = 12345u + t;
      for (int i = 0; i < 20000; ++i) {
        x = x * 1664525u + 1013904223u;
        const int k = (x >> 8) % kKernels, dev = (x >> 16) & 1, bytes = 1 + (x >> 20) % 200;
        if (table.allow(&kernels[k], dev, bytes, [&](int n) { attribute[dev][k] = n; return 0; }) != 0 || attribute[dev][k] < bytes) ++bad;
      }
    });
  for (auto& t : threads) t.join();
  CHECK(bad == 0);
}

static void a_failure_is_passed_on_and_not_noted() {
  static int kernel;
  CHECK(table.allow(&kernel, 1, 50, [](int) { return 7; }) == 7);
  int calls = 0;
  CHECK(table.allow(&kernel, 1, 50, [&](int) { ++calls; return 0; }) == 0 && calls == 1);
  CHECK(table.allow(&kernel, 1, 40, [&](int) { ++calls; return 0; }) == 0 && calls == 1);
  CHECK(table.allow(&kernel, 1, 60, [&](int) { ++calls; return 9; }) == 9 && calls == 2);
  CHECK(table.allow(&kernel, 1, 50, [&](int) { ++calls; return 0; }) == 0 && calls == 2);
  CHECK(table.allow(&kernel, 2, 50, [&](int) { ++calls; return 0; }) == 0 && calls == 3);       // another device
}

static void no_room() {
  static char kernels[SmemTable::kKernels + 1];
  for (int i = 0; i < SmemTable::kKernels; ++i) CHECK(table.allow(&kernels[i], 5, 10, [](int) { return 0; }) == 0);
  CHECK(table.allow(&kernels[SmemTable::kKernels], 5, 10, [](int) { return 0; }) == SmemTable::kNoRoom);
  CHECK(table.allow(&kernels[3], 5, 20, [](int) { return 0; }) == 0);
  CHECK(table.allow(&kernels[0], -1, 10, [](int) { return 0; }) == SmemTable::kNoRoom);
  CHECK(table.allow(&kernels[0], SmemTable::kDevices, 10, [](int) { return 0; }) == SmemTable::kNoRoom);
}

int main() {
  larger_is_noted_late();
  never_lowered();
  a_failure_is_passed_on_and_not_noted();
  no_room();
  return fails ? 1 : 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("smem_table")
    source, exe = at / "table.cpp", at / "table"
    source.write_text(PROGRAM)
    subprocess.check_call([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-pthread", "-I", lib_build.CSRC, str(source), "-o", str(exe)])
    return str(exe)


def test_sizes_that_were_allowed_stay_allowed(program):
    run = subprocess.run([program], stdout=subprocess.PIPE, text=True, timeout=120)
    assert run.returncode == 0, run.stdout
