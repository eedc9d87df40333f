"""The plan of an expert block's training step: the arithmetic that the host makes its launches from, run as a program of its own."""
import os
import subprocess

import pytest
import torch

from paper_2402_14800_amd import build
from tests.test_gpu_expert_ffn_forms import APART

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <utility>
#include <vector>
#include "ffn_plan.h"
using namespace moep;
static int failures = 0;
static int64_t T; static int H, F, dt;
#define CHECK(x) do { if (!(x) && ++failures < 20) std::printf("T %lld H %d F %d dtype %d: %s\n", (long long)T, H, F, dt, #x); } while (0)
static int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }

static void check_plan() {
  FfnBackwardPlan p;
  const moep_dtype type = (moep_dtype)dt;
  CHECK(plan_ffn_backward(T, H, F, type, &p));
  const bool bf16 = type == MOEP_BF16;
  const int64_t step = bf16 ? 64 : 32, size = bf16 ? 2 : 4, rows = bf16 ? 256 : 1;
  // every range of a product's K is whole steps of its GEMM; one range takes K as it is
  auto divides = [&](int64_t K, int ranges) { return ranges >= 1 && (ranges == 1 ? K % (bf16 ? 64 : 4) == 0 : K % (step * ranges) == 0); };
  CHECK(divides(H, p.dh_parts));
  CHECK(divides(2 * (int64_t)F, p.dx_parts));
  CHECK(divides(p.Tp, p.t_parts));
  CHECK(divides(p.Tp, p.t_parts13));
  CHECK(p.Tp >= T && (p.t_parts == 1 ? p.Tp < T + 64 : p.Tp < T + step * p.t_parts));
  CHECK(p.together ? bf16 && p.t_parts13 == p.t_parts : p.t_parts13 == (p.t_parts % 2 ? p.t_parts : p.t_parts / 2));
  CHECK(p.rows13 % 2 == 0 && p.rows13 / 2 >= F && (p.rows13 / 2) % rows == 0);
  CHECK(p.dh_parts * T < (int64_t)1 << 42 && p.t_parts < 65536 && p.dx_parts < 65536 && p.dh_parts < 65536);
  // what the kernels write at either end of every piece of the workspace lies within it, and the pieces do not overlap
  std::vector<std::pair<size_t, size_t>> at;
  auto piece = [&](size_t off, int64_t bytes) { if (bytes) at.push_back({off, off + (size_t)bytes}); };
  piece(p.dy, bf16 ? up(T, 256) * H * 2 : 0);
  piece(p.w2t, up(F, rows) * H * size);
  piece(p.dh, (int64_t)p.dh_parts * T * F * 4);
  piece(p.dab, up(T, rows) * 2 * F * size);
  piece(p.w13t, up(H, rows) * 2 * F * size);
  piece(p.x_t, up(H, rows) * p.Tp * size);
  piece(p.dy_t, up(H, rows) * p.Tp * size);
  piece(p.dadb_t, 2 * up(F, rows) * p.Tp * size);
  piece(p.h_t, up(F, rows) * p.Tp * size);
  if (p.dx_parts > 1) piece(p.dx_part, (int64_t)p.dx_parts * T * H * 4);
  if (p.t_parts13 > 1) piece(p.w13_part, p.together ? 2 * (int64_t)p.t_parts * F * H * 4 : (int64_t)p.t_parts13 * p.rows13 * H * 4);
  if (p.t_parts > 1) piece(p.w2_part, (int64_t)p.t_parts * H * F * 4);
  std::sort(at.begin(), at.end());
  for (size_t i = 0; i < at.size(); ++i) {
    CHECK(at[i].first % 256 == 0);
    CHECK(at[i].second <= (i + 1 < at.size() ? at[i + 1].first : p.total));
  }
}

int main(int argc, char** argv) {
  for (int i = 1; i + 3 < argc; i += 4) {                    // T H F dtype ...: the plans
    FfnBackwardPlan p;
    if (!plan_ffn_backward(std::atoll(argv[i]), std::atoi(argv[i + 1]), std::atoi(argv[i + 2]), (moep_dtype)std::atoi(argv[i + 3]), &p)) return 2;
    std::printf("%d %d %d %d %d\n", (int)p.together, p.dh_parts, p.dx_parts, p.t_parts, p.t_parts13);
  }
  if (argc > 1) return 0;
  const int64_t Ts[] = {1, 2, 3, 31, 32, 33, 63, 64, 65, 127, 129, 255, 256, 257, 300, 500, 777, 1000, 1023, 1501, 2049, 2305, 3000, 4001, 4096, 4099, 6001,
                        8192, 12345, 16385, 33000, 65537, 100003, 262144, 1000003, 16777216, 268435508, 1073741760};
  for (dt = 0; dt < 2; ++dt)
    for (int64_t t : Ts)
      for (int h = 1; h <= 1024; h = h < 40 ? h + 1 : h * 9 / 8)
        for (int f = 1; f <= 4096; f = f < 40 ? f + 1 : h < 40 ? f * 5 / 4 : f * 3 / 2) {
          T = t; H = h * (dt ? 64 : 4); F = f * (dt ? 64 : 4);
          check_plan();
        }
  std::srand(3);
  for (int i = 0; i < 20000; ++i) {
    dt = std::rand() % 2;
    const int unit = dt ? 64 : 4;
    T = 1 + (((int64_t)std::rand() << 31 | std::rand()) & (((int64_t)1 << (1 + std::rand() % 29)) - 1));
    H = unit * (1 + std::rand() % (65536 / unit >> std::rand() % 10));
    F = unit * (1 + std::rand() % (262144 / unit >> std::rand() % 12));
    check_plan();
  }
  if (!failures) std::puts("ok");
  return failures != 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover", "-I", os.path.join(ROOT, "include"), "-I", build.CSRC,
                    str(at / "plan.cpp"), "-o", str(at / "plan")], check=True)
    return str(at / "plan")


def test_ranges_divide_and_pieces_fit(program):
    r = subprocess.run([program], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


def test_tested_steps_take_the_forms_they_are_there_for(program):
    """The GPU tests' steps with products apart are so, in the ranges that the tests name; one of each kind is among them."""
    shapes = [str(v) for T, H, F, dtype in APART for v in (T, H, F, int(dtype == torch.bfloat16))]
    r = subprocess.run([program, *shapes], capture_output=True, text=True)
    plans = [tuple(int(v) for v in line.split()) for line in r.stdout.splitlines()]
    assert r.returncode == 0 and plans == [(0, *parts) for parts in APART.values()]
    bf16 = [parts for (_, _, _, dtype), parts in APART.items() if dtype == torch.bfloat16]
    for kind in (lambda dh, dx, t, t13: dh > 1, lambda dh, dx, t, t13: dx == 1, lambda dh, dx, t, t13: dx > 1, lambda dh, dx, t, t13: t == t13 == 1,
                 lambda dh, dx, t, t13: t > t13 == 1, lambda dh, dx, t, t13: t > t13 > 1, lambda dh, dx, t, t13: t == t13 > 1):
        assert any(kind(*parts) for parts in bf16)
