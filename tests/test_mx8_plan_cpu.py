"""Host arithmetic of the quantised attention's work split and of the launches' divisors, compiled with g++ under
sanitizers: every key range is covered once, parts stay within the chip and the scratch, n / d by multiplication
is exact."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_32518_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include "kernels.hpp"
#include "seg_table.hpp"
using namespace unstep;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main() {
  srand(1);
  for (uint64_t d = 1; d < (uint64_t(1) << 31); d = d < 3000 ? d + 1 : uint64_t(d * 1.001) + 1) {
    const FastDiv f = fast_div(uint32_t(d));
    const uint32_t top = 0x7fffffffu, q = top / uint32_t(d) * uint32_t(d);
    for (uint32_t n : {0u, 1u, uint32_t(d - 1), uint32_t(d), top, top - 1, q, q - 1})
      if (n <= top) CHECK(divide(n, f) == n / d);
    for (int i = 0; i < 30; ++i) {
      const uint32_t n = (uint32_t(rand()) << 1 ^ uint32_t(rand())) & top;
      CHECK(divide(n, f) == n / d);
    }
  }
  for (int i = 0; i < 20000; ++i) {
    const int B = 1 + rand() % 4, H = 1 + rand() % (rand() % 8 ? 40 : 400), N = 1 + rand() % 16;
    const int keys = 1 + rand() % (1 << (4 + rand() % 20));
    const size_t scratch = rand() % 3 ? kAttnMaxWorkspace : attn_workspace_bytes(rand() % 256);
    const AttnPlan p = attn_plan_mx8(B, H, N, keys, scratch);
    const int tk = (keys + kAttnBlockK - 1) / kAttnBlockK;
    CHECK(p.plain_groups == B * H);
    if (p.workspace == 0) {
      CHECK(p.groups == B * H && p.parts == 1);
      continue;
    }
    CHECK(p.workspace == attn_workspace_bytes(p.groups) && p.workspace <= scratch);
    CHECK(p.parts > 1 && p.parts <= tk && p.groups == p.parts * B * H && p.groups <= kAttnMaxGroups);
    for (int t = 0; t < B * H; t += B * H > 1 ? B * H - 1 : 1) {
      int next = 0;
      for (int j = 0; j < p.parts; ++j) {
        const Segment s = part_segment(tk, p.parts, t * p.parts + j);
        CHECK(s.t == t && s.k0 == next && s.k1 > s.k0 && s.k1 <= tk);
        next = s.k1;
      }
      CHECK(next == tk);
    }
  }
  // more queries: the split of the bf16 kernel
  for (int n : {17, 256, 1560, 4680}) {
    const AttnPlan a = attn_plan_mx8(1, 12, n, 18720), b = attn_plan(1, 12, n, 18720);
    CHECK(a.groups == b.groups && a.parts == b.parts && a.workspace == b.workspace);
  }
  // more query tiles than compute units: contiguous ranges of units, every unit once, at most two partials each
  int splits = 0;
  for (int i = 0; i < 3000; ++i) {
    const int H = 257 + rand() % 1200, keys = 1 + rand() % 20000;
    const AttnPlan p = attn_plan_mx8(1, H, 17 + rand() % 240, keys, rand() % 4 ? kAttnMaxWorkspace : kAttnMaxWorkspace - 16);
    if (p.workspace == 0) {
      CHECK(p.groups == H);
      continue;
    }
    ++splits;
    CHECK(p.groups == kAttnMaxGroups && p.parts == 0 && p.workspace == kAttnMaxWorkspace);
    Schedule sc;
    sc.Tk = (keys + kAttnBlockK - 1) / kAttnBlockK;
    sc.U = int64_t(H) * sc.Tk;
    sc.G = p.groups;
    int64_t next = sc.U;
    for (int g = kAttnMaxGroups - 1; g >= 0; --g) {
      int64_t hi = sc.start(g + 1);
      const int64_t lo = sc.start(g);
      CHECK(hi == next && lo < hi);
      int partials[2] = {0, 0};
      while (hi > lo) {
        const Segment s = take_segment(sc, lo, hi);
        CHECK(s.k0 < s.k1 && s.k1 <= sc.Tk && hi == s.t * sc.Tk + s.k0);
        if (!s.full) {
          CHECK(++partials[s.slot] == 1);
          const int64_t ga = sc.owner(s.t * sc.Tk), gb = sc.owner(s.t * sc.Tk + sc.Tk - 1);
          CHECK(ga <= g && g <= gb && ga < gb);
          CHECK(s.slot == (g == ga ? (sc.start(ga) >= s.t * sc.Tk ? 0 : 1) : 0));   // where the merge looks for it
        }
      }
      next = lo;
    }
    CHECK(next == 0);
  }
  CHECK(splits > 100);
  std::printf("ok\n");
}
"""


def test_plan_and_divisors(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime.h")):
        pytest.skip("needs g++ and the HIP headers")
    src, exe = tmp_path / "plan.cpp", str(tmp_path / "plan")
    src.write_text(SOURCE)
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{ROOT}/include", f"-I{CSRC}", str(src),
                        os.path.join(CSRC, "attn_plan.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


SMALL = r"""
#include <cstdio>
#include <cstdlib>
#include "kernels.hpp"
#include "seg_table.hpp"
using namespace unstep;
#define CHECK(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); return 1; } } while (0)
int main() {
  srand(2);
  int small = 0, cut = 0;
  for (int i = 0; i < 50000; ++i) {
    const int B = 1 + rand() % 3, H = 1 + rand() % 60, N = 17 + rand() % (1 << (3 + rand() % 10));
    const int keys = 1 + rand() % (1 << (4 + rand() % 13));
    if (!mx8_few(B, H, N, keys)) continue;
    ++small;
    const int tiles = (N + kMx8FewQueries - 1) / kMx8FewQueries;
    const int tiles256 = (N + kAttnBlockQ - 1) / kAttnBlockQ, tk = (keys + kAttnBlockK - 1) / kAttnBlockK;
    for (size_t scratch : {size_t(0), size_t(kAttnMaxWorkspace), attn_workspace_bytes(rand() % 256)}) {
      const AttnPlan p = attn_plan_mx8(B, H, N, keys, scratch);
      CHECK(p.plain_groups == B * H * tiles && p.parts >= 1 && p.parts <= tk && p.groups == p.plain_groups * p.parts);
      CHECK(p.groups <= kAttnMaxGroups && p.workspace <= scratch);
      if (p.parts == 1) {
        CHECK(p.workspace == 0);
        continue;
      }
      ++cut;
      CHECK(p.workspace == attn_workspace_bytes(B * H * tiles256 * p.parts));
      CHECK(p.part_o_floats == size_t(B) * H * tiles256 * p.parts * 2 * kAttnBlockQ * kHeadDim);
    }
  }
  CHECK(small > 1000 && cut > 1000);
  CHECK(mx8_few(1, 1, 1, 1) && mx8_few(4, 400, 16, 1 << 20));          // up to 16 queries always
  CHECK(mx8_few(1, 12, 27, 432) && mx8_few(1, 8, 512, 2048));
  CHECK(!mx8_few(1, 12, 17, 18720) && !mx8_few(1, 12, 4680, 18720) && !mx8_few(1, 60, 32, 19200) && !mx8_few(1, 257, 17, 64));
  std::printf("ok\n");
}
"""


def test_small_chunks(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime.h")):
        pytest.skip("needs g++ and the HIP headers")
    src, exe = tmp_path / "small.cpp", str(tmp_path / "small")
    src.write_text(SMALL)
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{ROOT}/include", f"-I{CSRC}", str(src),
                        os.path.join(CSRC, "attn_plan.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
