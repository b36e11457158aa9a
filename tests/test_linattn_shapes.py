"""That the GPU tests of linear attention reach every shape its rule (csrc/seq_internal.h, lin_shape) can choose: the rule
is compiled for the CPU, swept over sizes, and asked for the tests' cases."""
import os
import subprocess

from tests.test_gpu_linattn import CASES
from tests.test_gpu_linattn_shapes import SHAPES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include <stdio.h>
#include <stdlib.h>
#include <set>
#include <tuple>
#include "seq_internal.h"
using namespace pnn;
typedef std::tuple<int, int, int, int, int, int, int> Shape;

Shape shape(int f32, int B, int T, int H, int K, int V, int backward) {
  pnn_linattn_desc d = {};
  d.dtype = f32 ? PNN_F32 : PNN_BF16;
  d.batch = B, d.length = T, d.heads = d.kv_heads = H, d.key_width = K, d.value_width = V;
  const LinShape p = lin_shape(d, backward);
  const int many = lin_blocks(p, V) > 1 || (backward && lin_blocks(p, K) > 1);
  return Shape(backward, f32, p.pad, p.waves, p.tiny, many, p.segments > 1);
}

int main(int argc, char** argv) {
  std::set<Shape> can, are;
  for (int f32 = 0; f32 < 2; ++f32)
    for (int backward = 0; backward < 2; ++backward)
      for (int BH = 1; BH <= 1024; BH += BH < 40 ? 1 : 7)
        for (int T : {2, 31, 64, 127, 128, 256, 300, 777, 2048, 32768})
          for (int K = 1; K <= 256; K += K < 8 ? 1 : 5)
            for (int V = 1; V <= 256; V += V < 8 ? 1 : 5) can.insert(shape(f32, 1, T, BH, K, V, backward));
  for (int i = 1; i + 5 < argc; i += 6)
    for (int backward = 0; backward < 2; ++backward) {
      int v[6];
      for (int j = 0; j < 6; ++j) v[j] = atoi(argv[i + j]);
      if (v[2] > 1) are.insert(shape(v[0], v[1], v[2], v[3], v[4], v[5], backward));
    }
  int missing = 0;
  for (const Shape& s : can)
    if (!are.count(s)) {
      ++missing;
      printf("%s %s pad %d waves %d tiny %d blocks %d cut %d\n", std::get<0>(s) ? "backward" : "forward",
             std::get<1>(s) ? "f32" : "bf16", std::get<2>(s), std::get<3>(s), std::get<4>(s), std::get<5>(s), std::get<6>(s));
    }
  printf("%d of %d missing\n", missing, (int)can.size());
  return missing != 0 || can.size() < 30;
}
"""


def test_tests_reach_every_shape(tmp_path):
    src, exe = tmp_path / "shapes.cpp", tmp_path / "shapes"
    src.write_text(SOURCE)
    r = subprocess.run(["hipcc", "-x", "c++", "-D__HIP_PLATFORM_AMD__", "-std=c++17", "-O1", "-I/opt/rocm/include",
                        "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2103_08802_amd", "csrc"),
                        str(src), "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    asked = [str(x) for B, T, H, _, K, V, dtype, *_ in CASES + SHAPES for x in (int(dtype == "f32"), B, T, H, K, V)]
    r = subprocess.run([str(exe)] + asked, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout
