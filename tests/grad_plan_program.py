"""The gradient operators' host-side plans (csrc/iso_grad_plan.cpp, plain C++) as a program of their own."""
import os
import subprocess
from dataclasses import dataclass
from typing import List

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_19331_amd", "csrc")


def program(tmp_path, body):
    """Runs `body` (a C++ main) with the given arguments; returns the words of its output, a list per line."""
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text('#include "iso_grad_plan.h"\n#include <cstdio>\n#include <cstdlib>\n#include <vector>\nusing namespace iso;\n'
                   + body)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-I", os.path.join(ROOT, "include"), "-o", str(exe),
                    str(src), os.path.join(CSRC, "iso_grad_plan.cpp")], check=True)

    def run(*args):
        out = subprocess.run([str(exe), *map(str, args)], check=True, capture_output=True, text=True).stdout
        return [line.split() for line in out.splitlines()]
    return run


# dt accumulate base, then five words a layer: tokens rows cols ld_dy checkpoint (layers of one number share it)
WEIGHT_GRAD = r"""int main(int n, char** v) {
  std::vector<iso_weight_grad> g((n - 4) / 5);
  for (size_t j = 0; j < g.size(); ++j) {
    char** a = v + 4 + 5 * j;
    g[j].in.rows = atoll(a[0]), g[j].rows = atoll(a[1]), g[j].in.cols = atoll(a[2]), g[j].ld_dy = atoll(a[3]);
    g[j].in.q = (int8_t*)((uintptr_t)atoll(a[4]) << 32), g[j].in.e = (uint8_t*)g[j].in.q;
    g[j].dy = (void*)(((uintptr_t)j + 1) << 40), g[j].grad = (void*)(((uintptr_t)j + 1) << 44);
  }
  const int dt = atoi(v[1]);
  const WeightGradPlan P = plan_weight_grad(g.data(), (int)g.size(), dt, atoi(v[2]) != 0, (uint8_t*)(uintptr_t)atoll(v[3]));
  const LayerTable& L = P.layers;
  printf("%d %u %u %u %zu %zu %lld %d %u\n", P.tile, L.tiles, L.whole, L.split, P.total,
         weight_grad_workspace_bytes(g.data(), (int)g.size(), dt), (long long)(intptr_t)L.part, P.prep.n, P.prep.blocks);
  for (int j = 0; j < L.n; ++j) {
    const Layer& l = L.l[j];
    printf("layer %lld %lld %lld %lld %lld %lld %lld %d %d %d %d %d %d %u\n", (long long)(intptr_t)l.y, (long long)(intptr_t)l.x,
           (long long)((uintptr_t)l.g >> 44), (long long)l.y_ld, (long long)l.x_ld, (long long)l.y_bytes, (long long)l.x_bytes,
           l.rows, l.cols, l.across, l.down, l.steps, l.parts, l.tile0);
  }
  for (int j = 0; j < P.prep.n; ++j) {
    const Prep& p = P.prep.p[j];
    printf("prep %lld %lld %lld %lld %u %u %u %d\n", (long long)(intptr_t)p.dst, (long long)p.rows, (long long)p.ld,
           (long long)p.part, p.cols, p.per_row, p.block0, p.e != nullptr);
  }
}"""


@dataclass
class Schedule:
    tile: int
    tiles: int
    whole: int
    split: int
    total: int
    need: int
    part: int
    preps: int
    blocks: int
    layers: List[List[int]]
    prep: List[List[int]]


def schedule(run, layers, dt, accumulate=False, base=0):
    """layers: (tokens, rows, cols, ld_dy, checkpoint) each; dt 0 fp32, 1 bf16."""
    out = run(dt, int(accumulate), base, *[w for l in layers for w in l])
    rows = {"layer": [], "prep": []}
    for line in out[1:]:
        rows[line[0]].append([int(w) for w in line[1:]])
    return Schedule(*map(int, out[0]), rows["layer"], rows["prep"])
