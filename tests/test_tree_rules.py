"""The word of a tree's non-finite nodes: plain arithmetic, run by a host compiler."""
import os
import shutil
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_01278_amd", "csrc")
MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include "host_rules.hpp"
int main(int, char** v) {
  const int low = static_cast<int>(strtoul(v[1], nullptr, 0)), high = static_cast<int>(strtoul(v[2], nullptr, 0));
  printf("%llu\n", static_cast<unsigned long long>(pillar::nodes_of(low, high)));
}
"""


def test_each_node_names_itself_alone(tmp_path):
    """Node 31 is the sign of the low word: widened with it, nodes 32 to 63 would be looked up past the context."""
    (tmp_path / "main.cpp").write_text(MAIN)
    exe = str(tmp_path / "nodes")
    subprocess.run([shutil.which("g++") or "c++", "-std=c++17", "-D__host__=", "-D__device__=", "-I", CSRC, str(tmp_path / "main.cpp"), "-o", exe], check=True)
    nodes = lambda word: int(subprocess.run([exe, str(word & (2 ** 32 - 1)), str(word >> 32)], check=True, capture_output=True, text=True).stdout)
    for node in range(64):
        assert nodes(1 << node) == 1 << node, node
    for word in (0, 2 ** 64 - 1, 2 ** 63 | 2 ** 31, 2 ** 31 | 5):
        assert nodes(word) == word, hex(word)
