"""What the blocks of tree attention's tensor-core form load in a step, on the host (no GPU)."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2503_01586_b200", "csrc")


def test_every_block_loads_something_in_every_step(tmp_path):
    """A load warp that has nothing to wait for but a phase's parity may come two phases late and then waits for good: what
    holds it is that no step's products start without its bytes.  So each block's share is a box at least, it fits the block's
    part of a stage, together they hold all tokens or columns there are, and the announced sum is what is loaded."""
    src, exe = tmp_path / "steps.cpp", tmp_path / "steps"
    src.write_text('''#include "tree_steps.cuh"
#include <cstdio>
int main() {
  long long cases = 0, bad = 0;
  for (int cg = 1; cg <= 2; ++cg) {
    for (int box = 8; box <= 128; box *= 2)
      for (int left = 1; left <= 700; ++left) {
        const int half = 256 / cg;
        int sum = 0;
        for (int rank = 0; rank < cg; ++rank) {
          const int mine = tree_score_boxes(left - rank * half, half, box), tokens = left - rank * half;
          const int want = tokens < half ? tokens : half;
          bad += mine < 1 || mine * box > half || mine * box < want || (want > 0 && (mine - 1) * box >= want);
          sum += mine;
        }
        bad += sum != tree_score_boxes_all(left, 256, box, cg);
        ++cases;
      }
    for (int held = 1; held <= 4; ++held) {
      const int share = tree_value_share(held, cg);
      int sum = 0, in = 0;
      bad += share * cg != (held <= 2 ? 2 : 4);
      for (int rank = 0; rank < cg; ++rank) {
        const int ch = tree_value_chunks(held, cg, rank), real = held - share * rank;
        bad += ch < 1 || ch > share || ch > 4 / cg || (real > 0 && ch != (real < share ? real : share));
        sum += ch;
        in += real < 0 ? 0 : real < ch ? real : ch;
      }
      bad += in != held || sum != tree_value_chunks_all(held, cg);
      ++cases;
    }
  }
  std::printf("%lld %lld", cases, bad);
}''')
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout == f"{2 * (5 * 700 + 4)} 0"
