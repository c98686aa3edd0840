"""The record of the barriers that a copying lane has armed, compiled alone: wherever the lane stops, every phase that was armed and may still be open
is waited for, a use of the turn that it did not finish too."""
import os
import subprocess


ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r"""
#include <cassert>
#include <cstdio>
#include <vector>
#include "armed_ring.cuh"
using namespace laga;
template <uint32_t kSize> static void check() {
    // a lane that arms a use at the start of each turn and stops after `turns` of them, in the last one `before` or behind the arming
    for (uint32_t turns = 0; turns < 4 * kSize + 3; ++turns)
        for (int before = 0; before < 2; ++before) {
            ArmedRing<kSize> ring;
            std::vector<int> phase(kSize, -1);               // the last phase that was armed
            for (uint32_t t = 0; t <= turns; ++t) {
                if (t == turns && before) break;
                assert(ring.at() == t % kSize);
                phase[ring.at()] += 1;
                ring.arm();
            }
            std::vector<int> waited(kSize, -1);
            ring.last_phases([&](uint32_t i, uint32_t parity) {
                assert(i < kSize && waited[i] < 0);
                waited[i] = (int)parity;
            });
            for (uint32_t i = 0; i < kSize; ++i) assert(phase[i] < 0 ? waited[i] < 0 : waited[i] == (phase[i] & 1));
        }
}
int main() {
    check<1>(); check<2>(); check<3>(); check<4>();
    puts("ok");
}
"""


def test_every_armed_phase_is_waited_for(tmp_path):
    source, binary = tmp_path / "t.cpp", tmp_path / "t"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", f"-I{os.path.join(ROOT, 'paper_2607_17644_b200', 'csrc')}", str(source), "-o", str(binary)], check=True)
    out = subprocess.run([str(binary)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout == "ok\n", out.stdout + out.stderr


def test_the_decode_counts_scales_where_it_arms_them():
    """In the source: between arming a scales' barrier and the record of it there is nothing that could leave the loop."""
    with open(os.path.join(ROOT, "paper_2607_17644_b200", "csrc", "attn_decode8_sm100.cuh")) as f:
        lines = [line.strip() for line in f]
    at = [i for i, line in enumerate(lines) if line.startswith("mbar_arrive_expect_tx(c_bar,")]
    assert len(at) == 1 and lines[at[0] + 1] == "armed_scales.arm();"
    assert sum("armed_scales.last_phases(" in line for line in lines) == 1
