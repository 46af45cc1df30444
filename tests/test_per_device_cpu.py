"""csrc/per_device.h: a number per device, a failed question is not kept.  (Compiled here with the host compiler; on the GPU the streamed losses ask it for the clusters that fit.)"""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1811_02084_b200", "csrc")
PROGRAM = r"""
#include <cstdio>
#include "per_device.h"
int main() {
  mtf::KnownPerDevice known;
  int asked = 0, answer = 0;
  auto get = [&](int device) { return known.get(device, [&] { ++asked; return answer; }); };
  auto show = [&](int device) { const int n = get(device); std::printf("%d/%d ", n, asked); };
  show(0);                       // the question fails
  answer = 70; show(0); show(0); // asked again, and kept
  answer = 8; show(1); show(0);  // another device has its own
  answer = 0; show(1); show(2);
  answer = 5; show(-1); show(64);   // no device that is kept
}
"""


def test_a_failed_question_is_asked_again_and_devices_have_their_own(tmp_path):
    source, program = tmp_path / "known.cpp", tmp_path / "known"
    source.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", CSRC, "-o", str(program), str(source)], check=True)
    out = subprocess.run([str(program)], check=True, capture_output=True, text=True).stdout.split()
    assert out == ["0/1", "70/2", "70/2", "8/3", "70/3", "8/3", "0/4", "5/5", "5/6"]


def test_the_streamed_losses_keep_their_clusters_there():
    text = open(os.path.join(CSRC, "loss_rows.cu")).read()
    asked = text[text.index("int resident_clusters("):]
    asked = asked[:asked.index("\n}\n")]
    assert "known.get(device" in asked and "cudaOccupancyMaxActiveClusters" in asked and "static" not in asked
