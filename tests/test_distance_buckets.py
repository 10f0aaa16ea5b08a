"""Where the buckets of a position bias begin, as the library forms them, against the definition in whole numbers."""
import random
import subprocess

from oracle.layers import first_distances
from paper_2509_23241_amd import build

PROGRAM = r"""
#include <cstdio>
#include "local_attention.h"
int main() {
  int buckets, reach;
  while (scanf("%d %d", &buckets, &reach) == 2) {
    const tp::DistanceBuckets d = tp::make_distance_buckets(buckets, reach);
    for (int b = 0; b < d.count; ++b) printf("%d ", d.first[b]);
    printf("\n");
  }
}
"""

# A border lies this close above a whole number: 1e-9 (93 buckets), 1e-6 (127), between them; and the first found to be one distance off.
CLOSE = [(99, 255215), (63, 75881), (113, 25495), (93, 531804), (117, 425586), (69, 780600), (103, 724374), (99, 279648), (69, 1000294),
         (118, 834461), (126, 1030393), (62, 923422), (42, 1006612), (95, 1043926), (103, 963503), (127, 1045482)]


def test_first_distances_of_the_library(tmp_path):
    rng = random.Random(3)
    cases = list(CLOSE)
    for buckets in range(2, 129):
        half = buckets // 2
        cases += [(buckets, half + 1), (buckets, 2 * half), (buckets, 1 << 20), (buckets, max(half + 1, 128)), (buckets, max(half + 1, 1024))]
        cases += [(buckets, rng.randint(half + 1, 1 << rng.randint(7, 20))) for _ in range(12)]
    source, program = tmp_path / "buckets.hip", tmp_path / "buckets"
    source.write_text(PROGRAM)
    subprocess.run([build._hipcc(), "--offload-host-only", "-std=c++17", "-O1", "-I", build.CSRC, "-x", "hip", str(source), "-x", "none",
                    build.lib_path(), "-Wl,-rpath," + build.LIBDIR, "-o", str(program)], check=True, capture_output=True)
    run = subprocess.run([str(program)], input="\n".join("%d %d" % c for c in cases), capture_output=True, text=True, timeout=60, check=True)
    lines = run.stdout.splitlines()
    assert len(lines) == len(cases)
    wrong = [c for c, line in zip(cases, lines) if [int(v) for v in line.split()] != first_distances(*c)]
    assert not wrong, wrong
