"""Which kernel takes a product's rows: the quicker one of what both measured (no GPU)."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# rows of x, rows of the matrix, k, group, us on the device of the kernel of few rows and of the
# tensor cores', from a cold L2 on a GB300 with 152 SMs
MEASURED = [
    (9, 4096, 4096, 128, 13.5, 25.8), (16, 4096, 4096, 128, 13.4, 25.8), (32, 4096, 4096, 128, 15.5, 25.8),
    (64, 4096, 4096, 128, 21.6, 25.7), (96, 4096, 4096, 128, 28.8, 25.7), (112, 4096, 4096, 128, 38.0, 25.7),
    (64, 4096, 4096, 64, 23.7, 34.0), (96, 4096, 4096, 32, 29.8, 52.3), (16, 16384, 4096, 128, 23.7, 25.7),
    (24, 16384, 4096, 128, 34.0, 27.7), (32, 16384, 4096, 128, 36.0, 27.8), (24, 16384, 4096, 64, 34.0, 36.0),
    (32, 16384, 4096, 64, 38.0, 36.0), (24, 16384, 4096, 32, 36.0, 56.5), (64, 16384, 4096, 32, 66.7, 56.4),
    (16, 8192, 2048, 128, 13.4, 19.6), (32, 8192, 2048, 128, 17.5, 19.6), (48, 8192, 2048, 128, 29.9, 19.6),
    (64, 8192, 2048, 64, 27.8, 22.7), (64, 8192, 2048, 32, 27.8, 33.9), (16, 28672, 4096, 128, 30.4, 41.1),
    (32, 28672, 4096, 128, 46.2, 42.1), (32, 28672, 4096, 64, 48.3, 60.6), (48, 28672, 4096, 32, 95.4, 101.5),
    (96, 28672, 4096, 128, 117.9, 44.2),
]

SOURCE = """#include <cstdio>
#include <cstdlib>
#include "w4_rule.h"
int main(int n, char** v) {
  for (int i = 1; i + 3 < n; i += 4) {
    const int rows = atoi(v[i]), m = atoi(v[i + 1]), k = atoi(v[i + 2]), group = atoi(v[i + 3]);
    printf("%d\\n", (int)tre::few_is_quicker(rows, (m + 31) / 32 * 2, (k + 63) / 64, group, 152));
  }
}
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("rule")
    (d / "rule.cc").write_text(SOURCE)
    csrc = os.path.join(ROOT, "paper_2609_29160_gb300", "csrc")
    subprocess.run(["g++", "-std=c++17", "-I", csrc, str(d / "rule.cc"), "-o", str(d / "rule")], check=True)

    def ask(shapes):
        out = subprocess.run([str(d / "rule"), *(str(x) for s in shapes for x in s)], check=True, capture_output=True)
        return [bool(int(x)) for x in out.stdout.split()]

    return ask


def test_the_quicker_kernel_is_taken(rule):
    for few, m in zip(rule([m[:4] for m in MEASURED]), MEASURED):
        assert few == (m[4] <= m[5]), m


def test_ends(rule):
    """Up to eight rows always, past 96 never, whatever the matrix."""
    shapes = [(t, n, k, g) for t in (1, 8, 97, 4096) for n in (1, 4096, 1 << 20) for k in (128, 1 << 20) for g in (32, 64, 128)]
    assert all(few == (s[0] <= 8) for few, s in zip(rule(shapes), shapes))
