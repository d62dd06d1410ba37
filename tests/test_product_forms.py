"""Which of the products' kernels a call takes (product_forms.hpp), compiled for the CPU: every form is reached by the shapes
that the GPU tests run it with, and few rows go through registers only."""
import shutil
import subprocess
from pathlib import Path

import pytest

from tests.product_shapes import DISORDERED, SHAPES

CSRC = Path(__file__).resolve().parent.parent / "paper_2509_06362_amd" / "csrc"
UNITS = 256


@pytest.fixture(scope="module")
def form_of(tmp_path_factory):
    """(rows, experts or 0, channels, bytes of a row) to (form, whether tiles begin at unlike steps)."""
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    at = tmp_path_factory.mktemp("forms")
    src, exe = at / "forms.cpp", at / "forms"
    src.write_text("""#include <cstdio>
#include <cstdlib>
#include "product_forms.hpp"
using namespace maaso;
int main(int n, char** v) {
  const char* names[] = {"stream", "64", "128four", "128two", "256"};
  for (int i = 1; i + 4 < n; i += 5) {
    const ProductShape s{(uint32_t)atoll(v[i]), (uint32_t)atoll(v[i + 1]), (uint32_t)atoll(v[i + 2]), (uint32_t)atoll(v[i + 3]), v[i + 4][0] == '1'};
    printf("%s %d\\n", names[product_form(s, %UNITS%u)], begins_unlike(s) ? 1 : 0);
  }
  return 0;
}
""".replace("%UNITS%", str(UNITS)))
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", f"-I{CSRC}", str(src), "-o", str(exe)], check=True)

    def run(shapes):
        words = [str(x) for rows, experts, channels, n_bytes in shapes for x in (rows, max(experts, 1), channels, n_bytes, int(experts > 0))]
        out = subprocess.run([str(exe), *words], check=True, capture_output=True, text=True, timeout=60).stdout
        return [(name, flag == "1") for name, flag in (line.split() for line in out.splitlines())]

    return run


def test_shapes_reach_their_forms(form_of):
    assert form_of([s[3:4] + s[2:3] + s[4:] for s in SHAPES]) == [s[:2] for s in SHAPES]
    assert [f for f, _ in form_of([(rows, e, channels, n_bytes) for _, e, rows, channels, n_bytes in DISORDERED])] == [s[0] for s in DISORDERED]
    for form in ("stream", "64", "128four", "128two", "256"):
        of = [s for s in SHAPES if s[0] == form]
        assert any(s[1] for s in of) and any(s[2] == 0 for s in of) and any(s[2] > 1 for s in of), form
        assert any(s[2] > 64 for s in of) or form == "128four"  # (groups of more than 64 experts never take it)
        assert any(s[4] % 16 for s in of) and any(s[5] % 128 for s in of)
    assert all(s[4] % 2 == 0 and s[5] % 2 == 0 for s in SHAPES)


def test_few_rows_go_through_registers(form_of):
    one = 1 << 20
    for rows in range(1, 41):
        for experts, channels, n_bytes in ((0, 4096, 2048), (1, 300, 100), (7, 1200, 2048), (64, 1200, 2048), (8, 8192, 4096), (1024, 16, 16)):
            all_rows = rows * max(experts, 1)
            (form, unlike), = form_of([(all_rows, experts, channels, n_bytes)])
            weights = max(experts, 1) * channels * n_bytes
            assert (form == "stream") == (rows <= 4 or (rows <= 16 and weights <= 32 * one)), (rows, experts)
            assert unlike == (weights >= 96 * one)


def test_every_size_has_a_form(form_of):
    """The largest sizes there can be, which pass 32 bits on the way, and one row more or less than some."""
    most = 2 ** 31 - 1
    shapes = [(n, e, c, b) for n in (1, 17, 65, 4095, 4097, most) for e in (0, 1, 1024) for c in (1, 64, 65, 2 ** 28 - 2) for b in (1, 128, 129, 2 * 131071)]
    assert len(form_of(shapes)) == len(shapes)
    assert form_of([(most, 0, 8192, 4096), (most, 1024, 2 ** 28 - 2, 262142)]) == [("256", False), ("256", True)]
