"""Which slices of a tensor group norm keeps in registers (csrc/gn_shape.h, host arithmetic): each shape on the side where the measurements beside the rule put
it; and that a slice's rows are all covered by registers that exist."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.abspath(__file__)), "..", "paper_1901_06773_amd", "csrc")
MAIN = """
#include <cstdio>
#include "gn_shape.h"
int main() {
  int n, hw, c, groups, v, es, back;
  while (std::scanf("%d %d %d %d %d %d %d", &n, &hw, &c, &groups, &v, &es, &back) == 7) {
    const acc::SliceCfg f = acc::slice_cfg(n, hw, c, groups, v, es, back);
    std::printf("%d %d %d %d %d %d %d %d\\n", f.nt, f.r, f.sl.s * es, f.sl.all, f.sl.tpr, f.sl.rpi, f.sl.trips, f.sl.rest);
  }
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("gn_shape")
    (d / "main.cpp").write_text(MAIN)
    subprocess.check_call(["g++", "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-I", CSRC, str(d / "main.cpp"), "-o", str(d / "main")])

    def answer(cases):
        text = "".join(" ".join(str(int(x)) for x in c) + "\n" for c in cases)
        out = subprocess.run([str(d / "main")], input=text, capture_output=True, text=True, check=True)
        assert not out.stderr
        return [tuple(int(x) for x in line.split()) for line in out.stdout.splitlines()]
    return answer


F32, BF16 = (4, 4), (8, 2)


# images, positions, channels, groups, type, backward: workgroups of 32-byte slices, and whether they are taken
@pytest.mark.parametrize("n,hw,c,groups,kind,back,all_,taken", [
    (19, 3025, 128, 16, F32, True, 304, False), (16, 3025, 128, 16, F32, True, 256, True), (12, 3025, 128, 16, F32, True, 192, True),
    (17, 3025, 128, 16, F32, True, 272, False), (8, 3025, 128, 16, F32, True, 128, False), (32, 3025, 128, 16, F32, True, 512, False),
    (64, 3025, 128, 16, F32, True, 1024, False), (38, 3136, 64, 32, F32, True, 304, False), (32, 3136, 64, 32, F32, True, 256, True),
    (18, 3136, 256, 32, BF16, True, 288, False), (16, 3136, 256, 32, BF16, True, 256, True), (11, 3136, 256, 32, BF16, True, 176, True),
    (10, 3136, 256, 32, BF16, True, 160, False), (18, 6400, 256, 32, BF16, False, 288, False), (16, 6400, 256, 32, BF16, False, 256, True),
    (38, 6400, 128, 16, F32, False, 608, False), (16, 6400, 128, 16, F32, False, 256, True),
])
def test_narrow_slices_are_most_of_one_round_of_the_compute_units(ask, n, hw, c, groups, kind, back, all_, taken):
    nt, _, width, workgroups, *_ = ask([(n, hw, c, groups, *kind, back)])[0]
    assert (nt == 1024) == taken and (nt == 0) != taken
    assert (width, workgroups) == (32, all_)


@pytest.mark.parametrize("n,hw,c,groups,kind,back,threads", [
    (64, 3136, 256, 32, BF16, False, 1024), (64, 784, 512, 32, BF16, True, 512), (2, 49, 512, 32, F32, False, 256), (17, 3136, 256, 32, F32, False, 1024),
    (1, 1600, 512, 32, BF16, False, 512), (2, 3136, 256, 32, BF16, False, 0), (8, 3136, 256, 32, BF16, False, 1024), (1, 100000, 64, 32, F32, False, 0),
])
def test_wide_slices(ask, n, hw, c, groups, kind, back, threads):
    nt, _, width, *_ = ask([(n, hw, c, groups, *kind, back)])[0]
    assert nt == threads and (not nt or width >= 64)


def test_every_row_of_a_slice_has_a_register(ask):
    cases = [(n, hw, per * groups, groups, v, es, back) for n in (1, 3, 16, 200) for hw in (1, 2, 49, 196, 784, 1600, 3025, 3136, 6400, 9216, 20000)
             for groups in (1, 3, 8, 32) for per in (1, 2, 8, 15, 64, 300) for v, es in (F32, BF16) for back in (0, 1) if per * groups % v == 0]
    for (n, hw, c, groups, v, es, back), (nt, r, width, all_, tpr, rpi, trips, rest) in zip(cases, ask(cases)):
        if not nt:
            continue
        assert nt in (256, 512, 1024) and 1 <= tpr <= 256 and tpr * rpi <= nt and tpr * v * es == width
        assert trips * rpi + rest == hw and 0 <= rest < rpi and trips + (rest > 0) == r <= 20
        assert all_ * (width // es) == n * c
