"""The sizes of the GPU tests reach every tile shape that the library can choose, and several pieces of a vocabulary."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2510_15545_amd as tt
import util_head_sizes as sizes
from paper_2510_15545_amd import build

DRIVER = r"""
#include <cstdio>
#include "tiles.h"
using namespace tt::tiles;
template <int DT, Use U> void show(const char *what, long m, long n) {
    with_shape<DT, U>(m, n, [&](auto shape) { typedef decltype(shape) S; printf("%s %d %ld %ld %d %d\n", what, DT, m, n, S::TM, S::TN); });
}
template <int DT> void all(long n, long v, long h) {
    show<DT, kForward>("forward", v, n);
    if constexpr (DT != kI8) {
        show<DT, kGradLogits>("logits", v, n);
        show<DT, kGradHidden>("hidden", h, n);
        show<DT, kGradWeight>("weight", h, n);
    }
}
int main() {
    for (long n, v, h; scanf("%ld %ld %ld", &n, &v, &h) == 3;) {
        all<TT_BF16>(n, v, h);
        all<TT_F32>(n, v, h);
        all<kI8>(n, v, h);
        printf("rows 0 0 %ld %ld 0\n", n, (long)padded_rows(n));
    }
}
"""
HALF, SMALL, WIDE3, WIDE4 = (128, 128), (128, 64), (256, 192), (256, 256)
BF16, F32, I8 = 0, 2, 3


@pytest.fixture(scope="module")
def chosen(tmp_path_factory):
    """{(product, type, n, v or h): tile} and {n: rows with their padding}, from the library's own rule compiled for the host."""
    if not (os.environ.get("HIPCC") or os.path.exists("/opt/rocm/bin/hipcc") or shutil.which("hipcc")):
        pytest.skip("no compiler")
    folder = tmp_path_factory.mktemp("shapes")
    source, program = folder / "shapes.hip", folder / "shapes"
    source.write_text(DRIVER)
    subprocess.run([build.hipcc(), f"--offload-arch={build.ARCH}", "--offload-host-only", "-O0", "-std=c++17", "-I", os.path.join(build.ROOT, "include"),
                    "-I", os.path.join(build.HERE, "csrc"), str(source), "-o", str(program)], check=True, timeout=300)
    every = list(sizes.FORWARD + sizes.GRADIENT + sizes.PIECES) + [(a, v, 64) for a in (65, 128, 129, 200, 333, 500, 512, 513, 577, 700, 1100, 5000) for v in (300, 20011, 200003)]
    text = subprocess.run([str(program)], input="".join("%d %d %d\n" % s for s in every), capture_output=True, text=True, check=True, timeout=60).stdout
    tiles, rows = {}, {}
    for what, dt, m, n, a, b in (line.split() for line in text.splitlines()):
        if what == "rows":
            rows[int(n)] = int(a)
        else:
            tiles[what, int(dt), int(n), int(m)] = (int(a), int(b))
    return tiles, rows


def test_every_tile_of_the_forward_products_is_reached(chosen):
    tiles, _ = chosen
    for dt in (BF16, F32, I8):
        reached = {tiles["forward", dt, n, v] for n, v, _ in sizes.FORWARD}
        assert reached == {t for (what, d, n, _), t in tiles.items() if what == "forward" and d == dt and n > 64}, dt
        assert reached == ({SMALL, HALF} if dt == F32 else {SMALL, HALF, WIDE3, WIDE4})


def test_every_tile_of_the_gradients_products_is_reached(chosen):
    tiles, _ = chosen
    for what, wide in (("logits", {SMALL, HALF, WIDE3, WIDE4}), ("hidden", {HALF, WIDE3, WIDE4}), ("weight", {HALF, WIDE4})):
        for dt in (BF16, F32):
            reached = {tiles[what, dt, n, h if what != "logits" else v] for n, v, h in sizes.GRADIENT}
            assert reached >= {t for (w, d, n, _), t in tiles.items() if w == what and d == dt}, (what, dt)
            assert reached >= (wide if dt != F32 else {HALF}), (what, dt)


def test_several_pieces_are_reached(chosen):
    _, rows = chosen
    for n, v, h in sizes.PIECES:
        for dt in (0, 1, 2):
            used = ctypes.c_size_t(0)
            assert tt.lib().tt_head_logprobs_backward_workspace_used(n, v, h, dt, ctypes.byref(used)) == tt.TT_OK
            # one piece would hold a row of dz for every (padded) row, two beyond 64 rows of 16 bits, and a row of weights, each of whole steps
            one = v * ((2 if dt != 2 and n > 64 else 1) * rows[n] + max(h, 32 if dt == 2 else 64)) * (4 if dt == 2 else 2)
            assert used.value < one, (n, v, h, dt)
