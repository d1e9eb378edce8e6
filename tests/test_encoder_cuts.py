"""Which tiles and splits the gated feed-forward takes, without a GPU: the sizes that the GPU tests run
cover every choice, whatever the thresholds between them are."""
import ctypes
import importlib.util
import os
import subprocess

import pytest

from conftest import ROOT
from encoder_sizes import FFN_CUTS

SOURCE = '''
#include "%s"
extern "C" void cuts(int dtype, int64_t rows, int64_t n_in, int64_t n_out, int64_t *to) {
    const auto g = ndvm::ops::gated_cut(dtype, rows, n_in, n_out);
    const auto p = ndvm::ops::pieces(dtype, rows, n_in, n_out);
    const int64_t all[] = {g.ba, g.bb, g.splits, p.tile, p.dx, p.dw};
    for (int i = 0; i < 6; ++i) to[i] = all[i];
}
'''


@pytest.fixture(scope="module")
def cuts(tmp_path_factory):
    spec = importlib.util.spec_from_file_location("_b", os.path.join(ROOT, "paper_2607_03574_amd", "build.py"))
    b = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(b)
    if not os.path.exists(b.HIPCC):
        pytest.skip("no compiler")
    d = tmp_path_factory.mktemp("cuts")
    (d / "cuts.cpp").write_text(SOURCE % os.path.join(b.CSRC, "ffn_cut.h"))
    subprocess.run([b.HIPCC, "-O1", "-std=c++17", "-shared", "-fPIC", str(d / "cuts.cpp"), "-o", str(d / "cuts.so")],
                   check=True, capture_output=True)
    f = ctypes.CDLL(str(d / "cuts.so")).cuts
    f.argtypes, f.restype = [ctypes.c_int] + [ctypes.c_int64] * 3 + [ctypes.c_void_p], None

    def call(dtype, *size):
        to = (ctypes.c_int64 * 6)()
        f(dtype, *size, to)
        return tuple(to)

    return call


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_sizes_cover_every_cut(cuts, dtype):
    taken = [cuts(dtype, *size) for size in FFN_CUTS]
    assert {(a, b, s > 1) for a, b, s, *_ in taken} == {(256, 256, False), (256, 128, False), (128, 128, False), (128, 128, True)}
    assert {(t, x > 1, w > 1) for *_, t, x, w in taken} == {(t, x, w) for t in (128, 256) for x in (False, True) for w in (False, True)}


@pytest.mark.parametrize("dtype", [0, 1, 2])
def test_cuts_of_any_size_are_within_what_the_kernels_take(cuts, dtype):
    sizes = [1, 7, 63, 64, 65, 129, 1000, 5000, 30000, 1 << 21]
    for rows in [0] + sizes:
        for n_in in sizes:
            for n_out in sizes:
                a, b, splits, tile, dx, dw = cuts(dtype, rows, n_in, n_out)
                assert (a, b) in ((256, 256), (256, 128), (128, 128)) and tile in (128, 256)
                assert 1 <= splits <= 16 and (splits == 1 or (a, b) == (128, 128)) and 1 <= dx <= 32 and 1 <= dw <= 32
