"""The tiles and shares that the 8-bit products choose (csrc/fp8_choice.h, compiled here
as plain C++), among them where the device runs no clusters, and the products' entry
points where no device can be asked. No GPU."""
import ctypes as ct
import os
import random
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_23144_gb300", "csrc")
GB300 = (0, 152, 76, 46, 36, 28, 23, 15, 15)

DRIVER = r"""
#include "fp8_choice.h"
extern "C" void choose(int pairs, int rows, int blocks, int x_rows, const int* of, int* out) {
  awsrc::fp8::Clusters c;
  for (int i = 0; i < 9; ++i) c.of[i] = of[i];
  const auto r = pairs ? awsrc::fp8::choose_pairs(rows, blocks, x_rows, c) : awsrc::fp8::choose_few(rows, blocks, x_rows, c);
  out[0] = r.n;
  out[1] = r.split;
}
"""


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    d = tmp_path_factory.mktemp("choice")
    (d / "driver.cpp").write_text(DRIVER)
    so = str(d / "choice.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-shared", "-fPIC",
                    "-I", CSRC, "-o", so, str(d / "driver.cpp")], check=True)
    lib = ct.CDLL(so)

    def f(pairs, rows, blocks, x_rows, of=GB300):
        out = (ct.c_int * 2)()
        lib.choose(int(pairs), rows, blocks, x_rows, (ct.c_int * 9)(*of), out)
        return out[0], out[1]

    return f


def sizes(n):
    rng = random.Random(5)
    edge = [1, 2, 7, 8, 9, 127, 128, 129, 152 * 8, 152 * 8 + 1, 152 * 128, 152 * 128 + 1, 1 << 20, 1 << 30]
    for _ in range(n):
        yield rng.choice(edge + [rng.randrange(1, 40000)]), rng.choice([1, 2, 3, 15, 16, 17, 148, 1 << 17, rng.randrange(1, 200)])


@pytest.mark.parametrize("of", [GB300, (0, 152) + (0,) * 7, (0, 152, 76, 0, 36, 0, 0, 0, 15)])
def test_few_rows_have_a_tile_that_fits(choose, of):
    for rows, blocks in sizes(300):
        for x_rows in (1, 16, 17, 64):
            n, split = choose(False, rows, blocks, x_rows, of)
            assert n % 8 == 0 and 8 <= n <= 128 and 1 <= split <= 8 and split <= max(1, (blocks + 1) // 2)
            if split > 1:  # all shares run at the same time
                assert -(-rows // n) <= of[split]


@pytest.mark.parametrize("of", [GB300, (0, 152) + (0,) * 7, (0, 152, 76, 0, 36, 0, 0, 0, 15)])
def test_more_rows_have_a_tile_that_fits(choose, of):
    for rows, blocks in sizes(300):
        for x_rows in (65, 128, 1000, 100000, 1 << 30):
            n, split = choose(True, rows, blocks, x_rows, of)
            assert n in (64, 128, 192, 256) and 1 <= split <= 4
            if split > 1:
                assert 4 * split <= blocks and -(-rows // 256) * -(-x_rows // n) <= of[2 * split]


def test_no_clusters_means_no_shares(choose):
    none = (0, 152) + (0,) * 7
    for rows, blocks in sizes(100):
        assert choose(False, rows, blocks, 1, none)[1] == 1 and choose(True, rows, blocks, 300, none)[1] == 1


def test_shares_are_taken_where_rows_are_few(choose):
    assert choose(False, 256, 160, 1)[1] > 1 and choose(True, 512, 40, 100)[1] > 1
    assert choose(False, 40000, 16, 1)[1] == 1 and choose(True, 18944, 28, 8192) == (256, 1)


NO_DEVICE = r"""
import ctypes as ct
import paper_2608_23144_gb300 as aw
from paper_2608_23144_gb300 import _step
P = 1 << 20  # aligned addresses that nothing reads
def mat(rows, k):
    return ct.byref(_step._Fp8(rows=rows, cols=4096, codes=P << k, exps=P << (k + 1)))
for rows in (1, 16, 40, 300):
    for _ in range(2):
        assert aw.lib.awsrc_fp8_linear(P, 0, 4096, mat(rows, 4), mat(300, 6), P << 9, 0, 300, P << 8, 1 << 30, None) == 5
        assert aw.lib.awsrc_fp8_gemm(mat(rows, 4), mat(300, 6), P << 9, 0, 300, P << 8, 1 << 30, None) == 5
print("refused")
"""


def test_products_without_a_device_to_ask_are_errors():
    """Not a division by the clusters of a device that did not answer (which ends the process on x86)."""
    env = dict(os.environ, CUDA_VISIBLE_DEVICES="-1", PYTHONPATH=ROOT)
    r = subprocess.run([sys.executable, "-c", NO_DEVICE], env=env, cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "refused", r
