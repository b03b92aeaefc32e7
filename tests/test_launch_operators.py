"""The launches of the operators around the linear layer as the host decides on them (tests/launch_operators_driver.cpp)."""
import os
import subprocess

import pytest

from paper_2407_08296_amd import build as qg_build
from paper_2407_08296_amd import qgalore as qg

HERE = os.path.dirname(os.path.abspath(__file__))
up = lambda v, to: -(-v // to)


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    qg.lib()
    exe = str(tmp_path_factory.mktemp("launch") / "launch_operators_driver")
    lib_dir = os.path.dirname(os.path.abspath(qg.LIB_PATH))
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-x", "c++", "-std=c++17", "-O1",
                    "-I", os.path.join(qg_build.ROOT, "include"), os.path.join(HERE, "launch_operators_driver.cpp"), "-rdynamic",
                    "-L", lib_dir, "-l:" + os.path.basename(qg.LIB_PATH), "-Wl,-rpath," + lib_dir, "-o", exe], check=True)

    def run(what, *sizes):
        p = subprocess.run([exe, what, *map(str, sizes)], capture_output=True, text=True, timeout=300)
        assert p.returncode == 0, p.stdout[-500:] + p.stderr
        return [tuple(int(v) for v in line.split()) for line in p.stdout.splitlines()[:-1]]   # (workgroups in x, in y, threads)
    return run


@pytest.mark.parametrize("tokens,d", [(1, 1), (1, 16384), ((1 << 22) - 1, 1), ((1 << 22) - 1, 513), ((1 << 22) - 1, 16384)])
def test_norms_up_to_their_largest(driver, tokens, d):
    assert len(driver("norm_forward", tokens, d)) == 1
    main, cols = driver("norm_backward", tokens, d)
    assert main[0] <= 256 and cols == (up(2 * d, 32), 1, 1024)


@pytest.mark.parametrize("tokens,m,n", [(1, 1, 1), (1, 46340, 46340), ((1 << 31) - 1 >> 4, 8, 8), (8, (1 << 27) - 1, 8), (46340, 46340, 46340),
                                        (8, 8, (1 << 27) - 1)])
def test_linear_layers_up_to_their_largest(driver, tokens, m, n):
    for what in ("act_forward", "act_backward", "gated_forward", "gated_backward"):
        driver(what, tokens, m, n)


@pytest.mark.parametrize("tokens,h,vocab", [(1, 1, 1), ((1 << 24) - 1, 1, 16383), ((1 << 24) - 1, 1023, 16384), (16383, 8191, (1 << 24) - 1),
                                            (1, 8191, (1 << 24) - 1), (1, 65535, (1 << 21) - 1), ((1 << 18) - 1, 65535, 1), (400000, 64, 600000)])
def test_heads_up_to_their_largest(driver, tokens, h, vocab):
    driver("head_forward", tokens, h, vocab)
    driver("head_backward", tokens, h, vocab)


def test_the_head_takes_the_vocabulary_in_pieces(driver):
    """4096 tokens: two pieces of 16128 and 15872 entries, each with its dz (256 x 256 tiles), dx and dW (128 x 256); no join."""
    got = driver("head_backward", 4096, 4096, 32000)
    tiles = [(16 * up(w, 256), 1, 512) for w in (16128, 15872)]
    dw = [(up(w, 128) * 16, 1, 256) for w in (16128, 15872)]
    assert got[1:] == [tiles[0], (256, 1, 512), dw[0], tiles[1], (256, 1, 512), dw[1]]


def test_the_head_splits_the_contraction_of_dx(driver):
    """1000 tokens, 2048 wide: 128 tiles of 128 x 128, the contraction of 32003 in eight parts at most, then their sum."""
    got = driver("head_backward", 1000, 2048, 32003)
    assert got[2] == (128, 8, 256) and len(got) == 5


def test_two_weight_gradients_in_one_launch(driver):
    got = driver("gated_backward", 1000, 5461, 2048)
    assert got[1] == (128, 4, 256) and got[-1] == (up(43 * 8, 8) * 8, 2, 256)       # dx in four parts; G of both
    assert len(driver("gated_backward", 64, 2736, 1024)) == 5                       # few tiles: each in a launch of its own


@pytest.mark.parametrize("tokens,kernels", [(512, 2), (2048, 2), (2049, 3)])
def test_dbias_of_short_batches_takes_no_second_kernel(driver, tokens, kernels):
    assert len(driver("act_backward", tokens, 768, 256)) in (kernels, kernels + 1)
    first = driver("act_backward", tokens, 768, 256)[0]
    assert first == ((48, 1, 512) if tokens <= 2048 else (2, (2049 + 7) // 8, 256))


@pytest.mark.parametrize("tokens,m,n,want", [
    (1, 8192, 4096, (256, 512)), (64, 8192, 4096, (512, 256)),                       # contraction over eight waves, over four
    (150, 4095, 2047, (192, 512)), (500, 2048, 768, (256, 256)),                     # tiles of 64 tokens in two groups, in one
    (500, 4096, 2048, (256, 512)), (500, 4096, 512, (256, 256)),                     # of 128 tokens in two groups, in one
    (700, 2736, 2048, (480, 256)), (1000, 5461, 2048, (688, 256)),                   # 473 tiles of 64 tokens; 688 of 128
    (4096, 11008, 4096, (1376, 512)),                                                # 256 tokens, eight waves
])
def test_tiles_of_the_gated_pair(driver, tokens, m, n, want):
    assert driver("gated_forward", tokens, m, n) == [(want[0], 1, want[1])]
