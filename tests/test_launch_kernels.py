"""Which kernels the operators around the linear layer launch, as the host decides on it (tests/launch_kernels_driver.cpp)."""
import math
import random

import pytest

import launch_kernels


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    return launch_kernels.make(tmp_path_factory.mktemp("launch"))


def test_direct_loads_of_long_rows(launches):
    """The weight gradient by direct loads addresses 32 rows of an operand from one base in 31 bits: rows of up to 2^25 elements.  Longer ones
    (few columns or rows of the weight, or rows far apart) take the tiles that address each row in 64 bits."""
    at = 1 << 25
    short = [("act_backward", 32, at, 32, 0, 3, 7), ("act_backward", 32, 32, at, 0, 3, 7), ("act_backward", 31, 31, 65536, at, 3, 2),
             ("gated_backward", 32, at, 32, 0, 2, 3), ("gated_backward", 32, 32, at, 0, 2, 3), ("gated_backward", 31, 31, 65536, at, 2, 2)]
    long = [("act_backward", 32, at + 1, 32, 0, 3, 7), ("act_backward", 32, 32, at + 1, 0, 3, 7), ("act_backward", 32, 40000000, 32, 0, 3, 7),
            ("act_backward", 31, 31, 65536, at + 16, 3, 2), ("act_backward", 8, (1 << 27) - 1, 8, 0, 3, 2), ("act_backward", 8, 8, (1 << 27) - 1, 0, 3, 2),
            ("gated_backward", 32, at + 1, 32, 0, 2, 3), ("gated_backward", 32, 32, at + 1, 0, 2, 3), ("gated_backward", 31, 31, 65536, at + 16, 2, 2)]
    for call, got in zip(short, launches(short)):
        assert any(k[0].startswith("k_gemm_kslow_direct<unsigned short, true>") for k in got), call
    for call, got in zip(long, launches(long)):
        assert not any(k[0].startswith(("k_gemm_kslow_direct", "k_align_rows")) for k in got), call


# kernels of the operators around the linear layer (the weight gradient's by direct loads is theirs in its ragged form)
OWN = ("k_residual_norm", "k_act_backward", "k_column_sums", "k_gemm_epilogue", "k_ksplit_epilogue", "k_join_parts", "k_align_rows", "k_head",
       "k_gemm_kslow_direct<unsigned short, true>")


def test_every_kernel_is_launched_by_some_call(launches):
    """Sizes spread over their range, a third of them whatever comes, the rest multiples of 64 and of 256."""
    rng = random.Random(1)

    def size(most):
        v, r = int(round(math.exp(rng.uniform(0, math.log(most))))), rng.random()
        return max(1, v if r < 1 / 3 else v // 64 * 64 if r < 2 / 3 else v // 256 * 256)
    calls = [("kernels",), ("act_forward", 1024, 4096, 1024, 0), ("act_forward", 1000, 4090, 1024, 0)]   # (256 tiles of 128 x 128: the only
    # number of them that is taken in two groups of waves)
    for _ in range(12000):
        tokens, m, n = size(9000), size(12000), size(12000)
        calls += [("act_forward", tokens, m, n, 0), ("act_backward", tokens, m, n, 0, rng.randrange(4), rng.randrange(1, 8)),
                  ("gated_forward", tokens, m, n, 0), ("gated_backward", tokens, m, n, 0, 2, rng.randrange(1, 4))]
        calls += [("head_forward", tokens, n, size(130000), 0), ("head_backward", tokens, n, size(130000), 0, 0, rng.randrange(1, 4))]
        calls += [(w, tokens, size(16384), rng.randrange(2), rng.randrange(3)) for w in ("norm_forward", "norm_backward")]
    held, *got = launches(calls)
    launched = {k[0] for one in got for k in one}
    assert len(held) > 50 and [k[0] for k in held if k[0].startswith(OWN) and k[0] not in launched] == []


@pytest.mark.parametrize("tokens,vocab", [(1, (1 << 24) - 1), (64, 2000000), (65, 600000), (129, 520000), (513, 130000), (1000, 66000), (4096, 32000),
                                          (5000, 50304), (30000, 128256), (65536, 4100)])
def test_pieces_of_the_vocabulary(launches, tokens, vocab):
    """dz of a piece, of the rows that the tokens are padded to, takes 128 MiB at most, and the pieces cover the vocabulary."""
    got, = launches([("head_backward", tokens, 64, vocab, 0, 0, 2)])
    unit = 64 if tokens <= 64 else 128 if tokens <= 512 else 256
    padded = -(-tokens // unit) * unit
    covered = 0
    for name, grid, _, _ in (k for k in got if "DLogitsRun" in k[0]):
        a = [v.strip() for v in name[name.index("<") + 1:].split(",")]
        rows, cols = 32 * int(a[3]) * int(a[6]), int(a[4])
        down = -(-padded // rows)                                    # tiles; the grid is the next multiple of 8
        covered += grid // down * cols
        assert padded * max((grid - 7) // down, 1) * cols * 2 <= 1 << 27, (name, grid)
    assert covered >= vocab


def test_every_kernel_is_launched_by_a_test(launches):
    """The sizes of the tests on the GPU, by what the host makes of them."""
    import test_gpu_head_loss as head
    import test_gpu_linear_act as layer
    import test_gpu_operator_kernels as more
    import test_gpu_residual_norm as norm
    calls = [("kernels",)]
    calls += [("act_forward", *s, 0) for s in layer.CASES + more.ACT_FORWARD]
    calls += [("act_backward", *s, 0, act, out) for s in layer.CASES + layer.SLABS + more.ACT_DIRECT for act, out in ((0, 7), (3, 1), (3, 2), (3, 4), (3, 7))]
    calls += [("gated_forward", *s, 0) for s in layer.CASES + layer.GATED + more.GATED_FORWARD]
    calls += [("gated_backward", *s, 0, 2, out) for s in layer.CASES + more.GATED_DX + more.GATED_DIRECT for out in (1, 2, 3)]
    calls += [("head_forward", *s, 0) for s in head.CASES + more.TOGETHER + more.HEAD]
    calls += [("head_backward", *s, 0, 0, 3) for s in head.CASES + head.PARTS + more.HEAD]
    calls += [(w, *s, fp32, gate) for w in ("norm_forward", "norm_backward") for s in norm.SHAPES for fp32 in (0, 1) for gate in (0, 1, 2)]
    held, *got = launches(calls)
    launched = {k[0] for one in got for k in one}
    assert [k[0] for k in held if k[0].startswith(OWN) and k[0] not in launched] == []
    # ... and the forms of one kernel that its name does not tell apart
    of = dict(zip(calls[1:], got))
    names = lambda *call: [k[0] for k in of[call]]
    assert all("k_head_rows" in names("head_forward", *s, 0) for s in more.TOGETHER)
    for s in more.ACT_DIRECT:
        assert any(k.startswith("k_gemm_kslow_direct") for k in names("act_backward", *s, 0, 3, 2))
    for s in more.GATED_DIRECT:                                       # both weights' gradients in one launch
        assert [k[2] for k in of[("gated_backward", *s, 0, 2, 2)] if k[0].startswith("k_gemm_kslow_direct")] == [2]
    assert "k_align_rows" in names("act_backward", 65, 5463, 2051, 0, 3, 2) and "k_align_rows" in names("gated_backward", 33, 5461, 1027, 0, 2, 2)
