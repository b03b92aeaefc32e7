"""Which kernels the operators around the linear layer launch, as the host decides on it (tests/launch_kernels_driver.cpp)."""
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
