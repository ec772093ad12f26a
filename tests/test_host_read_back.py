"""What a call in two passes reads back between them, on a runtime that runs nothing (fake_hip.cpp): by a kernel, for a copy command waits for its turn at a
copy engine."""
import os
import shutil

import pytest

import fake_hip

pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"),
                                reason="needs g++ and the HIP headers")


@pytest.fixture(scope="module")
def runtime(tmp_path_factory):
    return fake_hip.build(str(tmp_path_factory.mktemp("fake_hip")))


@pytest.mark.parametrize("P,radix", [(100, 4), (100, 99), (256, 2), (300, 17)])
def test_the_counts_of_two_passes_are_written_by_a_kernel(runtime, P, radix):
    """Behind all metadata and ahead of the payload."""
    for kernels, _ in fake_hip.run(runtime, "early", [[P, radix, 4 << 20, 1, 0]] * 2):
        assert kernels.count("k_mirror_counts") == 1
        at = kernels.index("k_mirror_counts")
        assert not [k for k in kernels[:at] if k == "k_copy"] and not [k for k in kernels[at:] if k.startswith(("k_layout", "k_exchange"))]


def test_a_call_in_one_pass_reads_nothing_back(runtime):
    for kernels, _ in fake_hip.run(runtime, "early", [[100, 4, 300, 1, 0], [100, 100, 4 << 20, 1, 0], [100, 4, 300, 0, 0]]):
        assert "k_mirror_counts" not in kernels
