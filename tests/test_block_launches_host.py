"""The launches of a block's operators, recorded without a GPU (tests/native/block_launches.cpp): none leaves what the runtime takes, fewer than 2^32 threads in x and at most 65535 workgroups in y; operands
that no GPU holds, which would need more, are refused."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2511_16041_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM_INC = "/opt/rocm/include"
pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(ROCM_INC), reason="needs g++ and the HIP headers")
MOST_ROWS, MOST_PITCH, MOST_NORM = 2 ** 23, 2 ** 22 - 8, 2 ** 24


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """launches(operator, sizes ..) -> [[workgroups in x, in y, threads in x, in y]]"""
    lib = build.ensure_built()
    exe = str(tmp_path_factory.mktemp("launches") / "block_launches")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", ROCM_INC, "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "native", "block_launches.cpp"),
                    "-o", exe, "-rdynamic", lib, "-Wl,-rpath," + os.path.dirname(lib)], check=True)

    def run(*args, beyond=False):
        out = subprocess.run([exe] + [str(a) for a in args], capture_output=True, text=True, check=True, timeout=60).stdout.splitlines()
        found = [[int(x) for x in re.match(r"launch (\d+) (\d+) (\d+) (\d+)", line).groups()] for line in out[:-1]]
        assert out[-1] == "status 0" or (beyond and out[-1] == "status 5"), (args, out[-1])
        for x, y, threads, other in found:
            assert 1 <= x and x * threads < 2 ** 32 and 1 <= y <= 65535 and threads * other <= 1024, (args, found)
        return found
    return run


@pytest.mark.parametrize("M", [1, 8, 9, 32, 33, 100, 2048, 65536, MOST_ROWS])
@pytest.mark.parametrize("N,K", [(1, 8), (33, 64), (4096, 4096), (5001, 2056), (MOST_PITCH, 8), (8, MOST_PITCH)])
def test_linear(launches, M, N, K):
    beyond = max(M * N, M * K, N * K) > 2 ** 37          # 256 GiB each
    for act in (0, 3):
        for workspace in (0, 1):
            for more in (0, 1):
                assert len(launches("linear", M, N, K, act, workspace, more, beyond=beyond)) <= 2              # the product, and the join of its shares
    for asked in (1, 2, 4, 7):
        assert len(launches("linear_backward", M, N, K, 3, 1, 0, asked, beyond=beyond)) <= 6                    # dx and dw with a join each, the bias's gradient over rows and then over shares
        launches("linear_backward", M, N, K, 0, 1, 1, asked, beyond=beyond)


@pytest.mark.parametrize("D", [1, 64, 1000, 4096, 8192, 8193, 16384, 2 ** 20, MOST_NORM])
@pytest.mark.parametrize("M,groups", [(1, 1), (33, 1), (65536, 1), (65536, 8), (65535, 65535), (MOST_ROWS, 1), (MOST_ROWS, 32768)])
def test_residual_norm(launches, M, D, groups):
    for post, pre in ((1, 1), (2, 2), (0, 2), (1, 0)):
        assert len(launches("residual", M, D, groups, post, pre, 1)) == 1
        assert len(launches("residual_backward", M, D, groups, post, pre, 1, 0)) == 1
        launches("residual_backward", M, D, groups, post, pre, 1, 1, beyond=M * D > 2 ** 40 or groups * D > 2 ** 34)


@pytest.mark.parametrize("M", [1, 2, 16, 17, 64])
@pytest.mark.parametrize("D,F,experts,k", [(8, 8, 1, 1), (2048, 1408, 60, 4), (4096, 14336, 8, 2), (MOST_PITCH, 128, 256, 16), (128, MOST_PITCH, 2, 1)])
def test_moe(launches, M, D, F, experts, k):
    for group in (0, 32, 128):
        if group == 0 or (D % max(group, 8) == 0 and F % max(group, 8) == 0):
            assert 3 <= len(launches("moe", M, D, F, experts, k, group)) <= 5
