"""The launches of the feed-forward sublayer's operators, recorded without a GPU (tests/native/launches.cpp): none leaves what the runtime takes, fewer
than 2^32 threads in x and at most 65535 workgroups in y, and together they take every row once."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2511_16041_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM_INC = "/opt/rocm/include"
pytestmark = pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(ROCM_INC), reason="needs g++ and the HIP headers")
MOST_ROWS = 2 ** 23


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """launches(operator, sizes ..) -> [{"grid": workgroups in x and y, "block": threads in x and y, and what the program prints of the arguments}]"""
    lib = build.ensure_built()
    exe = str(tmp_path_factory.mktemp("launches") / "launches")
    subprocess.run(["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I", ROCM_INC, "-I", os.path.join(ROOT, "include"), "-I", build.CSRC,
                    os.path.join(ROOT, "tests", "native", "launches.cpp"), "-o", exe, "-rdynamic", lib, "-Wl,-rpath," + os.path.dirname(lib)], check=True)

    def run(*args):
        out = subprocess.run([exe] + [str(a) for a in args], capture_output=True, text=True, check=True, timeout=60).stdout.splitlines()
        assert out[-1] == "status 0", (args, out[-1])
        found = []
        for line in out[:-1]:
            n = [int(x) for x in re.match(r"launch (\d+) (\d+) (\d+) (\d+)", line).groups()]
            found.append({"grid": n[:2], "block": n[2:], **{k: int(x) for k, x in re.findall(r" ([a-z]+) (-?\d+)", line)}})
        for one in found:
            assert one["grid"][0] * one["block"][0] < 2 ** 32 and 1 <= one["grid"][1] <= 65535, (args, one)
        return found
    return run


def consecutive(found, M, pitches):
    """The launches take rows 0 .. M - 1 in order; pitches: bytes from a row to the next in each operand."""
    row = 0
    for one in found:
        for name, pitch in pitches.items():
            assert one[name] == row * pitch, (one, name)
        row += one["rows"]
    assert row == M


@pytest.mark.parametrize("type", [0, 1])
@pytest.mark.parametrize("D", [1, 64, 1000, 2049, 4097, 8192, 8193, 16384, 16385, 2 ** 24])
def test_layer_norm(launches, D, type):
    size = 4 if type else 2
    for M in (1, 1000, 2 ** 21 - 1, 2 ** 21, 2 ** 22 + 3, MOST_ROWS):
        found = launches("norm", M, D, type, D + 8, D + 16)
        consecutive(found, M, {"x": (D + 8) * size, "y": (D + 16) * size, "mean": 4, "rstd": 4})


@pytest.mark.parametrize("type", [0, 1])
@pytest.mark.parametrize("D", [1, 1000, 4097, 8193, 16384, 16385, 2 ** 24])
def test_layer_norm_backward(launches, D, type):
    size = 4 if type else 2
    for M in (1, 1000, 2 ** 22 + 3, MOST_ROWS):
        found = launches("norm_backward", M, D, type, D + 8, D + 16, D + 24, 0)
        consecutive(found, M, {"x": (D + 8) * size, "dy": (D + 16) * size, "dx": (D + 24) * size, "mean": 4, "rstd": 4})
        launches("norm_backward", M, D, type, D + 8, D + 16, D + 24, 1)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N", [1, 4096, 4097, 8192, 8193, 2 ** 24])
def test_products_with_4_bit_weights(launches, N, group):
    K = 2 * group
    for M in (1, 64, 2 ** 20 - 16, 2 ** 20 - 15, 2 ** 20, MOST_ROWS):
        for type in (0, 1):
            found = launches("q4", M, N, K, group, type, K + 8, N + 3)
            consecutive(found, M, {"x": 2 * (K + 8), "y": (4 if type else 2) * (N + 3)})
        consecutive(launches("q4_gated", M, N, K, group, K + 8, N + 3), M, {"x": 2 * (K + 8), "y": 2 * (N + 3)})


@pytest.mark.parametrize("type", [0, 1])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K", [(1, 128), (1000, 4096), (2 ** 13, 2 ** 20), (2 ** 14 - 1, 2 ** 20), (2 ** 14 + 7, 2 ** 20), (2 ** 24, 128), (2 ** 24, 4224), (2 ** 20 + 3, 2 ** 18), (2 ** 13 + 1, 2 ** 22)])
def test_quantising_and_decoding(launches, N, K, group, type):
    size, G = (4 if type else 2), K // group
    consecutive(launches("q4_quantize", N, K, group, type, K + 3), N, {"w": size * (K + 3), "packed": K // 2, "scales": 2 * G, "zeros": G})
    consecutive(launches("q4_decode", N, K, group, type), N, {"out": size * K, "packed": K // 2, "scales": 2 * G, "zeros": G})


BLOCKS = [(33, 1032, 1544), (129, 520, 4104), (257, 264, 7176), (500, 4096, 14336), (1000, 2048, 5504), (1500, 2056, 5000), (2000, 136, 72), (2600, 2056, 3592), (2600, 3592, 2056), (3600, 2056, 3080),
          (8192, 4096, 14336)]


@pytest.mark.parametrize("M,D,F", BLOCKS)
def test_shares_fit_the_workspace_of_a_gated_block(launches, M, D, F):
    import paper_2511_16041_amd as atb
    L = atb.lib()
    for name, size in (("ffn", L.atb_ffn_workspace(M, D, F, 1)), ("ffn_backward", L.atb_ffn_backward_workspace(M, D, F))):
        found = launches(name, M, D, F, 1, 1)
        assert max(one["parts"] * one["planes"] * one["m"] * one["n"] * 4 for one in found if one["parts"] > 1) == size if size else all(one["parts"] == 1 for one in found)


@pytest.mark.parametrize("M,D,F", BLOCKS)
def test_without_a_workspace_large_tiles_are_nearly_as_many_as_cus(launches, M, D, F):
    """Large tiles (512 threads) that are chosen because their shares fill the CUs have no business where there is no room for shares."""
    for name in ("ffn", "ffn_backward"):
        found = launches(name, M, D, F, 0, 1)
        assert all(one["parts"] == 1 for one in found)
        for one in found:
            assert one["block"][0] == 256 or one["grid"][0] * one["grid"][1] >= 192, one


@pytest.mark.parametrize("K,ldx", [(2 ** 22, 2 ** 22), (2 ** 22, 2 ** 26), (128, 2 ** 26), (128, 2 ** 22 + 8)])
def test_4_bit_weights_of_the_longest_rows(launches, K, ldx):
    """K up to 2^22 is documented, and with it rows of x at least that far apart."""
    consecutive(launches("q4", 40, 24, K, 128, 0, ldx, 24), 40, {"x": 2 * ldx, "y": 48})
    consecutive(launches("q4_gated", 40, 24, K, 128, ldx, 24), 40, {"x": 2 * ldx, "y": 48})
