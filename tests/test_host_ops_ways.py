"""Which way the sequence operators take, on a runtime without a GPU (test_host_ops): that the sizes of test_gpu_ops_turns are in
large and small tiles, and have workgroups take more than one tile, row or part."""
import ctypes as C
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
sys.path.insert(0, ROOT)

from tests.test_gpu_ops_turns import CHUNKS, LARGE, NORMS, SMALL  # noqa: E402
from tests.test_host_ops import OK, P, make_library, stub_path  # noqa: E402, F401

TILES = {"large": (b"4TileILi4ELi2ELi8E", 256, 256), "small": (b"4TileILi2ELi2ELi4E", 128, 512)}


def launched(stub):
    """(name, workgroups in the first dimension) of what was launched since the last call."""
    lines = [line.split() for line in stub.stub_log().splitlines()]
    stub.stub_clear()
    return [(name, int(x)) for name, x, _ in lines]


def products(stub, vf, ctx):
    stub.stub_clear()
    for sizes, way in ((LARGE, "large"), (SMALL, "small")):
        mark, side, at_once = TILES[way]
        for M, N, K in sizes:
            for af, ot in ((2, 1), (3, 1), (3, 0)):
                assert vf.vf_mx_matmul(ctx, af, P, P, P, P, M, N, K, None, ot, P, N) == OK
                (name, grid), = launched(stub)
                tiles = -(-M // side) * -(-N // side)
                assert b"k_mx_tile" in name and mark in name and grid == min(tiles, at_once), (name, grid)
                assert way == "small" or tiles > 2 * at_once
    assert -(-SMALL[1][0] // 128) * -(-SMALL[1][1] // 128) > 2 * 512


def norms(stub, vf, ctx):
    stub.stub_clear()
    for rows, width in NORMS:
        for ot in range(4):
            assert vf.vf_rms_norm(ctx, 1, P, width, P, width, None, 1e-5, rows, width, None, 0, ot, P, width, P if ot > 1 else None) == OK
            (name, grid), = launched(stub)
            waves = min(max(-(-width // 512), 1), 16)
            held = 4 // waves if waves < 4 else 1        # rows of a workgroup
            assert b"k_rms_norm" in name and grid * held < rows, (rows, width, grid)


def sequences(stub, vf, ctx):
    from paper_2011_14486_amd import binding
    stub.stub_clear()
    for (H, N_P, G, N, W), n in CHUNKS:
        channels = H * N_P + 2 * G * N
        layer = binding._Ssm(H, N_P, G, N, W, P, None, P, None, None)
        io = binding._SsmIo(1, n, n, n, 33 * n, 33, None, None, None, P, P, P, P, channels, H, H * N_P, H * N_P, P, P, 1 << 40, 1 << 40)
        assert vf.vf_ssm_scan(ctx, C.byref(layer), C.byref(io)) == OK
        (name, grid), = launched(stub)
        assert b"k_ssm_chunks" in name and grid < n * G, (name, grid)


@pytest.mark.parametrize("case", ["products", "norms", "sequences"])
def test_ways(stub_path, case):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), stub_path, case], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    globals()[sys.argv[2]](*make_library(sys.argv[1]))
