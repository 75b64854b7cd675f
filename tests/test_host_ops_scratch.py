"""The scan's scratch on a runtime without a GPU (test_host_ops): what a call may ask for, whatever its sizes."""
import ctypes as C
import os
import random
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
sys.path.insert(0, ROOT)

from tests.test_host_ops import OK, P, make_library, stub_path  # noqa: E402, F401

BOUND = 260 << 20     # states of the workgroups of four rounds, 256 MiB at most, and the logarithms of their decays


def bounded(stub, vf, ctx):
    """Calls over the whole range of sizes launch the same with allocations of more than BOUND refused as without, and a few of them
    need more than a quarter of it."""
    from paper_2011_14486_amd import binding
    vf.vf_destroy.argtypes = [C.c_void_p]
    rng = random.Random(4)
    large = split = 0
    for _ in range(4000):
        heads = rng.choice([1, 2, 3, 8, 32, 40, 64, 100, 256, 1024])
        groups = rng.choice([g for g in (1, 2, 4, heads) if heads % g == 0])
        p, n = rng.choice([1, 16, 31, 32, 64, 80, 128, 250, 256]), rng.choice([1, 16, 24, 32, 64, 100, 128, 160, 256])
        channels, n_seq = heads * p + 2 * groups * n, rng.choice([1, 1, 2, 3, 7, 50, 300])
        length = int(2 ** rng.uniform(4, 30)) // n_seq + 1
        layer = binding._Ssm(heads, p, groups, n, rng.choice([2, 4, 6]), P, None, P, None, None)
        io = binding._SsmIo(rng.randrange(2), n_seq, 0, 0, n_seq * length, length, None, None, None, P, P, None, P, channels, heads, 0, heads * p,
                            None, None, None, None)
        logs = []
        for refuse in (1 << 62, BOUND + 1, BOUND // 4):
            own = C.c_void_p()
            stub.stub_fail(1, 0)
            assert vf.vf_create(C.byref(own), 0, None) == 0
            stub.stub_fail(refuse, 1 << 62)
            stub.stub_clear()
            assert vf.vf_ssm_scan(own, C.byref(layer), C.byref(io)) == OK
            logs.append(stub.stub_log())
            stub.stub_fail(1, 0)
            vf.vf_destroy(own)
        assert logs[0] == logs[1], (heads, groups, p, n, n_seq, length)
        split += b"k_ssm_join" in logs[0]
        large += logs[0] != logs[2]
    assert split > 1000 and large > 20, (split, large)


def test_scratch_is_bounded(stub_path):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), stub_path], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    bounded(*make_library(sys.argv[1]))
