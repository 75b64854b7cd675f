"""Which attention kernel takes a head's size, and that no lane of it fetches past the end of a cache's row, on a runtime without a GPU.

A lane takes a fixed number of neighbouring numbers of a row; one whose first number lies in the row takes them from there, others from
the row's begin.  (Three numbers at a time, which rows of 80 and 88 do not consist of, are taken from before where they would end behind the row.)  So the
numbers from a first one inside have to lie inside too, for every width that comes to a kernel: the last row of the last page ends with the cache."""
import os
import re
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
sys.path.insert(0, ROOT)

from tests.kv_ref import width_of  # noqa: E402
from tests.test_host_kv import EIGHT, OK, call, library, make_library, names  # noqa: E402
from tests.test_host_ops import stub_path  # noqa: E402, F401


def fetches(name, w):
    """(first numbers, how many) of every fetch of a row of w numbers by the kernel's lanes, and the widest row that it holds."""
    m = re.search(r"k_attend_wideILi(\d)ELi(\d+)E", name)
    if m:
        fmt, DP = int(m[1]), int(m[2])
        VW = DP // 32
        values = [VW * n if VW * n >= w or VW != 3 else min(VW * n, w - VW) for n in range(32)]
        assert set(range(w)) <= {f + x for f in values for x in range(VW)}
        return [([8 * x + 4 * g for x in range(DP // 8) for g in range(2)], 4), (values, VW)], DP
    m = re.search(r"k_attend_rowsI([tf])Li(\d)ELi(\d+)E", name)
    if m:
        f32, fmt, DP = m[1] == "f", int(m[2]), int(m[3])
        VW = (4 if DP >= 64 else DP // 16) if f32 else (8 if DP >= 128 else DP // 16)
        values = [VW * n for n in range(DP // VW)]
        if f32:
            return [(list(range(0, DP, 4)), 4), (values, VW)], DP
        each = 16 if fmt == 2 and DP >= 64 else 8
        return [(list(range(0, DP, each)), each), (values, VW)], DP
    m = re.search(r"k_attend_tileILi(\d)ELi(\d+)E", name)
    assert m, name
    return [(list(range(0, int(m[2]), 8)), 8)], int(m[2])


def widths(stub, vf, ctx):
    """Every head size, type and format, few rows and many, few keys and many."""
    taken = set()
    for kind, fmt in ((0, 0), (1, 1), (0, 2), (1, 2)):
        for dim in range(1, 257):
            w = width_of(fmt, dim)
            for tokens, keys in ((1, 100), (1, 10 ** 5), (300, 100), (300, 5000)):
                stub.stub_clear()
                assert call(vf, ctx, "attend", **dict(EIGHT if fmt == 2 else {}, format=fmt), type=kind, head_dim=dim, n_seq=1, tokens=tokens, ldq=8 * dim, ldo=8 * dim,
                            longest_kv=keys, max_pages=1 << 14, ld_table=1 << 14) == OK
                name = names(stub)[0][0]
                each, widest = fetches(name, w)
                assert widest >= dim, (name, dim)
                for firsts, n in each:
                    assert all(f + n <= w for f in firsts if f < w), (name, dim, w)
                taken.add(re.search(r"k_attend_\w+?ILi\d+ELi\d+E|k_attend_rowsI[tf]Li\dELi\d+E", name)[0])
    assert len(taken) == 16 + 6 + 7, sorted(taken)   # every instance has been asked for


@pytest.mark.parametrize("case", ["widths"])
def test_host_kv_widths(stub_path, case):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), stub_path, case], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    globals()[sys.argv[2]](*library(*make_library(sys.argv[1])))
