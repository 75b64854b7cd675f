"""Sequence operators on a runtime without a GPU (hip_stub.c: launches are written down, not run): what they refuse, and
that a refused call launches nothing."""
import ctypes as C
import os
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
EINVAL, OK, BIG = -1, 0, 1 << 40
P = 1 << 20      # an address that nothing here reads


def make_library(stub_path):
    stub = C.CDLL(stub_path, mode=C.RTLD_GLOBAL)
    stub.stub_log.restype = C.c_char_p
    stub.stub_fail.argtypes = [C.c_size_t, C.c_size_t]
    from paper_2011_14486_amd import binding
    vf = C.CDLL(binding.LIB_PATH)
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    vf.vf_create.argtypes = [C.POINTER(vp), C.c_int, vp]
    vf.vf_rms_norm.argtypes = [vp, i32, vp, i64, vp, i64, vp, C.c_float, i64, i64, vp, i64, i32, vp, i64, vp]
    vf.vf_mx_quantize.argtypes = [vp, i32, vp, i64, i64, i64, i32, vp, vp]
    vf.vf_mx_dequantize.argtypes = [vp, i32, vp, vp, i64, i64, i32, vp, i64]
    vf.vf_mx_matmul.argtypes = [vp, i32, vp, vp, vp, vp, i64, i64, i64, vp, i32, vp, i64]
    vf.vf_ssm_scan.argtypes = vf.vf_ssm_step.argtypes = [vp, vp, vp]
    ctx = vp()
    assert vf.vf_create(C.byref(ctx), 0, None) == 0
    return stub, vf, ctx


def refusals(stub, vf, ctx, fn, good, changes, order):
    """fn(good) launches and returns OK; with any one of the changes it returns VF_EINVAL and launches nothing."""
    stub.stub_clear()
    assert fn(ctx, *(good[k] for k in order)) == OK and stub.stub_log() != b""
    stub.stub_clear()
    assert fn(None, *(good[k] for k in order)) == EINVAL
    for change in changes:
        args = dict(good, **change)
        assert fn(ctx, *(args[k] for k in order)) == EINVAL, change
    assert stub.stub_log() == b""


def norm(stub, vf, ctx):
    order = ["type", "x", "ldx", "res", "ldr", "gain", "eps", "rows", "width", "sum", "lds", "ot", "out", "ldo", "scales"]
    good = dict(type=1, x=P, ldx=100, res=2 * P, ldr=100, gain=3 * P, eps=1e-5, rows=4, width=100, sum=4 * P, lds=100, ot=1, out=5 * P,
                ldo=100, scales=None)
    refusals(stub, vf, ctx, vf.vf_rms_norm, good, [
        dict(type=2), dict(type=-1), dict(ot=4), dict(ot=-1), dict(x=None), dict(out=None), dict(rows=-1), dict(rows=BIG), dict(width=0),
        dict(width=32769, ldx=40000, ldr=40000, lds=40000, ldo=40000), dict(ldx=99), dict(ldr=99), dict(lds=99), dict(ldo=99),
        dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")), dict(x=P + 1), dict(res=P + 1), dict(sum=P + 1), dict(out=P + 1),
        dict(gain=P + 2), dict(sum=P, ldx=101), dict(sum=2 * P, ldr=101), dict(scales=P), dict(ldx=-100)], order)
    mx = dict(good, ot=2, scales=6 * P, ldo=0)
    refusals(stub, vf, ctx, vf.vf_rms_norm, mx, [dict(scales=None), dict(out=5 * P + 8)], order)
    for more in (dict(rows=0, x=None, out=None), dict(res=None, ldr=0, sum=None, lds=0, gain=None)):
        args = dict(good, **more)
        assert vf.vf_rms_norm(ctx, *(args[k] for k in order)) == OK


def microscaled(stub, vf, ctx):
    order = ["type", "x", "ld", "rows", "cols", "fmt", "codes", "scales"]
    good = dict(type=1, x=P, ld=100, rows=4, cols=100, fmt=3, codes=2 * P, scales=3 * P + 1)
    refusals(stub, vf, ctx, vf.vf_mx_quantize, good, [
        dict(type=2), dict(fmt=1), dict(fmt=4), dict(x=None), dict(codes=None), dict(scales=None), dict(codes=P + 8), dict(rows=-1),
        dict(rows=BIG), dict(cols=0), dict(cols=1 << 25, ld=1 << 25), dict(ld=99), dict(x=P + 1)], order)
    order = ["fmt", "codes", "scales", "rows", "cols", "type", "out", "ld"]
    good = dict(fmt=2, codes=2 * P, scales=3 * P, rows=4, cols=100, type=0, out=P, ld=100)
    refusals(stub, vf, ctx, vf.vf_mx_dequantize, good, [
        dict(type=3), dict(fmt=0), dict(codes=None), dict(scales=None), dict(out=None), dict(codes=P + 4), dict(rows=-1), dict(cols=0),
        dict(ld=99), dict(out=P + 2)], order)
    order = ["af", "a", "as", "w", "ws", "M", "N", "K", "bias", "ot", "out", "ld"]
    for M in (1, 40, 5000):
        good = {"af": 2, "a": P, "as": 2 * P, "w": 3 * P, "ws": 4 * P, "M": M, "N": 100, "K": 70, "bias": None, "ot": 1, "out": 5 * P, "ld": 100}
        refusals(stub, vf, ctx, vf.vf_mx_matmul, good, [
            dict(af=1), dict(ot=2), dict(a=None), {"as": None}, dict(w=None), dict(ws=None), dict(out=None), dict(M=-1), dict(M=BIG),
            dict(N=-1), dict(N=1 << 25, ld=1 << 25), dict(K=0), dict(K=1 << 25), dict(ld=99), dict(a=P + 8), dict(w=P + 8), dict(out=P + 1),
            dict(bias=P + 2)], order)
    for more in (dict(M=0), dict(N=0)):
        assert vf.vf_mx_matmul(ctx, *(dict(good, a=None, w=None, out=None, **more)[k] for k in order)) == OK


def scan(stub, vf, ctx):
    from paper_2011_14486_amd import binding
    layer = dict(heads=4, head_dim=64, groups=2, n_state=64, taps=4, conv_w_dev=P, conv_b_dev=None, a_dev=P, d_dev=None, dt_bias_dev=None)
    io = dict(type=1, n_seq=3, n_slots_in=3, n_slots_out=3, tokens=30, longest=10, offsets_dev=None, slots_in_dev=None, slots_out_dev=None,
              xbc_dev=P, dt_dev=P, z_dev=P, out_dev=P, ld_xbc=512, ld_dt=4, ld_z=256, ld_out=256, conv_in_dev=P, ssm_in_dev=P,
              conv_out_dev=9 * P, ssm_out_dev=9 * P)

    def call(fn, **more):
        la, a = dict(layer), dict(io)
        for k, v in more.items():
            (la if k in la else a)[k] = v
        return fn(ctx, C.byref(binding._Ssm(**la)), C.byref(binding._SsmIo(**a)))

    def bad(fn, *changes):
        stub.stub_clear()
        for change in changes:
            assert call(fn, **change) == EINVAL, change
        assert stub.stub_log() == b""

    one = dict(tokens=3)
    for fn, base in ((vf.vf_ssm_scan, {}), (vf.vf_ssm_step, one)):
        stub.stub_clear()
        assert call(fn, **base) == OK and stub.stub_log() != b""
        assert call(fn, offsets_dev=P if fn is vf.vf_ssm_scan else None, n_slots_in=1, slots_in_dev=P, n_slots_out=0, slots_out_dev=P,
                    **base) == OK
        assert call(fn, conv_in_dev=None, ssm_in_dev=None, conv_out_dev=None, ssm_out_dev=None, z_dev=None, ld_z=0, **base) == OK
        assert call(fn, taps=1, conv_in_dev=None, conv_out_dev=None, **base) == OK
        assert fn(None, None, None) == EINVAL and fn(ctx, None, None) == EINVAL
        bad(fn, *(dict(base, **c) for c in (
            dict(heads=0), dict(heads=5), dict(head_dim=0), dict(head_dim=257, ld_xbc=5000, ld_z=5000, ld_out=5000), dict(groups=0),
            dict(groups=3), dict(n_state=0), dict(n_state=257, ld_xbc=5000), dict(taps=0), dict(taps=9), dict(conv_w_dev=None),
            dict(a_dev=None), dict(a_dev=P + 2), dict(d_dev=P + 1), dict(type=2), dict(type=-1), dict(n_seq=-1), dict(tokens=-3),
            dict(tokens=1 << 31, n_seq=1 << 30), dict(longest=-1), dict(xbc_dev=None), dict(dt_dev=None), dict(out_dev=None), dict(xbc_dev=P + 1),
            dict(ld_xbc=511), dict(ld_dt=3), dict(ld_z=255), dict(ld_out=255), dict(conv_in_dev=None), dict(ssm_in_dev=None),
            dict(conv_out_dev=None), dict(ssm_out_dev=None), dict(n_slots_in=2), dict(n_slots_out=2), dict(ssm_in_dev=P + 2),
            dict(conv_in_dev=None, ssm_in_dev=None, slots_in_dev=P), dict(slots_in_dev=P + 2), dict(n_slots_in=-1, slots_in_dev=P))))
    bad(vf.vf_ssm_scan, dict(tokens=31), dict(offsets_dev=P + 2), dict(n_seq=0))
    bad(vf.vf_ssm_step, dict(tokens=30), dict(offsets_dev=P, tokens=3))
    stub.stub_clear()
    assert call(vf.vf_ssm_scan, n_seq=0, tokens=0) == OK and stub.stub_log() == b""


def captured(stub, vf, ctx):
    """A long sequence on a stream that is being captured: the call allocates nothing and launches what needs nothing; behind it the
    split form comes as without a capture."""
    from paper_2011_14486_amd import binding
    layer = binding._Ssm(2, 64, 1, 64, 4, P, None, P, None, None)
    io = binding._SsmIo(1, 1, 0, 0, 20000, 20000, None, None, None, P, P, None, P, 512, 64, 0, 256, None, None, None, None)
    for on in (1, 0):
        stub.stub_capture(on)
        stub.stub_fail(0, (1 << 62) if on else 0)
        if not on:
            stub.stub_fail(1, 0)
        assert vf.vf_ssm_scan(ctx, C.byref(layer), C.byref(io)) == OK
    # no memory for the split: the call goes on without
    stub.stub_capture(0)
    other = C.c_void_p()
    assert vf.vf_create(C.byref(other), 0, None) == 0
    stub.stub_fail(4096, 1 << 62)
    stub.stub_clear()
    assert vf.vf_ssm_scan(other, C.byref(layer), C.byref(io)) == OK and stub.stub_log() != b""
    stub.stub_fail(1, 0)
    vf.vf_destroy.argtypes = [C.c_void_p]
    vf.vf_destroy(other)


def refused_launch(stub, vf, ctx):
    """A launch that the runtime refuses is an error of the call."""
    stub.stub_fail_launch.argtypes = [C.c_char_p, C.c_int]
    stub.stub_fail_launch(b"k_rms_norm", 0)
    assert vf.vf_rms_norm(ctx, 1, P, 100, None, 0, None, 1e-5, 4, 100, None, 0, 1, P, 100, None) == -4
    assert vf.vf_last_hip_error(ctx) != 0
    stub.stub_fail_launch(b"k_mx_quantize", 0)
    assert vf.vf_mx_quantize(ctx, 1, P, 100, 4, 100, 3, P, P) == -4
    stub.stub_fail_launch(b"k_mx_", 0)
    assert vf.vf_mx_matmul(ctx, 3, P, P, P, P, 4, 100, 70, None, 1, P, 100) == -4


@pytest.fixture(scope="module")
def stub_path(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("stub") / "hip_stub.so")
    subprocess.run(["gcc", "-shared", "-fPIC", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-o", out,
                    os.path.join(HERE, "hip_stub.c")], check=True)
    from paper_2011_14486_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2011_14486_amd.build import build_lib
        build_lib()
    return out


@pytest.mark.parametrize("case", ["norm", "microscaled", "scan", "captured", "refused_launch"])
def test_host_ops(stub_path, case):
    # (a process of its own: the stub takes the place of the whole runtime)
    r = subprocess.run([sys.executable, os.path.abspath(__file__), stub_path, case], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


if __name__ == "__main__":
    sys.path.insert(0, ROOT)
    globals()[sys.argv[2]](*make_library(sys.argv[1]))
