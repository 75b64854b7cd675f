"""The attention operators on a runtime without a GPU (test_host_ops): what they refuse, that a refused call launches nothing, which way they
take, their scratch, captured streams and missing memory."""
import ctypes as C
import os
import random
import subprocess
import sys

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
sys.path.insert(0, ROOT)

from tests.test_host_ops import BIG, EINVAL, OK, P, make_library, stub_path  # noqa: E402, F401

BOUND = 260 << 20
NAN, INF = float("nan"), float("inf")


def library(stub, vf, ctx):
    vp, i32, i64 = C.c_void_p, C.c_int32, C.c_int64
    vf.vf_kv_append.argtypes = [vp, vp, vp, vp, i32, vp, i64, vp, i64, i32, vp, i64, vp, i64]
    vf.vf_kv_read.argtypes = [vp, vp, vp, i32, vp, i64, vp, i64]
    vf.vf_kv_attend.argtypes = [vp, vp, vp, i32, i32, vp, i64, i32, i32, C.c_float, i64, vp, i64]
    vf.vf_destroy.argtypes = [vp]
    return stub, vf, ctx


KV = dict(format=1, kv_heads=2, head_dim=64, page=16, pages=10, k_dev=P, v_dev=2 * P, k_scales_dev=None, v_scales_dev=None)
SEQS = dict(n_seq=3, max_pages=4, tokens=6, longest=2, ld_table=4, offsets_dev=None, lengths_dev=P, table_dev=P)
ROPE = dict(rotary=64, interleaved=0, freq_dev=P, magnitude=1.0)
APPEND = dict(type=1, k=3 * P, ldk=128, v=4 * P, ldv=128, heads=8, q=5 * P, ldq=512, qo=6 * P, ldqo=512)
READ = dict(type=1, k=3 * P, ldk=128, v=4 * P, ldv=128)
ATTEND = dict(type=1, heads=8, q=5 * P, ldq=512, causal=1, window=0, scale=0.125, longest_kv=64, out=6 * P, ldo=512)
EIGHT = dict(format=2, k_scales_dev=P + 1, v_scales_dev=P + 3)


def call(vf, ctx, what, **more):
    from paper_2011_14486_amd import binding as b
    parts = [dict(KV), dict(SEQS), dict(ROPE), dict({"append": APPEND, "read": READ, "attend": ATTEND}[what])]
    for k, v in more.items():
        hit = [p for p in parts if k in p]
        assert len(hit) == 1 or k == "rope", k
        for p in hit:
            p[k] = v
    kv, seqs = b._Kv(**parts[0]), b._KvSeqs(**parts[1])
    rope = None if more.get("rope", 1) is None else C.byref(b._Rope(**parts[2]))
    args = list(parts[3].values())
    fn = {"append": vf.vf_kv_append, "read": vf.vf_kv_read, "attend": vf.vf_kv_attend}[what]
    return fn(ctx, C.byref(kv), C.byref(seqs), *([rope] if what == "append" else []), *args)


def refused(stub, vf, ctx):
    cache = [dict(format=3), dict(format=-1), dict(kv_heads=0), dict(kv_heads=1 << 17), dict(head_dim=0), dict(head_dim=257, ldk=10 ** 4, ldv=10 ** 4),
             dict(page=8), dict(page=48), dict(page=2048), dict(page=0), dict(pages=0), dict(pages=-4), dict(k_dev=None), dict(v_dev=None),
             dict(k_dev=P + 8), dict(v_dev=P + 2), dict(k_scales_dev=P), dict(format=2), dict(EIGHT, v_scales_dev=None)]
    seqs = [dict(n_seq=-1), dict(tokens=-3), dict(tokens=7), dict(tokens=1 << 31, n_seq=1 << 30), dict(longest=-1), dict(max_pages=-1), dict(ld_table=3),
            dict(ld_table=BIG), dict(max_pages=1 << 27, ld_table=1 << 27), dict(lengths_dev=None), dict(table_dev=None), dict(lengths_dev=P + 2),
            dict(table_dev=P + 1), dict(offsets_dev=P + 2), dict(n_seq=0)]
    rows = [dict(ldk=127), dict(ldv=100), dict(k=P + 1), dict(v=P + 1), dict(ldk=-128), dict(ldk=BIG)]
    own = dict(
        append=[dict(k=None), dict(v=None), dict(heads=-1), dict(heads=0), dict(q=None), dict(qo=None), dict(ldq=511), dict(ldqo=511), dict(q=P + 1), dict(type=2),
                dict(type=-1), dict(type=0), dict(qo=5 * P, ldqo=513), dict(rotary=66), dict(rotary=63), dict(rotary=-2), dict(freq_dev=None),
                dict(freq_dev=P + 4), dict(magnitude=NAN), dict(magnitude=INF)],
        read=[dict(type=2), dict(type=-1)],
        attend=[dict(heads=0), dict(heads=7), dict(heads=-2), dict(q=None), dict(out=None), dict(ldq=511), dict(ldo=511), dict(q=P + 1), dict(out=P + 1), dict(causal=2),
                dict(window=-1), dict(causal=0, window=5), dict(scale=-1.0), dict(scale=NAN), dict(scale=INF), dict(scale=3e38), dict(ldo=-5), dict(longest_kv=-1), dict(type=0), dict(type=3)])
    for what in ("append", "read", "attend"):
        for good in ({}, EIGHT, dict(offsets_dev=P, tokens=7), dict(max_pages=0, ld_table=0, table_dev=None)):
            stub.stub_clear()
            assert call(vf, ctx, what, **good) == OK and stub.stub_log() != b"", (what, good)
        stub.stub_clear()
        for change in cache + seqs + (rows if what != "attend" else []) + own[what]:
            change = {k: v for k, v in change.items() if what != "attend" or k not in ("ldk", "ldv")}
            assert call(vf, ctx, what, **change) == EINVAL, (what, change)
        assert stub.stub_log() == b""
        assert call(vf, ctx, what, n_seq=0, tokens=0) == OK and call(vf, ctx, what, tokens=0) == OK and stub.stub_log() == b""
    for fn, n in ((vf.vf_kv_append, 13), (vf.vf_kv_read, 7), (vf.vf_kv_attend, 12)):
        kinds = fn.argtypes[1:]
        nothing = [None if k is C.c_void_p else 0 for k in kinds]
        assert len(kinds) == n and fn(None, *nothing) == EINVAL and fn(ctx, *nothing) == EINVAL
    # what is allowed
    for what, good in (("append", dict(rope=None)), ("append", dict(rotary=0, freq_dev=None)), ("append", dict(heads=0, q=None, qo=None)), ("append", dict(qo=5 * P)),
                       ("append", dict(tokens=0, k=None, v=None, q=None, qo=None)), ("read", dict(k=None)), ("read", dict(type=0)), ("read", dict(k=None, v=None)),
                       ("attend", dict(causal=0)), ("attend", dict(window=1 << 30)), ("attend", dict(scale=0.0)), ("attend", dict(longest_kv=BIG, longest=BIG)),
                       ("attend", dict(tokens=0, q=None, out=None))):
        assert call(vf, ctx, what, **good) == OK, (what, good)
    # rows of a cache's head are counted in 32 bits
    assert call(vf, ctx, "attend", heads=1 << 16, ldq=BIG >> 10, ldo=BIG >> 10, n_seq=1, tokens=1 << 17, max_pages=1, ld_table=1) == EINVAL


def names(stub):
    lines = [line.split() for line in stub.stub_log().splitlines()]
    stub.stub_clear()
    return [(name.decode(), int(x)) for name, x, _ in lines]


def ways(stub, vf, ctx):
    """Which kernels run, by the sizes that the host knows."""
    long = dict(max_pages=1 << 16, ld_table=1 << 16)
    kinds = {"few": "k_attend_rowsItLi1ELi64ELi1ELi4E", "share": "k_attend_rowsItLi1ELi64ELi1ELi0E", "sequences": "k_attend_rowsItLi1ELi64ELi1ELi2E",
             "group": "k_attend_rowsItLi1ELi64ELi1ELi3E", "find": "k_attend_group", "tile": "k_attend_tileILi1ELi64E", "join": "k_attend_join"}
    for sizes, want in (
            (dict(n_seq=1, tokens=1, longest_kv=64), ["share"]),
            (dict(n_seq=1, tokens=1, longest_kv=1000, **long), ["few"]),
            (dict(n_seq=1, tokens=4, longest_kv=1000, **long), ["few"]),
            (dict(n_seq=1, tokens=1, longest_kv=100000, **long), ["few", "join"]),
            (dict(n_seq=200, tokens=200, longest_kv=100, **long), ["share"]),
            (dict(n_seq=2000, tokens=2000, longest_kv=100, **long), ["sequences"]),
            (dict(n_seq=2000, tokens=2000, longest_kv=1000, **long), ["find", "group"]),
            (dict(n_seq=64, tokens=64, longest_kv=20000, **long), ["find", "group", "join"]),
            (dict(n_seq=5000, tokens=5000, longest_kv=1000, **long), ["sequences"]),          # too many to be sorted
            (dict(n_seq=2000, tokens=2000, offsets_dev=P, longest=1, longest_kv=1000, **long), ["sequences"]),
            (dict(n_seq=1, tokens=5, longest_kv=1000, **long), ["tile", "join"]),
            (dict(n_seq=1, tokens=5, longest_kv=100, **long), ["tile"]),
            (dict(n_seq=1, tokens=8192, longest_kv=8192, **long), ["tile"]),
            (dict(n_seq=1, tokens=1000, longest_kv=8192, **long), ["tile", "join"]),
            (dict(n_seq=100, tokens=5000, longest_kv=50, **long), ["tile"])):
        stub.stub_clear()
        assert call(vf, ctx, "attend", **sizes) == OK
        got = names(stub)
        assert len(got) == len(want) and all(kinds[w] in name for w, (name, _) in zip(want, got)), (sizes, got)
    # fp32: few rows share the keys, more have waves of 32, or of 16 with long heads
    for tokens, dim, way in ((4, 64, "k_attend_rowsIfLi0ELi64ELi1ELi4E"), (5, 64, "k_attend_wideILi0ELi64E"), (5, 96, "k_attend_wideILi0ELi96E"), (5, 200, "k_attend_rowsIfLi0ELi256ELi1ELi1E")):
        assert call(vf, ctx, "attend", type=0, format=0, n_seq=1, tokens=tokens, head_dim=dim, ldq=8 * dim, ldo=8 * dim, longest_kv=1000, **long) == OK
        assert any(way in name for name, _ in names(stub))
    assert call(vf, ctx, "attend", type=0, format=0, n_seq=1, tokens=50, longest_kv=500, **long) == OK
    assert "k_attend_rowsIfLi0ELi64ELi1ELi1E" in names(stub)[0][0]
    # a window bounds the keys that the work is split by
    assert call(vf, ctx, "attend", n_seq=1, tokens=1, longest_kv=100000, window=100, **long) == OK
    assert [("k_attend_rows" in name) for name, _ in names(stub)] == [True]


def scratch(stub, vf, ctx):
    """Over the whole range of sizes no call asks for more than the documented bound; captured, or without memory, it goes on without."""
    rng = random.Random(3)
    split = grouped = 0
    for _ in range(4000):
        kv = rng.choice([1, 2, 3, 8, 40, 128])
        heads, dim = kv * rng.choice([1, 2, 4, 7, 16, 64]), rng.choice([1, 16, 40, 64, 80, 128, 200, 256])
        fmt, n = rng.choice([0, 1, 2]), rng.choice([1, 2, 5, 16, 64, 300, 5000])
        kind = fmt if fmt < 2 else rng.choice([0, 1])
        rows, keys = min(int(2 ** rng.uniform(0, 14)), (1 << 30) // (n * heads // kv)), int(2 ** rng.uniform(0, 20))
        args = dict(EIGHT if fmt == 2 else {}, kv_heads=kv, head_dim=dim, format=fmt, n_seq=n, tokens=n * rows, type=kind, heads=heads, ldq=heads * dim, ldo=heads * dim,
                    longest_kv=keys, max_pages=1 << 16, ld_table=1 << 16)
        logs = []
        for refuse, capturing in ((1 << 62, 0), (BOUND + 1, 0), (4096, 0), (1 << 62, 1)):
            own = C.c_void_p()
            stub.stub_fail(1, 0)
            assert vf.vf_create(C.byref(own), 0, None) == 0
            stub.stub_fail(refuse, 1 << 62)
            stub.stub_capture(capturing)
            stub.stub_clear()
            assert call(vf, own, "attend", **args) == OK, args
            logs.append(stub.stub_log())
            stub.stub_capture(0)
            stub.stub_fail(1, 0)
            vf.vf_destroy(own)
        assert logs[0] == logs[1] and b"k_attend" in logs[2] and b"join" not in logs[3] and b"group" not in logs[3], args
        split += b"join" in logs[0]
        grouped += b"k_attend_group" in logs[0]
    assert split > 200 and grouped > 20, (split, grouped)


def failing(stub, vf, ctx):
    """A launch that the runtime refuses is an error of the call."""
    stub.stub_fail_launch.argtypes = [C.c_char_p, C.c_int]
    for name, what, more in ((b"k_kv_append", "append", {}), (b"k_kv_read", "read", {}), (b"k_attend_rows", "attend", {}),
                             (b"k_attend_tile", "attend", dict(tokens=300)), (b"k_attend_join", "attend", dict(n_seq=1, tokens=1, longest_kv=10 ** 5, max_pages=1 << 16, ld_table=1 << 16)),
                             (b"k_attend_group", "attend", dict(n_seq=2000, tokens=2000, longest_kv=1000, max_pages=1 << 10, ld_table=1 << 10))):
        stub.stub_fail_launch(name, 0)
        assert call(vf, ctx, what, **more) == -4 and vf.vf_last_hip_error(ctx) != 0, name
        assert call(vf, ctx, what, **more) == OK


@pytest.mark.parametrize("case", ["refused", "ways", "scratch", "failing"])
def test_host_kv(stub_path, case):  # noqa: F811
    r = subprocess.run([sys.executable, os.path.abspath(__file__), stub_path, case], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


def test_binding_refuses():
    """What the Python side looks at before the library is asked."""
    import torch
    from paper_2011_14486_amd import binding as vf

    class Ctx:
        pass

    ctx = Ctx()
    ctx.torch, ctx.device = torch, torch.device("cpu")
    cache = Ctx()
    cache.device, cache.head_dim, cache.kv_heads, cache.page, cache.tensors = ctx.device, 64, 2, 16, ()
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)   # noqa: E731
    table, lengths = i32(3, 4), i32(3)
    q, k = torch.zeros((6, 512), dtype=torch.bfloat16), torch.zeros((6, 128), dtype=torch.bfloat16)
    for more in (dict(table=i32(3, 4, 1)), dict(table=table.long()), dict(table=i32(4, 3).t()), dict(lengths=i32(4)), dict(lengths=lengths.long()),
                 dict(lengths=i32(6)[::2]), dict(offsets=i32(3)), dict(table=i32(4, 4), lengths=i32(4)), dict(q=q[:, :100]), dict(q=q.half()), dict(q=q[:, ::2]),
                 dict(window=(1 << 32) + 5), dict(window=-1)):
        args = dict(dict(q=q, table=table, lengths=lengths), **more)
        with pytest.raises(ValueError):
            vf.vf_kv_attend(ctx, cache, args.pop("q"), args.pop("table"), args.pop("lengths"), **args)
    for more in (dict(k=k[:, :64]), dict(v=k.float()), dict(v=k[:5]), dict(q_out=q), dict(q=q.float()), dict(q=q, q_out=k)):
        args = dict(dict(k=k, v=k), **more)
        with pytest.raises(ValueError):
            vf.vf_kv_append(ctx, cache, args.pop("k"), args.pop("v"), table, lengths, **args)
    with pytest.raises(ValueError):
        vf.vf_kv_read(ctx, cache, table, lengths, 7)
    with pytest.raises(ValueError):
        vf.vf_kv_read(ctx, cache, table, lengths, 6, out_type=2)
    other = Ctx()
    other.__dict__.update(cache.__dict__, device=torch.device("meta"))
    with pytest.raises(ValueError):
        vf.vf_kv_attend(ctx, other, q, table, lengths)
    for bad in (dict(fmt=3), dict(head_dim=0), dict(head_dim=300), dict()):   # (tensors that are not on a GPU)
        args = dict(dict(fmt=1, head_dim=64), **bad)
        with pytest.raises(ValueError):
            vf.KvCache(args["fmt"], args["head_dim"], torch.zeros(4, 2, 16, 64).bfloat16(), torch.zeros(4, 2, 16, 64).bfloat16())
    with pytest.raises(ValueError):
        vf.Rope(torch.zeros(4, dtype=torch.float64))


if __name__ == "__main__":
    globals()[sys.argv[2]](*library(*make_library(sys.argv[1])))
