"""Argument checks of the orthogonalised update, before anything touches a device."""
import ctypes
import os

import pytest

from paper_2108_00951_amd import binding

FAKE = 0x10000   # never dereferenced: validation fails first
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        pytest.fail("libefsparse.so is not built (run __graft_entry__.build())")
    return binding.declare(ctypes.CDLL(binding.LIB_PATH))


def i32(*v):
    return (ctypes.c_int32 * max(len(v), 1))(*v)


def i64(*v):
    return (ctypes.c_int64 * max(len(v), 1))(*v)


def test_workspace_bytes(lib):
    one = lib.muon_workspace_bytes(1, i32(96), i32(96))
    # two X, two X^T, A and B, four bytes a value
    assert one >= 6 * 96 * 96 * 4
    assert lib.muon_workspace_bytes(2, i32(96, 96), i32(96, 96)) > one
    assert lib.muon_workspace_bytes(1, i32(-1), i32(64)) == 0
    assert lib.muon_workspace_bytes(1, i32(65536), i32(32768)) == 0
    assert lib.muon_workspace_bytes(65537, None, None) == 0
    assert lib.muon_workspace_bytes(1, None, i32(4)) == 0


def test_orthogonalize_rejects_bad_arguments(lib):
    need = lib.muon_workspace_bytes(3, i32(80, 80, 80), i32(100, 100, 100))
    good = dict(g=FAKE, ldg=100, sg=8000, o=FAKE, ldo=100, so=8000, dtype=0, batch=3, rows=80, cols=100, steps=5,
                co=None, eps=1e-7, ws=FAKE, nb=need)
    bad = [dict(dtype=2), dict(dtype=-1), dict(batch=-1), dict(batch=65537), dict(rows=-1), dict(cols=-1),
           dict(rows=65536, cols=65536), dict(g=None), dict(o=None), dict(g=FAKE + 2), dict(o=FAKE + 1),
           dict(dtype=1, g=FAKE + 1), dict(ldg=99), dict(ldo=99), dict(sg=-1), dict(so=-8000), dict(so=7999), dict(so=0),
           dict(sg=2 ** 62), dict(steps=0), dict(steps=65), dict(eps=-1.0), dict(eps=NAN), dict(eps=INF),
           dict(co=(ctypes.c_float * 3)(1, NAN, 0)), dict(ws=None), dict(ws=FAKE + 8)]
    for over in bad + [dict(nb=need - 1)]:
        a = dict(good, **over)
        rc = lib.muon_orthogonalize(a["g"], a["ldg"], a["sg"], a["o"], a["ldo"], a["so"], a["dtype"], a["batch"],
                                    a["rows"], a["cols"], a["steps"], a["co"], a["eps"], a["ws"], a["nb"], None)
        assert rc == (binding.EFS_ESPACE if "nb" in over else binding.EFS_EINVAL), over
        assert lib.efs_last_error_message()
    # rows of the matrices in turn do not overlap: only the workspace is refused
    rc = lib.muon_orthogonalize(FAKE, 300, 100, FAKE, 300, 100, 0, 3, 80, 100, 5, None, 1e-7, FAKE, 0, None)
    assert rc == binding.EFS_ESPACE
    for batch, rows, cols in ((0, 80, 100), (3, 0, 100), (3, 80, 0)):
        assert lib.muon_orthogonalize(None, 100, 0, None, 100, 0, 0, batch, rows, cols, 5, None, 1e-7, None, 0,
                                      None) == binding.EFS_OK


def test_apply_rejects_bad_arguments(lib):
    rows, cols, off = i32(4, 70), i32(6, 75), i64(0, 24)
    need = lib.muon_workspace_bytes(2, rows, cols)
    a0, x0, m0 = FAKE, FAKE + 65536, FAKE + 131072
    good = dict(avg=a0, x=x0, m=m0, d=6000, n=2, off=off, rows=rows, cols=cols, beta=0.9, gamma=0.1, decay=0.0,
                nest=1, steps=5, eps=1e-7, ws=FAKE, nb=need)
    bad = [dict(avg=None), dict(x=None), dict(m=None), dict(avg=a0 + 2), dict(d=-1), dict(d=2 ** 31), dict(d=5273),
           dict(n=-1), dict(n=65537), dict(off=None), dict(rows=None), dict(cols=None), dict(off=i64(0, 23)),
           dict(off=i64(-1, 24)), dict(off=i64(24, 0)), dict(rows=i32(4, -70)), dict(rows=i32(4, 2 ** 30)),
           dict(beta=NAN), dict(gamma=INF), dict(decay=NAN), dict(nest=2), dict(steps=0), dict(steps=65),
           dict(eps=-1.0), dict(ws=None), dict(ws=FAKE + 4), dict(x=a0 + 23996), dict(m=x0), dict(m=a0 - 23996)]
    for over in bad + [dict(nb=need - 1)]:
        a = dict(good, **over)
        rc = lib.muon_apply(a["avg"], a["x"], a["m"], a["d"], a["n"], a["off"], a["rows"], a["cols"], a["beta"],
                            a["gamma"], a["decay"], a["nest"], a["steps"], a["eps"], a["ws"], a["nb"], None)
        assert rc == (binding.EFS_ESPACE if "nb" in over else binding.EFS_EINVAL), over
    assert lib.muon_apply(None, None, None, 0, 0, None, None, None, 0.9, 0.1, 0.0, 1, 5, 1e-7, None, 0,
                          None) == binding.EFS_OK


def test_orthogonalize_takes_g_itself_and_no_other_overlap(lib):
    def call(g, ldg, sg, o, ldo, so, batch=3):
        return lib.muon_orthogonalize(g, ldg, sg, o, ldo, so, 0, batch, 80, 100, 5, None, 1e-7, FAKE, 0, None)
    # accepted: only the workspace is refused
    for good in ((FAKE, 100, 8000, FAKE, 100, 8000), (FAKE, 100, 8000, FAKE + 96000, 100, 8000),
                 (FAKE, 100, 0, FAKE + 32000, 100, 8000),
                 (FAKE, 250, 20000, FAKE + 400, 250, 20000), (FAKE + 400, 250, 20000, FAKE, 250, 40000),
                 (FAKE, 100, 8000, FAKE + 4, 100, 8000, 1)):
        assert call(*good) == binding.EFS_ESPACE, good
    for bad in ((FAKE, 100, 0, FAKE, 100, 8000), (FAKE, 100, 8000, FAKE + 32000, 100, 8000),
                (FAKE + 95996, 100, 8000, FAKE, 100, 8000), (FAKE, 100, 8000, FAKE, 100, 16000),
                (FAKE, 250, 20000, FAKE + 396, 250, 20000), (FAKE + 604, 250, 20000, FAKE, 250, 20000),
                (FAKE, 250, 20100, FAKE + 400, 250, 20100)):
        assert call(*bad) == binding.EFS_EINVAL, bad
        assert b"overlaps g" in lib.efs_last_error_message()


def test_workspace_of_the_longest_axes(lib):
    """Where the padded axis passes 32 bits a matrix is still one of the large
    ones: two X of four bytes a value, and two X^T of 128 bytes a row."""
    for n in (2 ** 31 - 17, 2 ** 31 - 16, 2 ** 31 - 15, 2 ** 31 - 2, 2 ** 31 - 1):
        for rows, cols in ((1, n), (n, 1)):
            assert lib.muon_workspace_bytes(1, i32(rows), i32(cols)) > 2 * (4 + 128) * n, (rows, cols)
        # and a call with less is refused before it reaches a device
        assert lib.muon_orthogonalize(FAKE, n, 0, FAKE, n, 0, 0, 1, 1, n, 5, None, 1e-7, FAKE, 2 ** 20,
                                      None) == binding.EFS_ESPACE
        assert lib.muon_apply(FAKE, 2 ** 34, 2 ** 35, n, 1, i64(0), i32(1), i32(n), 0.9, 0.1, 0.0, 1, 5, 1e-7, FAKE,
                              2 ** 20, None) == binding.EFS_ESPACE


def test_workgroups_of_the_longest_axes_are_counted(lib):
    """A 1 x n of about 2^31 values takes 33.5 M tiles of 64 values, twice: more
    than a grid has in a batch of 200, at every n."""
    for n in (2 ** 31 - 1024, 2 ** 31 - 256, 2 ** 31 - 60, 2 ** 31 - 1):
        for rows, cols in ((1, n), (n, 1)):
            assert lib.muon_workspace_bytes(200, i32(*[rows] * 200), i32(*[cols] * 200)) == 0, (rows, cols)
            assert lib.muon_workspace_bytes(20, i32(*[rows] * 20), i32(*[cols] * 20)) > 20 * 264 * n, (rows, cols)


def test_orthogonalize_into_other_columns_of_the_same_rows(lib):
    def call(rows, ldg, sg, o, ldo, so):
        return lib.muon_orthogonalize(FAKE, ldg, sg, o, ldo, so, 0, 3, rows, 100, 5, None, 1e-7, FAKE, 0, None)
    # accepted (only the workspace is refused): matrices whose rows take turns, matrices of one row
    for good in ((80, 600, 100, FAKE + 1200, 600, 100), (1, 100, 200, FAKE + 400, 100, 200),
                 (1, 200, 200, FAKE + 400, 100, 200), (1, 100, 0, FAKE + 400, 100, 100)):
        assert call(*good) == binding.EFS_ESPACE, good
    for bad in ((80, 600, 100, FAKE + 1196, 600, 100), (80, 600, 100, FAKE + 1204, 600, 100),
                (80, 600, 100, FAKE + 1200, 500, 100), (1, 100, 200, FAKE + 396, 100, 200),
                (1, 100, 200, FAKE + 404, 100, 200), (1, 100, 50, FAKE + 400, 100, 200)):
        assert call(*bad) == binding.EFS_EINVAL, bad
        assert b"overlaps g" in lib.efs_last_error_message()


def test_the_workspace_meets_nothing_else(lib):
    need = lib.muon_workspace_bytes(2, i32(80, 80), i32(100, 100))
    for g, out, ws in ((FAKE, 2 ** 24, FAKE + 63984), (2 ** 24, FAKE, FAKE), (FAKE, 2 ** 24, 2 ** 24 - need // 16 * 16 + 16)):
        rc = lib.muon_orthogonalize(g, 100, 8000, out, 100, 8000, 0, 2, 80, 100, 5, None, 1e-7, ws, need, None)
        assert rc == binding.EFS_EINVAL and b"must not overlap" in lib.efs_last_error_message()
    need = lib.muon_workspace_bytes(1, i32(80), i32(100))
    for k in range(3):
        at = [2 ** 24, 2 ** 25, 2 ** 26]
        rc = lib.muon_apply(*at, 8000, 1, i64(0), i32(80), i32(100), 0.9, 0.1, 0.0, 1, 5, 1e-7, at[k] + 31984, need, None)
        assert rc == binding.EFS_EINVAL and b"must not overlap" in lib.efs_last_error_message()


def test_sizes_past_32_bits_do_not_wrap():
    for shape in ((2 ** 32 + 3, 5), (5, 2 ** 32 + 3), (2 ** 31, 1), (-2 ** 32 + 3, 5)):
        with pytest.raises(ValueError, match="32 bits"):
            binding.muon_workspace_bytes([(4, 4), shape])
        with pytest.raises(ValueError, match="32 bits"):
            binding.new_muon_workspace([shape], "cpu")


def test_no_workspace_for_matrices_that_no_call_takes():
    for shapes in ([(65536, 65536)], [(-1, 4)], [(2, 2)] * 65537):
        assert binding.muon_workspace_bytes(shapes) == 0
        with pytest.raises(ValueError, match="out of range"):
            binding.new_muon_workspace(shapes, "cpu")
    assert binding.new_muon_workspace([], "cpu").numel() >= 16
    assert binding.new_muon_workspace([(0, 5)], "cpu").numel() >= 16
