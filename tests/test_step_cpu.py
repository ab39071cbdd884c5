"""Argument checks of the lookup, the layer norm and the AdamW step, before
anything touches a device."""
import ctypes
import os

import pytest

from paper_2108_00951_amd import binding

FAKE = 1 << 20   # never dereferenced: validation fails first
OK, EINVAL, ESPACE = binding.EFS_OK, binding.EFS_EINVAL, binding.EFS_ESPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        pytest.fail("libefsparse.so is not built (run __graft_entry__.build())")
    return binding.declare(ctypes.CDLL(binding.LIB_PATH))


def refused(lib, call, good, bad, want=EINVAL):
    for over in bad:
        a = dict(good, **over)
        assert call(*a.values(), None) == (ESPACE if "nb" in over else want), over
        assert lib.efs_last_error_message()


LOOK = dict(table=FAKE, ld_table=64, table_dtype=0, ids=9 * FAKE, out=5 * FAKE, ld_out=64, dtype=0, tokens=10, vocab=1000,
            width=64, scale=1.0, ignore=-100, status=None)
SPREAD = dict(dout=FAKE, ld_dout=64, dtype=0, ids=9 * FAKE, dtable=5 * FAKE, ld_dtable=64, table_dtype=0, tokens=10, vocab=1000,
              width=64, scale=1.0, ignore=-100, accumulate=0, status=None, ws=12 * FAKE, nb=1 << 20)
BOTH = [dict(ids=None), dict(ids=9 * FAKE + 4), dict(dtype=2), dict(table_dtype=-1), dict(tokens=-1), dict(vocab=0),
        dict(width=0), dict(tokens=2 ** 22 + 1), dict(vocab=2 ** 24 + 1), dict(width=2 ** 18 + 1), dict(status=FAKE * 7 + 2),
        dict(scale=float("nan")), dict(scale=float("inf"))]


def test_lookup_rejects_bad_arguments(lib):
    refused(lib, lib.embed_forward, LOOK, BOTH + [
        dict(table=None), dict(out=None), dict(table=FAKE + 2), dict(out=FAKE + 1, dtype=1), dict(ld_table=63),
        dict(ld_out=63), dict(ld_out=2 ** 31), dict(out=FAKE), dict(out=FAKE + 4 * 63999), dict(ids=5 * FAKE + 8),
        dict(status=5 * FAKE), dict(status=FAKE + 4 * 63999), dict(status=9 * FAKE + 76)])
    assert lib.embed_forward(*dict(LOOK, tokens=0, table=None, ids=None, out=None).values(), None) == OK


def test_table_gradient_rejects_bad_arguments(lib):
    need = lib.embed_workspace_bytes(10, 1000, 64)
    refused(lib, lib.embed_backward, SPREAD, BOTH + [
        dict(dout=None), dict(dtable=None), dict(dout=FAKE + 2), dict(ld_dout=63), dict(ld_dtable=63), dict(ld_dtable=2 ** 31),
        dict(accumulate=2), dict(ws=None), dict(ws=12 * FAKE + 8), dict(nb=need - 1), dict(dtable=FAKE),
        dict(dout=5 * FAKE + 255996), dict(ids=5 * FAKE), dict(ws=5 * FAKE), dict(ws=FAKE), dict(ws=9 * FAKE),
        dict(status=12 * FAKE), dict(status=5 * FAKE + 4), dict(tokens=2 ** 22, vocab=2 ** 17)])
    # nothing to add: no memory is looked at but the table's
    assert lib.embed_backward(*dict(SPREAD, tokens=0, dout=None, ids=None, accumulate=1).values(), None) == OK


def test_other_columns_of_the_same_rows_are_no_overlap(lib):
    """Refused for the workspace alone, which comes after them."""
    a = dict(SPREAD, ld_dout=200, ld_dtable=200, dtable=FAKE + 256, vocab=10, tokens=10, ws=None)
    assert lib.embed_backward(*a.values(), None) == EINVAL
    assert b"workspace" in lib.efs_last_error_message()


def test_embed_workspace_bytes(lib):
    assert lib.embed_workspace_bytes(0, 5, 5) >= 16
    assert lib.embed_workspace_bytes(31, 1000, 4096) < 1024            # no word can be split
    # an eighth of the tokens' rows at most, and what sorting takes
    assert lib.embed_workspace_bytes(2 ** 16, 1000, 4096) <= 2 ** 16 * (4096 * 4 // 16 + 9) + 64
    for bad in ((-1, 5, 5), (2 ** 22 + 1, 5, 5), (5, 0, 5), (5, 2 ** 24 + 1, 5), (5, 5, 0), (5, 5, 2 ** 18 + 1), (2 ** 22, 2 ** 17, 5)):
        assert lib.embed_workspace_bytes(*bad) == 0, bad


NORM = dict(x=FAKE, ld_x=64, weight=2 * FAKE, bias=3 * FAKE, y=4 * FAKE, ld_y=64, dtype=0, weight_dtype=0, rows=100, width=64,
            eps=1e-5, mean=5 * FAKE, rstd=6 * FAKE)
BACK = dict(x=FAKE, ld_x=64, weight=2 * FAKE, mean=5 * FAKE, rstd=6 * FAKE, dy=7 * FAKE, ld_dy=64, dx=8 * FAKE, ld_dx=64,
            dtype=0, weight_dtype=0, rows=100, width=64, dweight=9 * FAKE, dbias=10 * FAKE, ws=11 * FAKE, nb=1 << 20)
SIZES = [dict(dtype=2), dict(weight_dtype=-1), dict(rows=-1), dict(width=0), dict(width=2 ** 18 + 1), dict(x=None),
         dict(x=FAKE + 2), dict(ld_x=63), dict(ld_x=2 ** 31), dict(weight=2 * FAKE + 2), dict(mean=5 * FAKE + 2), dict(rstd=5 * FAKE + 2)]


def test_norm_rejects_bad_arguments(lib):
    refused(lib, lib.layernorm_forward, NORM, SIZES + [
        dict(y=None), dict(ld_y=63), dict(bias=3 * FAKE + 1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
        dict(y=FAKE + 4), dict(y=FAKE, ld_y=65), dict(y=FAKE + 25596), dict(y=2 * FAKE + 4), dict(weight=4 * FAKE),
        dict(bias=4 * FAKE + 252), dict(mean=6 * FAKE + 4), dict(mean=FAKE + 400), dict(rstd=4 * FAKE), dict(rstd=3 * FAKE)])
    assert lib.layernorm_forward(*dict(NORM, rows=0, x=None, y=None).values(), None) == OK


def test_norm_gradients_reject_bad_arguments(lib):
    need = lib.layernorm_workspace_bytes(100, 64)
    refused(lib, lib.layernorm_backward, BACK, SIZES + [
        dict(dy=None), dict(dx=None), dict(mean=None), dict(rstd=None), dict(ld_dy=63), dict(ld_dx=63), dict(dx=7 * FAKE + 4),
        dict(dx=FAKE + 4), dict(dx=7 * FAKE, ld_dx=65), dict(dweight=9 * FAKE + 2), dict(dbias=9 * FAKE + 2), dict(dbias=9 * FAKE),
        dict(dweight=2 * FAKE), dict(dbias=7 * FAKE), dict(dweight=8 * FAKE + 400), dict(dx=5 * FAKE), dict(dweight=6 * FAKE),
        dict(ws=None), dict(ws=11 * FAKE + 8), dict(nb=need - 1), dict(ws=FAKE), dict(ws=9 * FAKE), dict(ws=5 * FAKE + 16)])
    assert lib.layernorm_backward(*dict(BACK, rows=0, x=None, dy=None, dx=None, dweight=None, dbias=None).values(), None) == OK
    for bad in ((-1, 5), (5, 0), (5, 2 ** 18 + 1)):
        assert lib.layernorm_workspace_bytes(*bad) == 0, bad


class Lists:
    """adamw_apply with three tensors, 300 floats each, every list in its own place."""

    def __init__(self, lib):
        self.lib = lib
        self.at = {k: [(i + 1) * 100 * FAKE + n * 8192 for n in range(3)] for i, k in enumerate("gxmvc")}
        self.good = dict(gtype=0, state=0, sizes=[300] * 3, decays=[0.1] * 3, count=3, lr=1e-3, b1=0.9, b2=0.99, eps=1e-8, step=1,
                         step_device=None, factors=None, seed=0)

    def call(self, lists=(), **over):
        a = dict(self.good, **over)
        at = {k: list(v) for k, v in self.at.items()}
        for k, n, p in lists:
            if n is None:
                at[k] = None
            else:
                at[k][n] = p
        arr = {k: None if v is None else (ctypes.c_void_p * 3)(*v) for k, v in at.items()}
        sizes = None if a["sizes"] is None else (ctypes.c_int64 * 3)(*a["sizes"])
        decays = None if a["decays"] is None else (ctypes.c_float * 3)(*a["decays"])
        return self.lib.adamw_apply(arr["g"], a["gtype"], arr["x"], arr["c"], arr["m"], arr["v"], a["state"], sizes, decays,
                                    a["count"], a["lr"], a["b1"], a["b2"], a["eps"], a["step"], a["step_device"], a["factors"],
                                    a["seed"], None)


def test_adamw_rejects_bad_arguments(lib):
    c = Lists(lib)
    inf, nan = float("inf"), float("nan")
    for over in (dict(gtype=2), dict(state=2), dict(state=-1), dict(sizes=None), dict(sizes=[1, -1, 1]),
                 dict(sizes=[1, 2 ** 31, 1]), dict(decays=[0.0, nan, 0.0]), dict(count=-1), dict(count=65537), dict(lr=nan),
                 dict(lr=inf), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=nan), dict(eps=-1e-8), dict(eps=nan),
                 dict(step=0), dict(step_device=FAKE + 4), dict(factors=FAKE + 2)):
        assert c.call(**over) == EINVAL, over
        assert lib.efs_last_error_message()
    for k in "gxmv":
        assert c.call([(k, None, None)]) == EINVAL
        assert c.call([(k, 1, None)]) == EINVAL
        assert c.call([(k, 1, c.at[k][1] + 2)]) == EINVAL
    assert c.call([("c", 1, c.at["c"][1] + 1)]) == EINVAL
    for k in "mv":   # states of 8 bits to 16 bytes
        assert c.call([(k, 1, c.at[k][1] + 8)], state=1) == EINVAL
    assert c.call(count=0, sizes=None) == OK
    assert c.call([(k, n, None) for k in "gxmv" for n in range(3)], sizes=[0, 0, 0]) == OK


@pytest.mark.parametrize("descending", [False, True])
def test_adamw_refuses_what_overlaps(lib, descending):
    c = Lists(lib)
    if descending:   # lists that are not in the order of their addresses
        c.at = {k: v[::-1] for k, v in c.at.items()}
    for written in "xmvc":
        for other in "gxmvc":
            for shift in (0, 4, 596 if "c" in (written, other) else 1196):
                for n in range(3):
                    if other == written:
                        lists = [(written, n, c.at[written][(n + 1) % 3] + shift)]
                    else:
                        lists = [(written, n, c.at[other][1] + shift)]
                    assert c.call(lists) == EINVAL, (written, other, shift, n)
                    assert b"must not overlap" in lib.efs_last_error_message()


def test_adamw_refuses_rates_among_what_it_writes(lib):
    c = Lists(lib)
    for k in "xmvc":
        for n in range(3):
            for at in (c.at[k][n], c.at[k][n] + 592):
                for what in ("step_device", "factors"):
                    assert c.call(**{what: at}) == EINVAL
                    assert b"must not overlap" in lib.efs_last_error_message()


def test_reading_states_rejects_bad_arguments(lib):
    at = {k: [(i + 1) * 100 * FAKE + n * 8192 for n in range(2)] for i, k in enumerate(("m8", "v8", "m", "v"))}

    def call(fn, over=None, sizes=(300, 300), count=2):
        a = {k: list(v) for k, v in at.items()}
        for k, n, p in over or ():
            a[k][n] = p
        arr = {k: (ctypes.c_void_p * 2)(*v) for k, v in a.items()}
        order = ("m8", "v8", "m", "v") if fn is lib.adamw_read_state else ("m", "v", "m8", "v8")
        return fn(*(arr[k] for k in order), (ctypes.c_int64 * 2)(*sizes), count, None)
    for fn in (lib.adamw_read_state, lib.adamw_write_state):
        assert call(fn, sizes=(300, -1)) == EINVAL
        assert call(fn, count=-1) == EINVAL
        assert call(fn, count=0) == OK
        for k in at:
            assert call(fn, [(k, 1, None)]) == EINVAL
            assert call(fn, [(k, 1, at[k][1] + (8 if k in ("m8", "v8") else 2))]) == EINVAL
        # 512 codes and two floats against 1,200 bytes
        assert call(fn, [("m", 0, at["m8"][1] + 516)]) == EINVAL
        assert call(fn, [("v8", 1, at["v"][0] + 1184)]) == EINVAL
        assert b"must not overlap" in lib.efs_last_error_message()


def test_state_bytes(lib):
    for n, want in ((0, 0), (1, 260), (256, 260), (257, 520), (1000, 4 * 260)):
        assert lib.adamw_state_bytes(n) == want
    assert lib.adamw_state_bytes(-1) == 0 and lib.adamw_state_bytes(2 ** 31) == 0
    assert lib.adamw_state_bytes(2 ** 31 - 1) == 2 ** 23 * 260


def test_sizes_past_32_bits_do_not_wrap():
    for sizes in ((2 ** 32 + 3, 50, 8), (3, 2 ** 32 + 50, 8), (3, 50, 2 ** 31)):
        with pytest.raises(ValueError, match="32 bits"):
            binding.embed_workspace_bytes(*sizes)
    for sizes in ((2 ** 32 + 3, 8), (3, 2 ** 31)):
        with pytest.raises(ValueError, match="32 bits"):
            binding.layernorm_workspace_bytes(*sizes)


def test_no_workspace_for_sizes_that_no_call_takes():
    for sizes in ((-1, 50, 8), (3, 0, 8), (3, 50, 2 ** 18 + 1)):
        with pytest.raises(ValueError, match="out of range"):
            binding.new_embed_workspace(*sizes, "cpu")
    for sizes in ((-1, 8), (3, 0)):
        with pytest.raises(ValueError, match="out of range"):
            binding.new_layernorm_workspace(*sizes, "cpu")
    with pytest.raises(ValueError, match="out of range"):
        binding.new_adamw_state([5, -1], "cpu")
    m, v = binding.new_adamw_state([5, 0, 300], "cpu")
    assert [t.numel() for t in m] == [260, 0, 520] and all(t.data_ptr() % 16 == 0 for t in m + v if t.numel())


def test_tensors_off_the_device_or_of_another_type_are_refused():
    import torch
    f, i = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(TypeError, match="device tensor"):
        binding.embed_forward(f, i, f.clone())
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        binding.embed_forward(f.half(), i, f.clone())
    with pytest.raises(ValueError, match="width"):
        binding.embed_forward(f, i, torch.zeros(4, 7))
    with pytest.raises(TypeError, match="device tensor"):
        binding.layernorm_forward(f, None, None, f.clone())
    with pytest.raises(TypeError, match="one dtype"):
        binding.layernorm_forward(f, None, None, f.bfloat16())
    with pytest.raises(ValueError, match="width"):
        binding.layernorm_backward(f, None, f[:, 0], f[:, 0], f[:, :7], f, None, None, None)


def test_lists_of_other_tensors_are_refused():
    import torch
    f = torch.zeros(3)
    for lists, error, match in ((([f], [f], [f], [f]), TypeError, "device tensor"), (([f.half()], [f], [f], [f]), TypeError, "must be"),
                                (([f], [f, f], [f], [f]), ValueError, "as many"), (([None], [f], [f], [f]), TypeError, "None")):
        with pytest.raises(error, match=match):
            binding.prepare_adamw_apply(*lists, lr=1e-3)
    with pytest.raises(ValueError, match="as many"):
        binding.adamw_read_state([], [], [f], [f])


@pytest.mark.parametrize("size", [2 ** 64 + 5, 2 ** 63, -2 ** 64 + 5])
def test_sizes_past_64_bits_do_not_wrap(size):
    with pytest.raises(ValueError, match="64 bits"):
        binding.adamw_state_bytes(size)
    with pytest.raises(ValueError, match="64 bits"):
        binding.new_adamw_state([3, size], "cpu")
