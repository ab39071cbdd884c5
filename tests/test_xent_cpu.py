"""Argument checks of the cross entropy, before anything touches a device."""
import ctypes
import os

import pytest

from paper_2108_00951_amd import binding

FAKE = 1 << 20   # never dereferenced: validation fails first


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        pytest.fail("libefsparse.so is not built (run __graft_entry__.build())")
    return binding.declare(ctypes.CDLL(binding.LIB_PATH))


def test_workspace_bytes(lib):
    forward = lib.xent_workspace_bytes(100, 5000, 64, 0, 0)
    assert 0 < forward < lib.xent_workspace_bytes(100, 5000, 64, 0, 1)
    assert lib.xent_workspace_bytes(0, 5000, 64, 1, 1) > 0
    for bad in ((-1, 5000, 64, 0, 0), (2 ** 22 + 1, 5, 64, 0, 0), (100, 0, 64, 0, 0), (100, 2 ** 24 + 1, 64, 0, 0),
                (100, 5000, 0, 0, 0), (100, 5000, 2 ** 18 + 1, 0, 0), (100, 5000, 64, 2, 0), (100, 5000, 64, 0, 2),
                (2 ** 22, 2 ** 17, 64, 0, 0)):
        assert lib.xent_workspace_bytes(*bad) == 0, bad
    # the logits are not kept: a large vocabulary's pieces stay far below them
    tokens, vocab = 65536, 131072
    assert lib.xent_workspace_bytes(tokens, vocab, 64, 1, 1) < 2 * tokens * vocab / 4


GOOD = dict(h=FAKE, ld_h=64, w=4 * FAKE, ld_w=64, target=FAKE, dtype=0, tokens=10, vocab=1000, hidden=64, ignore=-100)
BAD = [dict(h=None), dict(w=None), dict(h=FAKE + 2), dict(dtype=1, w=FAKE + 1), dict(ld_h=63), dict(ld_w=63),
       dict(ld_w=2 ** 31), dict(target=None), dict(target=FAKE + 4), dict(dtype=2), dict(tokens=-1), dict(vocab=0),
       dict(hidden=0), dict(tokens=2 ** 23), dict(ws=None), dict(ws=FAKE + 8)]


def test_forward_rejects_bad_arguments(lib):
    need = lib.xent_workspace_bytes(10, 1000, 64, 0, 0)
    good = dict(GOOD, loss=FAKE, lse=FAKE, ws=FAKE, nb=need)
    for over in BAD + [dict(loss=None), dict(lse=None), dict(lse=FAKE + 2), dict(nb=need - 1)]:
        a = dict(good, **over)
        rc = lib.xent_forward(*(a[k] for k in GOOD), a["loss"], a["lse"], a["ws"], a["nb"], None)
        assert rc == (binding.EFS_ESPACE if "nb" in over else binding.EFS_EINVAL), over
        assert lib.efs_last_error_message()
    assert lib.xent_forward(None, 64, None, 64, None, 0, 0, 1000, 64, -100, None, None, None, 0,
                            None) == binding.EFS_OK


def test_backward_rejects_bad_arguments(lib):
    need = lib.xent_workspace_bytes(10, 1000, 64, 0, 1)
    good = dict(GOOD, lse=FAKE, dloss=FAKE, dh=8 * FAKE, ld_dh=64, dw=16 * FAKE, ld_dw=64, ws=FAKE, nb=need)
    more = [dict(lse=None), dict(dloss=None), dict(dh=None), dict(dw=None), dict(dh=8 * FAKE + 2), dict(ld_dh=63),
            dict(ld_dw=63), dict(dh=FAKE), dict(dw=4 * FAKE), dict(dw=4 * FAKE + 255996), dict(dh=16 * FAKE + 512),
            dict(nb=need - 1)]
    for over in BAD + more:
        a = dict(good, **over)
        rc = lib.xent_backward(*(a[k] for k in GOOD), a["lse"], a["dloss"], a["dh"], a["ld_dh"], a["dw"], a["ld_dw"],
                               a["ws"], a["nb"], None)
        assert rc == (binding.EFS_ESPACE if "nb" in over else binding.EFS_EINVAL), over


def test_backward_refuses_shared_elements_of_the_same_rows(lib):
    need = lib.xent_workspace_bytes(10, 1000, 64, 0, 1)
    args = dict(GOOD, ld_h=128, ld_w=128)
    h, w = args["h"], args["w"]
    for dh, dw in ((h + 252, w + 256), (h + 256, w + 260), (h + 256, w - 252), (h + 256 + 512 * 9 + 4, w + 256 + 512 * 9 + 4)):
        rc = lib.xent_backward(*(args[k] for k in GOOD), FAKE, FAKE, dh, 128, dw, 128, FAKE, need, None)
        assert rc == binding.EFS_EINVAL, (dh - h, dw - w)
        assert b"must not overlap" in lib.efs_last_error_message()


def test_few_tokens_need_no_copy_of_the_head(lib):
    vocab, hidden = 131072, 4096
    for dtype, head in ((0, vocab * hidden * 4), (1, vocab * hidden * 2)):
        assert lib.xent_workspace_bytes(1, vocab, hidden, dtype, 0) < 2 ** 20
        assert lib.xent_workspace_bytes(64, vocab, hidden, dtype, 0) < head / 100
        assert lib.xent_workspace_bytes(1, vocab, hidden, dtype, 1) < head / 50
        assert lib.xent_workspace_bytes(64, vocab, hidden, dtype, 1) < head / 8
        # more tokens: a copy along the rows, and for the gradients one along the columns
        assert lib.xent_workspace_bytes(129, vocab, hidden, dtype, 0) > head
        assert lib.xent_workspace_bytes(65, vocab, hidden, dtype, 1) > 2 * head
    assert lib.xent_workspace_bytes(128, vocab, hidden, 0, 0) < vocab * hidden / 50
    assert lib.xent_workspace_bytes(65, vocab, hidden, 1, 0) > vocab * hidden * 2


def test_what_is_written_meets_nothing_else(lib):
    """h 2,560 bytes, w 256,000, the vectors 40 and 80, at places of their own;
    one of them moved into another by an element."""
    at = dict(h=FAKE, w=4 * FAKE, target=5 * FAKE, loss=6 * FAKE, lse=7 * FAKE, dloss=8 * FAKE, dh=9 * FAKE, dw=10 * FAKE,
              ws=12 * FAKE)

    def call(gradient, **over):
        a = dict(at, **over)
        head = (a["h"], 64, a["w"], 64, a["target"], 0, 10, 1000, 64, -100)
        need = lib.xent_workspace_bytes(10, 1000, 64, 0, int(gradient))
        if gradient:
            return lib.xent_backward(*head, a["lse"], a["dloss"], a["dh"], 64, a["dw"], 64, a["ws"], need, None)
        return lib.xent_forward(*head, a["loss"], a["lse"], a["ws"], need, None)
    forward = [dict(loss=at["lse"]), dict(loss=at["lse"] + 36), dict(lse=at["loss"] - 36), dict(loss=at["h"] + 2556),
               dict(lse=at["w"] - 36), dict(lse=at["w"] + 255996), dict(loss=at["target"] + 76), dict(loss=at["ws"]),
               dict(lse=at["ws"] - 36), dict(ws=at["h"]), dict(ws=at["w"] + 16), dict(ws=at["target"])]
    backward = [dict(lse=at["dh"]), dict(dloss=at["dh"] + 2556), dict(lse=at["dw"] - 36), dict(dloss=at["dw"] + 255996),
                dict(target=at["dw"]), dict(target=at["dh"] - 72), dict(dloss=at["ws"]), dict(lse=at["ws"] - 36),
                dict(ws=at["dw"]), dict(ws=at["dh"]), dict(ws=at["h"] + 2544), dict(dh=at["dw"]), dict(dw=at["w"])]
    for gradient, cases in ((False, forward), (True, backward)):
        for over in cases:
            assert call(gradient, **over) == binding.EFS_EINVAL, over
            assert b"must not overlap" in lib.efs_last_error_message(), over


def test_sizes_past_32_bits_do_not_wrap():
    import torch
    for sizes in ((2 ** 32 + 3, 50, 8), (3, 2 ** 32 + 50, 8), (3, 50, 2 ** 31)):
        with pytest.raises(ValueError, match="32 bits"):
            binding.xent_workspace_bytes(*sizes, torch.float32)


def test_no_workspace_for_sizes_that_no_call_takes():
    import torch
    for sizes in ((-1, 50, 8), (3, 0, 8), (3, 50, 2 ** 18 + 1)):
        with pytest.raises(ValueError, match="out of range"):
            binding.new_xent_workspace(*sizes, torch.float32, "cpu")
    assert binding.new_xent_workspace(0, 50, 8, torch.float32, "cpu").numel() >= 16
