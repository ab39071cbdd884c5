"""Lookup of words' vectors and the gradient of their table against plain 64-bit
forms."""
import numpy as np
import pytest

from tests import _step
from tests._checks import assert_bits_equal

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2108_00951_amd import binding as efs  # noqa: E402

DEV = "cuda"
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
PAIRS = [("fp32", "fp32"), ("bf16", "fp32"), ("fp32", "bf16"), ("bf16", "bf16")]


def say(*a):
    print(*a, flush=True)


def draw(rng, shape, kind):
    return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(TYPES[kind])


def words(rng, tokens, vocab, kind):
    if kind == "same":
        ids = np.full(tokens, vocab // 2)
    elif kind == "zipf":
        ids = np.minimum(np.exp(rng.random(tokens) * np.log(vocab)).astype(np.int64), vocab) - 1
    elif kind == "runs":   # words of 31, 32 and 33 tokens, and those of the table's ends
        ids = np.repeat(np.arange(vocab)[::-1], 31 + np.arange(vocab) % 3)[:tokens]
        ids = np.concatenate([ids, np.zeros(tokens - ids.size, np.int64)])[rng.permutation(tokens)]
    else:
        ids = rng.integers(0, vocab, tokens)
    ids = ids.astype(np.int64)
    if kind == "holes":
        ids[rng.random(tokens) < 0.4] = -100
        ids[rng.random(tokens) < 0.1] = vocab
        ids[rng.random(tokens) < 0.1] = -(2 ** 40)
    return ids


def check_forward(table, ids, out_dtype, scale=1.0, ignore=-100, status=None):
    out = torch.full((ids.size, table.shape[1]), 7.0, dtype=TYPES[out_dtype], device=DEV)
    efs.embed_forward(table.to(DEV), torch.from_numpy(ids).to(DEV), out, scale=scale, ignore_index=ignore, status=status)
    ok = (ids >= 0) & (ids < table.shape[0]) & (ids != ignore)
    want = (table[torch.from_numpy(np.where(ok, ids, 0))].float() * np.float32(scale)).to(out.dtype)
    want[torch.from_numpy(~ok)] = 0.0
    assert torch.equal(out.cpu(), want)


def gradient(dout, ids, vocab, to="fp32", scale=1.0, before=None, ignore=-100, status=None):
    dtable = torch.full((vocab, dout.shape[1]), 7.0, dtype=TYPES[to], device=DEV)
    if before is not None:
        dtable.copy_(before)
    ws = efs.new_embed_workspace(ids.size, vocab, dout.shape[1], DEV)
    ws.fill_(0xFF)
    efs.embed_backward(dout.to(DEV), torch.from_numpy(ids).to(DEV), dtable, ws, scale=scale, ignore_index=ignore,
                       accumulate=before is not None, status=status)
    return dtable


def check_backward(dout, ids, vocab, to="fp32", scale=1.0, before=None, ignore=-100):
    got = gradient(dout, ids, vocab, to, scale, before, ignore)
    want, limit = _step.embed_gradient(dout.float().numpy(), ids, vocab, float(np.float32(scale)), ignore,
                                       None if before is None else before.double().numpy(), to)
    _step.within(got.float().cpu().numpy(), (want, limit), "dtable")
    return got


@pytest.mark.parametrize("dtype, table", PAIRS)
@pytest.mark.parametrize("tokens, vocab, width", [(1, 1, 1), (1, 5, 7), (3, 9, 64), (65, 33, 130), (200, 50, 1000), (17, 300, 4097)])
def test_forward(tokens, vocab, width, dtype, table):
    rng = np.random.default_rng(tokens + width)
    check_forward(draw(rng, (vocab, width), table), words(rng, tokens, vocab, "holes"), dtype, 0.37)


def test_forward_of_strided_rows_leaves_what_lies_between():
    rng = np.random.default_rng(1)
    ids = torch.from_numpy(words(rng, 50, 20, "uniform")).to(DEV)
    table = draw(rng, (20, 91), "bf16").to(DEV)[:, 3:80]
    wide = torch.full((50, 101), 5.0, device=DEV)
    efs.embed_forward(table, ids, wide[:, 1:78])
    assert torch.equal(wide[:, 1:78], table[ids].float())
    assert torch.all(wide[:, :1] == 5.0) and torch.all(wide[:, 78:] == 5.0)


def test_forward_of_a_long_row():
    rng = np.random.default_rng(2)
    check_forward(draw(rng, (3, 2 ** 18), "fp32"), np.array([2, 0, 2, 1], np.int64), "fp32")


def test_an_ignored_word_may_lie_in_the_table():
    rng = np.random.default_rng(3)
    ids = np.array([0, 1, 2, 1, 0], np.int64)
    check_forward(draw(rng, (3, 40), "fp32"), ids, "fp32", ignore=1)
    got = check_backward(draw(rng, (5, 40), "fp32"), ids, 3, ignore=1)
    assert torch.all(got[1] == 0.0)


@pytest.mark.parametrize("kind", ["uniform", "same", "zipf", "runs", "holes"])
@pytest.mark.parametrize("tokens, vocab, width", [(1, 1, 1), (1, 40, 70), (31, 7, 33), (32, 7, 64), (33, 1, 129), (64, 3, 8),
                                                  (700, 1000, 65), (3000, 97, 257), (5000, 20000, 16), (9999, 1500, 33), (4096, 60, 40), (4097, 60, 40)])
def test_backward(tokens, vocab, width, kind):
    say("embed_backward", tokens, vocab, width, kind)
    rng = np.random.default_rng(tokens * 31 + vocab)
    check_backward(draw(rng, (tokens, width), "fp32"), words(rng, tokens, vocab, kind), vocab, scale=1.7)


@pytest.mark.parametrize("dtype, to", PAIRS)
@pytest.mark.parametrize("add", [False, True])
def test_backward_types(dtype, to, add):
    rng = np.random.default_rng(4)
    for tokens, vocab, width in ((20, 50, 70), (600, 90, 523), (4500, 700, 267)):
        before = draw(rng, (vocab, width), to) if add else None
        check_backward(draw(rng, (tokens, width), dtype), words(rng, tokens, vocab, "zipf"), vocab, to, 8.0, before)


# few tokens, and more than are handled without sorting
@pytest.mark.parametrize("tokens", [400, 5000])
def test_added_rows_without_a_token_keep_their_bits(tokens):
    rng = np.random.default_rng(5)
    vocab = 5 * tokens // 4
    before = draw(rng, (vocab, 30), "fp32")
    before[7] = float("nan")
    ids = words(rng, tokens, vocab, "holes")
    ids[ids == 7] = 8
    got = gradient(draw(rng, (tokens, 30), "fp32"), ids, vocab, before=before).cpu()
    left = torch.from_numpy(np.setdiff1d(np.arange(vocab), ids))
    assert_bits_equal(got[left].numpy(), before[left].numpy(), "rows without a token")


@pytest.mark.parametrize("tokens", [300, 6000])
def test_backward_of_strided_rows_leaves_what_lies_between(tokens):
    rng = np.random.default_rng(6)
    vocab = 40 if tokens < 1000 else 2000
    ids = torch.from_numpy(words(rng, tokens, vocab, "zipf")).to(DEV)
    dout = draw(rng, (tokens, 77), "fp32").to(DEV)
    wide = torch.full((vocab, 99), 5.0, device=DEV)
    ws = efs.new_embed_workspace(tokens, vocab, 60, DEV)
    efs.embed_backward(dout[:, 9:69], ids, wide[:, 1:61], ws)
    dense = gradient(dout[:, 9:69].contiguous(), ids.cpu().numpy(), vocab)
    assert torch.equal(wide[:, 1:61], dense)
    assert torch.all(wide[:, :1] == 5.0) and torch.all(wide[:, 61:] == 5.0)


def test_the_same_bits_each_time():
    rng = np.random.default_rng(7)
    dout, ids = draw(rng, (20000, 96), "bf16"), words(rng, 20000, 300, "zipf")
    first = gradient(dout, ids, 300)
    for _ in range(3):
        assert torch.equal(gradient(dout, ids, 300), first)


def test_no_tokens():
    out = torch.empty(0, 8, device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    efs.embed_forward(torch.ones(4, 8, device=DEV), none, out)
    dtable = torch.full((4, 8), 3.0, device=DEV)
    ws = efs.new_embed_workspace(0, 4, 8, DEV)
    efs.embed_backward(out, none, dtable, ws, accumulate=True)
    assert torch.all(dtable == 3.0)
    efs.embed_backward(out, none, dtable, ws)
    assert torch.all(dtable == 0.0)


def test_no_token_that_counts():
    rng = np.random.default_rng(8)
    for tokens in (5, 500, 5000):
        assert torch.all(check_backward(draw(rng, (tokens, 40), "fp32"), np.full(tokens, -100), 60) == 0.0)


@pytest.mark.parametrize("tokens", [300, 5000])
def test_rows_that_do_not_count_may_hold_anything(tokens):
    rng = np.random.default_rng(9)
    ids = words(rng, tokens, 50, "holes")
    dout = draw(rng, (tokens, 20), "fp32")
    clean = gradient(dout, ids, 50)
    dout[torch.from_numpy((ids < 0) | (ids >= 50))] = float("nan")
    assert torch.equal(gradient(dout, ids, 50), clean)


@pytest.mark.parametrize("tokens", [900, 5000])
def test_nan_stays_in_its_word(tokens):
    rng = np.random.default_rng(10)
    ids = words(rng, tokens, 20, "zipf")
    dout = draw(rng, (tokens, 70), "fp32")
    clean = gradient(dout, ids, 20)
    dout[450, 33] = float("nan")
    got = gradient(dout, ids, 20)
    where = torch.zeros_like(got, dtype=torch.bool)
    where[ids[450], 33] = True
    assert torch.equal(torch.isnan(got), where)
    assert torch.equal(got[~where], clean[~where])


def test_status_word():
    rng = np.random.default_rng(11)
    status = efs.new_embed_status(DEV)
    table, dout = draw(rng, (10, 6), "fp32"), draw(rng, (4, 6), "fp32")
    good, bad = np.array([1, -100, 9, 0]), np.array([1, 10, 9, 0])
    check_forward(table, good, "fp32", status=status)
    gradient(dout, good, 10, status=status)
    assert efs.embed_status(status) == 0
    check_forward(table, bad, "fp32", status=status)
    assert efs.embed_status(status) == efs.EMBED_BAD_ID
    check_forward(table, good, "fp32", status=status)   # not cleared
    assert efs.embed_status(status) == efs.EMBED_BAD_ID
    status.zero_()
    gradient(dout, np.array([1, -1, 2, 3]), 10, status=status)
    assert efs.embed_status(status) == efs.EMBED_BAD_ID
    many = np.full(5000, 3)
    for at, want in ((None, 0), (4999, efs.EMBED_BAD_ID)):
        status.zero_()
        if at is not None:
            many[at] = 10
        gradient(draw(rng, (5000, 6), "fp32"), many, 10, status=status)
        assert efs.embed_status(status) == want


def test_gradient_against_differences():
    """The sum of weight * out is linear in the table: its difference over a step
    is the gradient but for roundings."""
    rng = np.random.default_rng(12)
    table, ids, weight = draw(rng, (30, 16), "fp32"), words(rng, 80, 30, "zipf"), draw(rng, (80, 16), "fp32")

    def loss(tab):
        out = torch.empty(80, 16, device=DEV)
        efs.embed_forward(tab.to(DEV), torch.from_numpy(ids).to(DEV), out, scale=2.0)
        return float((out.cpu().double() * weight.double()).sum())
    grad = gradient(weight, ids, 30, scale=2.0).cpu().double()
    for v, c in ((0, 0), (3, 7), (29, 15), (11, 2)):
        up, down = table.clone(), table.clone()
        up[v, c] += 1.0
        down[v, c] -= 1.0
        # table +- 1 is rounded: 2^-24 of at most 8, times 2 and the weights' sum
        slack = 2.0 ** -20 * float(weight.abs()[:, c].sum())
        assert abs((loss(up) - loss(down)) / 2.0 - float(grad[v, c])) <= slack


@pytest.mark.parametrize("start", range(32))
def test_split_words_that_start_anywhere_in_a_piece(start):
    """Words that are summed piece by piece, of which one starts at each place of a
    piece of 32 sorted tokens; pieces without such a start lie between."""
    counts = [start, 33, 31, 32 + (32 - start) % 32, 700, 1, 0, 64, 3]
    counts.append(4300 - sum(counts))
    ids = np.repeat(np.arange(len(counts)), counts)
    rng = np.random.default_rng(start)
    rng.shuffle(ids)
    dout = torch.from_numpy(rng.integers(-9, 10, (len(ids), 70)).astype(np.float32))
    want = np.zeros((len(counts), 70))
    np.add.at(want, ids, dout.numpy())
    before = torch.ones(len(counts), 70)
    assert np.array_equal(gradient(dout, ids, len(counts)).cpu().numpy(), want)
    assert np.array_equal(gradient(dout, ids, len(counts), before=before).cpu().numpy(), want + 1.0)
