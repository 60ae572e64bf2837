"""The embedding gradient where its sums are exact: small whole numbers and a power of two as the scale, so that fp32 forms every sum
of up to 2^24 without rounding, in whatever order, and the result is compared for equality.  No gradient is zero and all have the
same sign, so a token that is left out, or taken twice, changes every column of its row -- however long the run of equal
tokens is.  Runs begin and end anywhere in the windows of 64 entries that the kernels sum by."""
import numpy as np
import pytest
import torch

from paper_2601_02360_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
MOST = 7                                 # the largest gradient; times the most tokens here it is below 2^24


def runs_of(lengths, seed):
    """Token k lengths[k] times, in a seeded order."""
    ids = np.repeat(np.arange(len(lengths)), lengths)
    return np.random.default_rng(seed).permutation(ids).astype(np.int32)


def check(lengths, d, spread=0, grad_type=F32, table_type=F32, accumulate=False, ignored=None, vocab=None, seed=0):
    """spread: so many more tokens, each of another row behind the runs'."""
    lengths = list(lengths) + [1] * spread
    vocab = len(lengths) + 3 if vocab is None else vocab
    ids = torch.as_tensor(runs_of(lengths, seed + sum(lengths) + d)).cuda()
    rows = len(ids)
    assert rows * MOST < 2 ** 24 and len(lengths) <= vocab
    g = torch.Generator(device="cuda").manual_seed(seed + rows)
    grad = torch.randint(1, MOST + 1, (rows, d), generator=g, device="cuda").to(grad_type)
    was = torch.randint(-9, 10, (vocab, d), generator=g, device="cuda").to(table_type)
    table = was.clone() if accumulate else torch.full_like(was, 12288.0)
    ws = B.embedding_grad_workspace(rows, vocab, d)
    ws.fill_(255)
    B.sparseloco_embedding_grad(grad, ids, table, ws, scale=0.5, ignore_id=-1 if ignored is None else ignored, accumulate=accumulate)
    want = torch.zeros(vocab, d, dtype=torch.int64)
    host, names = grad.cpu().to(torch.int64).numpy(), ids.cpu().numpy()
    order = np.argsort(names, kind="stable")
    first = np.concatenate([[0], np.cumsum(lengths)[:-1]])
    want[:len(lengths)] = torch.as_tensor(np.add.reduceat(host[order], first, axis=0))
    if ignored is not None:
        want[ignored] = 0
    want = want.double() * 0.5
    if accumulate:
        want += was.double().cpu()
    want = want.to(table_type)           # (exact in fp32; to bf16 one rounding to nearest even)
    got = table.cpu()
    wrong = (got != want).nonzero()
    assert len(wrong) == 0, "%d places, the first (%d, %d): %g instead of %g" % (
        len(wrong), *wrong[0], got[tuple(wrong[0])], want[tuple(wrong[0])])


WIDTHS = [3, 65, 257, 514]               # an element a lane in one and two slices, four a lane in two and three


# How far into a window the long run begins, and its length: about one window, the 64 windows that a wave looks at at once, twice
# that, the 64 windows whose sums are taken in one round, and more.
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("before", [0, 1, 37, 63, 64])
@pytest.mark.parametrize("run", [63, 64, 65, 127, 129, 4032, 4095, 4096, 4097, 4096 + 63, 4096 + 64, 8191, 8192, 8193, 8192 + 65, 16384])
def test_a_run_that_begins_inside_a_window(run, before, d):
    check(([before] if before else []) + [run, 5], d)


@pytest.mark.parametrize("accumulate,ignored", [(False, None), (True, None), (True, 1)])
@pytest.mark.parametrize("grad_type,table_type", [(F32, F32), (BF16, F32), (F32, BF16), (BF16, BF16)])
@pytest.mark.parametrize("d", WIDTHS)
def test_long_runs_in_every_type_and_added(d, grad_type, table_type, accumulate, ignored):
    for lengths, spread in (([29, 3000, 40], 20), ([29, 70, 4096 + 40, 64, 9001], 700), ([11, 20000, 300], 3000)):
        check(lengths, d, spread, grad_type, table_type, accumulate, ignored)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("run", [8 * 8 * 64 - 3, 8 * 8 * 64, 8 * 8 * 64 + 64 + 5, 2 * 64 * 64 * 8 + 17, 50000, 65537, 140000])
@pytest.mark.parametrize("d", [31, 258])
def test_the_longest_runs(d, run, accumulate):
    """Several rounds of windows' sums by all waves of a workgroup, and of looking for the run's end."""
    check([50, run, 77], d, 40, accumulate=accumulate)


@pytest.mark.parametrize("rows", [4096, 4097, 16384, 16385, 40000])
@pytest.mark.parametrize("d", [80, 300])
def test_frequencies_that_fall_like_one_over_the_rank(d, rows):
    n = 400
    share = 1.0 / np.arange(1, n + 1)
    lengths = np.maximum(1, (share / share.sum() * (rows - n)).astype(np.int64))
    lengths[0] += rows - lengths.sum()
    check(np.random.default_rng(rows).permutation(lengths), d)


@pytest.mark.parametrize("run,before", [(5000, 70), (9000, 1), (16000, 63)])
def test_long_runs_whose_order_is_merged_beside_the_zeros(run, before):
    """More than 64 MB of zeros: the tokens are ordered in runs of 2048 that are merged, although there are few."""
    check([before, run, 5], 300, 9, vocab=66000)


@pytest.mark.parametrize("rows", [4097, 6000, 16384])
def test_the_order_after_one_merge(rows):
    """Above 64 MB of zeros an order of up to 16384 tokens is merged once and lies in the second of the workspace's two stages,
    [rows, tokens] each, of whole blocks of 512 entries."""
    vocab, d = 2 ** 21, 16
    entries = -(-rows // 512) * 512
    ws = B.embedding_grad_workspace(rows, vocab, d)
    ws.fill_(255)
    ids = (torch.arange(rows, device="cuda") * 7919 % 1000).to(torch.int32)
    grad, table = torch.ones(rows, d, device="cuda"), torch.empty(vocab, d, device="cuda")
    B.sparseloco_embedding_grad(grad, ids, table, ws)
    row, token = ws[:16 * entries].view(torch.int32).view(4, entries)[2:]
    assert token.min().item() >= 0 and token.max().item() < rows
    want = ids.sort(stable=True)
    assert torch.equal(row[:rows], want.values) and torch.equal(token[:rows].long(), want.indices) and (row[rows:] >= vocab).all()
    assert torch.equal(table[:1000], torch.bincount(ids, minlength=1000).float()[:, None].expand(-1, d)) and not table[1000:].any()
