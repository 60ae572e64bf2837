"""The embedding lookup, bit for bit, and its gradient against the float64 oracle (oracle/inner.py).

Bars of the gradient: a row of n tokens is n additions of products with the scale, in whatever order, and at most three
roundings more (the product, a sum that was there, the result): (n + 3) 2^-24 of the magnitudes' sum; a bf16 result half a
unit of its 8 bits more."""
import numpy as np
import pytest
import torch

from oracle import inner as O
from paper_2601_02360_amd import binding as B

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U24, TINY = 2.0 ** -24, 2.0 ** -126
GUARD = 12288.0                          # (a bf16 number)


class Placed:
    """Tensors from element 65 (odd, so aligned to their elements and no more) of larger buffers with guard values around them."""
    EDGE = 65

    def __init__(self):
        self.buffers = []

    def __call__(self, values, dtype=F32):
        values = torch.as_tensor(values)
        buf = torch.full((values.numel() + 2 * self.EDGE,), GUARD if dtype.is_floating_point else 7, dtype=dtype, device="cuda")
        self.buffers.append(buf)
        return buf[self.EDGE:-self.EDGE].view(values.shape).copy_(values)

    def check(self):
        for buf in self.buffers:
            guard = GUARD if buf.dtype.is_floating_point else 7
            assert (buf[:self.EDGE] == guard).all() and (buf[-self.EDGE:] == guard).all(), "written beside an array"


def rounded(x, dtype):
    return torch.as_tensor(x).to(dtype).float().numpy()


def normal(rng, *shape):
    return rng.standard_normal(shape).astype(np.float32)


# ---------------------------------------------------------------- lookup

@pytest.mark.parametrize("rows,vocab,d", [(1, 1, 1), (1, 5, 2), (3, 7, 3), (37, 300, 768), (5, 50, 1023), (64, 50, 1024), (65, 50, 1025),
                                          (9, 20, 2050), (130, 1000, 257), (4099, 611, 30), (2, 3, 4096 + 6),
                                          (70, 40, 64), (1001, 33, 33), (129, 40, 127), (255, 40, 128), (257, 40, 129),
                                          (18, 40, 200), (1031, 99, 256), (7, 30, 512), (6, 30, 513), (5, 9, 1500), (3, 9, 2049), (21, 9, 5003), (9, 9, 8200), (8193, 99, 1024), (8195, 60, 1790)])
@pytest.mark.parametrize("table_type,out_type,perp,seq", [(F32, F32, False, 0), (F32, BF16, True, 5), (BF16, F32, True, 64), (BF16, BF16, False, 3)])
def test_lookup(rows, vocab, d, table_type, out_type, perp, seq):
    rng = np.random.default_rng(rows + d)
    table, t_perp, pos = (rounded(normal(rng, n, d), table_type) for n in (vocab, vocab, max(seq, 1)))
    ids = rng.integers(-2, vocab + 2, rows).astype(np.int32)             # those outside are clamped
    place = Placed()
    out = place(np.zeros((rows, d), np.float32), out_type)
    B.sparseloco_embedding_lookup(place(table, table_type), place(ids, torch.int32), out, scale=1.7,
                                  t_perp=place(t_perp, table_type) if perp else None, pos_embed=place(pos, table_type) if seq else None)
    want = torch.as_tensor(O.lookup(table, ids, t_perp if perp else None, pos if seq else None, 1.7)).to(out_type)
    assert torch.equal(out.cpu(), want)
    place.check()


def test_lookup_beyond_32_bit_offsets():
    """A table of 2.2 billion bf16 elements, 4.4 GB, and its last rows."""
    vocab, d = 1_100_000, 2000
    table = torch.zeros(vocab, d, dtype=BF16, device="cuda")
    at = torch.tensor([0, 1, 536_870, 536_871, 1_073_742, vocab - 1], dtype=torch.int32, device="cuda")
    for k, v in enumerate(at.tolist()):
        table[v] = k + 1
    out = torch.empty(len(at), d, dtype=F32, device="cuda")
    B.sparseloco_embedding_lookup(table, at, out, scale=2.0)
    assert torch.equal(out, (torch.arange(1, len(at) + 1, device="cuda") * 2.0)[:, None].expand(-1, d))


# ---------------------------------------------------------------- gradient

def tokens(rng, rows, vocab, how):
    if how == "same":
        return np.full(rows, vocab // 2, np.int32)
    if how == "text":                    # frequencies that fall like 1 / rank
        return np.minimum(np.exp(rng.random(rows) * np.log(vocab + 1)).astype(np.int64) - 1, vocab - 1).astype(np.int32)
    if how == "outside":
        return rng.integers(-3, vocab + 3, rows).astype(np.int32)
    return (np.arange(rows) * 7919 % vocab).astype(np.int32)


def check_grad(rows, vocab, d, how, grad_type=F32, table_type=F32, accumulate=False, ignore=None, scale=1.3, seed=0):
    rng = np.random.default_rng(seed + rows + vocab + d)
    ids = tokens(rng, rows, vocab, how)
    ignore_id = -1 if ignore is None else int(ignore if rows == 0 else ids[rows // 2])
    grad, before = rounded(normal(rng, rows, d), grad_type), rounded(normal(rng, vocab, d), table_type)
    place = Placed()
    g, t, x = place(grad, grad_type), place(before, table_type), place(ids, torch.int32)
    ws = B.embedding_grad_workspace(rows, vocab, d)
    ws.fill_(255)                        # (whatever it held is not to matter)
    call = lambda table: B.sparseloco_embedding_grad(g, x, table, ws, scale=scale, ignore_id=ignore_id, accumulate=accumulate)
    call(t)
    place.check()
    want, size, count = O.embedding_grad(grad, ids, vocab, scale, ignore_id)
    bar = (count[:, None] + 3) * U24 * (size + (np.abs(before) if accumulate else 0.0))
    if accumulate:
        want = before.astype(np.float64) + want
    if table_type == BF16:
        bar = bar + 2.0 ** -8 * np.abs(want)
    got = t.double().cpu().numpy()
    off = np.abs(got - want)
    assert np.all(off <= 1.01 * bar + TINY), "off by %.3g of the bar" % np.max(off / (1.01 * bar + TINY))
    empty = count == 0
    assert np.array_equal(got[empty], before[empty] if accumulate else np.zeros((int(empty.sum()), d)))
    again = place(before, table_type)
    call(again)
    assert torch.equal(t, again), "the same call gave other bits"


@pytest.mark.parametrize("rows", [0, 1, 2, 63, 64, 65, 1000, 1025])
@pytest.mark.parametrize("vocab,d", [(1, 1), (3, 2), (300, 3), (2560, 64), (2561, 255), (5121, 256), (777, 257), (50, 770), (33, 259)])
def test_gradient_of_few_tokens(rows, vocab, d):
    for how in ("text", "same", "outside", "spread"):
        check_grad(rows, vocab, d, how)


@pytest.mark.parametrize("rows,vocab,d", [(2048, 4000, 260), (4097, 300, 513), (16384, 32000, 64), (16383, 2000, 300), (16385, 2561, 257),
                                          (40000, 999, 65), (33000, 9000, 270), (50000, 3, 258), (2049, 40, 64),
                                          (65537, 700, 80), (140000, 5000, 66), (4096, 700, 300), (4097, 33000, 514), (16384, 66000, 260)])
@pytest.mark.parametrize("how", ["text", "same", "spread"])
def test_gradient_of_many_tokens(rows, vocab, d, how):
    """Long runs of one token, several blocks of the sort, one and two rounds of merging."""
    check_grad(rows, vocab, d, how)


@pytest.mark.parametrize("rows,vocab,d", [(700, 900, 130), (5000, 3000, 514), (20000, 5200, 259), (20000, 200, 31)])
@pytest.mark.parametrize("grad_type,table_type", [(F32, BF16), (BF16, F32), (BF16, BF16)])
@pytest.mark.parametrize("accumulate,ignore", [(False, 1), (True, None), (True, 1)])
def test_gradient_types_accumulation_and_padding(rows, vocab, d, grad_type, table_type, accumulate, ignore):
    for how in ("text", "outside"):
        check_grad(rows, vocab, d, how, grad_type, table_type, accumulate, ignore, scale=-0.7)


@pytest.mark.parametrize("rows,vocab,d", [(3000, 50304, 768), (17000, 32001, 2050), (300, 262144, 300), (18000, 262144, 256), (20, 2 ** 21 - 2, 3)])
def test_gradient_at_the_models_sizes_and_the_largest_tables(rows, vocab, d):
    check_grad(rows, vocab, d, "text")


@pytest.mark.parametrize("rows,vocab,d,accumulate", [(500, 40, 257, False), (20000, 3000, 300, True), (6000, 90, 20, False)])
def test_every_token_ignored_and_rows_with_nan(rows, vocab, d, accumulate):
    """Padding leaves every row empty whatever grad_out holds there; a NaN stays in its row and column."""
    ids = torch.full((rows,), 3, dtype=torch.int32, device="cuda")
    grad = torch.full((rows, d), float("nan"), device="cuda")
    table = torch.full((vocab, d), 5.0, device="cuda")
    ws = B.embedding_grad_workspace(rows, vocab, d)
    B.sparseloco_embedding_grad(grad, ids, table, ws, ignore_id=3, accumulate=accumulate)
    assert (table == (5.0 if accumulate else 0.0)).all()
    grad = torch.ones(rows, d, device="cuda")
    ids = (torch.arange(rows, device="cuda") % vocab).to(torch.int32)
    grad[rows - 1, d - 1] = float("nan")
    B.sparseloco_embedding_grad(grad, ids, table, ws, accumulate=accumulate)
    assert torch.isnan(table).nonzero().tolist() == [[(rows - 1) % vocab, d - 1]]


@pytest.mark.parametrize("rows,entries,stage", [(5, 512, 0), (2048, 2048, 0), (2049, 2560, 0), (16384, 16384, 0), (16384 + 7, 16896, 0)])
def test_no_entry_of_the_order_names_a_token_that_is_not_there(rows, entries, stage):
    """The workspace holds the order of the tokens ([rows, tokens] of two stages): every entry's token is one of the call's, also
    of those that only fill a block, whose rows of grad_out are read like the others'."""
    vocab, d = 50, 8
    ws = B.embedding_grad_workspace(rows, vocab, d)
    ws.fill_(255)
    ids = torch.arange(rows, device="cuda", dtype=torch.int32) % vocab
    grad, table = torch.ones(rows, d, device="cuda"), torch.empty(vocab, d, device="cuda")
    B.sparseloco_embedding_grad(grad, ids, table, ws)
    at = (2 * stage + 1) * entries
    row, token = (ws[:16 * entries].view(torch.int32)[at + k * entries:at + (k + 1) * entries] for k in (-1, 0))
    assert token.min().item() >= 0 and token.max().item() < rows
    assert torch.equal(row[:rows], ids.sort().values) and (row[rows:] >= vocab).all()
    assert torch.equal(ids[token[:rows].long()], row[:rows])
    assert torch.equal(table.sum(1), torch.bincount(ids, minlength=vocab).float() * d)


def test_gradient_against_differences():
    """The sum of weights times the looked-up rows, by differences in the table, in fp64 from fp32 lookups of powers of two
    that every step of the lookup forms exactly: the quotient of differences is the gradient exactly."""
    rows, vocab, d = 300, 40, 12
    rng = np.random.default_rng(1)
    ids = torch.as_tensor(tokens(rng, rows, vocab, "text")).cuda()
    weight = torch.as_tensor(rng.integers(-8, 9, (rows, d)).astype(np.float32)).cuda()
    table = torch.as_tensor(rng.integers(-64, 64, (vocab, d)).astype(np.float32)).cuda()
    grad = torch.empty(vocab, d, device="cuda")
    B.sparseloco_embedding_grad(weight, ids, grad, B.embedding_grad_workspace(rows, vocab, d), scale=0.5)

    def loss(t):
        out = torch.empty(rows, d, device="cuda")
        B.sparseloco_embedding_lookup(t, ids, out, scale=0.5)
        return (out.double() * weight.double()).sum().item()

    for v, c in [(0, 0), (0, d - 1), (1, 3), (5, 7), (vocab - 1, 2)]:
        up, down = table.clone(), table.clone()
        up[v, c] += 2.0
        down[v, c] -= 2.0
        assert (loss(up) - loss(down)) / 4.0 == grad[v, c].item()


@pytest.mark.parametrize("rows", [5000, 20000])
def test_a_larger_workspace_a_stream_and_a_graph(rows):
    vocab, d = 700, 257
    rng = np.random.default_rng(4)
    ws = B.embedding_grad_workspace(4 * rows, vocab, d)
    grad, ids = torch.empty(rows, d, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda")
    table, eager = torch.empty(vocab, d, device="cuda"), torch.empty(vocab, d, device="cuda")
    emb, out, out2 = torch.randn(vocab, d, device="cuda"), torch.empty(rows, d, device="cuda"), torch.empty(rows, d, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    ids.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        B.sparseloco_embedding_lookup(emb, ids, out, scale=3.0)
        B.sparseloco_embedding_grad(grad, ids, table, ws)
    for k in range(4):
        grad.copy_(torch.as_tensor(normal(rng, rows, d)))
        ids.copy_(torch.as_tensor(tokens(rng, rows, vocab, ("text", "same", "spread", "text")[k])))
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            B.sparseloco_embedding_lookup(emb, ids, out2, scale=3.0)
            B.sparseloco_embedding_grad(grad, ids, eager, ws)
        side.synchronize()
        assert torch.equal(table, eager) and torch.equal(out, out2)


def test_refusals():
    x, ids, table = torch.zeros(8, 16, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(5, 16, device="cuda")
    ws = B.embedding_grad_workspace(8, 5, 16)
    for call in (lambda: B.sparseloco_embedding_lookup(table, ids.long(), x), lambda: B.sparseloco_embedding_lookup(table, ids[:7], x),
                 lambda: B.sparseloco_embedding_lookup(table[:, :15], ids, x), lambda: B.sparseloco_embedding_lookup(table.half(), ids, x),
                 lambda: B.sparseloco_embedding_lookup(table, ids, x, t_perp=table.bfloat16()),
                 lambda: B.sparseloco_embedding_lookup(table, ids, x, t_perp=table[:4]),
                 lambda: B.sparseloco_embedding_lookup(table, ids, x, pos_embed=torch.zeros(4, 15, device="cuda")),
                 lambda: B.sparseloco_embedding_lookup(table, ids, x, pos_embed=torch.zeros(0, 16, device="cuda")),
                 lambda: B.sparseloco_embedding_lookup(table, ids, x.t()), lambda: B.sparseloco_embedding_lookup(table.cpu(), ids, x),
                 lambda: B.sparseloco_embedding_grad(x, ids, table, ws.float()), lambda: B.sparseloco_embedding_grad(x[:7], ids, table, ws),
                 lambda: B.sparseloco_embedding_grad(x, ids, table.double(), ws), lambda: B.sparseloco_embedding_grad(x, ids.cpu(), table, ws)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: B.sparseloco_embedding_lookup(table, ids, x, scale=float("nan")),
                 lambda: B.sparseloco_embedding_grad(x, ids, table, ws, scale=float("inf")),
                 lambda: B.sparseloco_embedding_grad(x, ids, table, ws[:8]),
                 lambda: B.embedding_grad_workspace(2 ** 28, 5, 16), lambda: B.embedding_grad_workspace(8, 0, 16),
                 lambda: B.embedding_grad_workspace(-1, 5, 16)):
        with pytest.raises(B.SparseLoCoError) as e:
            call()
        assert e.value.status == B.SPLC_EINVAL
    assert not table.any() and not x.any()
