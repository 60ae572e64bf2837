"""The inner step's entry points refuse bad arguments on the host, before anything touches a GPU, and the oracle's rounding to
8 bits keeps its own rules."""
import ctypes

import numpy as np
import pytest

from oracle import inner as O
from paper_2601_02360_amd import binding as B

ANY = ctypes.c_void_p(4096)              # never dereferenced: every call below is refused during validation


def how(**kw):
    n = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=1)
    n.update(kw)
    return ctypes.byref(B._AdamW(*(n[f] for f, _ in B._AdamW._fields_)))


def test_null_handles():
    L = B.lib()
    assert L.sparseloco_plan_num_flat_chunks(None) == B.SPLC_EINVAL
    assert L.sparseloco_grad_norm(None, None, 0, 1.0, ANY, ANY, None) == B.SPLC_EINVAL
    assert L.sparseloco_adamw_step(None, None, None, None, None, 0, how(), None, None, None, None) == B.SPLC_EINVAL
    assert L.sparseloco_adamw_step_8bit(None, None, None, 0, ANY, ANY, ANY, ANY, how(), None, None, None, None) == B.SPLC_EINVAL


def test_lookup_arguments():
    def call(table=ANY, perp=None, dtype=0, ids=ANY, vocab=5, pos=None, seq=0, scale=1.0, out=ANY, out_dtype=0, rows=4, d=8):
        return B.lib().sparseloco_embedding_lookup(table, perp, dtype, ids, vocab, pos, seq, scale, out, out_dtype, rows, d, None)

    for bad in (dict(table=None), dict(ids=None), dict(out=None), dict(vocab=0), dict(dtype=2), dict(out_dtype=-1), dict(rows=-1),
                dict(rows=2 ** 31), dict(d=0), dict(d=2 ** 24), dict(scale=float("inf")), dict(pos=ANY, seq=0)):
        assert call(**bad) == B.SPLC_EINVAL, bad
    odd = ctypes.c_void_p(4098)
    for bad in (dict(table=odd), dict(perp=odd), dict(pos=odd, seq=3), dict(ids=odd), dict(out=odd),
                dict(table=ctypes.c_void_p(4097), dtype=1), dict(out=ctypes.c_void_p(4097), out_dtype=1)):
        assert call(**bad) == B.SPLC_EALIGN, bad
    assert call(rows=0, ids=None, out=None) == B.SPLC_OK


def test_gradient_arguments():
    size = B.lib().sparseloco_embedding_grad_ws_bytes

    def call(g=ANY, gt=0, ids=ANY, rows=4, vocab=5, d=8, scale=1.0, ignore=-1, table=ANY, tt=0, acc=0, ws=ANY, n=1 << 30):
        return B.lib().sparseloco_embedding_grad(g, gt, ids, rows, vocab, d, scale, ignore, table, tt, acc, ws, n, None)

    for bad in (dict(g=None), dict(ids=None), dict(table=None), dict(ws=None), dict(gt=2), dict(tt=7), dict(rows=-1), dict(vocab=0),
                dict(d=0), dict(scale=float("nan")), dict(n=size(4, 5, 8) - 1)):
        assert call(**bad) == B.SPLC_EINVAL, bad
    for bad in (dict(g=ctypes.c_void_p(4098)), dict(table=ctypes.c_void_p(4097), tt=1), dict(ids=ctypes.c_void_p(4098)),
                dict(ws=ctypes.c_void_p(4100))):
        assert call(**bad) == B.SPLC_EALIGN, bad
    assert size(0, 5, 8) >= 0 and size(2 ** 30, 5, 8) == B.SPLC_EINVAL
    for rows, d in ((2 ** 28 - 1, 32), (2 ** 27, 127), (2 ** 19, 32767), (2 ** 10, 2 ** 24 - 1)):
        assert size(rows, 2 ** 31 - 1, d) > 0                             # rows max(d, 64) < 2^34
    for rows, d in ((2 ** 28, 1), (2 ** 27, 128), (2 ** 20, 2 ** 14), (4096, 2 ** 24 - 1)):
        assert size(rows, 5, d) == B.SPLC_EINVAL
    for vocab, d in ((5, 8), (50304, 768), (32001, 2050)):                # more rows never need less
        sizes = [size(rows, vocab, d) for rows in (0, 1, 100, 16384, 16385, 10 ** 6)]
        assert sizes == sorted(sizes)


@pytest.mark.parametrize("second", [False, True])
def test_rounding_to_8_bits_of_the_oracle(second):
    """What is held lies within a gap of the value, is an e4m3 number times the scale, and over many steps averages to it."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((4, 256)) * 10.0 ** rng.integers(-6, 1, (4, 256))
    x = np.abs(x) if second else x
    places = np.arange(x.size)
    total = np.zeros_like(x)
    for step in range(1, 513):
        numbers, scales, _ = O.held(x, places, step, second)
        assert np.abs(numbers).max() == 448.0
        y = numbers * scales[:, None]
        gap = scales[:, None] * np.ldexp(1.0, np.maximum(np.frexp(np.abs(x) / scales[:, None])[1] - 1, -6) - 3)
        assert np.all(np.abs(y - x) <= gap * (1 + 1e-12))
        assert np.all(np.abs(numbers) / np.ldexp(1.0, np.maximum(np.frexp(np.abs(numbers))[1] - 1, -6) - 3) % 1 == 0)
        if second:
            assert np.all(numbers[x > 0] > 0)
        total += y
    if not second:                       # (a root's least number is not the nearest one)
        assert np.all(np.abs(total / 512 - x) <= 0.02 * gap)
