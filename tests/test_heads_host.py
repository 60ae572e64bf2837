"""Queries and keys: bad arguments are refused on the host, before anything touches a GPU."""
import ctypes

import pytest
import torch

from paper_2601_02360_amd import binding as B

ANY, ODD = 4096, 4098                    # never dereferenced: every call below is refused during validation


def heads(data=ANY, token=64, head=16, n=4):
    return ctypes.byref(B._Heads(data, token, head, n))


def how(positions=ANY, frequencies=ANY, size=4, pairs=8, side=0, magnitude=1.0):
    return ctypes.byref(B._Rotation(positions, frequencies, size, pairs, side, magnitude))


def rotary(q=None, k=None, dtype=0, tokens=5, d=16, turn=None, q_out=None, k_out=None):
    return B.lib().sparseloco_rotary(q or heads(), k, dtype, tokens, d, turn or how(), 0, q_out or heads(), k_out, None)


def test_what_the_rotation_refuses():
    for bad in (dict(dtype=2), dict(tokens=-1), dict(tokens=2 ** 31), dict(d=15), dict(d=0), dict(d=514), dict(k=heads()), dict(k_out=heads()),
                dict(q=heads(n=-1)), dict(q=heads(None)), dict(q_out=heads(None)), dict(q_out=heads(n=5)), dict(q=heads(token=-1)),
                dict(q=heads(token=2 ** 61)), dict(turn=how(positions=None)), dict(turn=how(frequencies=None)), dict(turn=how(size=2)),
                dict(turn=how(pairs=0)), dict(turn=how(pairs=9)), dict(turn=how(magnitude=float("inf"))),
                dict(k=heads(2 * ANY), q_out=heads(2 * ANY), k_out=heads(3 * ANY)), dict(k=heads(2 * ANY), q_out=heads(3 * ANY), k_out=heads()),
                dict(k=heads(2 * ANY), q_out=heads(3 * ANY), k_out=heads(3 * ANY)), dict(q_out=heads(token=0)), dict(q_out=heads(head=15)), dict(q_out=heads(token=63)), dict(q_out=heads(token=16, head=64))):
        assert rotary(**bad) == B.SPLC_EINVAL, bad
    L = B.lib()
    assert L.sparseloco_rotary(None, None, 0, 5, 16, how(), 0, heads(), None, None) == B.SPLC_EINVAL
    assert L.sparseloco_rotary(heads(), None, 0, 5, 16, None, 0, heads(), None, None) == B.SPLC_EINVAL
    for bad in (dict(q=heads(ODD)), dict(q_out=heads(ODD)), dict(q=heads(ODD + 1), dtype=1), dict(turn=how(positions=ODD)),
                dict(turn=how(positions=ANY + 4, size=8)), dict(turn=how(frequencies=ANY + 4))):
        assert rotary(**bad) == B.SPLC_EALIGN, bad
    assert rotary(tokens=0) == B.SPLC_OK and rotary(tokens=0, q=heads(None), q_out=heads(None)) == B.SPLC_OK
    assert rotary(q=heads(n=0), q_out=heads(n=0)) == B.SPLC_OK


def test_what_the_norm_refuses():
    def call(gain=ANY, k_gain=ANY, kind=0, eps=1e-6, keys=True, at=ANY):
        k = heads(at) if keys else None
        return B.lib().sparseloco_qk_norm_rotary(heads(), k, 0, 5, 16, gain, k_gain, kind, eps, how(), heads(), k, None)
    assert call() == B.SPLC_EINVAL       # (keys where the queries are)
    for bad in (dict(gain=None), dict(k_gain=None), dict(kind=2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=1e300)):
        assert call(at=2 * ANY, **bad) == B.SPLC_EINVAL, bad
    assert call(at=2 * ANY, gain=ODD) == B.SPLC_EALIGN and call(at=2 * ANY, k_gain=ANY + 1, kind=1) == B.SPLC_EALIGN


def test_what_the_gradient_refuses():
    size = B.lib().sparseloco_qk_norm_rotary_grad_ws_bytes

    def call(dq=None, dk=None, q=None, k=None, gq=None, gk=None, sums=(ANY, ANY), ws=ANY, n=1 << 30, k_gain=ANY):
        dk, k, gk = (t or heads(2 * ANY) for t in (dk, k, gk))
        return B.lib().sparseloco_qk_norm_rotary_grad(dq or heads(), dk, q or heads(), k, 0, 5, 16, ANY, k_gain, 0, 1e-6, how(), gq or heads(), gk,
                                                      *sums, 0, ws, n, None)
    for bad in (dict(sums=(None, ANY)), dict(sums=(ANY, None)), dict(ws=None), dict(n=size(5, 4, 4, 16) - 1), dict(k_gain=None),
                dict(gq=heads(2 * ANY)), dict(gk=heads()), dict(gq=heads(head=3)), dict(dq=heads(n=3)), dict(k=heads(n=1))):
        assert call(**bad) == B.SPLC_EINVAL, bad
    for bad in (dict(sums=(ODD, ANY)), dict(ws=ODD), dict(gk=heads(ODD))):
        assert call(**bad) == B.SPLC_EALIGN, bad
    for bad in ((-1, 1, 1, 16), (2 ** 31, 1, 1, 16), (1, -1, 1, 16), (1, 1, 2 ** 17, 16), (1, 1, 1, 17), (1, 1, 1, 514)):
        assert size(*bad) == B.SPLC_EINVAL
    sizes = [size(n, 8, 8, 64) for n in (0, 1, 5, 1000, 1024, 1025, 10 ** 6)]
    assert sizes == sorted(sizes) and sizes[0] > 0


def test_what_is_written_lies_as_the_input_that_it_replaces():
    """In place is element for element: heads that begin where the input's do, at other strides, would be read after they are written."""
    by_head = dict(token=16, head=80)                                  # five tokens of a head, then the next head
    assert rotary(q_out=heads(**by_head)) == B.SPLC_EINVAL
    assert rotary(q_out=heads(head=32, token=128)) == B.SPLC_EINVAL
    assert rotary(q=heads(token=0)) == B.SPLC_EINVAL                    # (one token's heads for all, written over)
    assert rotary(k=heads(2 * ANY), q_out=heads(3 * ANY), k_out=heads(2 * ANY, **by_head)) == B.SPLC_EINVAL
    for place in ("grad", "in"):
        lists = [heads(ANY), heads(2 * ANY), heads(3 * ANY), heads(4 * ANY)]
        out = [heads(ANY if place == "grad" else 3 * ANY, **by_head), heads(5 * ANY)]
        assert B.lib().sparseloco_qk_norm_rotary_grad(*lists, 0, 5, 16, ANY, ANY, 0, 1e-6, how(), *out, ANY, ANY, 0, ANY, 1 << 30,
                                                      None) == B.SPLC_EINVAL


def test_what_the_binding_refuses():
    q, k = torch.zeros(5, 4, 16), torch.zeros(5, 2, 16)
    positions, f, w = torch.zeros(5, dtype=torch.int32), torch.zeros(8, dtype=torch.float64), torch.zeros(16)

    def call(q=q, k=k, positions=positions, f=f, q_out=q, k_out=k):
        return B.sparseloco_rotary(q, k, positions, f, q_out, k_out)
    for bad in (dict(q=q[0]), dict(q=q.half()), dict(k=k.bfloat16()), dict(k=k[:, :, :8]), dict(k=k[:4]), dict(q_out=k), dict(k_out=None),
                dict(k=None), dict(q=torch.zeros(5, 4, 32)[..., ::2]), dict(positions=positions.float()), dict(positions=positions[:4]),
                dict(positions=torch.zeros(10, dtype=torch.int32)[::2]), dict(f=f.float()), dict(f=f[None]), dict(q="q"), dict()):
        with pytest.raises(ValueError):
            call(**bad)
    for gains in ((w[:8], w), (w, w.bfloat16()), (w, None), (w.half(), w.half())):
        with pytest.raises(ValueError):
            B.sparseloco_qk_norm_rotary(q, k, *gains, positions, f, q, k)
    with pytest.raises(B.SparseLoCoError):
        B.qk_norm_rotary_workspace(2 ** 40, 1, 1, 16)
    for bad in (dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=8, factor=0.5), dict(rotary_dim=8, scaling="other"),
                dict(rotary_dim=2, scaling="base"), dict(rotary_dim=8, scaling="by_parts", fast=1.0)):
        with pytest.raises(ValueError):
            B.rotary_frequencies(device="cpu", **bad)


def test_native_calls_hand_back_what_is_not_plainly_right():
    native, x = B._native(), torch.zeros(5, 4, 16)
    for name in ("rotary", "qk_norm_rotary", "qk_norm_rotary_grad"):
        for args in ((), (None,), (x,) * 5, (x,) * 17, (None,) * 30, ("0",) * 12):
            assert getattr(native, name)(*args) is None


def test_gains_gradients_in_one_place():
    """Sums of queries and of keys are finished side by side: in one buffer one would be lost, or read too early to be added to."""
    lists = [heads(ANY * i) for i in range(1, 7)]

    def call(q_sum, k_sum, tokens=5):
        return B.lib().sparseloco_qk_norm_rotary_grad(*lists[:4], 0, tokens, 16, ANY, ANY, 0, 1e-6, how(), *lists[4:], q_sum, k_sum, 1, 64 * ANY, 1 << 30,
                                                      None)
    for tokens in (5, 0):
        for apart in (-60, -4, 0, 4, 60):
            assert call(32 * ANY, 32 * ANY + apart, tokens) == B.SPLC_EINVAL, apart
