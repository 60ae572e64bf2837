"""Orthogonalised updates: bad arguments are refused on the host, before anything touches a GPU."""
import ctypes

import pytest
import torch

from paper_2601_02360_amd import binding as B


def test_null_handles():
    L = B.lib()
    rows = (ctypes.c_int64 * 1)(4)
    how = B._Muon(1e-3, 0.9, 0.1, 1e-7, None, 5, 1, 0, B.SPLC_MATMUL_FP16)
    any_ = ctypes.c_void_p(4096)
    assert L.sparseloco_orthogonalize_ws_bytes(None, rows, B.SPLC_MATMUL_FP16) == B.SPLC_EINVAL
    assert L.sparseloco_orthogonalize(None, rows, any_, any_, 0, None, 5, 1e-7, B.SPLC_MATMUL_FP16, any_, 1 << 30, None) == B.SPLC_EINVAL
    assert L.sparseloco_muon_step(None, rows, any_, any_, any_, 0, ctypes.byref(how), None, None, None, any_, 1 << 30, None) == B.SPLC_EINVAL
    assert L.sparseloco_muon_step(any_, rows, any_, any_, any_, 0, None, None, None, None, any_, 1 << 30, None) == B.SPLC_EINVAL
    assert L.sparseloco_muon_step(any_, rows, any_, any_, any_, -1, ctypes.byref(how), None, None, None, any_, 1 << 30, None) == B.SPLC_EINVAL


def test_what_the_binding_refuses():
    ws = torch.zeros(100, dtype=torch.uint8)
    for bad in ([], [(1.0, 2.0)], [(1.0, 2.0, 3.0, 4.0)]):
        with pytest.raises(ValueError):
            B.sparseloco_orthogonalize(None, [], [], ws, coefficients=bad)
    for bad in (ws, ws.float(), ws[::2], None):
        with pytest.raises(ValueError):
            B.sparseloco_orthogonalize(None, [], [], bad)


@pytest.mark.gpu
def test_what_the_library_refuses():
    plan = B.Plan([(6, 8), (5, 3)], 32)
    x = [torch.ones(6, 8, device="cuda"), torch.ones(5, 3, device="cuda")]
    out = [t.clone() for t in x]
    ws = B.orthogonalize_workspace(plan)
    small = B.orthogonalize_workspace(plan, matmul=B.SPLC_MATMUL_FP16)
    assert small.numel() < ws.numel()

    def ortho(x=x, out=out, ws=ws, **how):
        with pytest.raises((ValueError, B.SparseLoCoError)):
            B.sparseloco_orthogonalize(plan, x, out, ws, **how)
    ortho(ws=ws[:-1])
    ortho(ws=small)
    ortho(ws=torch.empty(ws.numel() + 1, dtype=torch.uint8, device="cuda")[1:])
    for how in (dict(eps=-1.0), dict(eps=float("nan")), dict(matmul=B.SPLC_MATMUL_FP32), dict(matmul=7), dict(replica=-1), dict(replica=2 ** 31),
                dict(coefficients=[(1.0, 0.0, 0.0)] * 17), dict(coefficients=[(float("nan"), 0.0, 0.0)]), dict(coefficients=[(2e4, 0.0, 0.0)]),
                dict(coefficients=[(100.0, 0.0, 0.0)] * 2)):
        ortho(**how)
    ortho(x=x[:1])
    ortho(x=[x[0], x[1].half()])

    def step(**how):
        with pytest.raises((ValueError, B.SparseLoCoError)):
            B.sparseloco_muon_step(plan, out, x, x, ws, **dict(dict(lr=1e-3), **how))
    for how in (dict(lr=-1.0), dict(lr=float("nan")), dict(momentum=1.0), dict(momentum=-0.1), dict(weight_decay=-1.0), dict(adjust=3),
                dict(matmul=0), dict(eps=-1.0), dict(decay=torch.ones(1, device="cuda")), dict(grad_scale=torch.ones(2, device="cuda"))):
        step(**how)
    bad_rows = (ctypes.c_int64 * 2)(6, 4)
    assert B.lib().sparseloco_orthogonalize_ws_bytes(plan.handle, bad_rows, B.SPLC_MATMUL_FP16) == B.SPLC_EINVAL
    assert B.lib().sparseloco_orthogonalize_ws_bytes(plan.handle, None, B.SPLC_MATMUL_FP16) == B.SPLC_EINVAL
    long = B.Plan([2 ** 22 + 1], 32)
    with pytest.raises(B.SparseLoCoError):
        B.orthogonalize_workspace(long)
    torch.cuda.synchronize()
    assert all(bool((t == 1).all()) for t in out)


def test_how_products_are_cut_up():
    """The answer is host logic alone; tiles by how many of them there are, and several steps at once where that pays."""
    choice = B.orthogonalize_choice
    x3, one = B.SPLC_MATMUL_FP16X3, B.SPLC_MATMUL_FP16
    assert choice([]) == ([], 128)
    assert [c[2:] for c in choice([(300, 200)])[0]] == [(32, 32, 32)]
    assert {c[2:4] for c in choice([(1270, 1270)] * 17)[0]} == {(256, 256)} == {c[2:4] for c in choice([(1270, 1270)] * 17, matmul=one)[0]}
    for shapes in ([(5630, 2050)] * 3, [(2050, 5630)] * 3, [(768, 2048)] * 9 + [(768, 768)] * 12, [(2048, 5632)] * 48 + [(2048, 2048)] * 64):
        found, size = choice(shapes)
        assert [c[0] for c in found] == [r != c for r, c in shapes]
        other, small = choice(shapes, matmul=one)
        assert not any(c[0] for c in other) and 0 < small < size
    many, _ = choice([(3, 5)] * 300)
    assert [max(c[1] for c in many), min(c[1] for c in many)] == [2, 0] and all(sum(c[1] == i for c in many) <= 128 for i in range(3))
    L, sides = B.lib(), (ctypes.c_int64 * 2)(4, 4)
    for n, rows, columns, matmul in ((-1, sides, sides, x3), (2, None, sides, x3), (2, sides, None, x3), (2, sides, sides, B.SPLC_MATMUL_FP32),
                                     (1, (ctypes.c_int64 * 1)(0), sides, x3), (1, sides, (ctypes.c_int64 * 1)(2 ** 22 + 1), x3)):
        assert L.sparseloco_orthogonalize_choice(n, rows, columns, matmul, None) == B.SPLC_EINVAL
    assert L.sparseloco_orthogonalize_choice(2, sides, sides, x3, None) == choice([(4, 4), (4, 4)])[1]


@pytest.mark.parametrize("matmul", [B.SPLC_MATMUL_FP16X3, B.SPLC_MATMUL_FP16])
@pytest.mark.parametrize("shapes", [[(22000, 22000)] * 4, [(22000, 22000)] * 9, [(40000, 8000)] * 7 + [(20000, 20000)] * 3 + [(60000, 512)] * 40,
                                    [(30000, 30000)] * 2 + [(9000, 9000)] * 20, [(50000, 50000), (3, 3)], [(4096, 16384)] * 200], ids=str)
def test_batches_keep_their_bound(matmul, shapes):
    """16 GiB of operands at once, or one matrix."""
    choice, size = B.orthogonalize_choice(shapes, matmul=matmul)
    small = 8 * (len(shapes) + sum(-(-r * c // 4096) for r, c in shapes)) + 128
    operands = lambda shape: B.orthogonalize_choice([shape], matmul=matmul)[1]
    assert size <= max([2 ** 34] + [operands(s) for s in shapes]) + small
    assert sorted({c[1] for c in choice}) == list(range(1 + max(c[1] for c in choice)))
