"""Orthogonalised matrices on the paths that shapes choose: every size of tiles, and several steps at once in squares."""
import math

import pytest
import torch

from paper_2601_02360_amd import binding as B
from test_gpu_orthogonal import MODES, USUAL, agree, bound, in_squares, matrix, packed, plain, step_reference, tolerance

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("shapes", [[(300, 200)], [(768, 768)], [(1270, 1270)] * 4, [(1270, 1270)] * 17], ids=lambda s: "%d of %dx%d" % (len(s), *s[0]))
def test_the_same_call_gives_the_same_bits(mode, shapes):
    """Sums of a tile take its operands' place in LDS while the last fetches of operands are under way: what lands late would show as
    bits that differ from call to call, the more so where another call's workgroups run beside it."""
    matmul, _ = MODES[mode]
    x = [matrix(*s, "strong", 40 + i, torch.bfloat16) for i, s in enumerate(shapes)]
    plan = B.Plan(shapes, 32)
    ws = [B.orthogonalize_workspace(plan, matmul=matmul) for _ in range(2)]
    outs = [[torch.full_like(t, float("nan")) for t in x] for _ in range(4)]
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    B.sparseloco_orthogonalize(plan, x, outs[0], ws[0], matmul=matmul)
    torch.cuda.synchronize()
    B.sparseloco_orthogonalize(plan, x, outs[1], ws[0].fill_(255), matmul=matmul)
    torch.cuda.synchronize()
    for i in range(2):
        B.sparseloco_orthogonalize(plan, x, outs[2 + i], ws[i], matmul=matmul, stream=side[i])
    torch.cuda.synchronize()
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))
    assert all(bool(torch.isfinite(t).all()) for t in outs[0])


def orthogonalised(x, matmul, coefficients):
    shapes = [tuple(t.shape) for t in x]
    plan, out = B.Plan(shapes, 32), packed([torch.full_like(t, float("nan")) for t in x])
    ws = B.orthogonalize_workspace(plan, matmul=matmul)
    assert ws.numel() == B.orthogonalize_choice(shapes, matmul=matmul)[1]
    B.sparseloco_orthogonalize(plan, bound(plan, x), bound(plan, out), ws.fill_(255), coefficients=coefficients, matmul=matmul)
    return out


POLYNOMIALS = {
    "usual": USUAL, "one step": USUAL[:1], "three and one": USUAL[:4], "cubic": [(1.5, -0.5, 0.0)] * 8,
    "changing": [(8.2, -23.5, 17.3), (4.1, -2.95, 0.545), (1.875, -1.25, 0.375)], "large, then small": [(70.0, -50.0, 0.0), (0.02, 0.0, 0.0)],
    # 8 x 10 is above 64: a step by itself, then two
    "cut": [(8.0, -8.0, 0.0), (10.0, -0.8, 0.0), (0.1, 0.0, 0.0)]}


@pytest.mark.parametrize("polynomial", POLYNOMIALS)
@pytest.mark.parametrize("shapes,tiles", [([(70, 2241)], (32, 32, 64)), ([(2241, 70), (70, 2241)] * 24, (64, 64, 128)),
                                          ([(510, 1021), (1021, 510)] * 8 + [(510, 1021)], (128, 128, 128)),
                                          ([(900, 1801), (1801, 900)] * 12, (256, 256, 256))],
                         ids=lambda v: "%d of %dx%d" % (len(v), *v[0]) if isinstance(v, list) else "tiles %d" % v[1])
def test_steps_in_squares(polynomial, shapes, tiles):
    """Wide and tall matrices that take several steps at once, with every size of tiles for the products of squares (a third operand
    among them); single steps, pairs and triples, and where the product of the polynomials' first numbers ends one."""
    matmul, u = MODES["fp16x3"]
    assert all(c == (True, 0) + tiles for c in B.orthogonalize_choice(shapes, matmul=matmul)[0])
    x = packed([matrix(r, c, "noise" if i % 3 else "strong", 200 + i) for i, (r, c) in enumerate(shapes)])
    for t, o in zip(x, orthogonalised(x, matmul, POLYNOMIALS[polynomial])):
        agree(o, t, u, limit=in_squares(t, u, POLYNOMIALS[polynomial]), coefficients=POLYNOMIALS[polynomial])


@pytest.mark.parametrize("polynomial", POLYNOMIALS)
def test_steps_in_squares_beside_others(polynomial):
    """Matrices of both kinds in one call."""
    matmul, u = MODES["fp16x3"]
    shapes = [(767, 767)] * 12 + [(767, 2050)] * 9
    shapes[3], shapes[15] = shapes[15], shapes[3]
    assert [c[0] for c in B.orthogonalize_choice(shapes, matmul=matmul)[0]] == [c > 767 for _, c in shapes]
    x = packed([matrix(r, c, "strong", 300 + i) for i, (r, c) in enumerate(shapes)])
    c = POLYNOMIALS[polynomial]
    square = tolerance(x[0], u, c)                           # (the others' singular values are spread alike)
    for t, o in zip(x, orthogonalised(x, matmul, c)):
        agree(o, t, u, limit=in_squares(t, u, c) if t.shape[1] > 767 else square, coefficients=c)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("polynomial", ["usual", "changing"])
def test_symmetric_products_in_the_largest_tiles(mode, polynomial):
    """X X^T and A^2 in tiles of 256, where a wave has two blocks and those below the diagonal are another's mirror image, ragged."""
    matmul, u = MODES[mode]
    shapes = [(1270, 1271 - i % 2) for i in range(17)]
    assert all(c[2:4] == (256, 256) for c in B.orthogonalize_choice(shapes, matmul=matmul)[0])
    x = packed([matrix(r, c, "strong", 400 + i) for i, (r, c) in enumerate(shapes)])
    c = POLYNOMIALS[polynomial]
    limit = tolerance(x[0], u, c)
    for t, o in zip(x, orthogonalised(x, matmul, c)):
        agree(o, t, u, limit=limit, coefficients=c)


@pytest.mark.parametrize("mode,shapes", [("fp16x3", [(900, 1801), (1801, 900)] * 12), ("fp16x3", [(1270, 1271)] * 17), ("fp16", [(1270, 1271)] * 17)],
                         ids=["squares", "fp16x3", "fp16"])
def test_step_of_large_tiles(mode, shapes):
    matmul, u = MODES[mode]
    choice = B.orthogonalize_choice(shapes, matmul=matmul)[0]
    assert all(c[0] == (len(shapes) == 24) and c[2:4] == (256, 256) for c in choice)
    gen = torch.Generator(device="cuda").manual_seed(1)
    theta = packed([torch.randn(s, generator=gen, device="cuda") * 0.02 for s in shapes])
    g = packed([matrix(*s, "strong", 20 + i, torch.bfloat16) for i, s in enumerate(shapes)])
    m = packed([matrix(*s, "strong", 60 + i) for i, s in enumerate(shapes)])
    copy = packed([torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in shapes])
    old = [[t.clone() for t in x] for x in (theta, m)]
    plan, lr, wd = B.Plan(shapes, 32), 2e-2, 0.25
    B.sparseloco_muon_step(plan, bound(plan, theta), bound(plan, g), bound(plan, m), B.orthogonalize_workspace(plan, matmul=matmul).fill_(255),
                           lr=lr, weight_decay=wd, theta_bf16=bound(plan, copy), grad_scale=torch.full((1,), 0.5, device="cuda"), matmul=matmul)
    limit = None
    for i in range(len(shapes)):
        gradient = g[i].double() * 0.5
        want_m, update, want, f = step_reference(old[0][i], gradient, old[1][i], lr, 0.95, True, wd, B.SPLC_MUON_RMS)
        assert bool(((m[i].double() - want_m).abs() <= 5 * 2.0 ** -24 * (0.95 * old[1][i].double().abs() + 0.05 * gradient.abs())).all())
        if choice[i][0]:
            limit = in_squares(update, u)
        elif limit is None:
            limit = tolerance(update, u)
        off = theta[i].double() - want
        assert float(off.norm()) <= 4 * limit * lr * f + 2.0 ** -24 * 4 * float(want.norm())
        assert bool((off.norm(dim=1) <= 8 * limit * lr * f / math.sqrt(shapes[i][0]) + 2.0 ** -22 * want.norm(dim=1)).all())
        assert torch.equal(copy[i], theta[i].bfloat16())


# Bounds of X far below 1 on the way: shrunk and grown again, by steps alone and before usual ones, and in the cube of a small X.
SHRINKING = {
    "identity": [(1e-4, 0.0, 0.0)] * 3 + [(1e4, 0.0, 0.0)] * 3,
    "before usual ones": [(1e-3, 0.0, 0.0)] * 2 + [(1e4, 0.0, 0.0), (100.0, 0.0, 0.0)] + USUAL,
    "cubes": [(1e-3, 0.0, 0.0), (0.0, 1e4, 0.0), (1e4, 0.0, 0.0), (10.0, 0.0, 0.0)],
    "a little beside 1": [(1.0, 1e-35, 1e-38), (3.0, 0.0, -1e-30)],
    "far": [(1e-30, 0.0, 0.0)] + [(1e4, 0.0, 0.0)] * 7 + [(100.0, 0.0, 0.0)],
}


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("polynomial", SHRINKING)
@pytest.mark.parametrize("rows,columns", [(150, 260), (70, 2241)])
def test_polynomials_that_shrink(mode, polynomial, rows, columns):
    """X is held to 22 bits of its bound after every step (the fold over the tolerance that counts the first step's alone: the root of
    as many roundings as there are steps, and 4 times is allowed: up to 13 steps)."""
    matmul, u = MODES[mode]
    c = SHRINKING[polynomial]
    x = [matrix(rows, columns, "strong", 500)]
    (out,) = orthogonalised(x, matmul, c)
    limit = max(tolerance(x[0], u, c), math.sqrt(len(c) + 1) / 4 * 0.41 * 2.0 ** -22 * float(plain(x[0], c).norm()))
    if B.orthogonalize_choice([(rows, columns)], matmul=matmul)[0][0][0]:
        limit = max(limit, in_squares(x[0], u, c))
    agree(out, x[0], u, limit=limit, coefficients=c)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("share", [1e-4, 1e-5, 1e-7])
def test_matrices_that_are_small_beside_eps(mode, share):
    """X = M / (|M| + eps) with |M| a small share of eps: an element is held to 22 bits, but not below 2^-39 of the singular values' bound
    (half of fp16's smallest number, 2^-25, over the scale of 2^14; 2^-38 once they are between 1 and 2), and five usual steps make 3.4445
    times as much of that each, 2^-38 * 3.4445^5 * (1 + 1 / 3.4445 + ...) = 2^-38 * 690 an element at the most."""
    matmul, u = MODES[mode]
    x = matrix(150, 260, "noise", 600)
    eps = 2.0 ** -20
    x *= share * eps / float(x.double().norm())
    plan, out = B.Plan([x.shape], 32), torch.empty_like(x)
    B.sparseloco_orthogonalize(plan, [x], [out], B.orthogonalize_workspace(plan, matmul=matmul), matmul=matmul, eps=eps)
    want = plain(x, eps=eps)
    # the steps' terms beyond the first are share^2 (their operands' rounding counts as that part of u)
    off = (out.double() - want).abs()
    assert float(off.max()) <= 690 * 2.0 ** -38 + (2.0 ** -22 + 8 * u * share ** 2 * 3.4445 ** 10) * float(want.abs().max())
