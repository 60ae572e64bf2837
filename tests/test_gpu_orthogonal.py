"""Orthogonalised matrices and the step that takes them against a plain implementation in 64 bits.

Tolerances come from the inputs' singular values.  A step X' = a X + B X, B = b A + c A^2, A = X X^T, with operands rounded to
half steps u (2^-11 for FP16, 2^-22 for FP16X3) makes independent errors of rms 0.41 u (a relative error uniform in half a step,
over mantissas that are uniform in their logarithm); an error matrix E independent of X multiplies it to |E X| = |E| |X| / sqrt(n).  fp32
sums of K products are added 16 at a time: sqrt(3 K / 16) roundings of 2^-24 where three products make one.  An error in X goes on into
X' times the largest divided difference of the polynomial between singular values (and their negatives), the norm of the map's
derivative.  Four times the sum of squares is allowed for the whole, and eight times an even share for a single row or column."""
import math

import pytest
import torch

from paper_2601_02360_amd import binding as B

pytestmark = pytest.mark.gpu
USUAL = list(B.USUAL_COEFFICIENTS)
MODES = {"fp16": (B.SPLC_MATMUL_FP16, 2.0 ** -11), "fp16x3": (B.SPLC_MATMUL_FP16X3, 2.0 ** -22)}


def plain(m, coefficients=USUAL, eps=1e-7):
    x = m.double()
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / (x.square().sum().sqrt() + eps)
    for a, b, c in coefficients:
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return x.T if tall else x


def tolerance(m, u, coefficients=USUAL, eps=1e-7):
    """Expected 2-norm of the error."""
    s = torch.linalg.svdvals(m.double().cpu())
    s = s / (s.square().sum().sqrt() + eps)
    n, depth = len(s), max(m.shape)
    square = lambda *v: math.sqrt(sum(x * x for x in v))
    rho, total = 0.41 * u, 0.41 * u * float(s.norm())
    add = 2.0 ** -24 * math.sqrt(3 * depth / 16)
    for a, b, c in coefficients:
        f, fa = float(s.norm()), float(s.square().norm())
        new = a * s + b * s ** 3 + c * s ** 5
        fb = float((b * s ** 2 + c * s ** 4).norm())
        r, ra, rb = f / math.sqrt(n), fa / math.sqrt(n), fb / math.sqrt(n)
        in_a = square(math.sqrt(2) * r * rho * f, rho * fa, add * f * r)
        in_b = square(b * in_a, 2 * c * in_a * ra, rho * fb, add * c * fa * ra)
        step = square(in_b * r, rb * rho * f, add * fb * r)
        both, after = torch.cat([s, -s]), torch.cat([new, -new])
        gap = both[:, None] - both[None]
        slope = (after[:, None] - after[None]) / torch.where(gap.abs() < 1e-9, torch.ones_like(gap), gap)
        slope = torch.where(gap.abs() < 1e-9, (a + 3 * b * both ** 2 + 5 * c * both ** 4)[:, None].expand_as(slope), slope)
        total = square(float(slope.abs().max()) * total, step)
        s = new
    return total


def agree(got, m, u, want=None, limit=None, **how):
    want = plain(m, **how) if want is None else want
    limit = tolerance(m, u, **how) if limit is None else limit
    half = torch.finfo(got.dtype).eps / 2
    off = got.double() - want
    assert bool(torch.isfinite(off).all())
    size = float(want.norm())
    assert float(off.norm()) <= 4 * limit + half * size, (float(off.norm()) / max(size, 1e-30), limit / max(size, 1e-30))
    for k in (0, 1):
        lines = off.norm(dim=k)
        share = 8 * limit / math.sqrt(len(lines)) + half * want.norm(dim=k)
        assert bool((lines <= share).all()), (k, int((lines - share).argmax()), float((lines / share).max()))


def in_squares(m, u, coefficients=USUAL, eps=1e-7):
    """The error to expect where up to three steps at a time are taken in squares (A = X X^T; for each step B = b A + c A^2, Q = p Q, A = p A p
    with p = a + B; X = Q X; the product of the a's at most 64): of these formulas in 64 bits with every result off by independent
    relative errors of rms 0.41 u, as rounding it to hi + lo makes, and by what fp32 sums add."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    add = 2.0 ** -24 * math.sqrt(3 * max(m.shape) / 16)

    def off(t, sums=None):
        noise = torch.randn(t.shape, generator=gen, device="cuda", dtype=torch.float64) * 0.41 * u * t.abs()
        if sums is not None:                                 # rms of the terms' sum
            noise = noise + torch.randn(t.shape, generator=gen, device="cuda", dtype=torch.float64) * add * sums
        return t + noise

    def times(x, y, own=0.0, old=0.0):
        z = x @ y
        return off(own * old + z, (x.square() @ y.square()).sqrt())
    x = m.double()
    x = x.T if x.shape[0] > x.shape[1] else x
    x = off(x / (x.square().sum().sqrt() + eps))
    k = 0
    while k < len(coefficients):
        count, alpha = 1, coefficients[k][0]
        while count < 3 and k + count < len(coefficients) and abs(alpha * coefficients[k + count][0]) <= 64:
            alpha *= coefficients[k + count][0]
            count += 1
        g, q, of_one = times(x, x.T), None, 1.0
        for a, b, c in coefficients[k:k + count]:
            p = times(c * g, g, b, g)
            q = p if q is None else times(p, q, 1.0, a * q + of_one * p)
            of_one *= a
            t = times(p, g, a, g)
            g = times(p, t, a, t)
        x = times(q, x, of_one, x)
        k += count
    want = plain(m, coefficients, eps)
    return float(((x.T if m.shape[0] > m.shape[1] else x) - want).norm())


def matrix(rows, cols, kind, seed, dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    if kind == "strong":
        x += torch.randn(rows, 4, generator=gen, device="cuda") @ torch.randn(4, cols, generator=gen, device="cuda") * 2
    return (x * 1e-3).to(dtype)


SHAPES = [(1, 1), (1, 5), (700, 1), (2, 2), (3, 70), (64, 64), (65, 64), (63, 129), (128, 128), (129, 257), (300, 128), (127, 640),
          (513, 130), (256, 512), (40, 1000), (321, 320)]


def bound(plan, tensors):
    return plan.bind(tensors, dtype=tensors[0].dtype)


def packed(tensors, lead=1):
    """The tensors in one flat buffer, from 4 `lead` bytes on at multiples of 4 bytes, so that most start at no multiple of 8."""
    step = 4 // tensors[0].element_size()
    at = [lead * step]
    for t in tensors:
        at.append(at[-1] + -(-t.numel() // step) * step)
    flat = torch.zeros(at[-1], dtype=tensors[0].dtype, device="cuda")
    views = [flat[a:a + t.numel()].view(t.shape) for a, t in zip(at, tensors)]
    for v, t in zip(views, tensors):
        v.copy_(t)
    return views


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("kind", ["noise", "strong"])
def test_shapes(mode, kind):
    matmul, u = MODES[mode]
    x = packed([matrix(r, c, kind, 10 + i) for i, (r, c) in enumerate(SHAPES)])
    out = packed([torch.full_like(t, float("nan")) for t in x])
    plan = B.Plan(SHAPES, 32)
    ws = B.orthogonalize_workspace(plan, matmul=matmul).fill_(255)
    B.sparseloco_orthogonalize(plan, bound(plan, x), bound(plan, out), ws, matmul=matmul)
    for t, o in zip(x, out):
        agree(o, t, u)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("types", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16)])
def test_types(mode, types):
    matmul, u = MODES[mode]
    shapes = [(200, 136), (96, 333)]
    x = packed([matrix(*s, "noise", 3 + i, types[0]) for i, s in enumerate(shapes)])
    out = packed([torch.zeros(s, dtype=types[1], device="cuda") for s in shapes])
    plan = B.Plan(shapes, 32, tiled=True)
    B.sparseloco_orthogonalize(plan, x, out, B.orthogonalize_workspace(plan, matmul=matmul), matmul=matmul)       # plain lists
    for t, o in zip(x, out):
        agree(o, t, u)


@pytest.mark.parametrize("mode", MODES)
def test_other_polynomials(mode):
    """Cubic steps towards the polar factor, few and many, one that changes every step, and ranges far from 1."""
    matmul, u = MODES[mode]
    x = matrix(150, 260, "noise", 5)
    plan = B.Plan([x.shape], 32)
    ws, out = B.orthogonalize_workspace(plan, matmul=matmul), torch.empty_like(x)
    for c in ([(1.5, -0.5, 0.0)] * 16, [(3.4445, -4.7750, 2.0315)], [(8.2, -23.5, 17.3), (4.1, -2.95, 0.545), (1.875, -1.25, 0.375)],
              [(1.0, 0.0, 0.0)], [(20.0, 3.0, 0.0), (0.05, -0.001, 0.0)], [(0.001, 0.0, 0.5)]):
        B.sparseloco_orthogonalize(plan, [x], [out], ws, coefficients=c, matmul=matmul)
        agree(out, x, u, coefficients=c)


@pytest.mark.parametrize("kind", ["noise", "strong"])
def test_steps_taken_in_squares(kind):
    """Matrices of 512 rows or more that are half as wide again, wide and tall, beside others in one call; single steps, pairs, triples."""
    matmul, u = MODES["fp16x3"]
    shapes = [(512, 768), (700, 600), (520, 1600), (1700, 513), (65, 64), (513, 1025)]
    x = packed([matrix(r, c, kind, 60 + i) for i, (r, c) in enumerate(shapes)])
    plan = B.Plan(shapes, 32)
    ws = B.orthogonalize_workspace(plan, matmul=matmul)
    for c in (USUAL, USUAL[:1], USUAL[:4], [(1.5, -0.5, 0.0)] * 8, [(8.2, -23.5, 17.3), (4.1, -2.95, 0.545), (1.875, -1.25, 0.375)],
              [(70.0, -50.0, 0.0), (0.02, 0.0, 0.0)]):
        out = packed([torch.full_like(t, float("nan")) for t in x])
        B.sparseloco_orthogonalize(plan, bound(plan, x), bound(plan, out), ws.fill_(255), coefficients=c, matmul=matmul)
        for t, o in zip(x, out):
            wide = min(t.shape) >= 512 and 2 * max(t.shape) >= 3 * min(t.shape)
            agree(o, t, u, limit=in_squares(t, u, c) if wide else None, coefficients=c)


@pytest.mark.parametrize("mode", MODES)
def test_enough_matrices_for_the_largest_tiles(mode):
    """Ragged ones, square and tall, so many that products are cut into tiles of 256 and 128."""
    matmul, u = MODES[mode]
    shapes = [(1270, 1270)] * 24 + [(2601, 1270)] * 12
    x = packed([matrix(r, c, "strong", 80 + i) for i, (r, c) in enumerate(shapes)])
    out = packed([torch.full_like(t, float("nan")) for t in x])
    plan = B.Plan(shapes, 32)
    B.sparseloco_orthogonalize(plan, bound(plan, x), bound(plan, out), B.orthogonalize_workspace(plan, matmul=matmul).fill_(255), matmul=matmul)
    for i in (0, 23, 35):
        limit = tolerance(x[i], u)
        agree(out[i], x[i], u, limit=max(limit, in_squares(x[i], u)) if mode == "fp16x3" and i == 35 else limit)
    for i, t in enumerate(out):
        o = t.double() if i < 24 else t.T.double()           # O O^T has the squares of the result's singular values, 0.68^2 to 1.21^2
        assert float((o @ o.T).diagonal().sqrt().max()) < 1.22 and bool(torch.isfinite(o).all())


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("scale", [1e-30, 1.0, 1e30])
def test_matrices_whose_result_is_known(mode, scale):
    """c Q with Q's rows orthonormal becomes p(...p(1 / sqrt(n))) Q: permutations and a Hadamard matrix."""
    matmul, u = MODES[mode]
    n = 128
    gen = torch.Generator(device="cuda").manual_seed(0)
    q = torch.zeros(n, 200, device="cuda")
    q[torch.arange(n), torch.randperm(200, generator=gen, device="cuda")[:n]] = 1.0
    h = torch.ones(1, 1, device="cuda")
    while len(h) < n:
        h = torch.cat([torch.cat([h, h], 1), torch.cat([h, -h], 1)])
    for exact in (q, q.T.contiguous(), h / math.sqrt(n)):
        x = exact * scale
        plan = B.Plan([x.shape], 32)
        out = torch.empty_like(x)
        B.sparseloco_orthogonalize(plan, [x], [out], B.orthogonalize_workspace(plan, matmul=matmul), matmul=matmul, eps=0.0)
        s = 1 / math.sqrt(n)
        for a, b, c in USUAL:
            s = a * s + b * s ** 3 + c * s ** 5
        agree(out, x / scale, u, want=exact.double() * s, eps=0.0)


@pytest.mark.parametrize("mode", MODES)
def test_many_matrices_zeros_and_one_that_is_not_finite(mode):
    """More than a batch of them; what is wrong with one matrix stays there; empty tensors; the result in the input's place."""
    matmul, u = MODES[mode]
    shapes = [(7 + i % 5, 3 + i % 7) for i in range(301)]
    shapes[20] = (0, 4)
    x = [matrix(r, c, "noise", 100 + i) for i, (r, c) in enumerate(shapes)]
    plan = B.Plan(shapes, 32)
    ws = B.orthogonalize_workspace(plan, matmul=matmul)
    clean = [torch.empty_like(t) for t in x]
    B.sparseloco_orthogonalize(plan, x, clean, ws, matmul=matmul)
    for t, o in zip(x, clean):
        if t.numel():
            agree(o, t, u)
    bad = [t.clone() for t in x]
    bad[3].zero_()
    bad[50][1, 1], bad[60][0, 0] = float("nan"), float("inf")
    B.sparseloco_orthogonalize(plan, bad, bad, ws, matmul=matmul)
    for i, (a, b) in enumerate(zip(clean, bad)):
        if i == 3:
            assert bool((b == 0).all())
        elif i in (50, 60):
            assert bool(torch.isnan(b).all())
        else:
            assert torch.equal(a, b)


def step_reference(theta, g, m, lr, momentum, nesterov, decay, adjust, eps=1e-7):
    m = momentum * m.double() + (1 - momentum) * g
    u = momentum * m + (1 - momentum) * g if nesterov else m
    rows, cols = theta.shape
    f = {B.SPLC_MUON_NONE: 1.0, B.SPLC_MUON_ASPECT: math.sqrt(max(1.0, rows / cols)),
         B.SPLC_MUON_RMS: 0.2 * math.sqrt(max(rows, cols))}[adjust]
    return m, u, theta.double() * (1 - lr * decay) - lr * f * plain(u, eps=eps), f


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("nesterov,adjust,grads,clipped,copied", [
    (True, B.SPLC_MUON_RMS, torch.float32, True, True), (True, B.SPLC_MUON_ASPECT, torch.bfloat16, False, True),
    (False, B.SPLC_MUON_NONE, torch.bfloat16, True, False)])
def test_step(mode, nesterov, adjust, grads, clipped, copied):
    matmul, unit = MODES[mode]
    shapes = [(130, 200), (64, 64), (257, 96), (1, 33)]
    gen = torch.Generator(device="cuda").manual_seed(1)
    theta = packed([torch.randn(s, generator=gen, device="cuda") * 0.02 for s in shapes])
    g = packed([matrix(*s, "strong", 20 + i, grads) for i, s in enumerate(shapes)], 3)
    m = packed([matrix(*s, "strong", 30 + i) for i, s in enumerate(shapes)], 2)
    copy = packed([torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in shapes]) if copied else None
    old = [[t.clone() for t in x] for x in (theta, m)]
    scale = torch.full((1,), 0.375, device="cuda") if clipped else None
    decays = torch.tensor([1.0, 0.0, 2.0, 0.5], device="cuda")
    plan = B.Plan(shapes, 32)
    lr, wd = 2e-2, 0.25
    B.sparseloco_muon_step(plan, theta, g, m, B.orthogonalize_workspace(plan, matmul=matmul), lr=lr, momentum=0.9, nesterov=nesterov,
                           weight_decay=wd, adjust=adjust, grad_scale=scale, decay=decays, theta_bf16=copy, matmul=matmul)
    for i in range(len(shapes)):
        gradient = g[i].double() * (0.375 if clipped else 1.0)
        want_m, u, want, f = step_reference(old[0][i], gradient, old[1][i], lr, 0.9, nesterov, wd * float(decays[i]), adjust)
        # m: two products and a sum, and the coefficients' own roundings
        size = 0.9 * old[1][i].double().abs() + 0.1 * gradient.abs()
        assert bool(((m[i].double() - want_m).abs() <= 5 * 2.0 ** -24 * size).all())
        limit = tolerance(u, unit) * 4 * lr * f + 2.0 ** -24 * 4 * float(want.norm())
        assert float((theta[i].double() - want).norm()) <= limit
        lines = (theta[i].double() - want).norm(dim=1)
        assert bool((lines <= 8 * tolerance(u, unit) * lr * f / math.sqrt(shapes[i][0]) + 2.0 ** -22 * want.norm(dim=1)).all())
        if copied:
            assert torch.equal(copy[i], theta[i].bfloat16())


def test_a_factor_that_is_not_finite_leaves_everything():
    shapes = [(70, 90), (5, 5)]
    plan = B.Plan(shapes, 32)
    make = lambda seed, dtype=torch.float32: [matrix(*s, "noise", seed + i, dtype) for i, s in enumerate(shapes)]
    theta, g, m = make(1), make(5), make(9)
    copy = make(13, torch.bfloat16)
    old = [t.clone() for t in theta + m + copy]
    ws = B.orthogonalize_workspace(plan)
    for bad in (float("nan"), float("inf")):
        B.sparseloco_muon_step(plan, theta, g, m, ws, lr=0.1, grad_scale=torch.full((1,), bad, device="cuda"), theta_bf16=copy)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(old, theta + m + copy))
    zero = [torch.zeros_like(t) for t in theta]
    B.sparseloco_muon_step(plan, theta, zero, [t.zero_() for t in m], ws, lr=0.1, weight_decay=0.5)
    for a, b in zip(old, theta):
        assert float((a.double() * 0.95 - b.double()).abs().max()) <= 4 * 2.0 ** -24 * float(a.abs().max())


def test_replicas_streams_and_replays_of_a_graph():
    """Two sets of tensors; the calls on another stream; a captured step replayed with eager work between, every time the same bits."""
    shapes = [(200, 300), (160, 70)]
    plan = B.Plan(shapes, 32)
    make = lambda seed: [matrix(*s, "noise", seed + i) for i, s in enumerate(shapes)]
    sets = [make(1), make(3)]
    b_theta = plan.bind(sets)
    g, m = [make(5), make(7)], [make(9), make(11)]
    b_g, b_m = plan.bind(g), plan.bind(m)
    start = [[t.clone() for t in s] for s in sets], [[t.clone() for t in s] for s in m]

    def reset():
        for now, was in ((sets, start[0]), (m, start[1])):
            for a, b in zip(now, was):
                for x, y in zip(a, b):
                    x.copy_(y)
    ws = [B.orthogonalize_workspace(plan) for _ in range(2)]

    def step(replica, space, stream=None):
        B.sparseloco_muon_step(plan, b_theta, b_g, b_m, space, lr=0.05, replica=replica, stream=stream)
    step(0, ws[0])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(sets[1] + m[1], start[0][1] + start[1][1]))
    step(1, ws[0])
    torch.cuda.synchronize()
    want = [t.clone() for t in sets[0] + sets[1] + m[0] + m[1]]
    side = [torch.cuda.Stream() for _ in range(2)]
    reset()
    torch.cuda.synchronize()
    for replica in (0, 1):                                   # side by side, with a workspace each
        step(replica, ws[replica], side[replica])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, sets[0] + sets[1] + m[0] + m[1]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0, ws[0])
        step(1, ws[0])
    for _ in range(4):
        reset()
        B.orthogonalize_workspace(plan).fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, sets[0] + sets[1] + m[0] + m[1]))
