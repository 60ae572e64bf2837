"""The inner step's operators for attention heads and matrices, one after another as a replica runs them."""
import math

import pytest
import torch

from paper_2601_02360_amd import binding as B
from test_gpu_heads import gradient, normed, turned
from test_gpu_orthogonal import USUAL, plain, tolerance

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("matmul,unit", [(B.SPLC_MATMUL_FP16X3, 2.0 ** -22), (B.SPLC_MATMUL_FP16, 2.0 ** -11)])
def test_a_replicas_step(matmul, unit):
    """Lookup, a packed projection, normed and rotated heads, the way back into the packed gradient, the gradients' norm and the
    clipped step of both optimisers.  Gradients against 64 bits: rounding along products of 96 and 200 terms and through the heads
    (32 u and 104 u) makes (96 + 32 + 104 + 200) u at the worst, and the heads' gradient changes by up to four times what the heads
    are off: 1700 u, 1e-4.  Updates against the formulas on the gradients that are there."""
    vocab, d, tokens, hq, hk, hd = 50, 96, 200, 4, 2, 32
    gen = torch.Generator(device="cuda").manual_seed(0)
    table = torch.randn(vocab, d, generator=gen, device="cuda") * 0.5
    w = torch.randn((hq + 2 * hk) * hd, d, generator=gen, device="cuda") * 0.1
    gains = [1 + 0.1 * torch.randn(hd, generator=gen, device="cuda") for _ in range(2)]
    ids = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda", dtype=torch.int32)
    up = [torch.randn(tokens, h, hd, generator=gen, device="cuda") for h in (hq, hk)]
    positions = torch.arange(tokens, device="cuda") % 77
    f, magnitude = B.rotary_frequencies(hd, scaling="by_parts", factor=4.0, trained_length=32)

    def lists(packed):
        return packed[:, :hq * hd].unflatten(1, (hq, hd)), packed[:, hq * hd:(hq + hk) * hd].unflatten(1, (hk, hd))
    x, packed, d_packed = torch.empty(tokens, d, device="cuda"), torch.empty(tokens, len(w), device="cuda"), torch.zeros(tokens, len(w), device="cuda")
    B.sparseloco_embedding_lookup(table, ids, x)
    torch.mm(x, w.T, out=packed)
    q, k = lists(packed)
    outs, sums = [torch.empty(t.shape, device="cuda") for t in (q, k)], [torch.empty(hd, device="cuda") for _ in range(2)]
    B.sparseloco_qk_norm_rotary(q, k, *gains, positions, f, *outs, magnitude=magnitude)
    B.sparseloco_qk_norm_rotary_grad(*up, q, k, *gains, positions, f, *lists(d_packed), *sums, B.qk_norm_rotary_workspace(tokens, hq, hk, hd),
                                     magnitude=magnitude)
    d_w, d_table = torch.mm(d_packed.T, x), torch.empty_like(table)
    B.sparseloco_embedding_grad(torch.mm(d_packed, w), ids, d_table, B.embedding_grad_workspace(tokens, vocab, d))

    wx = table.double()[ids.long()]
    exact, found = wx @ w.double().T, torch.zeros(tokens, len(w), dtype=torch.float64, device="cuda")
    for side, (t, slot) in enumerate(zip(lists(exact), lists(found))):
        y = turned(normed(t, gains[side].double(), 1e-6), positions, f, magnitude, False)
        assert float((outs[side] - y).norm()) <= 1700 * U * float(y.norm())
        dx, dgain, _, _ = gradient(up[side].double(), t, gains[side].double(), positions, f, magnitude, False, 1e-6)
        slot.copy_(dx)
        assert float((sums[side] - dgain).norm()) <= 1700 * U * math.sqrt(tokens) * float(dgain.norm())
    assert bool((d_packed[:, (hq + hk) * hd:] == 0).all())
    for got, want in ((d_w, found.T @ wx), (d_table, torch.zeros_like(table, dtype=torch.float64).index_add(0, ids.long(), found @ w.double()))):
        assert float((got - want).norm()) <= 1700 * U * float(want.norm())

    plan, rows = B.Plan([w.shape], 32), B.Plan([table.shape], 32)
    norm, m = torch.empty(2, device="cuda"), torch.randn(w.shape, generator=gen, device="cuda") * float(d_w.std())
    B.sparseloco_grad_norm(plan, [d_w], norm, B.grad_norm_workspace(), max_norm=1.0)
    factor = float(norm[1])
    assert 0 < factor < 1
    old_w, old_m, copy = w.clone(), m.clone(), torch.empty_like(w, dtype=torch.bfloat16)
    lr, decay = 0.01, 0.1
    B.sparseloco_muon_step(plan, [w], [d_w], [m], B.orthogonalize_workspace(plan, matmul=matmul), lr=lr, weight_decay=decay, matmul=matmul,
                           grad_scale=norm[1:], theta_bf16=[copy])
    g = d_w.double() * factor
    want_m = 0.95 * old_m.double() + 0.05 * g
    u = 0.95 * want_m + 0.05 * g
    size = lr * 0.2 * math.sqrt(max(w.shape))
    want = old_w.double() * (1 - lr * decay) - size * plain(u)
    assert float((m - want_m).norm()) <= 8 * U * float(want_m.norm())
    assert float((w - want).norm()) <= 4 * tolerance(u, unit, USUAL) * size + 4 * U * float(want.norm())
    assert torch.equal(copy, w.bfloat16())
    first = [torch.zeros_like(table) for _ in range(2)]
    old = table.double()
    B.sparseloco_adamw_step(rows, [table], [d_table], [first[0]], [first[1]], lr=lr, step=1, eps=0.0, weight_decay=0.0, grad_scale=norm[1:])
    seen = d_table != 0                                      # (a first step is the gradient's sign)
    assert bool(((table.double() - old + lr * d_table.sign())[seen].abs() <= 32 * U * (lr + old[seen].abs())).all())


def test_native_calls_take_plain_arguments(monkeypatch):
    native, made = B._native(), []

    class Recorded:
        def __getattr__(self, name):
            def call(*args):
                made.append((name, getattr(native, name)(*args)))
                return made[-1][1]
            return call
    monkeypatch.setattr(B, "_native", lambda: Recorded())
    gen = torch.Generator(device="cuda").manual_seed(0)
    packed = torch.randn(30, 5, 16, generator=gen, device="cuda")
    f, _ = B.rotary_frequencies(16)
    results = []
    for stream, number, wide in ((None, float, False), (torch.cuda.Stream(), float, True), (None, int, False)):
        for keys in (True, False):
            q, k = packed[:, :3], packed[:, 3:] if keys else None
            positions = torch.arange(30, dtype=torch.int64 if wide else torch.int32, device="cuda")
            w = torch.linspace(1, 2, 16, device="cuda").bfloat16()
            like = lambda t: None if t is None else torch.zeros(t.shape, device="cuda")
            a, b, c, e, s = like(q), like(k), like(q), like(k), [torch.zeros(16, device="cuda") for _ in range(2)]
            ws = B.qk_norm_rotary_workspace(30, 3, 2, 16)
            torch.cuda.synchronize()
            made.clear()
            how = dict(magnitude=number(1), stream=stream)
            B.sparseloco_rotary(q, k, positions, f, a, b, inverse=True, **how)
            B.sparseloco_qk_norm_rotary(q, k, w, w if keys else None, positions, f, c, e, **how)
            torch.cuda.synchronize()
            results.append([t.clone() for t in (a, b, c, e) if t is not None])
            B.sparseloco_qk_norm_rotary_grad(a, b, q, k, w, w if keys else None, positions, f, c, e, s[0], s[1] if keys else None, ws, **how)
            torch.cuda.synchronize()
            results[-1] += [t.clone() for t in [c, e, s[0], s[1] if keys else None] if t is not None]
            if number is float:
                assert made == [(name, B.SPLC_OK) for name in ("rotary", "qk_norm_rotary", "qk_norm_rotary_grad")]
    for i, r in enumerate(results):
        assert all(torch.equal(x, y) for x, y in zip(r, results[i % 2]))


def test_a_matrix_of_more_than_two_to_the_31_elements():
    """Tall, with rows whose offsets pass 2^31 elements in every operand: against Q(M^T M) in 64 bits on rows from all over it."""
    rows, cols = 2 ** 22 - 5, 516
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.empty(rows, cols, device="cuda")
    for part in x.split(1 << 18):
        part.copy_(torch.randn(part.shape, generator=gen, device="cuda"))
    x[-300:] *= 50.0
    gram = torch.zeros(cols, cols, dtype=torch.float64, device="cuda")
    for part in x.split(1 << 18):
        wide = part.double()
        gram += wide.T @ wide
    size = float(gram.trace().sqrt()) + 1e-7
    a, q = gram / size ** 2, torch.eye(cols, dtype=torch.float64, device="cuda") / size
    for c in USUAL:
        p = c[0] * torch.eye(cols, dtype=torch.float64, device="cuda") + c[1] * a + c[2] * (a @ a)
        q, a = p @ q, p @ a @ p
    plan = B.Plan([(rows, cols)], 32)
    out = torch.empty_like(x)
    B.sparseloco_orthogonalize(plan, [x], [out], B.orthogonalize_workspace(plan))
    # A's sums of 2^22 products are off by the roundings of as many additions of 16, in three parts; its singular values are within a
    # factor of 1.2 of each other but for the last rows' directions, so that p maps errors on with slopes of 3.5 at most, of which a
    # result near 1 keeps few: 16 times is allowed.
    add = U * math.sqrt(3 * rows / 16)
    for at in (0, 1000, rows // 2, rows - 400):
        cut = slice(at, at + 300)
        want = x[cut].double() @ q
        assert float((out[cut] - want).norm()) <= 16 * add * float(want.norm()), at
    assert bool(torch.isfinite(out[::4097]).all())
