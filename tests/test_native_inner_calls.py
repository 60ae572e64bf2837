"""The native way (csrc/calls.cpp) of the inner step's calls: it makes the call or hands the arguments back to Python's checks."""
import numpy as np
import pytest
import torch

from paper_2601_02360_amd import binding as B

X, IDS, TABLE = torch.zeros(8, 16), torch.zeros(8, dtype=torch.int32), torch.zeros(5, 16)
NUMBERS = (1e-3, 0.9, 0.95, 1e-8, 0.1)


def test_arguments_that_are_not_plainly_right_are_handed_back():
    native = B._native()
    for name in ("grad_norm", "adamw_step", "adamw_step_8bit", "embedding_lookup", "embedding_grad"):
        for args in ((), (None,), (X,) * 5, (None,) * 30, ("0",) * 12):
            assert getattr(native, name)(*args) is None
    assert native.embedding_lookup(TABLE, IDS, X, None, None, 1.0, 0) is None            # on the host
    assert native.adamw_step(None, None, None, None, None, 0, *NUMBERS, 1 << 70, None, 0, None, None, 0) is None
    assert native.adamw_step(None, None, None, None, None, 0, *NUMBERS, 1, X, 0, None, None, 0) is None
    assert native.adamw_step(None, None, None, None, None, 0, 1, *NUMBERS[1:], 1, None, 0, None, None, 0) is None


def test_null_handles_are_refused_by_the_library():
    assert B._native().adamw_step(None, None, None, None, None, 0, *NUMBERS, 1, None, 0, None, None, 0) == B.SPLC_EINVAL


@pytest.mark.gpu
def test_plain_calls_are_taken_and_every_form_of_argument_gives_the_same(monkeypatch):
    native, made = B._native(), []

    class Recorded:
        def __getattr__(self, name):
            def call(*args):
                made.append((name, getattr(native, name)(*args)))
                return made[-1][1]
            return call
    monkeypatch.setattr(B, "_native", lambda: Recorded())
    n, rows, vocab, d = 2 * 4096 + 5, 70, 9, 33
    g = torch.Generator(device="cuda").manual_seed(1)
    first = [torch.rand(n, generator=g, device="cuda") for _ in range(4)]
    plan = B.Plan([n], 32)
    scale, decay = torch.full((1,), 0.5, device="cuda"), torch.full((1,), 2.0, device="cuda")
    x = torch.randn(rows, d, generator=g, device="cuda")
    ids = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    table = torch.nn.Parameter(torch.randn(vocab, d, generator=g, device="cuda"))
    side = torch.cuda.Stream()
    results = []
    for stream, number, lists in ((None, float, False), (side, float, False), (side.cuda_stream, float, False),
                                  (None, np.float64, False), (None, float, True)):
        theta, grad, m, v = (t.clone() for t in first)
        copy = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
        state = plan.adamw_8bit_buffers()
        out, ws = torch.zeros(2, device="cuda"), B.grad_norm_workspace()
        looked, summed = torch.empty(rows, d, device="cuda"), torch.empty(vocab, d, dtype=torch.bfloat16, device="cuda")
        gws = B.embedding_grad_workspace(rows, vocab, d)
        h = (lambda t: [t]) if lists else (lambda t: plan.bind([t], dtype=t.dtype, stream=stream))
        a, b, c, e, f = h(theta), h(grad), h(m), h(v), h(copy)
        torch.cuda.synchronize()
        made.clear()
        how = dict(lr=number(1e-3), step=2, grad_scale=scale, decay=decay, theta_bf16=f, stream=stream)
        B.sparseloco_grad_norm(plan, b, out, ws, max_norm=number(0.25), stream=stream)
        B.sparseloco_adamw_step(plan, a, b, c, e, **how)
        B.sparseloco_adamw_step_8bit(plan, a, b, *state, **how)
        B.sparseloco_embedding_lookup(table, ids, looked, t_perp=table, pos_embed=x, scale=number(2.0), stream=stream)
        B.sparseloco_embedding_grad(x, ids, summed, gws, scale=number(0.5), stream=stream)
        torch.cuda.synchronize()
        names = ("grad_norm", "adamw_step", "adamw_step_8bit", "embedding_lookup", "embedding_grad")
        if number is float and not lists:
            assert made == [(name, B.SPLC_OK) for name in names]
        results.append([theta, m, v, copy, out, looked, summed] + [s.view(torch.uint8) for s in state])
    for r in results[1:]:
        assert all(torch.equal(p, q) for p, q in zip(r, results[0]))
