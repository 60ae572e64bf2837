"""Integers that do not fit the type in which the library takes them are refused by the inner step's calls: nothing runs with their
lower bits (an ignore_id of 2^32 + 3 would leave out token 3, a step of 2^64 + 1 would be the first)."""
import pytest
import torch

from paper_2601_02360_amd import binding as B

LARGE = {"step": [2 ** 63, 2 ** 64 + 1, -2 ** 63 - 1], "replica": [2 ** 31, 2 ** 32, -2 ** 31 - 1, 2 ** 64],
         "ignore_id": [2 ** 31, 2 ** 32 + 3, -2 ** 31 - 1, 2 ** 64]}
CASES = [(call, argument, value) for call, arguments in (("grad_norm", ["replica"]), ("adamw_step", ["step", "replica"]),
                                                         ("adamw_step_8bit", ["step", "replica"]), ("embedding_grad", ["ignore_id"]))
         for argument in arguments for value in LARGE[argument]]


def calls(plan, theta, g, m, v, state, out, ws, grad, ids, table, grad_ws):
    return {"grad_norm": lambda **kw: B.sparseloco_grad_norm(plan, g, out, ws, **kw),
            "adamw_step": lambda **kw: B.sparseloco_adamw_step(plan, theta, g, m, v, **{"lr": 1e-2, "step": 1, **kw}),
            "adamw_step_8bit": lambda **kw: B.sparseloco_adamw_step_8bit(plan, theta, g, *state, **{"lr": 1e-2, "step": 1, **kw}),
            "embedding_grad": lambda **kw: B.sparseloco_embedding_grad(grad, ids, table, grad_ws, **kw)}


class FakePlan:
    numels, num_flat_chunks, handle = [8], 1, None


@pytest.mark.parametrize("call,argument,value", CASES)
def test_they_are_refused_before_the_library_is_called(call, argument, value, monkeypatch):
    class Library:
        def __getattr__(self, name):
            assert name == "sparseloco_strerror", "called with " + argument
            return lambda status: b"refused"
    monkeypatch.setattr(B, "lib", lambda: Library())
    monkeypatch.setattr(B, "_check_flat", lambda specs: None)
    monkeypatch.setattr(B, "_check_matrices", lambda specs: None)
    x, ids = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(B.SparseLoCoError) as e:
        calls(FakePlan(), None, None, None, None, [x] * 4, x, x, x, ids, x, torch.zeros(9, dtype=torch.uint8))[call](**{argument: value})
    assert e.value.status == B.SPLC_EINVAL


@pytest.mark.parametrize("sizes", [(2 ** 64 + 5, 5, 16), (8, 2 ** 32 + 5, 16), (8, 5, 2 ** 32 + 16)])
def test_workspaces_of_sizes_that_do_not_fit(sizes):
    with pytest.raises(B.SparseLoCoError):
        B.embedding_grad_workspace(*sizes)


@pytest.mark.gpu
def test_nothing_is_written_by_a_refused_call_and_other_integers_are_taken():
    import numpy as np
    n, rows, vocab, d = 5000, 70, 9, 33
    plan = B.Plan([n], 32)
    theta, g, m, v = (plan.bind([torch.rand(n, device="cuda")]) for _ in range(4))
    every = [b._keep[0][0] for b in (theta, g, m, v)]
    state, out, table = plan.adamw_8bit_buffers(), torch.full((2,), 7.0, device="cuda"), torch.full((vocab, d), 7.0, device="cuda")
    every += [out, table] + [s.view(torch.uint8) for s in state]
    grad, ids = torch.ones(rows, d, device="cuda"), (torch.arange(rows, device="cuda") % vocab).to(torch.int32)
    c = calls(plan, theta, g, m, v, state, out, B.grad_norm_workspace(), grad, ids, table, B.embedding_grad_workspace(rows, vocab, d))
    before = [t.clone() for t in every]
    for call, argument, value in CASES:
        with pytest.raises(B.SparseLoCoError):
            c[call](**{argument: value})
    assert all(torch.equal(a, b) for a, b in zip(before, every))
    c["grad_norm"](replica=np.int64(0))
    c["adamw_step"](step=np.int32(3), replica=np.int64(0))
    c["embedding_grad"](ignore_id=np.int64(3))
    assert not table[3].any() and table[:3].all() and table[4:].all()
