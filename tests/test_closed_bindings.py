"""A closed binding is refused, also where the argument is optional: it is not taken for one that was left out."""
import ctypes

import pytest
import torch

from paper_2601_02360_amd import binding as B


class FakePlan:
    numels = [8]
    handle = ctypes.c_void_p(4096)
    _h = handle
    _num_flat_chunks = num_flat_chunks = 1

    def _tensors(self, x, dtype=torch.float32, stream=None):
        return x

    def _messages(self, pairs, aux, stream=None):
        return pairs


class Bindings:
    """Makes handles that nothing was bound for; they are never dereferenced, and emptied at the end so that nothing releases them."""
    def __init__(self):
        self.made = []

    def __call__(self, open_: bool, kind=B.Tensors):
        t = kind.__new__(kind)
        t._h, t.dtype, t.n_sets = ctypes.c_void_p(4096 if open_ else None), torch.float32, 1
        self.made.append(t)
        return t


@pytest.fixture
def binding():
    made = Bindings()
    yield made
    for t in made.made:
        t._h = ctypes.c_void_p()


class Recorded:
    """In the place of the library and of its native calls: takes every call."""
    def __init__(self):
        self.made = []

    def __getattr__(self, name):
        def call(*args):
            if name != "sparseloco_strerror":
                self.made.append(name)
                return B.SPLC_OK
            return b"refused"
        return call


def calls(plan, o, messages, optional, state):
    """The calls that take an optional binding."""
    step = dict(lr=1e-3, step=1, theta_bf16=optional)
    return {"adamw_step": lambda: B.sparseloco_adamw_step(plan, *o, **step),
            "adamw_step_8bit": lambda: B.sparseloco_adamw_step_8bit(plan, o[0], o[1], *state, **step),
            "aggregate_update delta_bar_out": lambda: B.sparseloco_aggregate_update(plan, messages, o[0], 1.0, delta_bar_out=optional),
            "aggregate_update reset": lambda: B.sparseloco_aggregate_update(plan, messages, o[0], 1.0, reset=optional),
            "outer_step_batch": lambda: B.sparseloco_outer_step_batch(plan, o[0], o[1], o[2], messages, 0.9, 1.0, delta_bar_out=optional)}


@pytest.mark.parametrize("name", list(calls(*[None] * 5)))
def test_an_optional_binding_that_is_closed_is_refused(name, monkeypatch, binding):
    recorded = Recorded()
    monkeypatch.setattr(B, "lib", lambda: recorded)
    monkeypatch.setattr(B, "_native", lambda: recorded)
    monkeypatch.setattr(B, "_stream", lambda stream: None)
    monkeypatch.setattr(B, "_check_flat", lambda specs: None)
    o, messages, state = [binding(True) for _ in range(4)], binding(True, B.Messages), [torch.zeros(1)] * 4

    def call(optional):
        calls(FakePlan(), o, messages, optional, state)[name]()

    with pytest.raises(B.SparseLoCoError) as e:
        call(binding(False))
    assert e.value.status == B.SPLC_EINVAL and not recorded.made
    call(binding(True))                                      # open, and left out
    call(None)
    assert len(recorded.made) == 2


@pytest.mark.gpu
@pytest.mark.parametrize("eight", [False, True])
def test_a_step_with_a_closed_copy_changes_nothing(eight):
    n = 5000
    plan = B.Plan([n], 32)
    theta, g, m, v = (torch.rand(n, device="cuda") for _ in range(4))
    copy = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    state = list(plan.adamw_8bit_buffers())
    every = [theta, m, v, copy] + [s.view(torch.uint8) for s in state]
    before = [t.clone() for t in every]
    closed = plan.bind([copy], dtype=torch.bfloat16)
    closed.close()
    kw = dict(lr=1e-3, step=1, theta_bf16=closed)
    for bound in (plan.bind, lambda tensors: tensors):
        with pytest.raises(B.SparseLoCoError) as e:
            if eight:
                B.sparseloco_adamw_step_8bit(plan, bound([theta]), bound([g]), *state, **kw)
            else:
                B.sparseloco_adamw_step(plan, bound([theta]), bound([g]), bound([m]), bound([v]), **kw)
        assert e.value.status == B.SPLC_EINVAL
    assert all(torch.equal(a, b) for a, b in zip(before, every))
