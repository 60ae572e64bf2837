"""Calls that take plain lists bind them on the fly, and let go of the bindings and of the tensors when their work is done: a
training loop that passes fresh gradients at every step holds those of a few calls, not of all."""
import ctypes
import gc

import pytest
import torch

from paper_2601_02360_amd import binding as B


# ---------------------------------------------------------------- what is held and when it is let go, on the host

class Event:
    """An event that has passed when the test says so; waiting for it makes it pass."""
    made = []

    def __init__(self):
        self.stream, self.passed, self.waited = None, False, False
        Event.made.append(self)

    def record(self, stream):
        self.stream = stream

    def query(self):
        return self.passed

    def synchronize(self):
        self.waited = self.waited or not self.passed
        self.passed = True


class Library:
    """Counts handles; every call succeeds."""
    def __init__(self):
        self.made, self.alive, self.rebound = 0, set(), 0

    def __getattr__(self, name):
        if name.startswith("sparseloco_plan_num"):
            return lambda *args: 1
        return lambda *args: B.SPLC_OK

    def bind(self, out, *args):
        self.made += 1
        out._obj.value = 4096 * self.made
        self.alive.add(out._obj.value)
        return B.SPLC_OK

    def rebind(self, handle, *args):
        assert handle.value in self.alive
        self.rebound += 1
        return B.SPLC_OK

    def release(self, handle):
        self.alive.remove(handle.value)

    sparseloco_tensors_bind = sparseloco_messages_bind = bind
    sparseloco_tensors_rebind = sparseloco_messages_rebind = rebind
    sparseloco_tensors_release = sparseloco_messages_release = release


@pytest.fixture
def plan(monkeypatch):
    Event.made = []
    library = Library()
    monkeypatch.setattr(torch.cuda, "Event", Event)
    monkeypatch.setattr(B, "_torch_stream", lambda stream: stream)
    monkeypatch.setattr(B, "_capturing", lambda stream: stream == "captured")
    monkeypatch.setattr(B, "_check_tensor", lambda *args, **kw: None)
    monkeypatch.setattr(B, "_stream", lambda stream: None)
    monkeypatch.setattr(B, "lib", lambda: library)
    plan = B.Plan([8], 32)
    plan.library = library
    yield plan
    plan.close()
    assert not library.alive


def call(plan, lists=1, stream="one", sets=1):
    with B._Lists(plan, stream) as made:
        return [made.tensors([[torch.zeros(8)]] * sets) for _ in range(lists)]


def test_bindings_of_a_call_are_let_go_when_its_work_is_done(plan):
    first = call(plan, 5)
    assert Event.made[0].stream == "one" and all(b._keep for b in first)
    Event.made[0].passed = True
    second = call(plan)
    assert not any(b._keep or b._h.value for b in first) and all(b._keep for b in second)
    assert not any(e.waited for e in Event.made)


def test_who_is_far_ahead_waits_for_the_oldest_call_only(plan):
    calls = [call(plan) for _ in range(plan.CALLS_IN_FLIGHT + 3)]
    assert [bool(c[0]._keep) for c in calls] == [False] * 3 + [True] * plan.CALLS_IN_FLIGHT
    assert [e.waited for e in Event.made] == [True] * 3 + [False] * plan.CALLS_IN_FLIGHT


def test_handles_are_used_again_and_stay_few(plan):
    recorded = call(plan, 2, "captured")
    for k in range(1, 200):
        call(plan, 5)
        Event.made[-1].passed = True
    assert plan.library.made <= 2 + 5 * 2 and plan.library.rebound >= 5 * 190
    assert all(b._keep and b._h.value for b in recorded)     # a graph may still replay it
    for k in range(1, 200):                                  # always more than before
        call(plan, 5, sets=k)
        Event.made[-1].passed = True
    assert len(plan.library.alive) <= 2 + plan._spares.MOST + 10


def test_a_spare_handle_without_the_room_is_left(plan):
    call(plan, 1, sets=3)
    Event.made[-1].passed = True
    call(plan, 1, sets=4)
    Event.made[-1].passed = True
    assert plan.library.rebound == 0
    call(plan, 2, sets=3)                                    # (the first call's handle is spare, the second's will be)
    assert plan.library.rebound == 1
    with B._Lists(plan, "one") as made:                      # tensors' handles do not serve messages
        made.messages([torch.zeros(1)], [torch.zeros(1)])
    assert plan.library.rebound == 1


def test_a_call_that_is_refused_holds_what_it_had_bound(plan):
    with pytest.raises(RuntimeError):
        with B._Lists(plan, "one") as made:
            b = made.tensors([torch.zeros(8)])
            raise RuntimeError
    assert b._keep and plan._in_flight[0][1] == [b]


def test_null_handles_are_not_rebound():
    L = B.lib()
    assert L.sparseloco_tensors_rebind(None, None, 1, None, B.SPLC_F32, None) == B.SPLC_EINVAL
    assert L.sparseloco_messages_rebind(None, None, 1, None, None, None) == B.SPLC_EINVAL


# ---------------------------------------------------------------- on the GPU

def open_bindings():
    gc.collect()
    every = gc.get_objects()
    return (sum(1 for o in every if type(o) in (B.Tensors, B.Messages) and o._h.value)
            + sum(len(o._spares.handles) for o in every if type(o) is B.Plan))


def norms(plan, n, calls, stream=None):
    """A call with fresh gradients each: ones times the call's number."""
    outs, ws = torch.zeros(calls, 2, device="cuda"), B.grad_norm_workspace()
    torch.cuda.synchronize()
    most = 0
    for k in range(calls):
        with torch.cuda.stream(stream) if isinstance(stream, torch.cuda.Stream) else torch.cuda.stream(None):
            g = [torch.full((n,), float(k), device="cuda")]
        B.sparseloco_grad_norm(plan, g, outs[k], ws, stream=stream)
        del g
        most = max(most, torch.cuda.memory_allocated())
    torch.cuda.synchronize()
    assert torch.equal(outs[:, 0], torch.arange(calls, device="cuda") * float(n) ** 0.5)
    return most


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["current", "side"])
def test_memory_of_a_loop_with_fresh_gradients_is_bounded(kind):
    n, calls = 1 << 20, 300                                  # 4 MiB a call; its square root is a power of two
    plan = B.Plan([n], 32)
    before, bindings = torch.cuda.memory_allocated(), open_bindings()
    most = norms(plan, n, calls, torch.cuda.Stream() if kind == "side" else None)
    assert most - before < 10 * 4 * n
    assert open_bindings() - bindings <= plan.CALLS_IN_FLIGHT + 1
    plan.close()
    assert open_bindings() <= bindings


@pytest.mark.gpu
def test_bindings_outlive_calls_that_wait_on_their_stream():
    """Every call waits behind a kernel of some milliseconds: tables and tensors have to be there when it runs."""
    n = 1 << 14
    plan, side = B.Plan([n], 32), torch.cuda.Stream()
    outs, ws = torch.zeros(12, 2, device="cuda"), B.grad_norm_workspace()
    torch.cuda.synchronize()
    for k in range(12):
        with torch.cuda.stream(side):
            torch.cuda._sleep(5_000_000)
            g = [torch.full((n,), float(k), device="cuda")]
        B.sparseloco_grad_norm(plan, g, outs[k], ws, stream=side.cuda_stream)
        del g
        torch.full((n,), 1e3, device="cuda")                 # (memory that is free to the current stream is written)
    torch.cuda.synchronize()
    assert torch.equal(outs[:, 0], torch.arange(12, device="cuda") * float(n) ** 0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("eight", [False, True])
def test_a_loop_of_whole_steps_with_lists_and_with_bindings_gives_the_same(eight):
    numels, steps = [5000, 37], 40
    plan = B.Plan(numels, 32)
    g = torch.Generator(device="cuda").manual_seed(1)
    make = lambda: [torch.rand(n, generator=g, device="cuda") for n in numels]
    first, grads = [make() for _ in range(3)], [make() for _ in range(steps)]
    results = []
    for lists in (False, True):
        theta, m, v = ([t.clone() for t in s] for s in first)
        state = list(plan.adamw_8bit_buffers()) if eight else None
        copy = [torch.zeros(n, dtype=torch.bfloat16, device="cuda") for n in numels]
        out, ws = torch.zeros(2, device="cuda"), B.grad_norm_workspace()
        bind = (lambda s: s) if lists else (lambda s: plan.bind(s, dtype=s[0].dtype))
        for k in range(steps):
            fresh = [t.clone() for t in grads[k]]
            B.sparseloco_grad_norm(plan, bind(fresh), out, ws)
            moments = state if eight else [bind(m), bind(v)]
            (B.sparseloco_adamw_step_8bit if eight else B.sparseloco_adamw_step)(
                plan, bind(theta), bind(fresh), *moments, lr=1e-2, step=k + 1, grad_scale=out[1:], theta_bf16=bind(copy))
        results.append(theta + m + v + copy + [s.view(torch.uint8) for s in state or []])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert len(plan._in_flight) <= plan.CALLS_IN_FLIGHT and len(plan._spares.handles) <= plan._spares.MOST


@pytest.mark.gpu
def test_outer_steps_with_lists_are_let_go_too():
    numels, R, steps = [4096 * 3, 100], 2, 20
    plan = B.Plan(numels, 32)
    bindings = open_bindings()
    theta = [torch.rand(n, device="cuda") for n in numels]
    ef = [[torch.zeros(n, device="cuda") for n in numels] for _ in range(R)]
    pairs, aux = zip(*(plan.message_buffers() for _ in range(R)))
    for _ in range(steps):
        local = [[t + 1e-3 for t in theta] for _ in range(R)]
        for r in range(R):
            B.sparseloco_compress(plan, ef[r], pairs[r], aux[r], 0.9, theta_outer=theta, theta_local=local[r])
        B.sparseloco_aggregate_update(plan, list(pairs), theta, 1.0, aux=list(aux))
        B.sparseloco_outer_step_batch(plan, theta, local, ef, list(pairs), 0.9, 1.0, aux_out=list(aux))
    torch.cuda.synchronize()
    assert open_bindings() - bindings <= plan._spares.MOST + 4 * plan.CALLS_IN_FLIGHT
    assert all(torch.isfinite(t).all() for t in theta)


@pytest.mark.gpu
def test_a_handle_is_pointed_at_other_tensors_or_left_as_it_is():
    L, plan, other = B.lib(), B.Plan([4096, 10], 32), B.Plan([7], 32)
    sets = [[torch.full((n,), float(k), device="cuda") for n in (4096, 10)] for k in (1, 2, 3, 4)]
    out, ws = torch.zeros(2, device="cuda"), B.grad_norm_workspace()
    pointers = lambda sets: (ctypes.c_void_p * sum(map(len, sets)))(*[t.data_ptr() for s in sets for t in s])
    bound = plan.bind(sets[:2])

    def norm(replica, plan=plan):
        rc = L.sparseloco_grad_norm(plan.handle, bound.handle, replica, 1.0, out.data_ptr(), ws.data_ptr(), None)
        torch.cuda.synchronize()
        return out[0].item() if rc == B.SPLC_OK else rc

    def rebind(plan, sets, dtype=B.SPLC_F32, shift=0):
        p = pointers(sets)
        p[0] += shift
        return L.sparseloco_tensors_rebind(bound.handle, plan.handle, len(sets), p, dtype, None)

    want = lambda k, n=4106: pytest.approx(k * n ** 0.5, rel=1e-6)
    assert [norm(0), norm(1)] == [want(1), want(2)]
    assert rebind(plan, sets[:3]) == B.SPLC_ETOOBIG
    assert rebind(plan, sets[2:], dtype=7) == B.SPLC_EINVAL
    assert rebind(plan, sets[2:], shift=2) == B.SPLC_EALIGN
    assert [norm(0), norm(1)] == [want(1), want(2)]          # as it was
    assert rebind(plan, sets[2:]) == B.SPLC_OK
    assert [norm(0), norm(1)] == [want(3), want(4)]
    assert rebind(plan, sets[1:2]) == B.SPLC_OK              # one set, which serves every replica
    assert [norm(0), norm(1)] == [want(2), want(2)]
    one = [[torch.full((7,), 5.0, device="cuda")]] * 4       # another plan's, as many pointers as there is room for
    assert rebind(other, one) == B.SPLC_OK
    assert norm(0) == B.SPLC_EPLAN and norm(3, other) == want(5, 7)
    assert rebind(plan, sets[:2]) == B.SPLC_OK
    assert [norm(0), norm(1)] == [want(1), want(2)]


@pytest.mark.gpu
def test_message_lists_use_handles_again_whatever_their_buffers():
    """Aggregations of other buffers at every call, of fewer and of more replicas than before."""
    numels, rng = [4096 + 100], torch.Generator(device="cuda").manual_seed(3)
    plan = B.Plan(numels, 32)
    for R in (3, 1, 2, 4, 2, 3, 1, 4):
        ef = [[torch.randn(n, generator=rng, device="cuda") for n in numels] for _ in range(R)]
        zero = [torch.zeros(n, device="cuda") for n in numels]
        pairs, aux = zip(*(plan.message_buffers() for _ in range(R)))
        for r in range(R):
            B.sparseloco_compress(plan, ef[r], pairs[r], aux[r], 1.0, delta=zero)
        mean, again = ([torch.empty(n, device="cuda") for n in numels] for _ in range(2))
        B.sparseloco_aggregate(plan, list(pairs), mean, aux=list(aux))
        B.sparseloco_aggregate(plan, plan.bind_messages(list(pairs), list(aux)), plan.bind(again))
        assert torch.equal(mean[0], again[0]) and mean[0].any()


@pytest.mark.gpu
def test_a_graph_that_was_recorded_with_lists_keeps_its_tables():
    """Replayed between other calls with lists, which must not take the tables that the graph reads."""
    numels = [5000, 37]
    plan, other = B.Plan(numels, 32), torch.zeros(2, device="cuda")
    g, ws = [torch.zeros(n, device="cuda") for n in numels], B.grad_norm_workspace()
    out, graph = torch.zeros(2, device="cuda"), torch.cuda.CUDAGraph()
    B.sparseloco_grad_norm(plan, g, out, ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, capture_error_mode="relaxed"):          # (binding may allocate)
        B.sparseloco_grad_norm(plan, g, out, ws)
    for k in range(1, 5):
        for t in g:
            t.fill_(float(k))
        for _ in range(10):
            B.sparseloco_grad_norm(plan, [torch.ones(n, device="cuda") for n in numels], other, ws)
        graph.replay()
        torch.cuda.synchronize()
        assert out[0].item() == pytest.approx(k * sum(numels) ** 0.5, rel=1e-6)
