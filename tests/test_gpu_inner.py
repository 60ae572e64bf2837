"""The gradient norm and both forms of the AdamW step against the float64 oracle (oracle/inner.py).

Bars.  Every result may be off by the roundings of the terms it is made of (the oracle returns their sizes, in units of
2^-24) times 1.25 for second-order terms, plus the smallest fp32 number for what vanishes.  Moments in 8 bits: the number that
is held is the oracle's, but where the value lies nearer than 2^-15 gaps to the point where its rounding changes (sixteen
roundings of a value of up to sixteen gaps, and the 2^-20 to which the rule looks at it)."""
import numpy as np
import pytest
import torch

from oracle import inner as O
from paper_2601_02360_amd import binding as B

pytestmark = pytest.mark.gpu
U24, TINY = 2.0 ** -24, 2.0 ** -126
HOW = dict(lr=3e-3, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=7)
SETS = [[1], [3], [255], [257], [4096], [4095, 4097], [8192 + 1023, 5, 0, 4096, 700], [2, 1, 3], [70000, 33]]
GUARD = 12288.0                          # (a bf16 number)


class Placed:
    """Tensors at `shift` elements into larger buffers, guard values on both sides."""

    def __init__(self, shift):
        self.shift, self.buffers = shift, []

    def __call__(self, values, dtype=torch.float32):
        n = len(values)
        buf = torch.full((n + 2 * self.shift + 64,), GUARD, dtype=dtype, device="cuda")
        self.buffers.append((buf, n))
        view = buf[self.shift:self.shift + n]
        view.copy_(torch.as_tensor(values))
        return view

    def check(self):
        for buf, n in self.buffers:
            assert (buf[:self.shift] == GUARD).all() and (buf[self.shift + n:] == GUARD).all(), "written beside a tensor"


def draw(n, rng, scale):
    return (rng.standard_t(3, n) * scale).astype(np.float32)


def bf16(x):
    return torch.as_tensor(x).to(torch.bfloat16).float().numpy()


def f64(t):
    return t.detach().double().cpu().numpy()


def within(got, want, bar, what):
    off = np.abs(got - want)
    assert np.all(off <= 1.25 * U24 * bar + TINY), "%s: off by %.3g of its bar" % (what, np.max(off / (1.25 * U24 * bar + TINY)))


# ---------------------------------------------------------------- norm

@pytest.mark.parametrize("numels", SETS + [[4096 * 2100 + 17]])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm(numels, dtype):
    rng = np.random.default_rng(sum(numels))
    host = [draw(n, rng, 1e-2) for n in numels]
    if dtype == torch.bfloat16:
        host = [bf16(h) for h in host]
    plan, place = B.Plan(numels, 32), Placed(2)
    grads = plan.bind([place(h, dtype) for h in host], dtype=dtype)
    out, ws = torch.full((2,), 7.0, device="cuda"), B.grad_norm_workspace()
    for max_norm in (1e-3, 1e9, float("inf")):
        B.sparseloco_grad_norm(plan, grads, out, ws, max_norm=max_norm)
        want = O.norm(host, max_norm)
        got = f64(out)
        assert abs(got[0] - want[0]) <= 1.01 * U24 * want[0]             # sums in 64 bits, one rounding
        assert abs(got[1] - want[1]) <= 2.02 * U24 * want[1]             # and the quotient's
    place.check()


@pytest.mark.parametrize("scale", [1e-30, 1e-42, 1e25, 3e38])
def test_norm_of_gradients_whose_squares_leave_fp32(scale):
    g = np.array([scale] * 9, np.float32)
    plan = B.Plan([9], 32)
    out, ws = torch.empty(2, device="cuda"), B.grad_norm_workspace()
    B.sparseloco_grad_norm(plan, [torch.as_tensor(g).cuda()], out, ws, max_norm=1.0)
    want = O.norm([g], 1.0)
    got = f64(out)
    if want[0] > 3.4e38:
        assert np.isinf(got[0]) and np.isnan(got[1])
    else:
        assert abs(got[0] - want[0]) <= 1.01 * U24 * want[0] + 2.0 ** -149
        assert abs(got[1] - want[1]) <= 2.02 * U24 * want[1] + 2.0 ** -149


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("at", [0, 4095, 4096, 9999])
def test_norm_shows_what_is_not_finite(bad, at):
    g = torch.zeros(10000, device="cuda")
    g[at] = bad
    plan = B.Plan([10000], 32)
    out, ws = torch.empty(2, device="cuda"), B.grad_norm_workspace()
    B.sparseloco_grad_norm(plan, [g], out, ws)
    assert not torch.isfinite(out[0]) and torch.isnan(out[1])


def test_norm_of_nothing_and_of_zeros():
    out, ws = torch.full((2,), 7.0, device="cuda"), B.grad_norm_workspace()
    B.sparseloco_grad_norm(B.Plan([0, 0], 32), [None, None], out, ws)
    assert out.tolist() == [0.0, 1.0]
    out.fill_(7.0)
    B.sparseloco_grad_norm(B.Plan([5000], 32), [torch.zeros(5000, device="cuda")], out, ws)
    assert out.tolist() == [0.0, 1.0]


# ---------------------------------------------------------------- AdamW, fp32 moments

def inputs(numels, seed, grad_dtype):
    rng = np.random.default_rng(seed)
    theta, g, m = ([draw(n, rng, s) for n in numels] for s in (0.02, 1e-3, 3e-4))
    v = [np.square(draw(n, rng, 1e-3)) for n in numels]
    if grad_dtype == torch.bfloat16:
        g = [bf16(x) for x in g]
    return theta, g, m, v


def step_tensor(values, decay, scale, how):
    """The oracle's step of one tensor."""
    theta, g, m, root = (np.asarray(x, np.float64) for x in values)
    return O.adamw(theta, g, m, root, scale=float(np.float32(scale)), decay=float(np.float32(decay)), **how)


@pytest.mark.parametrize("numels", SETS)
@pytest.mark.parametrize("grad_dtype,copy,scaled,tiled", [(torch.float32, False, False, False), (torch.bfloat16, True, True, False),
                                                         (torch.float32, True, True, True)])
def test_adamw(numels, grad_dtype, copy, scaled, tiled):
    theta, g, m, v = inputs(numels, sum(numels), grad_dtype)
    shapes = [(n // 7, 7) if tiled and n % 7 == 0 and n else n for n in numels]
    plan, place = B.Plan(shapes, 32, tiled=tiled), Placed(2)
    put = lambda arrays, dtype=torch.float32: [place(a, dtype) for a in arrays]
    t_theta, t_g, t_m, t_v = put(theta), put(g, grad_dtype), put(m), put(v)
    t_copy = put([np.zeros(n, np.float32) for n in numels], torch.bfloat16) if copy else None
    scale = 0.37 if scaled else 1.0
    decays = [1.0 if i % 2 == 0 else 0.25 * i for i in range(len(numels))] if scaled else [1.0] * len(numels)
    B.sparseloco_adamw_step(plan, plan.bind(t_theta), plan.bind(t_g, dtype=grad_dtype), plan.bind(t_m), plan.bind(t_v),
                            grad_scale=torch.full((1,), scale, device="cuda") if scaled else None,
                            decay=torch.tensor(decays, device="cuda") if scaled else None,
                            theta_bf16=plan.bind(t_copy, dtype=torch.bfloat16) if copy else None, **HOW)
    place.check()
    for i, n in enumerate(numels):
        want = step_tensor((theta[i], g[i], m[i], np.sqrt(v[i].astype(np.float64))), decays[i], scale, HOW)
        for got, k, what in ((t_theta[i], 0, "theta"), (t_m[i], 1, "m"), (t_v[i], 2, "v")):
            if n:
                within(f64(got), want[k], want[k + 3], "%s of tensor %d" % (what, i))
        assert torch.equal(t_g[i].float().cpu(), torch.as_tensor(g[i])), "gradients were changed"
        if copy:
            assert torch.equal(t_copy[i], t_theta[i].to(torch.bfloat16))


@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shifts", [(1, 1, 2, 1, 2), (63, 63, 62, 63, 62), (64, 64, 64, 64, 64), (33, 2, 4, 0, 6), (0, 5, 2, 63, 34), (32, 32, 32, 32, 32)])
def test_adamw_of_arrays_at_any_place(shifts, grad_dtype):
    """Workgroups begin where theta has a multiple of 256 bytes: theta, m, v, gradients and copy at this many elements past one,
    together and each by itself, tensors that end inside, at and just behind a chunk's end, and beside each other in memory."""
    numels = [4096 * 3, 4096 * 2 + 1, 4096 * 2 + 64, 4096, 4095, 4033, 64, 63, 1, 4097, 4096 * 2 - 63]
    theta, g, m, v = inputs(numels, sum(shifts), grad_dtype)
    plan = B.Plan(numels, 32)
    arrays = [theta, m, [np.zeros(n, np.float32) for n in numels], v, g]
    dtypes = [torch.float32, torch.float32, torch.bfloat16, torch.float32, grad_dtype]
    shifts = list(shifts[:4]) + [shifts[4] if grad_dtype == torch.bfloat16 else shifts[0]]
    tens, buffers = [], []
    for host, dtype, shift in zip(arrays, dtypes, shifts):
        step = 2 if dtype == torch.bfloat16 else 1           # (a bf16 tensor starts at a dword)
        shift = shift // step * step
        buf = torch.full((shift + sum(-(-n // step) * step for n in numels) + 64,), GUARD, dtype=dtype, device="cuda")
        assert buf.data_ptr() % 256 == 0
        at, views, mine = shift, [], torch.zeros(buf.numel(), dtype=torch.bool, device="cuda")
        for h, n in zip(host, numels):
            views.append(buf[at:at + n].copy_(torch.as_tensor(h)))
            mine[at:at + n] = True
            at += -(-n // step) * step
        tens.append(views)
        buffers.append((buf, mine))
    t_theta, t_m, t_copy, t_v, t_g = tens
    B.sparseloco_adamw_step(plan, plan.bind(t_theta), plan.bind(t_g, dtype=grad_dtype), plan.bind(t_m), plan.bind(t_v),
                            theta_bf16=plan.bind(t_copy, dtype=torch.bfloat16), **HOW)
    for buf, mine in buffers:
        assert (buf[~mine] == GUARD).all(), "written beside a tensor"
    for i, n in enumerate(numels):
        want = step_tensor((theta[i], g[i], m[i], np.sqrt(v[i].astype(np.float64))), 1.0, 1.0, HOW)
        for got, k, what in ((t_theta[i], 0, "theta"), (t_m[i], 1, "m"), (t_v[i], 2, "v")):
            within(f64(got), want[k], want[k + 3], "%s of tensor %d" % (what, i))
        assert torch.equal(t_copy[i], t_theta[i].to(torch.bfloat16))
        assert torch.equal(t_g[i].float().cpu(), torch.as_tensor(g[i])), "gradients were changed"


@pytest.mark.parametrize("how", [dict(HOW, step=1), dict(HOW, beta1=0.0, beta2=0.0), dict(HOW, weight_decay=0.0, eps=1e-3),
                                 dict(HOW, step=100000, beta2=0.999), dict(HOW, lr=0.0)])
def test_adamw_numbers(how):
    theta, g, m, v = inputs([5000], 3, torch.float32)
    tens = [torch.as_tensor(x[0]).cuda() for x in (theta, g, m, v)]
    plan = B.Plan([5000], 32)
    B.sparseloco_adamw_step(plan, [tens[0]], [tens[1]], [tens[2]], [tens[3]], **how)
    want = step_tensor((theta[0], g[0], m[0], np.sqrt(v[0].astype(np.float64))), 1.0, 1.0, how)
    for got, k, what in ((tens[0], 0, "theta"), (tens[2], 1, "m"), (tens[3], 2, "v")):
        within(f64(got), want[k], want[k + 3], what)


def test_first_steps_from_zero_moments_with_zero_gradients():
    """A row that no token touched: 0 / (0 + eps) is no change, and no NaN."""
    theta = torch.linspace(-1, 1, 4500, device="cuda")
    plan, zeros = B.Plan([4500], 32), lambda: torch.zeros(4500, device="cuda")
    m, v, before = zeros(), zeros(), theta.clone()
    B.sparseloco_adamw_step(plan, [theta], [zeros()], [m], [v], lr=1e-3, step=1, weight_decay=0.0)
    assert torch.equal(theta, before) and not m.any() and not v.any()
    state = plan.adamw_8bit_buffers()
    B.sparseloco_adamw_step_8bit(plan, [theta], [zeros()], *state, lr=1e-3, step=1, weight_decay=0.0)
    assert torch.equal(theta, before) and not any(s.float().any() for s in state)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("factor", [float("nan"), float("inf")])
def test_a_factor_that_is_not_finite_skips_the_step(eight, factor):
    n = 4096 + 77
    rng = np.random.default_rng(0)
    tens = [torch.as_tensor(draw(n, rng, 1e-2)).cuda() for _ in range(3)] + [torch.rand(n, device="cuda")]
    plan = B.Plan([n], 32)
    state = list(plan.adamw_8bit_buffers()) if eight else tens[2:]
    copy = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    every = tens[:1] + state + [copy]
    before = [t.clone() for t in every]
    kw = dict(lr=1e-3, step=3, grad_scale=torch.full((1,), factor, device="cuda"), theta_bf16=[copy])
    if eight:
        B.sparseloco_adamw_step_8bit(plan, [tens[0]], [tens[1]], *state, **kw)
    else:
        B.sparseloco_adamw_step(plan, [tens[0]], [tens[1]], [state[0]], [state[1]], **kw)
    for was, is_ in zip(before, every):
        assert torch.equal(was.view(torch.uint8), is_.view(torch.uint8))


@pytest.mark.parametrize("eight", [False, True])
def test_a_gradient_that_is_not_finite_shows_without_a_factor(eight):
    """Not finite in one element: that element of theta (8 bits: and its block after the next step) is NaN, no other tensor's."""
    plan = B.Plan([5000, 300], 32)
    theta = [torch.ones(n, device="cuda") for n in (5000, 300)]
    g = [torch.full((n,), 1e-3, device="cuda") for n in (5000, 300)]
    g[0][777] = float("nan")
    if eight:
        state = plan.adamw_8bit_buffers()
        for step in (1, 2):
            B.sparseloco_adamw_step_8bit(plan, theta, g, *state, lr=1e-3, step=step)
    else:
        m, v = ([torch.zeros(n, device="cuda") for n in (5000, 300)] for _ in range(2))
        B.sparseloco_adamw_step(plan, theta, g, m, v, lr=1e-3, step=1)
    bad = torch.isnan(theta[0]).nonzero().flatten()
    assert 777 in bad.tolist() and (len(bad) == 1 if not eight else bad.min() >= 768 and bad.max() < 1024)
    assert torch.isfinite(theta[1]).all()


def test_sets_of_replicas_and_a_stream_of_ones_own():
    numels, R = [4100, 9], 3
    rng = np.random.default_rng(5)
    host = [[[draw(n, rng, 1e-2) for n in numels] for _ in range(R)] for _ in range(4)]
    tens = [[[torch.as_tensor(np.abs(a) if k == 3 else a).cuda() for a in s] for s in sets] for k, sets in enumerate(host)]
    plan = B.Plan(numels, 32)
    bound = [plan.bind(sets) for sets in tens]
    before = [[[t.clone() for t in s] for s in sets] for sets in tens]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    B.sparseloco_adamw_step(plan, *bound, replica=1, stream=side, **HOW)
    out, ws = torch.empty(2, device="cuda"), B.grad_norm_workspace()
    B.sparseloco_grad_norm(plan, bound[1], out, ws, replica=2, stream=side)
    side.synchronize()
    assert abs(f64(out)[0] - O.norm(host[1][2], 1.0)[0]) <= 1.01 * U24 * f64(out)[0]
    for k in range(4):
        for r in range(R):
            changed = not all(torch.equal(a, b) for a, b in zip(before[k][r], tens[k][r]))
            assert changed == (r == 1 and k != 1)
    with pytest.raises(B.SparseLoCoError):
        B.sparseloco_adamw_step(plan, *bound, replica=3, **HOW)


# ---------------------------------------------------------------- AdamW, moments in 8 bits

def chunked(arrays):
    """Tensors as flat chunks, zeros behind the end of each: the layout of the codes."""
    parts = [np.pad(np.asarray(a), (0, -len(a) % 4096)) for a in arrays]
    return np.concatenate(parts) if parts else np.zeros(0)


def random_state(plan, seed, present):
    g = torch.Generator(device="cuda").manual_seed(seed)
    m, m_scale, v, v_scale = plan.adamw_8bit_buffers()
    n = m.numel()
    m.copy_((torch.randn(n, generator=g, device="cuda") * 120).clamp_(-448, 448) * present)
    v.copy_((torch.rand(n, generator=g, device="cuda") * 440 + 1) * present)
    m_scale.copy_(torch.rand(n // 256, generator=g, device="cuda") * 2e-6)
    v_scale.copy_(torch.rand(n // 256, generator=g, device="cuda") * 4e-6)
    return m, m_scale, v, v_scale


@pytest.mark.parametrize("numels", SETS)
@pytest.mark.parametrize("grad_dtype,copy,scaled,tiled", [(torch.float32, False, False, False), (torch.bfloat16, True, True, False),
                                                         (torch.float32, True, True, True)])
def test_adamw_8bit(numels, grad_dtype, copy, scaled, tiled):
    theta, g, _, _ = inputs(numels, sum(numels) + 1, grad_dtype)
    shapes = [(n // 7, 7) if tiled and n % 7 == 0 and n else n for n in numels]
    plan, place = B.Plan(shapes, 32, tiled=tiled), Placed(2)
    put = lambda arrays, dtype=torch.float32: [place(a, dtype) for a in arrays]
    t_theta, t_g = put(theta), put(g, grad_dtype)
    t_copy = put([np.zeros(n, np.float32) for n in numels], torch.bfloat16) if copy else None
    present = chunked([np.ones(n, np.float32) for n in numels])
    assert len(present) == plan.num_flat_chunks * 4096
    state = random_state(plan, 11, torch.as_tensor(present).cuda())
    was = [s.float().cpu().numpy().astype(np.float64) for s in state]
    scale = 0.37 if scaled else 1.0
    decays = [1.0 if i % 2 == 0 else 0.25 * i for i in range(len(numels))] if scaled else [1.0] * len(numels)
    B.sparseloco_adamw_step_8bit(plan, plan.bind(t_theta), plan.bind(t_g, dtype=grad_dtype), *state,
                                 grad_scale=torch.full((1,), scale, device="cuda") if scaled else None,
                                 decay=torch.tensor(decays, device="cuda") if scaled else None,
                                 theta_bf16=plan.bind(t_copy, dtype=torch.bfloat16) if copy else None, **HOW)
    place.check()
    per = lambda i: chunked([np.full(n, decays[j]) for j, n in enumerate(numels)])
    m0, r0 = (was[k] * np.repeat(was[k + 1], 256) for k in (0, 2))
    full = [chunked(x).astype(np.float64) for x in (theta, g)]
    want = O.adamw(full[0], full[1], m0, r0, scale=float(np.float32(scale)), decay=per(0), **HOW)
    at = 0
    for i, n in enumerate(numels):
        if n:
            # (two roundings more: what the 8 bits stand for, and its square)
            within(f64(t_theta[i]), want[0][at:at + n], (want[3] + 4 * np.abs(want[0] - full[0]))[at:at + n], "theta of tensor %d" % i)
        if copy:
            assert torch.equal(t_copy[i], t_theta[i].to(torch.bfloat16))
        at += -(-n // 4096) * 4096
    places = np.arange(len(present))
    for k, x, second in ((0, want[1], False), (2, np.sqrt(want[2]), True)):
        numbers, scales, edge = O.held(x.reshape(-1, 256), places, HOW["step"], second)
        got = f64(state[k].float()).reshape(-1, 256)
        assert np.all(np.abs(f64(state[k + 1]) - scales) <= 12 * U24 * scales)
        differ = got != numbers
        assert np.all(edge[differ] <= 2.0 ** -15), "a number that is not the nearest on its side"
        assert not got.reshape(-1)[present == 0].any()


def test_8bit_numbers_read_and_write_all_codes():
    """Every code comes back as it is when the step changes nothing: beta = 1 - 2^-30 keeps both moments, and a value that is
    an e4m3 number times the scale is rounded to itself whatever the threshold."""
    plan = B.Plan([4096], 32)
    m, m_scale, v, v_scale = plan.adamw_8bit_buffers()
    codes = torch.arange(256, device="cuda", dtype=torch.int32)
    codes = torch.where((codes & 127) == 127, codes - 1, codes).to(torch.uint8)          # no NaN
    m.view(torch.uint8).copy_(codes.repeat(16))
    v.view(torch.uint8).copy_((codes & 127).repeat(16))
    m_scale.fill_(2.0 ** -20)
    v_scale.fill_(2.0 ** -18)
    before = [t.clone() for t in (m, m_scale, v, v_scale)]
    theta, g = torch.zeros(4096, device="cuda"), torch.zeros(4096, device="cuda")
    for step in (1, 2, 1000):
        B.sparseloco_adamw_step_8bit(plan, [theta], [g], m, m_scale, v, v_scale, lr=0.0, step=step, beta1=1 - 2.0 ** -30,
                                     beta2=1 - 2.0 ** -30)
        got = (m.float(), m_scale, v.float(), v_scale)
        for is_, was in zip(got, (before[0].float(), before[1], before[2].float(), before[3])):
            assert torch.equal(is_, was)


def test_8bit_moments_follow_their_averages():
    """A thousand steps of a gradient that drops to a hundredth after the first fifty: v falls by 5 % a step then, the root by
    2.5 %, less than half a gap (3 to 6 %); a rounding to nearest would hold it.  The mean over a block's elements of what is held stays
    within a gap (12.5 %) of the average that fp32 moments keep."""
    n = 4096
    plan = B.Plan([n], 32)
    theta, theta8 = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    state = plan.adamw_8bit_buffers()
    size = torch.logspace(-3, -1, n, device="cuda")
    steady = torch.zeros(n, device="cuda")
    steady[::64] = 1.0                   # keeps the scale of every block where it is
    for step in range(1, 251):
        g = size * (1.0 if step <= 50 else 0.01) * (1 - steady) + steady
        B.sparseloco_adamw_step(plan, [theta], [g], [m], [v], lr=1e-3, step=step)
        B.sparseloco_adamw_step_8bit(plan, [theta8], [g], *state, lr=1e-3, step=step)
        if step in (50, 100, 150, 250):
            held = state[2].float().view(-1, 256) * state[3][:, None]
            want = v.sqrt().view(-1, 256)
            calm = (steady == 0).view(-1, 256)
            ratio = ((held / want) * calm).sum(1) / calm.sum(1)
            assert ((ratio - 1).abs() < 0.125).all(), (step, ratio.min().item(), ratio.max().item())
            held = state[0].float().view(-1, 256) * state[1][:, None]
            assert ((held * calm).sum(1) / (m.view(-1, 256) * calm).sum(1) - 1).abs().max() < 0.125


# ---------------------------------------------------------------- as a program uses them

def test_an_inner_step_replays_from_a_hip_graph():
    """Norm, clip and step recorded once and replayed with new gradients, eager work between the replays."""
    numels = [4096 * 5 + 9, 700]
    plan = B.Plan(numels, 32)
    rng = np.random.default_rng(2)
    fresh = lambda: [[torch.as_tensor(draw(n, rng, 1e-2)).cuda() for n in numels]] + [[torch.zeros(n, device="cuda") for n in numels] for _ in range(3)]
    a = fresh()
    b = [[t.clone() for t in s] for s in a]
    out, ws, how = torch.empty(2, device="cuda"), B.grad_norm_workspace(), dict(lr=1e-2, step=5)

    def step(p, bound):
        B.sparseloco_grad_norm(p, bound[1], out, ws, max_norm=0.5)
        B.sparseloco_adamw_step(p, *bound, grad_scale=out[1:], **how)

    bound = [plan.bind(s) for s in a]
    other = [plan.bind(s) for s in b]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(plan, bound)
    for _ in range(4):
        new = [torch.as_tensor(draw(n, rng, 1e-2)).cuda() for n in numels]
        for s in (a, b):
            for t, x in zip(s[1], new):
                t.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        step(plan, other)
        torch.cuda.synchronize()
        for s, t in zip(a, b):
            for x, y in zip(s, t):
                assert torch.equal(x, y)


def test_refusals():
    plan = B.Plan([4096, 10], 32)
    f = lambda dtype=torch.float32: [torch.zeros(4096, dtype=dtype, device="cuda"), torch.zeros(10, dtype=dtype, device="cuda")]
    out, ws = torch.zeros(2, device="cuda"), B.grad_norm_workspace()
    theta, g, m, v = f(), f(), f(), f()
    ok = dict(lr=1e-3, step=1)

    def refused(status, call, *args, **kw):
        with pytest.raises(B.SparseLoCoError) as e:
            call(*args, **kw)
        assert e.value.status == status

    for max_norm in (0.0, -1.0, float("nan")):
        refused(B.SPLC_EINVAL, B.sparseloco_grad_norm, plan, g, out, ws, max_norm=max_norm)
    refused(B.SPLC_EINVAL, B.sparseloco_grad_norm, plan, plan.bind([g, g]), out, ws, replica=2)
    refused(B.SPLC_EPLAN, B.sparseloco_grad_norm, B.Plan([4096], 32), plan.bind(g), out, ws)
    for change in (dict(step=0), dict(step=-3), dict(lr=float("nan")), dict(lr=-1.0), dict(beta1=1.0), dict(beta2=1.0),
                   dict(beta1=-0.1), dict(eps=-1e-8), dict(eps=float("inf")), dict(weight_decay=float("nan")), dict(replica=-1)):
        refused(B.SPLC_EINVAL, B.sparseloco_adamw_step, plan, theta, g, m, v, **dict(ok, **change))
        refused(B.SPLC_EINVAL, B.sparseloco_adamw_step_8bit, plan, theta, g, *plan.adamw_8bit_buffers(), **dict(ok, **change))
    refused(B.SPLC_EPLAN, B.sparseloco_adamw_step, plan, plan.bind(f(torch.bfloat16), dtype=torch.bfloat16), g, m, v, **ok)
    refused(B.SPLC_EPLAN, B.sparseloco_adamw_step, plan, theta, g, m, plan.bind(f(torch.bfloat16), dtype=torch.bfloat16), **ok)
    refused(B.SPLC_EPLAN, B.sparseloco_adamw_step, plan, theta, g, m, v, theta_bf16=plan.bind(f()), **ok)
    state = list(plan.adamw_8bit_buffers())
    for k, wrong in ((0, state[0][:-1]), (0, state[0].view(torch.uint8)), (1, state[1][:-1]), (2, state[2].float()), (3, state[3].double())):
        with pytest.raises(ValueError):
            B.sparseloco_adamw_step_8bit(plan, theta, g, *(wrong if i == k else s for i, s in enumerate(state)), **ok)
    for scale in (torch.zeros(2, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda"), torch.zeros(1)):
        with pytest.raises(ValueError):
            B.sparseloco_adamw_step(plan, theta, g, m, v, grad_scale=scale, **ok)
    with pytest.raises(ValueError):
        B.sparseloco_adamw_step(plan, theta, g, m, v, decay=torch.ones(3, device="cuda"), **ok)
    with pytest.raises(ValueError):
        B.sparseloco_grad_norm(plan, g, out, ws[:100])
    assert not any(t.any() for s in (theta, m, v) for t in s)
