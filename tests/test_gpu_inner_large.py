"""The inner step's operators where offsets pass 32 bits: one tensor of more than 2^31 elements, tables and gradients of more than
4 GiB.  Checked where it can go wrong -- at both ends and around every power of two of bytes and elements from 2^31 on -- and by sums."""
import numpy as np
import pytest
import torch

from oracle import inner as O
from paper_2601_02360_amd import binding as B
from test_gpu_inner import HOW, U24, f64, within

pytestmark = pytest.mark.gpu
N = 2 ** 31 + 4096 * 3 + 77


def places(n):
    """Runs of 512 elements around the powers of two and at the ends."""
    at = [0, n - 512] + [p - 256 for p in (2 ** 29, 2 ** 30, 2 ** 31) if p + 256 <= n]
    return [slice(a, a + 512) for a in at]


def filled(n, dtype, scale, seed):
    """A pattern that no two places of interest share, without 64-bit copies of it."""
    x = torch.empty(n, dtype=dtype, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    for a in range(0, n, 1 << 28):
        part = x[a:a + (1 << 28)]
        part.copy_(torch.rand(part.numel(), generator=g, device="cuda").sub_(0.5).mul_(scale))
    return x


@pytest.mark.parametrize("shift", [0, 1])
def test_norm_and_adamw_over_a_tensor_of_more_than_two_to_the_31_elements(shift):
    plan = B.Plan([N], 32)
    theta_all = filled(N + shift, torch.float32, 0.1, 1)
    theta, g = theta_all[shift:], filled(N, torch.bfloat16, 1e-3, 2)
    m, v = filled(N, torch.float32, 1e-3, 3), filled(N, torch.float32, 1e-3, 4).square_()
    out, ws = torch.empty(2, device="cuda"), B.grad_norm_workspace()
    B.sparseloco_grad_norm(plan, [g], out, ws, max_norm=1.0)
    want = sum(float(g[a:a + (1 << 28)].double().square().sum()) for a in range(0, N, 1 << 28)) ** 0.5
    assert abs(out[0].item() - want) <= 1.01 * U24 * want
    before = [[f64(t[s].float()) for t in (theta, g, m, v)] for s in places(N)]
    B.sparseloco_adamw_step(plan, [theta], [g], [m], [v], **HOW)
    for s, (t0, g0, m0, v0) in zip(places(N), before):
        want = O.adamw(t0, g0, m0, np.sqrt(v0), **HOW)
        for got, k, what in ((theta, 0, "theta"), (m, 1, "m"), (v, 2, "v")):
            within(f64(got[s]), want[k], want[k + 3], "%s from %d" % (what, s.start))


def test_moments_in_8_bits_of_more_than_two_to_the_31_elements():
    plan = B.Plan([N], 32)
    theta, g = filled(N, torch.float32, 0.1, 1), filled(N, torch.bfloat16, 1e-3, 2)
    state = plan.adamw_8bit_buffers()
    before = [[f64(t[s].float()) for t in (theta, g)] for s in places(N)]
    B.sparseloco_adamw_step_8bit(plan, [theta], [g], *state, **HOW)
    for s, (t0, g0) in zip(places(N), before):
        zero = np.zeros_like(t0)
        want = O.adamw(t0, g0, zero, zero, **HOW)
        within(f64(theta[s]), want[0], want[3], "theta from %d" % s.start)
        if s.start % 256:                # (the blocks at the tensor's end do not begin with the run)
            continue
        for k, x, second in ((0, want[1], False), (2, np.sqrt(want[2]), True)):
            numbers, scales, edge = O.held(x.reshape(-1, 256), np.arange(s.start, s.stop), HOW["step"], second)
            got = f64(state[k][s].float()).reshape(-1, 256)
            assert np.all(np.abs(f64(state[k + 1][s.start // 256:s.stop // 256]) - scales) <= 12 * U24 * scales)
            differ = got != numbers
            assert np.all(edge[differ] <= 2.0 ** -15)
    codes = plan.num_flat_chunks * 4096
    assert not state[0][N:codes].float().any() and not state[2][N:codes].float().any()


@pytest.mark.parametrize("accumulate", [False, True])
def test_embedding_gradient_of_more_than_four_gib_into_a_table_of_more_than_four_gib(accumulate):
    rows, vocab, d = 700_000, 1_100_000, 2000
    grad = torch.zeros(rows, d, dtype=torch.bfloat16, device="cuda")
    ids = (torch.arange(rows, device="cuda", dtype=torch.int64) * 999_983 % vocab).to(torch.int32)
    at = [0, 1, 268_435, 536_870, 536_871, rows - 1]         # (2^30 and 2^31 bytes in, and behind)
    for k, r in enumerate(at):
        grad[r] = k + 1
    ids[at[2]] = ids[at[5]] = vocab - 1
    table = torch.full((vocab, d), 0.5 if accumulate else 7.0, dtype=torch.bfloat16, device="cuda")
    ws = B.embedding_grad_workspace(rows, vocab, d)
    B.sparseloco_embedding_grad(grad, ids, table, ws, accumulate=accumulate)
    base = 0.5 if accumulate else 0.0
    want = {}
    for k, r in enumerate(at):
        v = ids[r].item()
        want[v] = want.get(v, base) + (k + 1)
    for v, x in want.items():
        assert (table[v] == x).all(), (v, table[v, 0].item(), x)
    others = torch.ones(vocab, dtype=torch.bool, device="cuda")
    others[list(want)] = False
    for a in range(0, vocab, 100_000):
        part = table[a:a + 100_000][others[a:a + 100_000]]
        assert (part == base).all()
