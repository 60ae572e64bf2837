"""The AdamW step with moments in 8 bits over a tensor of more than 2^31 elements, from a state whose codes and scales differ from
block to block: a code or a scale that is read from or written to another place shows."""
import numpy as np
import pytest
import torch

from oracle import inner as O
from paper_2601_02360_amd import binding as B
from test_gpu_inner import HOW, U24, f64, within
from test_gpu_inner_large import N, filled

pytestmark = pytest.mark.gpu
BLOCK = 256
LAST = N // BLOCK * BLOCK                # the last block's first element; the tensor ends inside it


def codes(n, low, high, seed):
    """Values that e4m3 holds, at random."""
    x = torch.empty(n, dtype=torch.float8_e4m3fn, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(seed)
    for a in range(0, n, 1 << 28):
        part = x[a:a + (1 << 28)]
        part.copy_(torch.rand(part.numel(), generator=g, device="cuda").mul_(high - low).add_(low))
    return x


def test_every_block_has_its_own_codes_and_scales():
    plan = B.Plan([N], 32)
    total = plan.num_flat_chunks * 4096
    theta, g = filled(N, torch.float32, 0.1, 1), filled(N, torch.bfloat16, 1e-3, 2)
    m, v = codes(total, -448, 448, 3), codes(total, 1, 448, 4)
    m[N:].view(torch.uint8).zero_()
    v[N:].view(torch.uint8).zero_()
    block = torch.arange(total // BLOCK, device="cuda")
    m_scale = ((block % 977).float() / 977 + 0.5) * 2e-6     # (prime: no power of two further is the same)
    v_scale = ((block % 983).float() / 983 + 0.5) * 4e-6
    state = (m, m_scale, v, v_scale)
    assert total - LAST >= BLOCK
    starts = [0, LAST - 512] + [p - 256 for p in (2 ** 28, 2 ** 29, 2 ** 30, 2 ** 31)]
    before = {}
    for a in starts:
        s, b = slice(a, min(a + 768, N)), slice(a // BLOCK, a // BLOCK + 3)
        before[a] = [f64(t[s].float()) for t in (theta, g)] + [f64(t.float()) for t in (m[a:a + 768], m_scale[b], v[a:a + 768], v_scale[b])]
    B.sparseloco_adamw_step_8bit(plan, [theta], [g], *state, **HOW)
    for a, (t0, g0, mc, ms, vc, vs) in before.items():
        n = len(t0)
        t0, g0 = (np.pad(x, (0, 768 - n)) for x in (t0, g0))
        want = O.adamw(t0, g0, mc * np.repeat(ms, BLOCK), vc * np.repeat(vs, BLOCK), **HOW)
        # (two roundings more: what the 8 bits stand for, and its square)
        within(f64(theta[a:a + n]), want[0][:n], (want[3] + 4 * np.abs(want[0] - t0))[:n], "theta from %d" % a)
        for k, x, second in ((0, want[1], False), (2, np.sqrt(want[2]), True)):
            numbers, scales, edge = O.held(x.reshape(-1, BLOCK), np.arange(a, a + 768), HOW["step"], second)
            got = f64(state[k][a:a + 768].float()).reshape(-1, BLOCK)
            assert np.all(np.abs(f64(state[k + 1][a // BLOCK:a // BLOCK + 3]) - scales) <= 12 * U24 * scales)
            assert np.all(edge[got != numbers] <= 2.0 ** -15), "codes from %d" % a
            assert not got.reshape(-1)[n:].any()
    assert not m[N:].float().any() and not v[N:].float().any()
