"""Orthogonalised matrices on the paths that shapes choose: every size of tiles, and several steps at once in squares."""
import pytest
import torch

from paper_2601_02360_amd import binding as B
from test_gpu_orthogonal import MODES, matrix

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
