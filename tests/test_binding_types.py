"""Tensors are bound as fp32 or bf16 and as nothing else: elements of another type would be read as one of these, and fp16 ones
past the end of their tensor.  The calls that take the type of a list from the list refuse it in the same way."""
import pytest
import torch

from paper_2601_02360_amd import binding as B

OTHERS = [torch.float16, torch.float64, torch.int32, torch.int16, torch.float8_e4m3fn, torch.complex64]


class FakePlan:
    """What Tensors reads from a plan before it calls the library."""
    numels = [8, 3]
    handle = None


@pytest.mark.parametrize("dtype", OTHERS)
def test_other_element_types_are_refused_before_anything_is_bound(dtype):
    tensors = [torch.zeros(n).to(dtype) for n in FakePlan.numels]
    for lists in (tensors, [tensors, tensors]):
        assert B._dtype_of(lists) == dtype
        with pytest.raises(ValueError, match="float32 or bfloat16"):
            B.Tensors(FakePlan(), lists, B._dtype_of(lists))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", OTHERS)
def test_calls_refuse_lists_of_other_element_types(dtype):
    plan = B.Plan([4096, 10], 32)
    theta, m, v = ([torch.zeros(n, device="cuda") for n in (4096, 10)] for _ in range(3))
    other = [torch.zeros(n, device="cuda").to(dtype) for n in (4096, 10)]
    out, pairs = torch.full((2,), 7.0, device="cuda"), plan.message_buffers()
    for call in (lambda: plan.bind(other, dtype=dtype),
                 lambda: B.sparseloco_grad_norm(plan, other, out, B.grad_norm_workspace()),
                 lambda: B.sparseloco_adamw_step(plan, theta, other, m, v, lr=1e-3, step=1),
                 lambda: B.sparseloco_adamw_step_8bit(plan, theta, other, *plan.adamw_8bit_buffers(), lr=1e-3, step=1),
                 lambda: B.sparseloco_compress(plan, m, *pairs, 0.9, delta=other)):
        with pytest.raises(ValueError, match="float32 or bfloat16"):
            call()
    assert out.tolist() == [7.0, 7.0] and not any(t.any() for s in (theta, m, v) for t in s)
