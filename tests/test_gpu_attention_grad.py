"""The calls have no gradient: tensors that want one are refused, not answered without a graph."""

import pytest
import torch

from paper_2605_07238_amd import fate

pytestmark = pytest.mark.gpu


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def calls():
    """Names of the tensors a call takes, the tensors, and the call."""
    row = lambda h: torch.randn(6, h, 64, device="cuda").half()  # noqa: E731
    cache = lambda: torch.zeros(2, 2, 16, 64, dtype=torch.float16, device="cuda")  # noqa: E731
    off, kv, pages = ints(0, 6), ints(6), ints(0).view(1, 1)
    table = fate.rotation_table(16, 64)
    return {
        "append": (dict(q=row(4), k=row(2), v=row(2), k_cache=cache(), v_cache=cache(), table=table),
                   lambda x: fate.fate_kv_append(x["q"], x["k"], x["v"], x["k_cache"], x["v_cache"], off, kv, pages, x["table"])),
        "paged": (dict(q=row(4), k_cache=cache(), v_cache=cache()),
                  lambda x: fate.fate_attn_paged(x["q"], x["k_cache"], x["v_cache"], off, kv, pages)[0]),
        "prompt": (dict(q=row(4), k=row(2), v=row(2)), lambda x: fate.fate_attn_prompt(x["q"], x["k"], x["v"], off)[0]),
    }


@pytest.mark.parametrize("name", ["append", "paged", "prompt"])
def test_tensors_that_want_a_gradient(name):
    tensors, call = calls()[name]
    good = call(tensors)
    for key in tensors:
        tensors[key].requires_grad_()
        with pytest.raises(ValueError, match="gradient"):
            call(tensors)
        with torch.no_grad():
            assert torch.equal(call(tensors), good)
        with torch.inference_mode():
            assert torch.equal(call(tensors), good)
        tensors[key].requires_grad_(False)
    assert torch.equal(call(tensors), good)
    # what a graph made of them wants one too
    leaf = torch.randn(6, 4, 64, device="cuda", requires_grad=True)
    with pytest.raises(ValueError, match="gradient"):
        call(dict(tensors, q=leaf.half()))
    call(dict(tensors, q=leaf.half().detach()))
