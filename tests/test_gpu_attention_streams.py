"""Attention calls on a stream that is not the tensors' own: memory let go after the call is handed out behind it."""

import pytest
import torch

from paper_2605_07238_amd import fate

pytestmark = pytest.mark.gpu


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def calls(side):
    """What makes an input, and the call that reads it on `side`."""
    new = lambda: torch.randn(2048, 8, 64, device="cuda").half()  # noqa: E731
    off, pages = ints(0, 2048), torch.arange(128, dtype=torch.int32, device="cuda").view(1, -1)
    cache = [torch.zeros(128, 8, 16, 64, dtype=torch.float16, device="cuda") for _ in range(2)]
    return {
        "prompt": (new, lambda x: fate.fate_attn_prompt(x, x, x, off, stream=side)),
        "paged": (new, lambda x: fate.fate_attn_paged(x, *cache, off, ints(2048), pages, stream=side)),
        "append": (new, lambda x: fate.fate_kv_append(x, x, x, *cache, off, ints(2048), pages, stream=side)),
    }


@pytest.mark.parametrize("name", ["prompt", "paged", "append"])
def test_inputs_let_go_after_the_call(name):
    side = torch.cuda.Stream()
    new, call = calls(side)[name]
    much = torch.empty(1 << 31, dtype=torch.uint8, device="cuda")
    x = new()
    side.wait_stream(torch.cuda.current_stream())
    call(x)  # kernels load at the first call
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(50):  # the side stream is behind: about 20 ms
            much.zero_()
    x = new()
    side.wait_stream(torch.cuda.current_stream())
    kept = call(x)
    at, shape, dtype = x.data_ptr(), x.shape, x.dtype
    del x
    other = torch.empty(shape, dtype=dtype, device="cuda")
    assert not side.query()  # still behind, so what it will read cannot be anyone else's yet
    assert other.data_ptr() != at
    side.synchronize()
    del kept


def test_heads_of_no_elements_are_refused():
    x, off = torch.empty(2, 4, 0, dtype=torch.float16, device="cuda"), ints(0, 2)
    cache = torch.empty(1, 4, 16, 0, dtype=torch.float16, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    for call in (lambda: fate.fate_attn_prompt(x, x, x, off),
                 lambda: fate.fate_attn_paged(x, cache, cache, off, ints(2), ints(0).view(1, 1), ws=ws)):
        with pytest.raises(fate.FateError) as e:
            call()
        assert e.value.status == fate.FATE_EINVAL
