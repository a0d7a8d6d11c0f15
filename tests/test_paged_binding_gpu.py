"""The paged operators' binding on the GPU: one tensor of a call on the host is refused before any launch; a stream of the
tensors' device, the current one and a given one, is taken."""
import pytest
import torch

from gpu_helpers import log
from test_paged_binding_host import CALLS

pytestmark = pytest.mark.gpu


def on_gpu(call):
    import paper_2602_15922_amd as w
    f, args = CALLS[call]
    a = {n: x.cuda() if isinstance(x, torch.Tensor) else x for n, x in args().items()}
    if "cache" in a:
        k, v, _ = a["cache"]._keep
        a["cache"] = w.make_paged_cache(k.cuda(), v.cuda())
    return f, a


@pytest.mark.parametrize("call", list(CALLS))
def test_a_tensor_left_on_the_host(call):
    f, a = on_gpu(call)
    for n, x in a.items():
        if isinstance(x, torch.Tensor):
            log(f"{call}: {n} on the host")
            with pytest.raises(ValueError):
                f(**{**a, n: x.cpu()})
    if "cache" in a:
        with pytest.raises(ValueError, match="one device"):
            f(**{**a, "cache": CALLS[call][1]()["cache"]})


@pytest.mark.parametrize("call", list(CALLS))
def test_streams(call):
    f, a = on_gpu(call)
    log(f"{call}: streams")
    torch.cuda.synchronize()
    f(**a)
    f(**a, stream=torch.cuda.Stream())
    with torch.cuda.stream(torch.cuda.Stream()):
        f(**a)
    torch.cuda.synchronize()
