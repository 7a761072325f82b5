"""Norms and products on the GPU: memory that streams hand to one another, in place calls, scales that no rounding makes, and
more work than small grids hold."""
import numpy as np
import pytest
import torch

from paper_2609_25405_amd import linear as L

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu(request):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print(f"\n[case] {request.node.name}", flush=True)


# ------------------------------------------------------------------------------ streams
@pytest.mark.parametrize("side", ["pool", "default"])
def test_weights_packed_on_another_stream(side):
    """Weights packed on a stream of the caller's, into memory that the current stream has just given back and still has a
    kernel queued on."""
    m = torch.randn((512, 1024), device="cuda").to(torch.bfloat16)
    want = L.LinearWeights(m).packed.clone()
    torch.cuda.synchronize()
    default = torch.cuda.default_stream()
    here, there = (default, torch.cuda.Stream()) if side == "pool" else (torch.cuda.Stream(), default)
    with torch.cuda.stream(here):
        for _ in range(3):
            block = torch.empty_like(want)
            torch.cuda._sleep(20_000_000)
            block.fill_(7)
            del block
            w = L.LinearWeights(m, stream=there.cuda_stream)
            torch.cuda.synchronize()
            assert torch.equal(w.packed, want)
            # dropped at once: the memory is not another's before it is packed
            torch.cuda._sleep(1)
            there.wait_stream(here)
            with torch.cuda.stream(there):
                torch.cuda._sleep(20_000_000)
            L.LinearWeights(m, stream=there.cuda_stream)
            after = torch.full_like(want, 9)
            torch.cuda.synchronize()
            assert (after == 9).all()
