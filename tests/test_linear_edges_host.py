"""Norms and products on the CPU: calls whose tensors or sizes would have a kernel read or write what is not theirs, or what
another call holds.  No GPU work: every call below is rejected by host checks."""
import pytest
import torch

from paper_2609_25405_amd import _abi as A
from paper_2609_25405_amd import linear as L
from paper_2609_25405_amd import ops


def weights_of(n, k, groups=1, gated=False):
    """LinearWeights as a call on the host sees them: nothing is packed."""
    w = L.LinearWeights.__new__(L.LinearWeights)
    w._sizes, w._device = (n, k, groups, gated), -1
    return w


@pytest.mark.parametrize("workspace", [torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(64, dtype=torch.uint8)[::2],
                                       torch.zeros((4, 8)).t()])
def test_workspaces_whose_bytes_are_not_side_by_side_are_refused(workspace):
    x, y = torch.zeros((3, 64), dtype=torch.bfloat16), torch.zeros((3, 48), dtype=torch.bfloat16)
    with pytest.raises(A.OrthrusError, match="workspace"):
        L.linear(weights_of(48, 64), x, y, workspace=workspace)
    with pytest.raises(A.OrthrusError, match="workspace"):
        L.linear_grouped(weights_of(48, 64, 2), x, torch.zeros(3, dtype=torch.int32), y, workspace=workspace)
    with pytest.raises(A.OrthrusError, match="workspace"):
        ops.logprobs(torch.zeros((2, 8)), logprob=torch.zeros(2), workspace=workspace)


@pytest.mark.parametrize("name", ["codes", "scales", "shape"])
def test_rows_in_blocks_stay_what_they_were_made_of(name):
    """A call hands over the addresses that were taken when the object was made: none of its tensors can be exchanged."""
    m, other = L.Mx8.empty(3, 64, device="cpu"), L.Mx8.empty(5, 64, device="cpu")
    before = bytes(m._ref)
    with pytest.raises(AttributeError):
        setattr(m, name, getattr(other, name))
    assert bytes(m._ref) == before and m.shape == m.codes.shape == (3, 64)
    at = [int.from_bytes(before[8 * i:8 * i + 8], "little") for i in range(2)]
    assert at == [m.codes.data_ptr(), m.scales.data_ptr()]


@pytest.mark.parametrize("name", ["packed", "n", "k", "groups", "gated"])
def test_weights_stay_what_was_packed(name):
    w = weights_of(48, 64, 2, True)
    with pytest.raises(AttributeError):
        setattr(w, name, 1)
    assert (w.n, w.k, w.groups, w.gated) == (48, 64, 2, True)
