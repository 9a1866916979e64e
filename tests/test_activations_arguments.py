"""What the activation calls and their binding refuse, where it is not the obvious: decided from the arguments alone, without a GPU."""
import pytest

import paper_2303_02868_amd as apm
from test_activations_host import join, matrix, refused


def test_a_gate_for_all_tokens_is_looked_at_as_one_row():
    """It is read for a batch without tokens too (the sums' factors), and no distance between rows counts."""
    forward = lambda **o: apm.lib().apm_norm_join_forward(join(gate_kind=apm.APM_GATE_CHANNEL, **o), None)
    refused(forward(rows=0, gate=matrix(dtype=7)), apm.APM_EINVAL, "gate: bad dtype")
    refused(forward(rows=0, gate=matrix(1 << 20 | 1)), apm.APM_EINVAL, "gate is not aligned")
    refused(forward(gate=matrix(stride=1 << 55), y=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "x and y have different types")
    assert forward(rows=0) == apm.APM_OK


def test_a_workspace_is_as_large_as_the_memory_behind_it():
    """A tensor of stride 0 has more elements than memory: no call may take their number for the workspace's size."""
    torch = pytest.importorskip("torch")
    few = torch.zeros(16, 1, dtype=torch.uint8)
    for room in (few.expand(16, 1 << 20), few[::2]):
        room.is_pinned = lambda: True              # past the check of where it is
        grads = apm.apm_norm_join_grads()
        with pytest.raises(ValueError, match="workspace.*contiguous"):
            apm.apm_norm_join_backward(join(rows=0), grads, room)
        with pytest.raises(ValueError, match="workspace.*contiguous"):
            apm.apm_ckpt_weight_grad(apm.apm_weight_grad(), room)
