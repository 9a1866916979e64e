"""What the activation calls and their binding refuse, where it is not the obvious: decided from the arguments alone, without a GPU."""
import paper_2303_02868_amd as apm
from test_activations_host import join, matrix, refused


def test_a_gate_for_all_tokens_is_looked_at_as_one_row():
    """It is read for a batch without tokens too (the sums' factors), and no distance between rows counts."""
    forward = lambda **o: apm.lib().apm_norm_join_forward(join(gate_kind=apm.APM_GATE_CHANNEL, **o), None)
    refused(forward(rows=0, gate=matrix(dtype=7)), apm.APM_EINVAL, "gate: bad dtype")
    refused(forward(rows=0, gate=matrix(1 << 20 | 1)), apm.APM_EINVAL, "gate is not aligned")
    refused(forward(gate=matrix(stride=1 << 55), y=matrix(dtype=apm.APM_F32)), apm.APM_EINVAL, "x and y have different types")
    assert forward(rows=0) == apm.APM_OK
