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


class OnGpu:
    """What the binding asks a tensor on a GPU for."""

    def __init__(self, torch, device, *shape, dtype=None):
        self.t, self.device = torch.zeros(*shape, dtype=dtype or torch.bfloat16), device

    is_cuda = True

    def get_device(self):
        return self.device

    def __getattr__(self, name):
        return getattr(self.t, name)

    def __getitem__(self, i):
        return self.t[i]


def test_tensors_of_another_gpu_than_the_current_one(monkeypatch):
    """Kernels run on the current device: what lies on another one is refused, where a structure is made and where it is used."""
    torch = pytest.importorskip("torch")
    from paper_2303_02868_amd import binding
    here = [0]
    monkeypatch.setattr(binding, "_here", lambda: here[0])
    byte = torch.uint8
    there = lambda *s, **k: OnGpu(torch, 1, *s, **k)
    near = lambda *s, **k: OnGpu(torch, 0, *s, **k)
    kept = apm.make_ckpt(near(4, 64, dtype=byte), near(4, 2, dtype=byte), apm.APM_CKPT_I8)
    for wrong in (lambda: apm.make_matrix("x", there(4, 64), 4, 64), lambda: apm.make_vector("w", there(64), 64),
                  lambda: apm.make_ckpt(near(4, 64, dtype=byte), there(4, 2, dtype=byte), apm.APM_CKPT_I8),
                  lambda: apm.apm_ckpt_write(there(4, 64), kept), lambda: apm.apm_ckpt_read(kept, there(4, 64)),
                  lambda: apm.make_norm_join(4, 64, x=near(4, 64), pre_weight=there(64)),
                  lambda: apm.make_norm_join(4, 64, x=near(4, 64), pre_rstd=there(4, dtype=torch.float32)),
                  lambda: apm.make_weight_grad(near(4, 32), kept, there(32, 64)),
                  lambda: apm.make_weight_grad(near(4, 32), kept, near(32, 64), db=there(32)),
                  lambda: apm.apm_ckpt_weight_grad(apm.apm_weight_grad(), there(64, dtype=byte))):
        with pytest.raises(ValueError, match="on GPU 1, the current one is 0"):
            wrong()
    made = apm.make_norm_join(4, 64, x=near(4, 64), pre_ckpt=kept)
    grads = apm.make_norm_join_grads(made, dn=near(4, 64))
    grad = apm.make_weight_grad(near(4, 32), kept, near(32, 64))
    here[0] = 1
    for wrong in (lambda: apm.apm_norm_join_forward(made), lambda: apm.make_norm_join_grads(made), lambda: apm.apm_norm_join_backward(made, grads, None),
                  lambda: apm.apm_ckpt_weight_grad(grad), lambda: apm.apm_ckpt_write(there(4, 64), kept), lambda: apm.apm_ckpt_read(kept, there(4, 64))):
        with pytest.raises(ValueError, match="looked at for GPU 0, the current one is 1"):
            wrong()
