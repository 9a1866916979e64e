"""What the binding of the calls on tokens takes for what: types of words, and structures laid out as the header has them."""
import pytest

import paper_2303_02868_amd as apm
from test_activations_arguments import OnGpu


def test_the_seed_is_a_whole_number(monkeypatch):
    torch = pytest.importorskip("torch")
    from paper_2303_02868_amd import binding
    monkeypatch.setattr(binding, "_here", lambda: 0)
    on = lambda *s, dtype=torch.bfloat16: OnGpu(torch, 0, *s, dtype=dtype)
    make = lambda word: apm.make_dropout(on(4, 64), on(4, 64), p=0.5, seed=1, seed_at=word)
    for dtype in (torch.int64, torch.uint64):
        assert make(on(1, dtype=dtype)).seed_at
    for dtype in (torch.float64, torch.complex64, torch.int32, torch.uint32):
        with pytest.raises(ValueError, match="seed_at"):
            make(on(1, dtype=dtype))
    with pytest.raises(ValueError, match="seed_at"):
        make(on(2, dtype=torch.int64))
