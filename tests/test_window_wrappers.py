"""Host side of the Python wrappers of the query/key preparation, without a device."""
import pytest
import torch


def _rope(**kw):
    """A Rope whose tensors lie on the host (device -1), as they may look after somebody has replaced or converted them."""
    from paper_2305_17118_b200 import binding as sh
    r = object.__new__(sh.Rope)
    r.inv_freq, r.q_weight, r.k_weight = torch.ones(32), torch.ones(64, dtype=torch.bfloat16), None
    r._head = (64, 1, 32, 0, 0, 0, 0, 1e-6)
    for name, value in kw.items():
        setattr(r, name, value)
    return r


def test_a_rope_as_it_was_made_is_taken():
    assert len(_rope()._packed(64, torch.bfloat16, -1)) == 64
    assert len(_rope(q_weight=None)._packed(64, torch.float16, -1)) == 64


@pytest.mark.parametrize("name,value", [
    ("inv_freq", torch.ones(32, dtype=torch.float16)), ("inv_freq", torch.ones(32, dtype=torch.float64)), ("inv_freq", torch.ones(64)[::2]),
    ("inv_freq", torch.ones(16)), ("inv_freq", torch.ones(1, 32)), ("q_weight", torch.ones(64)), ("q_weight", torch.ones(128, dtype=torch.bfloat16)),
    ("q_weight", torch.ones(128, dtype=torch.bfloat16)[::2]), ("k_weight", torch.ones(128, dtype=torch.bfloat16)[::2]),
])
def test_a_rope_whose_tensors_changed_is_looked_at_again(name, value):
    """A kernel reads frequencies and weights as contiguous vectors of their types: others would be read past their end."""
    with pytest.raises(ValueError):
        _rope(**{name: value})._packed(64, torch.bfloat16, -1)
