"""Rotations are copied and saved, as the modules that hold one are."""
import copy
import io
import pickle

import pytest
import torch

from paper_2510_18121_amd import binding as B
from paper_2510_18121_amd import rotary as R


def saved(r):
    f = io.BytesIO()
    torch.save(r, f)
    f.seek(0)
    return torch.load(f, weights_only=False)  # (written above)


COPIES = [copy.copy, copy.deepcopy, lambda r: pickle.loads(pickle.dumps(r)), saved]


@pytest.mark.parametrize("copied", COPIES)
@pytest.mark.parametrize("kw", [{"rot_dim": 64, "interleaved": True, "factor": 1.5}, {"rot_dim": 0}])
def test_copies(copied, kw):
    r = R.Rotation(128, device="cpu", **kw)
    c = copied(r)
    for name in ("head_dim", "rot_dim", "interleaved", "factor", "device"):
        assert getattr(c, name) == getattr(r, name)
    assert torch.equal(c.turns, r.turns) and (c.frequencies == r.frequencies).all()
    assert c.desc is not r.desc and c.desc.turns == (c.turns.data_ptr() if r.rot_dim else None)
    assert [getattr(c.desc, f) for f, _ in R.RotationDesc._fields_[:4]] == [getattr(r.desc, f) for f, _ in R.RotationDesc._fields_[:4]]


def test_a_module_that_holds_one():
    class Layer(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.rotation, self.gain = R.Rotation(64, device="cpu"), torch.nn.Parameter(torch.ones(64))

    layer = Layer()
    again = copy.deepcopy(layer)
    assert again.rotation.turns.data_ptr() != layer.rotation.turns.data_ptr() and again.rotation.desc.turns == again.rotation.turns.data_ptr()


@pytest.mark.gpu
@pytest.mark.parametrize("copied", COPIES)
def test_copies_turn_alike(copied):
    r = R.Rotation(64, device="cuda:0")
    q = torch.randn(5, 2, 64, device="cuda:0").to(torch.bfloat16)
    pos, y, z = torch.arange(5, dtype=torch.int32, device="cuda:0"), torch.empty_like(q), torch.empty_like(q)
    B.ca_rotate(r, q, None, y, None, pos)
    c = copied(r)
    del r
    torch.cuda.synchronize()
    B.ca_rotate(c, q, None, z, None, pos)
    assert torch.equal(y, z)
