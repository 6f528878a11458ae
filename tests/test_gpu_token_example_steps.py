"""A step of the replicas in examples/token_replicas.py: parameters move against their gradients, replicas part between restarts, and a restart is the mean of what they held."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def E():
    spec = importlib.util.spec_from_file_location("token_replicas", os.path.join(ROOT, "examples", "token_replicas.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _trainer(E, interval):
    return E.Trainer(E.shards(3, 400, 37, "cuda"), 40, 2, 37, 4, 21, interval, share=0.25)


def _near(a, b):
    """The same operations once more: products of the library may be summed in another order."""
    return bool(((a - b).abs() <= 1e-5 * b.abs().max()).all())


def test_parameters_move_against_their_gradients(E):
    t, other = _trainer(E, 100), _trainer(E, 100)
    before = {k: v.clone() for k, v in t.p.items()}
    t.step()
    other.t = 1
    _, grads = other.gradients(*other.minibatch())
    for k, g in grads.items():
        assert bool(g.any()), k
        moved = t.p[k] - before[k]
        if k[0] in "ab":
            assert bool(((moved * g).flatten(1).sum(1) < 0).all()), k       # along -U V^T of the gradient U S V^T
        else:
            assert _near(t.p[k], before[k] - t.rate * g), k


def test_replicas_part_and_a_restart_is_their_mean(E):
    t, alone = _trainer(E, 3), _trainer(E, 100)
    for _ in range(2):
        t.step()
        alone.step()
    for k, v in t.p.items():
        assert not torch.equal(v[0], v[1]) and not torch.equal(v[0], v[2]), k
    t.step()
    alone.step()
    for k, v in t.p.items():
        mean = alone.p[k].mean(0)
        assert all(torch.equal(v[0], v[i]) for i in range(3)) and _near(v[0], mean), k
        assert not torch.equal(alone.p[k][0], alone.p[k][1]), k
