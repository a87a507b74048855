"""Modules with a seed number their calls; a run that is resumed from its state goes on with the next one (no GPU needed)."""
import copy

import pytest
import torch

from paper_1908_06077_amd.dropout import Draws, Dropout
from paper_1908_06077_amd.norm import ResidualNorm


def model(seed):
    return torch.nn.Sequential(Dropout(0.1, seed=seed), ResidualNorm(8, dropout=0.2, seed=None if seed is None else seed + 1))


def draws_of(m):
    return [m[0].draws, m[1].draws]


def test_a_resumed_run_goes_on():
    m = model(5)
    for _ in range(7):
        draws_of(m)[0].next()
    draws_of(m)[1].next()
    saved = copy.deepcopy(m.state_dict())
    want = [d.next() for d in draws_of(m)]
    other = model(5)
    other.load_state_dict(saved)
    assert [d.calls for d in draws_of(other)] == [7, 1] and [d.next() for d in draws_of(other)] == want
    assert [d.calls for d in draws_of(m)] == [8, 2]           # (not shared)
    copied = copy.deepcopy(other)
    assert [d.next() for d in draws_of(copied)] == [d.next() for d in draws_of(m)]
    copied.load_state_dict(saved)                             # a copy's state is its own
    assert [d.calls for d in draws_of(copied)] == [7, 1] and [d.calls for d in draws_of(other)] == [8, 2]


def test_state_of_tensors(tmp_path):
    m = model(5)
    draws_of(m)[0].next()
    assert all(isinstance(v, torch.Tensor) for v in m.state_dict().values())
    torch.save(m.state_dict(), tmp_path / "state")
    other = model(5)
    other.load_state_dict(torch.load(tmp_path / "state", weights_only=True))
    assert draws_of(other)[0].calls == 1


def test_states_without_calls_and_modules_without_seeds():
    """A state that was saved without the number of calls loads and leaves it; without a seed there is nothing to save."""
    plain = model(None)
    names = set(plain.state_dict())
    assert names == {"1.outer_weight", "1.outer_bias"}
    m = model(5)
    draws_of(m)[0].next()
    m.load_state_dict(plain.state_dict())
    assert [d.calls for d in draws_of(m)] == [1, 0]
    plain.load_state_dict(m.state_dict())
    with pytest.raises(RuntimeError, match="Unexpected"):     # what else is wrong with a state is still said
        m.load_state_dict({**m.state_dict(), "0.draws.other": torch.zeros(1)})
    with pytest.raises(RuntimeError, match="Missing"):
        m.load_state_dict({k: v for k, v in m.state_dict().items() if k != "1.outer_bias"})


def test_numbers_are_as_they_were():
    d = Draws(0.5, 3, None)
    assert [d.next() for _ in range(2)] == [(3 + k * 0xA0761D6478BD642F) % 2 ** 64 for k in (1, 2)]
    assert [n for n, _ in model(5).named_parameters()] == ["1.outer_weight", "1.outer_bias"]
