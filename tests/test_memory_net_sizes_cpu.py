"""Calls on a network with a memory whose tensors are smaller than what the library reads or writes are refused before it is called."""
import pytest
import torch

import paper_1611_06256_amd as g
from paper_1611_06256_amd import binding


class Called(Exception):
    pass


class Library:
    def __getattr__(self, name):
        def call(*_):
            raise Called(name)
        return call


@pytest.fixture
def net(monkeypatch):
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype, what: None)
    monkeypatch.setattr(binding, "_stream", lambda s: None)
    n = object.__new__(g.Ga3c)
    n._lib, n._ctx, n.desc, n.memory, n.n_actions = Library(), None, g.SMALL_NET(6), g.MemoryDesc(), 6
    monkeypatch.setattr(g.Ga3c, "__del__", lambda self: None, raising=False)
    return n


def test_predictions(net):
    frames, states = torch.zeros(5, 4, 84, 84, dtype=torch.uint8), torch.zeros(5, 4, 32, 16)
    good = {"uniforms": torch.zeros(5), "logits": torch.zeros(5, 6), "values": torch.zeros(5), "probs": torch.zeros(5, 6), "actions": torch.zeros(5)}
    with pytest.raises(Called):
        net.predict_memory(frames, states, **good)
    with pytest.raises(Called):
        net.predict_memory(frames, states, logits=torch.zeros(8, 6))            # room for more is the caller's business
    for what, t in good.items():
        with pytest.raises(g.Ga3cError, match=what):
            net.predict_memory(frames, states, **{**good, what: t.flatten()[:-1]})
    for bad in (frames[:, :3], frames[..., :83], frames.flatten(2)):
        with pytest.raises(g.Ga3cError, match="frames"):
            net.predict_memory(bad, states)


def test_updates(net):
    hp = g.HParams()
    frames = torch.zeros(3, 5, 4, 84, 84, dtype=torch.uint8)
    rest = [torch.zeros(3, 5) for _ in range(3)]
    with pytest.raises(Called):
        net.train_step_memory(frames, *rest, None, hp)
    with pytest.raises(Called):
        net.train_step_memory(frames.flatten(0, 1), *rest, torch.zeros(2), hp, seg_start=torch.zeros(3))
    for bad, kw in ((frames[:, :, :3], {}), (frames[..., :80, :], {}), (frames.flatten(0, 1), {}), (frames, {"seg_start": torch.zeros(3)}),
                    (frames.flatten(0, 1)[..., :83], {"seg_start": torch.zeros(3)})):
        with pytest.raises(g.Ga3cError, match="frames"):
            net.train_step_memory(bad, *rest, None, hp, **kw)
