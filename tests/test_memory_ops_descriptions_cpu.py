"""Descriptions of the memory operators are kept by the numbers in them, not by the objects that hold these."""
import torch

from paper_1611_06256_amd import binding


def test_numbers_that_change_in_place_are_read_at_each_call(monkeypatch):
    monkeypatch.setattr(binding, "_element_type", lambda t, what: 0)
    q, decay, scale, eps = torch.zeros(4, 2, 16), [torch.tensor(0.5), torch.tensor(0.75)], torch.tensor(0.25), torch.tensor(0.5)
    d, n = binding._decay_desc(q, q, decay, scale), binding._norm_desc(q, 4, "none", eps)[0]
    assert list(d.decay[:2]) == [0.5, 0.75] and d.scale == 0.25 and n.eps == 0.5
    decay[1].fill_(0.25), scale.fill_(2.0), eps.fill_(0.125)
    d, n = binding._decay_desc(q, q, decay, scale), binding._norm_desc(q, 4, "none", eps)[0]
    assert list(d.decay[:2]) == [0.5, 0.25] and d.scale == 2.0 and n.eps == 0.125
    d = binding._decay_desc(q, q, torch.tensor([1.0, 0.125]), 1)
    assert list(d.decay[:2]) == [1.0, 0.125] and d.scale == 1.0
