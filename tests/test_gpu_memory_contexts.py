"""A network with a memory predicts the same in contexts of any capacity: the kernels behind a prediction, and so its rounding, go by the
frames of the call."""
import pytest
import torch

import paper_1611_06256_amd as g
from test_gpu_memory_net import SMALL, net_of, random_frames

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("frames", [1, 8, 42])
@pytest.mark.parametrize("capacity,train", [(0, 0), (0, 40), (1000, 0)], ids=["least", "least_training", "large"])
def test_predictions_do_not_depend_on_the_capacity(frames, capacity, train):
    print(f"memory contexts {frames} {capacity} {train}", flush=True)
    desc, memory = SMALL
    got = []
    for most, updates in ((max(capacity, frames), train), (512, 40)):
        net, _ = net_of(desc, memory, most, updates)
        net.profile_enable(True)
        states = torch.rand(frames, 4, 32, 16, generator=torch.Generator().manual_seed(2)).cuda()
        out = torch.empty(frames, desc.n_actions, device="cuda"), torch.empty(frames, device="cuda")
        net.predict_memory(random_frames(4, frames, desc).cuda(), states, logits=out[0], values=out[1])
        got.append((out, states, set(net.profile_read())))
        torch.cuda.synchronize()
        net.close()
    (a, x, stages), (b, y, others) = got
    assert stages == others
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and torch.equal(x, y)
