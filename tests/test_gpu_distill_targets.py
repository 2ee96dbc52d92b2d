"""The teacher's targets where the worker and its caller are on different
streams."""
import numpy as np
import pytest

from oracle import rows
from paper_2509_26092_amd import binding as B
from paper_2509_26092_amd import inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("worker_aside", [True, False])
def test_teacher_targets_across_streams(worker_aside):
    """The images are still being made on the caller's stream when the call
    is made, and what it returns is read there at once: the same as with one
    stream, for several batches of different images."""
    import torch
    from paper_2509_26092_amd import distill
    n, k = 64, 7
    side = torch.cuda.Stream()
    w = B.Worker("cifar", 100, "fp32", stream=side if worker_aside else None)
    state = torch.zeros(w.n_state, device="cuda")
    B.rn18_destroy(B.rn18_init(w.cfg, 3, state))
    base = torch.from_numpy(inputs.images(1, n, 32, 32)).cuda()
    torch.cuda.synchronize()
    got = []
    with torch.cuda.stream(torch.cuda.current_stream() if worker_aside else side):
        for i in range(4):
            x = base
            for _ in range(50):                     # a queue of work before the last image is there
                x = x * 1.01 if i % 2 else x.flip(0)
            x = (x + 0.1 * i).contiguous()
            vals, idx = distill.teacher_targets(w, state, x, k)
            got.append((x, vals + 0.0, idx + 0))
    torch.cuda.synchronize()
    for x, vals, idx in got:
        z = torch.empty((n, 100), device="cuda")
        w.eval_logits(state, x, z)
        torch.cuda.synchronize()
        v, i = rows.topk(z.cpu().numpy(), k)
        assert np.array_equal(idx.cpu().numpy(), i) and np.array_equal(vals.cpu().numpy(), v)
    w.close()
