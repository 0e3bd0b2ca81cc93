"""Status words on the GPU: every call's own report arrives, however soon it follows the last one."""
import numpy as np
import pytest
import torch

import paper_2609_37772_amd as U
import uad_workloads as W
from tests import paged_oracle as P
from tests.test_gpu_paged import dev, handle

pytestmark = pytest.mark.gpu


def test_an_experts_status_is_reported_once_each_time(gpu):
    """Clearing it does not clear what a prefix that is queued right after it raises."""
    c = P.Cache(2, 2, 2, 64, 16, [40, 40], poison=0.0)
    side = torch.cuda.Stream()
    kv = handle(c, 2, stream=side)
    ex = U.ActionExpert(W.ModelShape(2, 128, 4, 2, 64, 256, 7), 2, 3, 64, stream=side)
    try:
        bad, lens = dev(np.full_like(c.table, c.n_pages)), dev(c.lens)
        torch.cuda.synchronize()
        for _ in range(50):
            ex.set_prefix_paged(kv, bad, lens, 40)
            with pytest.raises(U.UadError) as e:
                ex.synchronize()
            assert e.value.status == 9
        ex.synchronize()
    finally:
        ex.close()


def test_a_replay_on_another_stream_is_reported_each_time(gpu):
    """The handle's stream has nothing to do with where its graph runs."""
    c = P.Cache(9, 1, 1, 64, 16, [40])
    c.fill(4)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    kv = handle(c, 4, stream=side)
    with torch.cuda.stream(side):
        q, lens, table = torch.ones((1, 4, 64), device="cuda"), dev(c.lens), dev(np.full_like(c.table, -1))
        out = torch.empty_like(q)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            kv.attend(0, q, table, lens, out=out)
    for _ in range(50):
        with torch.cuda.stream(other):
            graph.replay()
        other.synchronize()
        with pytest.raises(U.UadError) as e:
            kv.synchronize()
        assert e.value.status == 9
    kv.synchronize()
