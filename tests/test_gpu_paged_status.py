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
