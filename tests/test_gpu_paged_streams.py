"""Calls made from another stream than the handle's: memory that queued work still uses is not handed out again."""
import numpy as np
import pytest
import torch

import paper_2609_37772_amd as U
import uad_workloads as W
from tests import paged_oracle as P
from tests.test_gpu_paged import check_attend, dev, draw, handle

pytestmark = pytest.mark.gpu
LATE = 200_000_000  # clock ticks that the handle's stream waits before its work


def taken_again(tensors):
    """Whether new tensors of the current stream get the memory of these, which are given up."""
    sizes = [(t.shape, t.dtype) for t in tensors]
    used = {t.data_ptr() for t in tensors}
    tensors.clear()
    new = [torch.empty(s, dtype=d, device="cuda") for s, d in sizes]
    return bool(used & {t.data_ptr() for t in new})


@pytest.fixture
def case(gpu):
    c = P.Cache(9, 1, 2, 64, 16, [300, 20])
    c.fill(4)
    side = torch.cuda.Stream()
    kv = handle(c, 4, stream=side)
    torch.cuda.synchronize()
    yield c, kv, side
    torch.cuda.synchronize()


def test_memory_given_up_is_taken_again_otherwise(case):
    assert taken_again([torch.zeros((300, 2, 64), device="cuda")])


@pytest.mark.parametrize("new", [[300, 20], [1, 1]], ids=["prompts", "tokens"])
def test_append_keeps_its_inputs(case, new):
    c, kv, side = case
    n = sum(new)
    k, v = draw(1, n, 2, 64), draw(2, n, 2, 64)
    args = [dev(k), dev(v), dev(c.table), dev(c.lens), dev(np.array([0, new[0], n], np.int32)), dev(np.arange(n, dtype=np.int32))]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LATE)
    kv.append(0, *args)
    assert not taken_again(args)
    kv.synchronize()
    pg, off = c.slot(1, 19)
    assert torch.equal(kv.v[0, pg, :, :, off].cpu(), v[-1].to(torch.bfloat16))


def test_attend_keeps_its_inputs_and_output(case):
    c, kv, side = case
    q = draw(1, 2, 4, 64)
    args = [dev(q), dev(c.table), dev(c.lens)]
    positions = dev(c.lens - 1)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(LATE)
    out = kv.attend(0, *args, positions=positions)
    args.append(positions)
    del positions
    assert not taken_again(args)
    # the output is the handle's stream's, and read on this one
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(LATE)
    got = out + 0
    at = out.data_ptr()
    del out
    with torch.cuda.stream(side):
        assert torch.empty((2, 4, 64), device="cuda").data_ptr() != at
    check_attend(c, kv, 0, q, got, 0, False)
    kv.synchronize()


def test_the_experts_prefix_keeps_its_inputs(gpu):
    shape = W.ModelShape(2, 128, 4, 2, 64, 256, 7)
    c = P.Cache(2, 2, 2, 64, 16, [40, 40])
    side = torch.cuda.Stream()
    kv = handle(c, 2)
    ex = U.ActionExpert(shape, 2, 3, 64, stream=side)
    try:
        args = [dev(c.table), dev(c.lens)]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(LATE)
        ex.set_prefix_paged(kv, *args, 40)
        assert not taken_again(args)
        ex.synchronize(), kv.synchronize()
    finally:
        ex.close()
