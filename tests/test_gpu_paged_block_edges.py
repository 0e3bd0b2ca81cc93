"""Appends to blocks whose scale the caller has set: any positive finite one, also where 448 times it is more than fp32 holds."""
import numpy as np
import pytest
import torch

import paper_2609_37772_amd as U
from tests.test_gpu_paged import BF16, F32, F8, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [2.0 ** 119, 2.0 ** 120, 2.0 ** 127, 1.5 * 2.0 ** 118, 1.5 * 2.0 ** 121, 3.4028234e38, 0.75])
@pytest.mark.parametrize("given", [BF16, F32])
@pytest.mark.parametrize("hd", [64, 256])
@pytest.mark.parametrize("starts", [False, True])
def test_rows_are_cut_to_448_scales(gpu, scale, given, hd, starts):
    """Three tokens of a block are held, a fourth comes: infinities are cut, a NaN stays one, other values are divided."""
    scale = float(np.float32(scale))
    kv = U.PagedKV(1, 1, 1, hd, 16, 2, 1, dtype=F8, block_scales=True)
    held = torch.linspace(-448, 448, hd).to(F8)
    kv.k.view(torch.uint8).fill_(0x7F), kv.v.view(torch.uint8).fill_(0x7F)
    kv.k[0, 1, 0, :3], kv.v[0, 1, 0, :, :3] = held.cuda(), held.cuda()[:, None]
    kv.k_scales.fill_(float("nan")), kv.v_scales.fill_(float("nan"))
    kv.k_scales[0, 1], kv.v_scales[0, 1] = scale, scale
    row = torch.zeros(hd, dtype=torch.float64)
    # beside what is not finite only values that need no larger power of two than the scale
    power = 2.0 ** np.floor(np.log2(scale))
    odd = [np.inf, -np.inf, np.nan, -np.nan, 1.0, -3.0, min(power * 300, 3e38), -min(power * 448, 3e38), min(power * 17, 1e38)]
    row[:len(odd)] = torch.tensor(odd, dtype=torch.float64)
    row[hd - 3:] = torch.tensor([np.inf, -np.inf, np.nan], dtype=torch.float64)
    row = row.to(given)
    x = dev(row)[None, None].contiguous()
    ints = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    kv.append(0, x, x, ints(1)[None].contiguous(), ints(4), ints(0, 1) if starts else None)
    kv.synchronize()
    assert float(kv.k_scales[0, 1, 0, 0]) == float(kv.v_scales[0, 1, 0, 0]) == scale
    want = (row.double() / scale).clamp(-448, 448)
    want = torch.where(row.isnan(), row.double(), want).float().to(F8).float()  # half way in 64 bits: none of these are
    for got, old in ((kv.k[0, 1, 0, 3], kv.k[0, 1, 0, :3]), (kv.v[0, 1, 0, :, 3], kv.v[0, 1, 0, :, :3].t())):
        assert torch.equal(got.float().cpu().nan_to_num(999), want.nan_to_num(999)), (got.float().cpu()[:12], want[:12])
        assert torch.equal(old.float().cpu(), held.float().expand(3, hd))
