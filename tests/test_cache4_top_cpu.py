"""The plain reference of the cache in 4 bits at the top of the storage types' range: a finite number is held as one."""
import numpy as np
import pytest
import torch

from tests import cache4_util as C4


def test_worked_blocks_at_the_top():
    # 3.5 to 4 times the greatest scale would be 4 times it, which the types do not have: 3 times it is held
    for dtype, e, values in ((torch.float16, 14, [57344.0, 60000.0, -65504.0]),
                             (torch.bfloat16, 126, [1.75 * 2.0 ** 127, -(2.0 - 2.0 ** -7) * 2.0 ** 127])):
        for x in values:
            block = torch.zeros(32, dtype=torch.float64)
            # (beside it half and a quarter of it, which are not changed by that, and the last number below)
            block[:4] = torch.tensor([x, 2.0 ** e, -1.5 * 2.0 ** e, 3.25 * 2.0 ** e], dtype=torch.float64)
            block = block.to(dtype)
            codes, scales = C4.quantise(block)
            held = C4.values(codes, scales)
            assert int(scales[0]) == 127 + e
            assert held[:4].tolist() == [np.sign(x) * 3 * 2.0 ** e, 2.0 ** e, -1.5 * 2.0 ** e, 3 * 2.0 ** e]
    # the largest blocks below: 6 times the scale before that
    assert C4.values(*C4.quantise(torch.full((32,), 57312.0, dtype=torch.float16)))[0] == 49152.0


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_a_finite_number_is_held_as_one(dtype):
    """Every finite number as its block's largest: a fifth of it off at most, a quarter where 4 times the scale is not a
    number of the type (from 3.5 scales on the largest goes to 3, 1/7 to 1/4 of it), or a quarter of the least scale."""
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(dtype)
    every = every[torch.isfinite(every)]
    block = torch.zeros(every.numel(), 32, dtype=dtype)
    block[:, 0], block[:, 1] = every, every / 3
    held = torch.from_numpy(C4.values(*C4.quantise(block)))
    assert torch.equal(held.to(dtype).double(), held)
    largest = every.double().abs()
    top = largest >= 1.75 * 2.0 ** (15 if dtype == torch.float16 else 127)
    assert int(top.sum()) > 60
    bound = torch.maximum(torch.where(top, largest / 4, largest / 5), torch.tensor(2.0 ** C4.LEAST[dtype] / 4))
    assert ((held - block.double()).abs() <= bound[:, None]).all()
