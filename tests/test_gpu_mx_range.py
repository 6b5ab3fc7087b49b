"""Microscaled records at the ends of the number range (needs a B200)."""
import numpy as np
import pytest
import torch

import mx_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_04991_b200 import binding as rac
    rac.load()
    return type("Env", (), dict(rac=rac, dev=torch.device("cuda:0")))


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("d", [64, 2880])
def test_blocks_far_below_the_largest_value_of_their_row(env, d, block):
    """Every power of two as the largest value of one block and of the row: a block's scale byte is 0 only where all of it is 0, however
    small it is beside the row's largest block."""
    rac, dev = env.rac, env.dev
    power = 2.0 ** torch.arange(-133, 128, dtype=torch.float64)        # all that bf16 has
    large = torch.tensor([2.0 ** k for k in (127, 126, 100, 50, 20, 0, -60, -110)], dtype=torch.float64)
    X = torch.zeros((large.numel(), power.numel(), d), dtype=torch.float64)
    X[:, :, 3] = large[:, None]
    X[:, :, 32] = power
    X[:, :, 33] = -power * 1.75
    X[:, :, d - 1] = power * 0.5
    X = X.view(-1, d).clamp(-3e38, 3e38).to(torch.bfloat16)
    cfg = rac.MxCfg(d, block)
    want, bad = ref.encode(X.double().numpy(), block)
    assert not bad
    pay = torch.zeros(want.shape, dtype=torch.uint8, device=dev)
    xh = torch.empty(X.shape, dtype=torch.bfloat16, device=dev)
    rac.rac_mx_encode(cfg, X.to(dev), X.shape[0], pay, pay.numel(), xh, None)
    assert np.array_equal(pay.cpu().numpy(), want)
    top = torch.finfo(torch.bfloat16).max
    values = torch.from_numpy(np.clip(ref.decode(want, d, block), -top, top)).to(torch.bfloat16)
    assert torch.equal(xh.cpu().view(torch.int16), values.view(torch.int16))
