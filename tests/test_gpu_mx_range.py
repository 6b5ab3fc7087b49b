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


def integers(T, d, block, seed, dev):
    """Every code, and scales of 1 and 2 that differ from block to block and row to row."""
    rng = np.random.default_rng(seed)
    rec, n = ref.random_records(T, d, block, rng), d // block
    rec[:, d // 2: d // 2 + n] = (127 if block == 32 else 0x38) + rng.integers(0, 2, (T, n)) * (1 if block == 32 else 8)
    if block == 16:
        rec[:, d // 2 + n] = rng.integers(0, 3, T)
    return torch.from_numpy(rec).to(dev), torch.from_numpy(ref.decode(rec, d, block)).to(dev)


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("M,N,d", [(3, 200, 32), (20, 40, 96), (40, 50, 32768), (1, 130, 32736), (300, 300, 16416), (200, 520, 8224), (700, 72, 320)])
def test_every_channel_scale_and_lane_counts(env, M, N, d, block):
    """Products that binary32 holds exactly up to the longest rows, 32 channels behind the last 64 and none: one code, one scale or one
    lane that were left out would show."""
    rac, dev = env.rac, env.dev
    (A, a), (B, b) = integers(M, d, block, M + d, dev), integers(N, d, block, N + d + 1, dev)
    # multiples of 1/4 (row exponents multiply by 16 at most, which costs no digits): every partial sum is exact below 2^22
    assert float((a.abs() @ b.abs().T).max()) < 2.0 ** 22 * (16 if block == 16 else 1)
    Y = torch.empty((M, N), dtype=torch.float32, device=dev)
    rac.rac_mx_product(rac.MxCfg(d, block, y_type=torch.float32), A, M, B, N, Y, None)
    assert torch.equal(Y.double(), a @ b.T)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_products_of_the_smallest_and_largest_scales(env, M):
    """Sums of one sign with scales at their ends: what binary32 holds is exact, above it an infinity, below it 0; codes of 0 and sums
    that cancel within a block give 0 beside any scale."""
    rac, dev = env.rac, env.dev
    d, block = 64, 32
    ones, mixed, zeros = 0x22, 0xA2, 0x00
    scales = (0, 1, 60, 127, 200, 253, 254)
    Y = torch.empty((M, M), dtype=torch.float32, device=dev)
    cfg = rac.MxCfg(d, block, y_type=torch.float32)
    for codes in (ones, mixed, zeros):
        for sa in scales:
            for sb in scales:
                A, B = (np.zeros((M, ref.record_bytes(d, block)), dtype=np.uint8) for _ in range(2))
                A[:, :32], B[:, :32] = codes, ones
                A[:, 32:34], B[:, 32:34] = sa, sb
                rac.rac_mx_product(cfg, torch.from_numpy(A).to(dev), M, torch.from_numpy(B).to(dev), M, Y, None)
                want = torch.tensor(64 * 2.0 ** (sa + sb - 254) if codes == ones else 0.0, dtype=torch.float64).to(torch.float32)
                assert bool((Y == want.to(dev)).all()), (codes, sa, sb)
