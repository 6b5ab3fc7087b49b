"""Products of microscaled records where the order of copies, sums and stores matters: call after call, every value
(needs a B200)."""
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


def exact_operand(T, d, block, seed, dev):
    """Records with all scales 1: every partial sum is a multiple of 1/4 below 2^22 (36 d, d up to 32768), which binary32 holds in
    any order."""
    rec = ref.random_records(T, d, block, np.random.default_rng(seed))
    rec[:, d // 2: d // 2 + d // block] = 127 if block == 32 else 0x38
    if block == 16:
        rec[:, d // 2 + d // block] = 0
    return torch.from_numpy(rec).to(dev), torch.from_numpy(ref.decode(rec, d, block)).to(dev)


def product_of(a, b, yt):
    return (a @ b.T).to(torch.float32).to(yt)       # exact in binary32, then the one rounding


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("y", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,N,off", [
    (256 + 149, 10240, None), (256 + 20, 10240, None), (256 + 255, 20480, None),           # a pair's second tile is not full
    (768 + 149, 4736, None),                                                                 # the same with tiles of 256 x 128
    (5000, 2048, [0, 300, 700, 1001, 1500, 2300, 2333, 3700, 5000]),                         # tiles that are not full anywhere
])
def test_rows_that_end_inside_a_tile_leave_the_tile_before_alone(env, M, N, off, block, y):
    """A pair of CTAs goes from full tiles, which copies store, to others, which lanes store, through the same buffers; few channels,
    so that the next sums are there at once."""
    rac, dev = env.rac, env.dev
    d = 64
    n = 1 if off is None else len(off) - 1
    A, a = exact_operand(M, d, block, 1, dev)
    B, b = exact_operand(n * N, d, block, 2, dev)
    cfg = rac.MxCfg(d, block, y_type=y)
    if off is None:
        want = product_of(a, b, y)
    else:
        want = torch.cat([product_of(a[off[s]:off[s + 1]], b[s * N:(s + 1) * N], y) for s in range(n)])
        seg_off = torch.tensor(off, dtype=torch.int32, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    wrong = torch.zeros(1, dtype=torch.int64, device=dev)
    Y = torch.empty((M, N), dtype=y, device=dev)
    for _ in range(100):
        Y.fill_(-7)
        if off is None:
            rac.rac_mx_product(cfg, A, M, B, N, Y, status)
        else:
            rac.rac_mx_product_segments(cfg, A, M, seg_off, n, B, N, Y, status)
        wrong += (Y != want).sum()
    assert int(wrong) == 0 and int(status) == 0


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("M,N,d,n", [(64, 6000, 4096, 1), (33, 40000, 1280, 1), (2000, 1000, 1792, 40), (16, 40000, 1280, 1), (200, 1000, 1792, 40)])
def test_rings_of_three_and_four_stages_keep_in_step(env, M, N, d, n, block):
    """The narrow form, split over clusters and not, odd numbers of stages a tile, while other calls on another stream take turns on
    the same SMs."""
    rac, dev = env.rac, env.dev
    A, a = exact_operand(M, d, block, 3, dev)
    B, b = exact_operand(n * N, d, block, 4, dev)
    cfg = rac.MxCfg(d, block)
    off = [i * M // n for i in range(n + 1)]
    seg_off = torch.tensor(off, dtype=torch.int32, device=dev)
    want = torch.cat([product_of(a[off[s]:off[s + 1]], b[s * N:(s + 1) * N], torch.bfloat16) for s in range(n)])
    side = torch.cuda.Stream()
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    wrong = torch.zeros(1, dtype=torch.int64, device=dev)
    Y, Z = torch.empty_like(want), torch.empty_like(want)
    X = torch.ones((4000, d), dtype=torch.bfloat16, device=dev)
    pay = torch.empty((4000, rac.rac_mx_record_bytes(cfg)), dtype=torch.uint8, device=dev)
    torch.cuda.synchronize()

    def call(out, **k):
        if n == 1:
            rac.rac_mx_product(cfg, A, M, B, N, out, status, **k)
        else:
            rac.rac_mx_product_segments(cfg, A, M, seg_off, n, B, N, out, status, **k)
    for _ in range(60):
        for _ in range(3):
            call(Z, stream=side)
            rac.rac_mx_encode(cfg, X, 4000, pay, pay.numel(), None, None, stream=side)
        Y.fill_(-7)
        call(Y)
        wrong += (Y != want).sum()
    torch.cuda.synchronize()
    assert int(wrong) == 0 and int(status) == 0 and torch.equal(Z, want)


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("M,N,d", [(4096, 4096, 256), (4096, 4096, 4096), (3328, 1408, 512)])
def test_waits_that_cannot_complete_end_with_a_status_before_the_last_tile(env, M, N, d, block):
    """Pairs of CTAs with more tiles to go (256 x 256 and 256 x 128): their warps give up at different times."""
    rac, dev = env.rac, env.dev
    A, a = exact_operand(M, d, block, 1, dev)
    B, b = exact_operand(N, d, block, 2, dev)
    cfg = rac.MxCfg(d, block)
    Y = torch.empty((M, N), dtype=torch.bfloat16, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    rac.rac_mx_selftest_bounded_wait(cfg, A, M, B, N, Y, status)
    torch.cuda.synchronize()
    assert int(status) == rac.STATUS_TIMEOUT
    status.zero_()
    rac.rac_mx_product(cfg, A, M, B, N, Y, status)          # the device is as it was
    assert int(status) == 0 and torch.equal(Y, product_of(a, b, torch.bfloat16))


@pytest.mark.parametrize("block", [16, 32])
def test_short_products_back_to_back(env, block):
    """One tile a pair or cluster and the next call's CTAs behind it on the same SMs: what one still sends to its neighbour must not
    reach those.  Every result of a row of calls of all forms."""
    rac, dev = env.rac, env.dev
    d = 256
    cfg = rac.MxCfg(d, block)
    B, b = exact_operand(2304, d, block, 2, dev)
    ops = [exact_operand(m, d, block, m, dev) for m in (300, 5, 2048, 40, 512, 700)]
    want = [product_of(a, b, torch.bfloat16) for _, a in ops]
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    wrong = torch.zeros(1, dtype=torch.int64, device=dev)
    outs = [[torch.empty_like(w) for w in want] for _ in range(8)]
    for _ in range(20):
        for row in outs:
            for y in row:
                y.fill_(-7)
        for row in outs:
            for (A, _), y in zip(ops, row):
                rac.rac_mx_product(cfg, A, A.shape[0], B, 2304, y, status)
        for row in outs:
            for w, y in zip(want, row):
                wrong += (y != w).sum()
    assert int(wrong) == 0 and int(status) == 0


@pytest.mark.parametrize("M", [3, 64, 300])
def test_products_beside_other_kernels_that_use_tensor_memory(env, M):
    """A library's matrix products before, behind and beside these, captured and replayed: both want the SMs' tensor memory."""
    rac, dev = env.rac, env.dev
    cfg = rac.MxCfg(1280, 16)
    (A, a), (B, b) = exact_operand(M, 1280, 16, 1, dev), exact_operand(2000, 1280, 16, 2, dev)
    want = product_of(a, b, torch.bfloat16)
    U = torch.eye(2048, dtype=torch.bfloat16, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    outs = [torch.empty_like(want) for _ in range(6)]

    def run():
        V = U
        for y in outs:
            rac.rac_mx_product(cfg, A, M, B, 2000, y, status)
            V = V @ U
        return V
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        V = run()
    side = torch.cuda.Stream()
    for _ in range(30):
        for y in outs:
            y.fill_(-7)
        graph.replay()
        with torch.cuda.stream(side):
            U @ U
        torch.cuda.synchronize()
        assert all(torch.equal(y, want) for y in outs)
    assert int(status) == 0 and torch.equal(V, U)
