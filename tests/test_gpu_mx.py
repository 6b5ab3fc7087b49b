"""Microscaled records and their products against the 64-bit restatement (needs a B200)."""
import numpy as np
import pytest
import torch

import mx_reference as ref

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def env():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_04991_b200 import binding as rac
    rac.load()
    return type("Env", (), dict(rac=rac, dev=torch.device("cuda:0")))


def states(T, d, x, seed, dev):
    """Ordinary rows, and rows for the borders: middles between codes, zeros, the smallest and largest numbers."""
    gen = torch.Generator().manual_seed(seed)
    dt = TYPES[x]
    v = torch.randn((T, d), generator=gen) * torch.exp(torch.randn((1, d), generator=gen))
    v = v.to(dt)
    top = torch.finfo(dt).max
    rows = [
        lambda: torch.randint(-28, 29, (d,), generator=gen) * 0.25,                         # many exact middles
        lambda: torch.randint(-40, 41, (d,), generator=gen) * 0.25 * 2.0 ** -5 * 1.375,
        lambda: torch.zeros(d),
        lambda: -torch.zeros(d),
        lambda: torch.where(torch.arange(d) % 48 == 7, top, 1.0),
        lambda: torch.randn(d, generator=gen) * top / 8,
        lambda: torch.randint(-9, 10, (d,), generator=gen) * torch.finfo(dt).smallest_normal * torch.finfo(dt).eps,
        lambda: torch.exp(8 * torch.randn(d, generator=gen)),
        lambda: torch.where(torch.arange(d) == d - 1, 1.0, 0.0),
        lambda: torch.full((d,), 6.0) * 2.0 ** torch.randint(-6, 7, (d,), generator=gen).float(),
    ]
    for i in range(min(T - 1, 4 * len(rows))):
        v[i + 1] = rows[i % len(rows)]().clamp(-top, top).to(dt)
    return v.to(dev)


def typed(v, x):
    """float64 numpy -> the type of X, saturating (as decode does)."""
    top = torch.finfo(TYPES[x]).max
    return torch.from_numpy(np.clip(v, -top, top)).to(TYPES[x])       # float64 to a narrower type rounds once


def same_bits(a, b):
    return torch.equal(a.contiguous().cpu().view(torch.int16), b.contiguous().cpu().view(torch.int16))


ROWS = [(1, 32), (2, 64), (7, 96), (45, 32), (5, 544), (41, 2880), (3, 4096), (33, 5120), (129, 224), (2, 8192), (3, 16416), (2, 32768)]


@pytest.mark.parametrize("x", ["bf16", "fp16"])
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("T,d", ROWS)
def test_encode_writes_the_records_of_the_definition(env, T, d, block, x):
    rac, dev = env.rac, env.dev
    X = states(T, d, x, T * 7 + d, dev)
    cfg = rac.MxCfg(d, block, x_type=TYPES[x])
    rec = rac.rac_mx_record_bytes(cfg)
    want, bad = ref.encode(X.double().cpu().numpy(), block)
    assert not bad
    pay = torch.full((T * rec + 64,), 0xA5, dtype=torch.uint8, device=dev)
    xh = torch.full((T + 1, d), 7.0, dtype=TYPES[x], device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    rac.rac_mx_encode(cfg, X, T, pay, T * rec, xh, status)
    got = pay.cpu().numpy()
    assert np.array_equal(got[: T * rec].reshape(T, rec), want)
    assert (got[T * rec:] == 0xA5).all() and bool((xh[T] == 7).all()) and int(status) == 0
    values = typed(ref.decode(want, d, block), x)
    assert same_bits(xh[:T], values)
    # without x_hat the same records, and the receiver has the same values
    alone = torch.full_like(pay, 0x5A)
    rac.rac_mx_encode(cfg, X, T, alone, T * rec, None, None)
    assert torch.equal(alone[: T * rec], pay[: T * rec])
    out = torch.full_like(xh, 7.0)
    rac.rac_mx_decode(cfg, pay, T, out, status)
    assert same_bits(out[:T], values) and bool((out[T] == 7).all())
    # in place
    Y = X.clone()
    rac.rac_mx_encode(cfg, Y, T, alone, T * rec, Y, None)
    assert same_bits(Y, values) and torch.equal(alone[: T * rec], pay[: T * rec])


@pytest.mark.parametrize("x", ["bf16", "fp16"])
@pytest.mark.parametrize("block", [16, 32])
def test_every_number_of_the_type_has_the_code_of_the_definition(env, block, x):
    """All 63 thousand finite values, each as a block's largest and beside smaller ones."""
    rac, dev = env.rac, env.dev
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16)
    v = bits.view(TYPES[x])
    v = v[torch.isfinite(v)]
    gen = torch.Generator().manual_seed(1)
    d = 64
    X = v[:, None] * torch.rand((v.numel(), d), generator=gen).to(TYPES[x])
    X[:, 5] = v
    X[:, 37] = v
    cfg = rac.MxCfg(d, block, x_type=TYPES[x])
    want, _ = ref.encode(X.double().numpy(), block)
    pay = torch.zeros(want.shape, dtype=torch.uint8, device=dev)
    xh = torch.empty(X.shape, dtype=TYPES[x], device=dev)
    rac.rac_mx_encode(cfg, X.to(dev), X.shape[0], pay, pay.numel(), xh, None)
    assert np.array_equal(pay.cpu().numpy(), want)
    assert same_bits(xh, typed(ref.decode(want, d, block), x))


@pytest.mark.parametrize("x", ["bf16", "fp16"])
@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("d", [96, 4096])
def test_values_that_are_not_finite_stay_in_their_block(env, d, block, x):
    rac, dev = env.rac, env.dev
    X = states(30, d, x, 3, dev)
    clean = X.clone()
    for t, c, v in [(0, 0, float("nan")), (2, d - 1, float("inf")), (3, 17, -float("inf")), (5, 40, float("nan"))]:
        X[t, c] = v
        b = c // block
        clean[t, b * block:(b + 1) * block] = 0
    X[7] = float("nan")
    clean[7] = 0
    cfg = rac.MxCfg(d, block, x_type=TYPES[x])
    want, bad = ref.encode(X.double().cpu().numpy(), block)
    assert bad
    pay = torch.zeros(want.shape, dtype=torch.uint8, device=dev)
    xh = torch.empty_like(X)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    rac.rac_mx_encode(cfg, X, 30, pay, pay.numel(), xh, status)
    assert int(status) == rac.STATUS_NONFINITE
    assert np.array_equal(pay.cpu().numpy(), want)
    values = typed(ref.decode(want, d, block), x)
    nan = torch.isnan(values)
    assert torch.equal(torch.isnan(xh).cpu(), nan) and same_bits(torch.where(nan, 0, xh.cpu()), torch.where(nan, 0, values))
    assert same_bits(typed(ref.decode(ref.encode(clean.double().cpu().numpy(), block)[0], d, block), x)[~nan], values[~nan])
    out = torch.empty_like(X)
    rac.rac_mx_decode(cfg, pay, 30, out, status)
    assert torch.equal(torch.isnan(out).cpu(), nan) and same_bits(torch.where(nan, 0, out.cpu()), torch.where(nan, 0, values))
    # the row of a product is NaN, the others are finite
    Y = torch.empty((30, 30), dtype=torch.float32, device=dev)
    cfg32 = rac.MxCfg(d, block, x_type=TYPES[x], y_type=torch.float32)
    w = torch.from_numpy(ref.random_records(30, d, block, np.random.default_rng(1))).to(dev)
    ok = torch.tensor([t for t in range(30) if t not in (0, 2, 3, 5, 7)], device=dev)
    rac.rac_mx_product(cfg32, pay, 30, w, 30, Y, status)
    assert bool(torch.isnan(Y[[0, 2, 3, 5, 7]]).all())
    y = ref.decode(want, d, block)
    fit = np.abs(y).max(-1) < 1e30
    assert bool(torch.isfinite(Y[[int(t) for t in ok if fit[int(t)]]]).all())
    rac.rac_mx_product(cfg32, w, 30, pay, 30, Y, status)
    assert bool(torch.isnan(Y[:, [0, 2, 3, 5, 7]]).all())
    assert int(status) == rac.STATUS_NONFINITE                         # what encode left, nothing more


@pytest.mark.parametrize("x", ["bf16", "fp16"])
@pytest.mark.parametrize("block", [16, 32])
def test_decode_of_any_bytes(env, block, x):
    """Records that no encoder wrote: every scale byte and exponent."""
    rac, dev = env.rac, env.dev
    d = 32 * 24
    rng = np.random.default_rng(9)
    rec = rng.integers(0, 256, (256, ref.record_bytes(d, block)), dtype=np.uint8)
    rec[:, d // 2 + d // block] = np.arange(256)       # block 16: the exponent; block 32: padding
    cfg = rac.MxCfg(d, block, x_type=TYPES[x])
    out = torch.empty((256, d), dtype=TYPES[x], device=dev)
    rac.rac_mx_decode(cfg, torch.from_numpy(rec).to(dev), 256, out, None)
    values = typed(ref.decode(rec, d, block), x)
    nan = torch.isnan(values)
    assert torch.equal(torch.isnan(out).cpu(), nan) and same_bits(torch.where(nan, 0, out.cpu()), torch.where(nan, 0, values))


def check_product(Y, a, b, yt):
    """Y against the 64-bit product.  The sums are binary32 in some order: every one of at most d additions is off by no more
    than 2^-23 of the sum of magnitudes (one unit in the last place: the tensor cores may cut instead of rounding); then one
    rounding to the type of Y, half a unit, and half its smallest number below the normal ones."""
    want = a @ b.T
    size = a.abs() @ b.abs().T
    fi = torch.finfo(yt)
    tol = a.shape[1] * 2.0 ** -23 * size + (fi.eps / 2 * want.abs() if yt != torch.float32 else 2.0 ** -24 * want.abs()) + fi.smallest_normal * fi.eps / 2
    tol = tol * (1 + fi.eps)
    # what rounds beyond the largest finite value is an infinity: the border is that value and half a unit more
    border = fi.max * (1 + fi.eps / 4)
    inf = torch.isinf(Y)
    assert bool((want.abs()[inf] + tol[inf] >= border).all()) and torch.equal(torch.sign(Y[inf]).double(), torch.sign(want[inf]))
    assert bool((want.abs()[~inf] - tol[~inf] <= border).all())
    err = torch.where(inf, 0.0, (Y.double() - want).abs())
    assert bool((err <= tol).all()), f"{float((err / tol).max())} of the tolerance"


def operand(T, d, block, seed, dev):
    rec = ref.random_records(T, d, block, np.random.default_rng(seed))
    return torch.from_numpy(rec).to(dev), torch.from_numpy(ref.decode(rec, d, block)).to(dev)


SIZES = [(1, 1, 32), (1, 16, 64), (2, 7, 96), (3, 130, 160), (9, 64, 256), (16, 128, 288), (17, 129, 512), (33, 40, 544), (64, 257, 1024),
         (65, 384, 2880), (128, 128, 256), (129, 255, 992), (130, 1000, 4096), (257, 513, 1056), (1, 4096, 4096), (8, 2880, 2880),
         (700, 72, 320), (1000, 1, 640), (1, 5000, 8192), (300, 300, 16416), (40, 50, 32768), (2051, 640, 736)]


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("M,N,d", SIZES)
def test_product(env, M, N, d, block):
    rac, dev = env.rac, env.dev
    A, a = operand(M, d, block, M * 31 + d, dev)
    B, b = operand(N, d, block, N * 37 + d, dev)
    for y, yt in TYPES.items():
        cfg = rac.MxCfg(d, block, y_type=yt)
        Y = torch.full((M + 1, N), 77.0, dtype=yt, device=dev)
        status = torch.zeros(1, dtype=torch.int32, device=dev)
        rac.rac_mx_product(cfg, A, M, B, N, Y, status)
        assert int(status) == 0
        assert bool((Y[M] == 77).all())
        check_product(Y[:M], a, b, yt)
        again = torch.full_like(Y, 5.0)
        rac.rac_mx_product(cfg, A, M, B, N, again, None)
        assert torch.equal(again[:M], Y[:M])                          # the same on every run


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("M,N,d", [(5, 300, 4096), (200, 300, 4096), (64, 5000, 2880)])
def test_product_of_small_integers_is_exact(env, M, N, d, block):
    """Scales of 1 and 2: every partial sum is a multiple of 1/4 below 2^22 (d * 12 * 12), which binary32 holds in any order."""
    rac, dev = env.rac, env.dev
    A, _ = operand(M, d, block, 5, dev)
    B, _ = operand(N, d, block, 6, dev)
    one, n = (127, d // block) if block == 32 else (0x38, d // block)
    for R in (A, B):
        R[:, d // 2: d // 2 + n] = one + (torch.arange(n, device=dev) % 2) * (1 if block == 32 else 8)
        if block == 16:
            R[:, d // 2 + n] = 0
    a, b = (torch.from_numpy(ref.decode(R.cpu().numpy(), d, block)).to(dev) for R in (A, B))
    Y = torch.empty((M, N), dtype=torch.float32, device=dev)
    rac.rac_mx_product(rac.MxCfg(d, block, y_type=torch.float32), A, M, B, N, Y, None)
    assert torch.equal(Y.double(), a @ b.T)


def test_row_exponents_at_their_ends(env):
    """Exponents that a single factor of binary32 would not hold: they cancel between the operands."""
    rac, dev = env.rac, env.dev
    d, M, N = 160, 40, 33
    A, _ = operand(M, d, 16, 1, dev)
    B, _ = operand(N, d, 16, 2, dev)
    A[:, d // 2 + d // 16] = 110
    B[:, d // 2 + d // 16] = 256 - 100
    a, b = (torch.from_numpy(ref.decode(R.cpu().numpy(), d, 16)).to(dev) for R in (A, B))
    for p, q, u, v, m, n in ((A, B, a, b, M, N), (B, A, b, a, N, M)):
        Y = torch.empty((m, n), dtype=torch.float32, device=dev)
        rac.rac_mx_product(rac.MxCfg(d, 16, y_type=torch.float32), p, m, q, n, Y, None)
        check_product(Y, u, v, torch.float32)


SEGMENTS = [
    (200, 130, 288, [0, 200]), (200, 70, 160, [0, 0, 1, 1, 130, 200]), (200, 70, 160, [0, 64, 128, 192, 200]),
    (50, 33, 96, [7, 20, 20, 41]),                       # rows before and behind the segments
    (50, 33, 96, [-5, 20, 90, 100]), (50, 33, 96, [0, 30, 10, 40]),       # clipped; descending
    (7, 300, 512, [0, 1, 2, 3, 4, 5, 6, 7]), (3, 40, 64, [0, 0, 0, 3, 3]), (5, 40, 64, [2, 2]), (1, 513, 2880, [0, 0, 1]),
    (400, 200, 1056, [0, 129, 130, 386, 400]), (1500, 257, 544, [0, 3, 700, 701, 701, 1100, 1499]),
    (64, 2880, 2880, list(range(0, 65, 2))),
]


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("M,N,d,off", SEGMENTS)
def test_product_by_segments(env, M, N, d, off, block):
    rac, dev = env.rac, env.dev
    n = len(off) - 1
    A, a = operand(M, d, block, M + d, dev)
    B, b = operand(n * N, d, block, N + d, dev)
    seg_off = torch.tensor(off, dtype=torch.int32, device=dev)
    for y, yt in TYPES.items():
        Y = torch.full((M, N), 77.0, dtype=yt, device=dev)
        status = torch.zeros(1, dtype=torch.int32, device=dev)
        rac.rac_mx_product_segments(rac.MxCfg(d, block, y_type=yt), A, M, seg_off, n, B, N, Y, status)
        assert int(status) == 0
        inside = torch.zeros(M, dtype=torch.int32)
        for s in range(n):
            inside[max(off[s], 0):max(0, min(off[s + 1], M))] += 1
        assert bool((Y[(inside == 0).to(dev)] == 77).all())
        for s in range(n):
            rows = torch.arange(max(off[s], 0), max(max(off[s], 0), min(off[s + 1], M)))
            rows = rows[inside[rows] == 1].to(dev)
            if rows.numel():
                check_product(Y[rows], a[rows], b[s * N:(s + 1) * N], yt)


def test_many_segments(env):
    """More segments than a warp or a block of threads counts at once, most of them empty."""
    rac, dev = env.rac, env.dev
    n, N, d, M = 2500, 16, 64, 900
    gen = torch.Generator().manual_seed(4)
    off = torch.sort(torch.randint(0, M + 1, (n + 1,), generator=gen)).values
    off[0], off[-1] = 0, M
    off[100:1400] = off[100]
    A, a = operand(M, d, 16, 1, dev)
    B, b = operand(n * N, d, 16, 2, dev)
    Y = torch.empty((M, N), dtype=torch.float32, device=dev)
    rac.rac_mx_product_segments(rac.MxCfg(d, 16, y_type=torch.float32), A, M, off.to(torch.int32).to(dev), n, B, N, Y, None)
    of = torch.searchsorted(off, torch.arange(M), right=True) - 1
    want = torch.einsum("td,tnd->tn", a, b.view(n, N, d)[of.to(dev)])
    size = torch.einsum("td,tnd->tn", a.abs(), b.view(n, N, d)[of.to(dev)].abs())
    assert bool(((Y.double() - want).abs() <= (d + 1) * 2.0 ** -23 * size).all())


@pytest.mark.parametrize("M", [1, 70, 300])
@pytest.mark.parametrize("block", [16, 32])
def test_states_through_the_boundary_into_the_next_partition(env, M, block):
    """The calls as they are used together: on a stream of its own, captured once and replayed on new states."""
    rac, dev = env.rac, env.dev
    d, N, n = 2880, 500, 4
    cfg = rac.MxCfg(d, block)
    rec = rac.rac_mx_record_bytes(cfg)
    gen = torch.Generator().manual_seed(M)
    W = (torch.randn((n * N, d), generator=gen) / 54).to(torch.bfloat16).to(dev)
    wpay = torch.empty((n * N, rec), dtype=torch.uint8, device=dev)
    rac.rac_mx_encode(cfg, W, n * N, wpay, wpay.numel(), None, None)
    X = torch.zeros((M, d), dtype=torch.bfloat16, device=dev)
    xs, xr = torch.empty_like(X), torch.empty_like(X)
    pay = torch.empty((M, rec), dtype=torch.uint8, device=dev)
    Y, Z = (torch.empty((M, N), dtype=torch.bfloat16, device=dev) for _ in range(2))
    seg_off = torch.tensor([0, M // 3, M // 3, M // 2, M], dtype=torch.int32, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)

    def step():
        rac.rac_mx_encode(cfg, X, M, pay, pay.numel(), xs, status)
        rac.rac_mx_decode(cfg, pay, M, xr, status)
        rac.rac_mx_product(cfg, pay, M, wpay, N, Y, status)
        rac.rac_mx_product_segments(cfg, pay, M, seg_off, n, wpay, N, Z, status)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    w = torch.from_numpy(ref.decode(wpay.cpu().numpy(), d, block)).to(dev)
    for seed in (1, 2):
        X.copy_(states(M, d, "bf16", seed, dev).clamp(-1e4, 1e4))
        graph.replay()
        torch.cuda.synchronize()
        values = ref.decode(ref.encode(X.double().cpu().numpy(), block)[0], d, block)
        assert same_bits(xs, typed(values, "bf16")) and same_bits(xr, xs) and int(status) == 0
        a = torch.from_numpy(values).to(dev)
        check_product(Y, a, w[:N], torch.bfloat16)
        off = seg_off.tolist()
        for s in range(n):
            if off[s + 1] > off[s]:
                check_product(Z[off[s]:off[s + 1]], a[off[s]:off[s + 1]], w[s * N:(s + 1) * N], torch.bfloat16)


def test_two_products_at_once(env):
    """Two streams, operands shared: nothing is kept between calls that they could disturb."""
    rac, dev = env.rac, env.dev
    cfg = rac.MxCfg(4096, 16)
    B, _ = operand(2000, 4096, 16, 1, dev)
    ops = [operand(m, 4096, 16, m, dev)[0] for m in (3, 40, 500)]
    alone = []
    for R in ops:
        alone.append(torch.empty((R.shape[0], 2000), dtype=torch.bfloat16, device=dev))
        rac.rac_mx_product(cfg, R, R.shape[0], B, 2000, alone[-1], None)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ops]
    outs = [torch.empty_like(y) for y in alone]
    for _ in range(20):
        for st, R, y in zip(streams, ops, outs):
            rac.rac_mx_product(cfg, R, R.shape[0], B, 2000, y, None, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(alone, outs))


def test_offsets_beyond_32_bits(env):
    """Records, states and products whose bytes pass 2^32."""
    rac, dev = env.rac, env.dev
    d, T = 8192, 930000
    cfg = rac.MxCfg(d, 16)
    rec = rac.rac_mx_record_bytes(cfg)
    X = torch.zeros((T, d), dtype=torch.bfloat16, device=dev)
    pay = torch.empty((T, rec), dtype=torch.uint8, device=dev)
    assert pay.numel() > 1 << 32
    last = states(50, d, "bf16", 8, dev).clamp(-1e4, 1e4)
    X[-50:] = last
    rac.rac_mx_encode(cfg, X, T, pay, pay.numel(), X, None)
    want, _ = ref.encode(last.double().cpu().numpy(), 16)
    assert np.array_equal(pay[-50:].cpu().numpy(), want)
    assert same_bits(X[-50:], typed(ref.decode(want, d, 16), "bf16"))
    X[-50:] = 0
    rac.rac_mx_decode(cfg, pay, T, X, None)
    assert same_bits(X[-50:], typed(ref.decode(want, d, 16), "bf16"))
    del X
    B, b = operand(40, d, 16, 2, dev)
    Y = torch.empty((T, 40), dtype=torch.bfloat16, device=dev)
    rac.rac_mx_product(cfg, pay, T, B, 40, Y, None)
    a = torch.from_numpy(ref.decode(want, d, 16)).to(dev)
    check_product(Y[-50:], a, b, torch.bfloat16)
    assert bool((Y[:-50] == 0).all())
    # as weights: a segment far behind, and Y beyond 2^32 bytes
    seg_off = torch.tensor([0] * 23249 + [0, 40], dtype=torch.int32, device=dev)
    Z = torch.empty((40, 40), dtype=torch.bfloat16, device=dev)
    rac.rac_mx_product_segments(cfg, B, 40, seg_off, 23250, pay, 40, Z, None)
    check_product(Z, b, a[-40:], torch.bfloat16)
    del Y
    big = torch.empty((3000, T), dtype=torch.bfloat16, device=dev)
    assert big.numel() * 2 > 1 << 32
    C, c = operand(3000, d, 16, 5, dev)
    rac.rac_mx_product(cfg, C, 3000, pay, T, big, None)
    check_product(big[-30:, -50:], c[-30:], a, torch.bfloat16)


def test_binding_checks_types_and_devices(env):
    rac, dev = env.rac, env.dev
    cfg = rac.MxCfg(64, 16, x_type=torch.float16, y_type=torch.float32)
    pay = torch.zeros(64 * 2, dtype=torch.uint8, device=dev)
    h = torch.zeros((2, 64), dtype=torch.float16, device=dev)
    with pytest.raises(TypeError, match="X: expected torch.float16, got BFloat16"):
        rac.rac_mx_encode(cfg, h.to(torch.bfloat16), 2, pay, pay.numel(), None, None)
    with pytest.raises(TypeError, match="X_hat: expected torch.float16"):
        rac.rac_mx_decode(cfg, pay, 2, h.float(), None)
    with pytest.raises(TypeError, match="Y: expected torch.float32, got Half"):
        rac.rac_mx_product(cfg, pay, 2, pay, 2, h, None)
    with pytest.raises(ValueError, match="X: must be contiguous"):
        rac.rac_mx_encode(cfg, torch.zeros((64, 2), dtype=torch.float16, device=dev).t(), 2, pay, pay.numel(), None, None)
    rac.rac_mx_encode(cfg, h, 0, pay, 0, None, None)
    rac.rac_mx_product(cfg, pay, 2, pay, 0, torch.empty((2, 0), dtype=torch.float32, device=dev), None)


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("M,N", [(1, 40), (30, 1000), (100, 130), (700, 300)])
def test_waits_that_cannot_complete_end_with_a_status(env, M, N, block):
    rac, dev = env.rac, env.dev
    d = 4096
    A, a = operand(M, d, block, 1, dev)
    B, b = operand(N, d, block, 2, dev)
    cfg = rac.MxCfg(d, block)
    Y = torch.empty((M, N), dtype=torch.bfloat16, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    rac.rac_mx_selftest_bounded_wait(cfg, A, M, B, N, Y, status)
    torch.cuda.synchronize()
    assert int(status) == rac.STATUS_TIMEOUT
    status.zero_()
    rac.rac_mx_product(cfg, A, M, B, N, Y, status)          # the device is as it was
    assert int(status) == 0
    check_product(Y, a, b, torch.bfloat16)


@pytest.mark.parametrize("M,N,d,n", [(4000, 2048, 1280, 8), (2600, 700, 768, 40), (1500, 3000, 1280, 1), (3000, 5000, 256, 1), (60, 5000, 1792, 16),
                                     (5000, 1000, 2304, 3)])
@pytest.mark.parametrize("block", [16, 32])
def test_calls_in_a_row_agree(env, M, N, d, n, block):
    """Many tiles per CTA, odd and even numbers of stages, call after call: the same sums every time and no wait that runs out."""
    rac, dev = env.rac, env.dev
    A, a = operand(M, d, block, 3, dev)
    B, b = operand(n * N, d, block, 4, dev)
    cfg = rac.MxCfg(d, block)
    off = [i * M // n for i in range(n + 1)]
    seg_off = torch.tensor(off, dtype=torch.int32, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    Ys = [torch.empty((M, N), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    for i in range(60):
        Y = Ys[min(i, 1)]
        if n == 1:
            rac.rac_mx_product(cfg, A, M, B, N, Y, status)
        else:
            rac.rac_mx_product_segments(cfg, A, M, seg_off, n, B, N, Y, status)
        if i == 0:
            for s in range(n):
                check_product(Y[off[s]:off[s + 1]], a[off[s]:off[s + 1]], b[s * N:(s + 1) * N], torch.bfloat16)
        else:
            assert torch.equal(Ys[0], Ys[1])
    assert int(status) == 0


def test_receiver_enters_the_next_partition(env):
    """The link's path: reconstruct what crossed, code it, first projection behind the boundary."""
    from paper_2608_04991_b200 import link, synth
    rac, dev = env.rac, env.dev
    d, T, N = 1024, 200, 300
    cfg = rac.CodecCfg(d, 128, 4, 0, scale_mode=1, topk_group=1)
    a, b = link.Loopback.pair()
    sender, receiver = link.Sender(link.DeviceCodec(cfg, dev, 2 * T), a), link.Receiver(link.DeviceCodec(cfg, dev, 2 * T, with_index=False), b)
    gen = synth.generator(5, dev)
    W = (torch.randn((N, d), generator=gen, device=dev) / 32).to(torch.bfloat16)
    for block in (16, 32):
        entry = link.EntryProduct(W, block)
        with pytest.raises(RuntimeError, match="no request in flight"):
            receiver.enter(entry)
        X = synth.activations(T, d, synth.channel_scale(d, 5, dev), gen)
        sender.uplink(torch.arange(T, dtype=torch.int32, device=dev), X)
        x_hat = receiver.uplink()
        Y = receiver.enter(entry)
        entry.check()
        values = [torch.from_numpy(ref.decode(ref.encode(v.double().cpu().numpy(), block)[0], d, block)).to(dev) for v in (x_hat, W)]
        check_product(Y, values[0], values[1], torch.bfloat16)
        sender.finish_without_downlink()
        receiver.finish_without_downlink()


@pytest.mark.parametrize("x", ["bf16"])
def test_sweep_reports_the_direct_records(env, x):
    from paper_2608_04991_b200 import sweep, synth
    dev = env.dev
    T, d = 300, 1024
    X = synth.activations(T, d, synth.channel_scale(d, 6, dev), synth.generator(6, dev))
    rows = sweep.sweep_direct(X)
    v = X.double().cpu().numpy()
    for block, r in zip((16, 32), rows):
        e = typed(ref.decode(ref.encode(v, block)[0], d, block), x).double().numpy() - v
        assert r["status"] == 0 and r["record_bytes"] == ref.record_bytes(d, block) and r["qgroup"] == block
        assert abs(r["rel_rms_error"] - np.sqrt((e ** 2).sum() / (v ** 2).sum())) < 1e-9 and r["max_abs_error"] == np.abs(e).max()
    assert rows[0]["rel_rms_error"] < rows[1]["rel_rms_error"]          # smaller blocks, finer scales


@pytest.mark.parametrize("M,N,d", [(300, 300, 160), (2000, 131, 992)])
def test_row_exponents_at_their_ends_in_large_products(env, M, N, d):
    """The large tiles apply the exponents apart from one another where a single factor would not hold them."""
    rac, dev = env.rac, env.dev
    A, _ = operand(M, d, 16, 1, dev)
    B, _ = operand(N, d, 16, 2, dev)
    A[:, d // 2 + d // 16] = 110
    B[:, d // 2 + d // 16] = 256 - 100
    A[5:9, d // 2 + d // 16] = 256 - 20
    a, b = (torch.from_numpy(ref.decode(R.cpu().numpy(), d, 16)).to(dev) for R in (A, B))
    for p, q, u, v, m, n in ((A, B, a, b, M, N), (B, A, b, a, N, M)):
        Y = torch.empty((m, n), dtype=torch.float32, device=dev)
        rac.rac_mx_product(rac.MxCfg(d, 16, y_type=torch.float32), p, m, q, n, Y, None)
        check_product(Y, u, v, torch.float32)


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("M,N,d,off", [(40, 100, 1024, [0, 40, 0, 40, 0, 40]), (200, 100, 1536, [0, 200, 0, 200, 0, 200, 0, 200]),
                                       (900, 300, 512, [0, 900, 0, 900])])
def test_segments_that_overlap_and_share_a_matrix(env, M, N, d, off, block):
    """More tiles than the sizes promise, in the form that splits the channels over clusters too."""
    rac, dev = env.rac, env.dev
    n = len(off) - 1
    A, a = operand(M, d, block, 1, dev)
    B, b = operand(N, d, block, 2, dev)
    Y = torch.full((M, N), 77.0, dtype=torch.bfloat16, device=dev)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    for _ in range(5):
        rac.rac_mx_product_segments(rac.MxCfg(d, block), A, M, torch.tensor(off, dtype=torch.int32, device=dev), n, B.repeat(n, 1), N, Y, status)
        check_product(Y, a, b, torch.bfloat16)
        Y.fill_(77)
    assert int(status) == 0


@pytest.mark.parametrize("block", [16, 32])
@pytest.mark.parametrize("T,d", [(5, 96), (70, 2880), (400, 544)])
def test_buffers_that_start_at_16_bytes_only(env, T, d, block):
    """Every pointer a multiple of 16 bytes and of no more."""
    rac, dev = env.rac, env.dev
    cfg = rac.MxCfg(d, block)
    rec = rac.rac_mx_record_bytes(cfg)

    def at16(shape, dtype):
        n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
        raw = torch.zeros(n + 64, dtype=torch.uint8, device=dev)
        skip = (16 - raw.data_ptr()) % 32
        v = raw[skip: skip + n].view(dtype).view(shape)
        assert v.data_ptr() % 32 == 16
        return v
    X, xh, out, pay = at16((T, d), torch.bfloat16), at16((T, d), torch.bfloat16), at16((T, d), torch.bfloat16), at16((T, rec), torch.uint8)
    X.copy_(states(T, d, "bf16", 1, dev).clamp(-1e4, 1e4))
    rac.rac_mx_encode(cfg, X, T, pay, pay.numel(), xh, None)
    want, _ = ref.encode(X.double().cpu().numpy(), block)
    values = ref.decode(want, d, block)
    assert np.array_equal(pay.cpu().numpy(), want) and same_bits(xh, typed(values, "bf16"))
    rac.rac_mx_decode(cfg, pay, T, out, None)
    assert same_bits(out, xh)
    a = torch.from_numpy(values).to(dev)
    for N in (T, T // 2):
        Y = at16((T, N), torch.bfloat16)
        rac.rac_mx_product(cfg, pay, T, pay, N, Y, None)
        check_product(Y, a, a[:N], torch.bfloat16)


def test_a_long_encode_in_place_and_odd_counts(env):
    """CTAs that go through several rows: the last ones of a count that no split divides, in place."""
    rac, dev = env.rac, env.dev
    for T, d, block in ((20011, 1056, 16), (20011, 1056, 32), (9001, 4128, 16), (4999, 16416, 16), (200003, 96, 16)):
        X = torch.randn((T, d), generator=torch.Generator(device=dev).manual_seed(T), device=dev).to(torch.bfloat16)
        cfg = rac.MxCfg(d, block)
        pay = torch.empty((T, rac.rac_mx_record_bytes(cfg)), dtype=torch.uint8, device=dev)
        Y = X.clone()
        rac.rac_mx_encode(cfg, Y, T, pay, pay.numel(), Y, None)
        pick = torch.cat((torch.arange(0, 40), torch.arange(T // 2, T // 2 + 40), torch.arange(T - 80, T))).to(dev)
        want, _ = ref.encode(X[pick].double().cpu().numpy(), block)
        assert np.array_equal(pay[pick].cpu().numpy(), want)
        out = torch.empty_like(X)
        rac.rac_mx_decode(cfg, pay, T, out, None)
        assert same_bits(out, Y)
        few = torch.empty_like(pay)                     # the same records from calls of other sizes
        for t in range(0, T, 4096):
            n = min(4096, T - t)
            rac.rac_mx_encode(cfg, X[t:t + n], n, few[t:t + n], n * few.shape[1], None, None)
        assert torch.equal(few, pay)
