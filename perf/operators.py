"""Microscaled 4-bit floating point as its users run it, for timing and for comparing results.

A row of ``d`` values travels as one record: e2m1 codes (two per byte, the even channel in the low half), one scale byte
per block, and, for blocks of 16, one exponent per row.  Blocks of 32 carry a power of two (e8m0), blocks of 16 an e4m3
scale times 2 to the row's exponent.  A case is a dict of plain values; ``kind`` says which calls one pass makes:

* ``encode``    states to records with the sender's own reconstruction in the same pass; returns the reconstruction.
* ``decode``    records to states.
* ``link``      encode without the sender's reconstruction and decode at the other end; returns what the receiver has.
* ``product``   records of ``T`` rows times records of an ``[N, d]`` weight matrix, transposed.
* ``entry``     encode of fresh states and the product with the first weight matrix behind the boundary.
* ``segments``  rows in segments, each with a weight matrix of its own (adapters, experts); some segments are empty.

``x`` and ``y`` are the types of the states and of the product.  Sizes are those of the tests and of the benchmark, or
generic.
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
_CHUNK = 1 << 26      # values at a time where inputs and 64-bit results are made


def _case(kind, T, d, block, N=0, segments=0, empty=0, x="bf16", y="bf16"):
    return {"kind": kind, "T": T, "d": d, "block": block, "N": N, "segments": segments, "empty": empty, "x": x, "y": y}


def listed():
    def named(name, *a, **k):
        return {"name": name, **_case(*a, **k)}
    return [
        # the first decode step of one conversation, which has no reference yet: the smallest call
        named("encode_1x4096_b32", "encode", 1, 4096, 32),
        # the same for 64 conversations at the receiving end
        named("decode_64x5120_b16", "decode", 64, 5120, 16),
        # a prompt of odd length in binary16
        named("encode_2051x4096_b16_fp16", "encode", 2051, 4096, 16, x="fp16"),
        # an ordinary batch of prompts, both ends
        named("link_16384x4096_b32", "link", 16384, 4096, 32),
        # long context: the sender with its own reconstruction, and the receiver
        named("encode_131072x5120_b16", "encode", 131072, 5120, 16),
        named("decode_131072x5120_b16", "decode", 131072, 5120, 16),
        # one conversation's token through a square projection: the weights are all there is to read
        named("product_1x4096x4096_b16", "product", 1, 4096, 16, N=4096),
        # 64 conversations: states arrive, are coded and enter the next partition
        named("entry_64x5120x5120_b16", "entry", 64, 5120, 16, N=5120),
        # a prompt through a projection of odd width
        named("product_2051x4096x2887_b32", "product", 2051, 4096, 32, N=2887),
        # a long prompt: the largest product
        named("product_16384x5120x5120_b16", "product", 16384, 5120, 16, N=5120),
        # a decode step spread over 32 experts, a few tokens each
        named("segments_128x2880x2880_b32", "segments", 128, 2880, 32, N=2880, segments=32, empty=6),
        # a prompt's tokens sorted by expert
        named("segments_8192x4096x2048_b16", "segments", 8192, 4096, 16, N=2048, segments=16, empty=2),
    ]


def draw(rng):
    def size(lo, hi):
        return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    kind = rng.choice(["encode", "decode", "link", "product", "entry", "segments"])
    block = rng.choice([16, 32])
    d = 32 * size(2, 256)
    x, y = rng.choice(["bf16", "bf16", "fp16"]), rng.choice(["bf16", "bf16", "fp16"])
    if kind in ("encode", "decode", "link"):
        return _case(kind, size(1, min(131072, 131072 * 5120 // d)), d, block, x=x)
    if kind != "segments":
        return _case(kind, size(1, 16384), d, block, N=size(16, min(5120, 5120 * 5120 // d)), x=x, y=y)
    n = size(1, 64)
    return _case(kind, size(1, 8192), d, block, N=size(16, min(4096, (1 << 28) // (n * d))), segments=n, empty=rng.randrange(0, n), x=x, y=y)


def _record(d, block):
    return -(-(d // 2 + d // block + (block == 16)) // 32) * 32


# ------------------------------------------------------------------------------------------ the operators, plainly
_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
# a value has code i where i borders are below it; where two codes are equally near the one of even index has the border,
# so the border below such a code is the binary32 number before the middle
_BORDERS = [0.25, 0.75 - 2.0 ** -24, 1.25, 1.75 - 2.0 ** -23, 2.5, 3.5 - 2.0 ** -22, 5.0]


def _power(k):
    """2 to the k, k an integer tensor within -149..127, without rounding."""
    return torch.tensor([2.0 ** i for i in range(-149, 128)], device=k.device)[k.int() + 149]


def _e4m3_values(device):
    """The 127 finite e4m3 values that are not negative, ascending: value i has byte i."""
    b = torch.arange(127, device=device)
    e, m = b >> 3, (b & 7).float()
    return torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2(e.float() - 7))


def _plain_scales(x, block, values):
    """Scale byte of every block, the scale itself, and the exponent of every row, of x [T, d] in binary32."""
    T, d = x.shape
    a = x.abs().view(T, d // block, block)
    fine = torch.isfinite(a).all(-1)
    amax = torch.where(fine, a.amax(-1), 0.0)
    if block == 32:
        m, e = torch.frexp(amax)
        k = torch.where(amax > 0, (e - 3 + (m > 0.75).int()).clamp(min=-127), -127)
        byte = torch.where(fine, k + 127, 255)
        s = _power(k)
        return byte.to(torch.uint8), torch.where(fine, s, float("nan")), None
    top = amax.amax(-1)
    m, e = torch.frexp(top)
    r = torch.where(top > 0, (e - 12 + (m > 0.65625).int()).clamp(min=-100), 0)
    byte = torch.searchsorted(6 * values, amax * _power(-r)[:, None])
    s = values[byte.clamp(max=126)] * _power(r)[:, None]
    return torch.where(fine, byte, 127).to(torch.uint8), torch.where(fine, s, float("nan")), r.to(torch.int8)


def _plain_codes(x, s, block, r):
    """Code 0..15 of every value of x [T, d] under the scales s [T, d / block]."""
    T, d = x.shape
    if r is not None:     # both divided by 2 to the row's exponent: no small scale is lost to underflow
        p = _power(-r.int())[:, None]
        x, s = x * p, s * p
    y = x.view(T, d // block, block) / torch.where(s > 0, s, 1.0)[..., None]
    y = torch.where(torch.isfinite(y), y, 0.0).view(T, d)
    c = torch.bucketize(y.abs(), torch.tensor(_BORDERS, device=x.device), out_int32=True)
    return (c + 8 * torch.signbit(y)).to(torch.uint8)


def _plain_encode(x, block):
    """Records of x [T, d]: codes, scales, exponent."""
    T, d = x.shape
    x = x.float()
    byte, s, r = _plain_scales(x, block, _e4m3_values(x.device))
    c = _plain_codes(x, s, block, r)
    out = torch.zeros((T, _record(d, block)), dtype=torch.uint8, device=x.device)
    out[:, : d // 2] = c[:, 0::2] | c[:, 1::2] << 4
    out[:, d // 2: d // 2 + d // block] = byte
    if r is not None:
        out[:, d // 2 + d // block] = r.view(torch.uint8)
    return out


def _plain_decode(rec, d, block):
    """Values [T, d] of records, in binary32."""
    T = rec.shape[0]
    table = torch.tensor(_E2M1 + [-v for v in _E2M1], device=rec.device)
    codes = rec[:, : d // 2].int()
    v = torch.stack((table[codes & 15], table[codes >> 4]), -1).view(T, d // block, block)
    byte = rec[:, d // 2: d // 2 + d // block].int()
    nan = torch.tensor(float("nan"), device=rec.device)
    if block == 32:
        s = torch.where(byte == 255, nan, _power((byte - 127).clamp(max=127)))
    else:
        s = torch.cat((_e4m3_values(rec.device), nan[None]))[byte & 127]
        s = s * _power(rec[:, d // 2 + d // block].view(torch.int8))[:, None]
    return (v * s[..., None]).view(T, d)


def _plain_round(v, dtype):
    top = torch.finfo(dtype).max
    return v.clamp(-top, top).to(dtype)


def _plain_product(a, b, d, block, dtype):
    return (_plain_decode(a, d, block) @ _plain_decode(b, d, block).t()).to(dtype)


def _plain_segments(a, b, seg_off, d, block, dtype):
    off = seg_off.tolist()
    return torch.cat([_plain_product(a[i:j], w, d, block, dtype) for i, j, w in zip(off, off[1:], b) if j > i])


# ------------------------------------------------------------------------------------------ inputs
def _states(T, d, gen, dtype, device):
    """Hidden states: heavy-tailed channels, a few of them twenty times as large, tokens of different sizes."""
    scale = torch.exp(0.5 * torch.randn(d, generator=gen, device=device))
    scale[torch.randperm(d, generator=gen, device=device)[: max(1, d // 256)]] *= 20
    x = torch.randn((T, d), generator=gen, device=device, dtype=torch.float32)
    x *= scale
    x *= torch.exp(0.3 * torch.randn((T, 1), generator=gen, device=device))
    return x.to(dtype)


def _coded(T, d, block, gen, make):
    """Records of T rows, made a piece at a time (the plain form wants a dozen copies of its input)."""
    step = max(1, _CHUNK // d)
    return torch.cat([_plain_encode(make(min(step, T - t), gen), block) for t in range(0, T, step)])


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=dev).manual_seed(seed * 1000003 + 17)
    kind, T, d, block, N = case["kind"], case["T"], case["d"], case["block"], case["N"]
    st = {"case": dict(case)}
    xt, yt = _TYPES[case["x"]], _TYPES[case["y"]]

    def states(t, g):
        return _states(t, d, g, xt, dev)

    def weights(n, g):
        return (torch.randn((n, d), generator=g, device=dev) * d ** -0.5).to(torch.bfloat16)
    if kind in ("encode", "link", "entry"):
        st["X"] = states(T, gen)
        st["records"] = torch.zeros((T, _record(d, block)), dtype=torch.uint8, device=dev)
    else:
        st["records"] = _coded(T, d, block, gen, states)
    if kind in ("encode", "decode", "link"):
        st["X_hat"] = torch.empty((T, d), dtype=xt, device=dev)
    if N:
        n = max(1, case["segments"])
        st["W"] = _coded(n * N, d, block, gen, weights)
        st["Y"] = torch.empty((T, N), dtype=yt, device=dev)
    if kind == "segments":
        # lengths as a router gives them: uneven, some none
        share = torch.rand(n, generator=gen, device=dev).double() ** 2 + 0.02
        share[torch.randperm(n, generator=gen, device=dev)[: case["empty"]]] = 0
        off = torch.round(torch.cumsum(share, 0) / share.sum() * T).to(torch.int32)
        off[-1] = T
        st["seg_off"] = torch.cat((torch.zeros(1, dtype=torch.int32, device=dev), off))
    st["status"] = torch.zeros(1, dtype=torch.int32, device=dev)
    return st


# ------------------------------------------------------------------------------------------ one pass
def _run_plain(st, case):
    kind, d, block = case["kind"], case["d"], case["block"]
    xt, yt = _TYPES[case["x"]], _TYPES[case["y"]]
    if kind in ("encode", "link"):
        return _plain_round(_plain_decode(_plain_encode(st["X"], block), d, block), xt)
    if kind == "decode":
        return _plain_round(_plain_decode(st["records"], d, block), xt)
    if kind == "product":
        return _plain_product(st["records"], st["W"], d, block, yt)
    if kind == "entry":
        return _plain_product(_plain_encode(st["X"], block), st["W"], d, block, yt)
    return _plain_segments(st["records"], st["W"].view(case["segments"], case["N"], -1), st["seg_off"], d, block, yt)


def _run_own(st, case):
    from paper_2608_04991_b200 import binding as rac
    kind, T, N = case["kind"], case["T"], case["N"]
    if "cfg" not in st:      # a program holds its configuration
        st["cfg"] = rac.MxCfg(case["d"], case["block"], x_type=_TYPES[case["x"]], y_type=_TYPES[case["y"]])
    cfg = st["cfg"]
    rec, status = st["records"], st["status"]
    if kind == "encode":
        rac.rac_mx_encode(cfg, st["X"], T, rec, rec.numel(), st["X_hat"], status)
        return st["X_hat"]
    if kind == "link":
        rac.rac_mx_encode(cfg, st["X"], T, rec, rec.numel(), None, status)
        rac.rac_mx_decode(cfg, rec, T, st["X_hat"], status)
        return st["X_hat"]
    if kind == "decode":
        rac.rac_mx_decode(cfg, rec, T, st["X_hat"], status)
        return st["X_hat"]
    if kind == "segments":
        rac.rac_mx_product_segments(cfg, rec, T, st["seg_off"], case["segments"], st["W"], N, st["Y"], status)
        return st["Y"]
    if kind == "entry":
        rac.rac_mx_encode(cfg, st["X"], T, rec, rec.numel(), None, status)
    rac.rac_mx_product(cfg, rec, T, st["W"], N, st["Y"], status)
    return st["Y"]


def run(state):
    return _run_own(state, state["case"]) if own else _run_plain(state, state["case"])


def work(case):
    kind, T, d, block, N = case["kind"], case["T"], case["d"], case["block"], case["N"]
    rec = _record(d, block)
    if kind == "encode":
        return {"bytes": T * (4 * d + rec), "flops": 2 * T * d}
    if kind == "decode":
        return {"bytes": T * (2 * d + rec), "flops": T * d}
    if kind == "link":
        return {"bytes": T * (4 * d + 2 * rec), "flops": 3 * T * d}
    # of a segmented product only the matrices whose segments hold rows are needed
    n = max(1, min(case["segments"] - case["empty"], T)) if kind == "segments" else 1
    states = T * (2 * d + rec) if kind == "entry" else 0
    return {"bytes": states + (T + n * N) * rec + 2 * T * N, "flops": 2 * T * N * d}


# ------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_numbers(device):
    code = torch.tensor([0, 1, 2, 3, 4, 6, 8, 12], dtype=torch.float64, device=device) / 2
    e4m3 = [(m / 512 if e == 0 else (8 + m) / 8 * 2.0 ** (e - 7)) for e in range(16) for m in range(8)][:127]
    return code, torch.tensor(e4m3, dtype=torch.float64, device=device)


def _exact_power_above(v, unit, lowest):
    """The smallest power of two p, 2 to the `lowest` at least, with unit * p >= v."""
    p = torch.tensor([2.0 ** i for i in range(lowest, 130)], dtype=torch.float64, device=v.device)
    return p[torch.searchsorted(unit * p, v).clamp(max=p.numel() - 1)]


def _exact_quantised(x, block):
    """Values of x [T, d] after the microscaled quantisation: the nearest code to x / scale by distance, the one with an
    even index of two that are equally near."""
    T, d = x.shape
    code, e4m3 = _exact_numbers(x.device)
    x = x.double().view(T, d // block, block)
    amax = x.abs().amax(-1)
    if block == 32:
        s = _exact_power_above(amax, 6, -127)
    else:
        top = amax.amax(-1, keepdim=True)
        p = torch.where(top > 0, _exact_power_above(top, 2688, -100), 1.0)
        s = e4m3[torch.searchsorted(6 * e4m3, amax / p)] * p
    y = x.abs() / torch.where(s > 0, s, 1.0)[..., None]
    even_first = torch.tensor([0, 2, 4, 6, 1, 3, 5, 7], device=x.device)
    near = (y[..., None] - code[even_first]).abs().argmin(-1)      # the first of equals
    return (torch.copysign(code[even_first][near], x) * s[..., None]).view(T, d)


def _exact_values(rec, d, block):
    """Values of records, in 64 bits."""
    code, e4m3 = _exact_numbers(rec.device)
    T = rec.shape[0]
    pair = rec[:, : d // 2].long()
    nib = torch.stack((pair % 16, pair // 16), 2).view(T, d)
    v = torch.where(nib >= 8, -code[nib % 8], code[nib % 8]).view(T, d // block, block)
    scale = rec[:, d // 2: d // 2 + d // block].long()
    if block == 32:
        s = torch.exp2(scale.double() - 127)
    else:
        r = rec[:, d // 2 + d // block].long()
        s = e4m3[scale] * torch.exp2((r - 256 * (r >= 128)).double())[:, None]
    return (v * s[..., None]).view(T, d)


def exact(case, seed):
    st = prepare(case, seed)
    kind, T, d, block = case["kind"], case["T"], case["d"], case["block"]
    step = max(1, (_CHUNK // 4) // d)      # the distances to all codes are eight times as many

    def by_piece(f, n):
        return torch.cat([f(slice(i, min(n, i + step))) for i in range(0, n, step)])
    if kind in ("encode", "link"):
        return by_piece(lambda t: _exact_quantised(st["X"][t], block), T)
    if kind == "decode":
        return by_piece(lambda t: _exact_values(st["records"][t], d, block), T)
    if kind == "entry":
        a = by_piece(lambda t: _exact_quantised(st["X"][t], block), T)
    else:
        a = by_piece(lambda t: _exact_values(st["records"][t], d, block), T)
    if kind != "segments":
        return a @ _exact_values(st["W"], d, block).t()
    off = st["seg_off"].tolist()
    w = st["W"].view(case["segments"], case["N"], -1)
    return torch.cat([a[off[s]: off[s + 1]] @ _exact_values(w[s], d, block).t() for s in range(case["segments"])])
