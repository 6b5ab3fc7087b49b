"""Microscaled records without a GPU: geometry, refusals, marshalling, and the tests' own reference."""
import ctypes as C

import numpy as np
import pytest
import torch

import mx_reference as ref

A = 0x10000      # a 16-byte aligned fake address: never dereferenced, the call is refused first
FAR = 1 << 40    # another one, far from it


@pytest.fixture(scope="module")
def rac():
    from paper_2608_04991_b200 import build, binding
    build.build()
    binding.load()
    return binding


@pytest.mark.parametrize("d,block,want", [(32, 16, 32), (32, 32, 32), (64, 16, 64), (4096, 16, 2336), (4096, 32, 2176),
                                          (5120, 16, 2912), (5120, 32, 2720), (2880, 32, 1536), (32768, 16, 18464)])
def test_record_geometry(rac, d, block, want):
    cfg = rac.MxCfg(d, block)
    assert rac.rac_mx_record_bytes(cfg) == want == ref.record_bytes(d, block)
    assert rac.rac_mx_payload_bytes(cfg, 1000) == 1000 * want and rac.rac_mx_payload_bytes(cfg, -1) == 0


def raw(rac, d=4096, block=16, x=0, y=0, flags=0):
    cfg = rac.MxCfg(32)
    cfg.d, cfg.block, cfg.x_type, cfg.y_type, cfg.flags = d, block, x, y, flags
    return cfg


def test_configurations_that_are_refused(rac):
    lib = rac.load()
    for cfg, code in [(raw(rac, d=0), -1), (raw(rac, d=-32), -1), (raw(rac, d=48), -4), (raw(rac, d=32800), -4), (raw(rac, block=8), -4),
                      (raw(rac, block=64), -4), (raw(rac, x=2), -4), (raw(rac, x=-1), -4), (raw(rac, y=3), -4), (raw(rac, flags=1), -4)]:
        assert rac.rac_mx_record_bytes(cfg) == 0 and rac.rac_mx_payload_bytes(cfg, 5) == 0
        c = C.byref(cfg)
        assert lib.rac_mx_encode(c, A, 1, FAR, 1 << 20, None, None, 0) == code
        assert lib.rac_mx_decode(c, A, 1, FAR, None, 0) == code
        assert lib.rac_mx_product(c, A, 1, A, 1, FAR, None, 0) == code
        assert lib.rac_mx_product_segments(c, A, 1, A, 1, A, 1, FAR, None, 0) == code
    assert lib.rac_mx_encode(None, A, 1, FAR, 1 << 20, None, None, 0) == -1
    with pytest.raises(TypeError):
        rac.MxCfg(4096, 16, x_type=torch.float64)
    assert C.sizeof(rac.MxCfg) == 20


def test_arguments_that_are_refused(rac):
    lib = rac.load()
    cfg = rac.MxCfg(4096, 16)
    rec = rac.rac_mx_record_bytes(cfg)

    def enc(X=A, T=4, pay=FAR, cap=4 * rec, xh=None):
        return lib.rac_mx_encode(C.byref(cfg), X, T, pay, cap, xh, None, 0)
    assert enc(X=None) == -1 and enc(pay=None) == -1 and enc(T=-1) == -1 and enc(T=1 << 31, cap=1 << 60) == -4
    assert enc(X=A + 8) == -2 and enc(pay=FAR + 4) == -2 and enc(xh=A + (1 << 30) + 2) == -2
    assert enc(cap=4 * rec - 1) == -3
    assert enc(pay=A) == -1 and enc(pay=A + 16) == -1                                # payload over X
    assert enc(xh=A + 16) == -1 and enc(xh=FAR) == -1                                # x_hat half over X, over the payload
    assert enc(T=0, X=None, pay=None, cap=0) == 0

    def dec(pay=A, T=4, xh=FAR):
        return lib.rac_mx_decode(C.byref(cfg), pay, T, xh, None, 0)
    assert dec(pay=None) == -1 and dec(xh=None) == -1 and dec(T=-1) == -1 and dec(T=1 << 31) == -4
    assert dec(pay=A + 1) == -2 and dec(xh=FAR + 8) == -2 and dec(xh=A + 32) == -1 and dec(T=0, pay=None, xh=None) == 0

    def mul(a=A, M=4, b=A + (1 << 20), N=8, y=FAR):
        return lib.rac_mx_product(C.byref(cfg), a, M, b, N, y, None, 0)
    assert mul(a=None) == -1 and mul(b=None) == -1 and mul(y=None) == -1 and mul(M=-1) == -1 and mul(N=-1) == -1
    assert mul(a=A + 8) == -2 and mul(b=A + (1 << 20) + 8) == -2 and mul(y=FAR + 2) == -2
    assert mul(y=A) == -1 and mul(y=A + (1 << 20)) == -1 and mul(M=1 << 31) == -4 and mul(N=1 << 31) == -4
    assert mul(M=0, a=None, b=None, y=None) == 0 and mul(N=0, a=None, b=None, y=None) == 0

    def seg(a=A, M=4, off=A, n=2, b=A + (1 << 20), N=8, y=FAR):
        return lib.rac_mx_product_segments(C.byref(cfg), a, M, off, n, b, N, y, None, 0)
    assert seg(off=None) == -1 and seg(off=A + 2) == -2 and seg(n=-1) == -1 and seg(n=65536) == -4 and seg(n=65535, N=1 << 20) == -4
    assert seg(y=A + (1 << 20) + 15 * rec + 16 - (15 * rec) % 16) == -1              # over the last matrix row
    assert seg(n=0, a=None, off=None, b=None, y=None) == 0 and seg(M=0, a=None, off=None, b=None, y=None) == 0


def test_binding_tells_types_and_configurations_apart(rac):
    cfg = rac.MxCfg(4096, 32, x_type=torch.float16, y_type=torch.float32)
    assert repr(cfg) == "MxCfg(d=4096, block=32, x_type=float16, y_type=float32)"
    with pytest.raises(TypeError, match="cfg: expected an MxCfg"):
        rac.rac_mx_decode(rac.CodecCfg(4096, 128, 4, 0), A, 0, FAR, None, stream=0)
    with pytest.raises(TypeError):
        rac.rac_decode_reconstruct(cfg, A, 0, A, 0, None, None, None, A, A, None, stream=0)
    with pytest.raises(ValueError, match="X_hat: must be a CUDA tensor"):
        rac.rac_mx_decode(cfg, A, 1, torch.zeros(4096, dtype=torch.float16), None, stream=0)
    with pytest.raises(TypeError, match="B: expected a torch tensor, an address or None"):
        rac.rac_mx_product(cfg, A, 1, "w", 1, FAR, None, stream=0)
    with pytest.raises(rac.RacError) as e:
        rac.rac_mx_product(cfg, A, 1, A + 8, 1, FAR, None, stream=0)
    assert e.value.code == -2 and "rac_mx_product" in str(e.value)
    rac.rac_mx_product_segments(cfg, A, 0, A, 1, A, 1, FAR, None, stream=0)       # no rows
    assert rac.prepare(rac.rac_mx_encode, cfg, A, 0, FAR, 0, None, None, stream=0)() is None


@pytest.mark.parametrize("block", [16, 32])
def test_reference_rounds_to_the_nearest_code_and_clips_nothing(block):
    """The restatement itself against a search over all codes."""
    rng = np.random.default_rng(block)
    x = np.clip(rng.standard_normal((20, 96)) * np.exp(3 * rng.standard_normal((20, 96))), -6e4, 6e4).astype(np.float16).astype(np.float64)
    x[3] = 0
    x[4, :block] = 0
    rec, bad = ref.encode(x, block)
    assert not bad
    v = ref.decode(rec, 96, block)
    s = ref.decode(np.where(np.arange(rec.shape[1]) < 48, 0x22, rec).astype(np.uint8), 96, block)     # every code 1.0
    all_codes = np.concatenate((ref.MAGNITUDE, -ref.MAGNITUDE))
    best = np.abs(all_codes * s[..., None] - x[..., None]).min(-1)
    assert np.array_equal(np.abs(v - x), best)
    assert (np.abs(x) <= 6 * s).all()
    assert np.array_equal(np.signbit(v), np.signbit(x) & (v != 0))


def narrow_ring(stages, own_only, both_arrive, steps=9):
    """Every order of events in the narrow product's ring: copies (issued when a stage is free, landing in any order), one warp of
    either scale team, the matrix thread.  A wait for copy i's phase of its stage ends as soon as the parity of the stage's
    finished phases says so.  Returns what goes wrong, or None."""
    start = (frozenset(), 0, 0, 0, 0)             # landed, issued, multiplied, the teams' places
    seen, todo = {start}, [start]
    while todo:
        landed, issued, done, *at = state = todo.pop()
        after = []
        if issued < steps and (issued < stages or done > issued - stages):
            after.append((landed, issued + 1, done, *at))
        after += [(landed | {i}, issued, done, *at) for i in range(issued) if i not in landed]
        for team in (0, 1):
            i = at[team]
            if i == steps:
                continue
            on = (landed, issued, done, *(at[k] + (k == team) for k in (0, 1)))
            phases = sum(1 for j in landed if j % stages == i % stages)
            if own_only and i % 2 != team:
                after.append(on)
            elif phases % 2 != i // stages % 2:
                if i not in landed:
                    return "a phase was taken for another"
                after.append(on)
        if done in landed and at[done % 2] > done and (not both_arrive or min(at) > done):
            after.append((landed, issued, done + 1, *at))
        if not after and (done, *at) != (steps, steps, steps):
            return "a wait can only run out"
        for s in after:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    return None


def test_the_rings_of_the_narrow_product_cannot_miss_a_phase():
    """As the kernel has them (3 stages: both teams arrive; 4: a team looks at its own stages only), and why not otherwise."""
    assert narrow_ring(3, own_only=False, both_arrive=True) is None
    assert narrow_ring(4, own_only=True, both_arrive=False) is None
    assert narrow_ring(3, own_only=False, both_arrive=False) == "a wait can only run out"
    assert narrow_ring(4, own_only=False, both_arrive=False) == "a wait can only run out"
    assert narrow_ring(3, own_only=True, both_arrive=False) == "a phase was taken for another"


def test_entry_product_takes_rows_of_its_weights_width_only(rac, monkeypatch):
    """States of another width would be read with the weights' record length, out of range where they are narrower."""
    from paper_2608_04991_b200 import link
    calls = []
    for name in ("rac_mx_encode", "rac_mx_product"):
        monkeypatch.setattr(rac, name, lambda *a, name=name, **k: calls.append(name))
    entry = link.EntryProduct(torch.zeros((40, 128), dtype=torch.bfloat16))
    calls.clear()
    for shape in ((7, 96), (7, 160), (128,), (2, 7, 128), (7, 0)):
        with pytest.raises(ValueError, match="128"):
            entry(torch.zeros(shape, dtype=torch.bfloat16))
    assert calls == []
    for T in (0, 1, 7):
        assert entry(torch.zeros((T, 128), dtype=torch.bfloat16)).shape == (T, 40)
    assert calls == ["rac_mx_encode", "rac_mx_product"] * 3
    for bad in (torch.zeros(128, dtype=torch.bfloat16), torch.zeros((4, 40), dtype=torch.bfloat16), torch.zeros((4, 32800), dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            link.EntryProduct(bad)
