"""The 8-bit paged KV cache on the GPU against its plain form in float64: the
append's bytes, scales and the read's values exactly."""
import numpy as np
import pytest
import torch

from oracle import q8
from paper_2504_09345_amd import binding as pb
from q8_util import Batch, same_bytes

from parity_util import announce

pytestmark = pytest.mark.gpu

LENS = [(1, 1), (16, 16), (17, 3), (40, 40), (33, 1), (70, 6), (0, 0), (5, 5), (129, 30), (48, 47)]


# --- the cache write and read ------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H_kv", [1, 3, 8])
def test_append_and_read_varlen(dtype, D, H_kv):
    announce(f"q8 append varlen {dtype} D={D} H_kv={H_kv}")
    b = Batch(LENS, H_q=H_kv, H_kv=H_kv, D=D, dtype=dtype, seed=H_kv)
    kn, vn = b.new_rows(1, odd=True), b.new_rows(2, odd=True)
    ref = b.written(kn, vn)
    d = b.upload()
    b.append(d, kn, vn)
    assert same_bytes(d, ref) == ""
    got = b.read(d)
    assert np.array_equal(got.astype(np.float64), q8.read(*ref, b.bt, b.ctx, D, b.qsl), equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_append_and_read_decode(dtype, D):
    announce(f"q8 append decode {dtype} D={D}")
    b = Batch([(c, 1) for c in (1, 0, 16, 17, 300, 0, 31, 32, 33)], H_q=4, H_kv=4, D=D, dtype=dtype, varlen=False)
    live = b.ctx > 0
    d = b.upload()
    for seed in range(3):  # (the same positions again: scales that grow, and that stay)
        kn, vn = b.new_rows(seed, odd=seed == 2), b.new_rows(seed + 9)
        b.k, b.v, b.scales = ref = b.written(kn, vn)
        b.append(d, kn, vn)
        assert same_bytes(d, ref) == ""
    got = b.read(d)
    assert np.array_equal(got[:, live].astype(np.float64), q8.read(*ref, b.bt, b.ctx, D)[:, live], equal_nan=True)
    assert (got[:, ~live] == -3.0).all()  # no row: left as it was


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_pages_filled_token_by_token(dtype, D):
    """Every slot of a page, the scale growing by anything from nothing to all of its range."""
    announce(f"q8 append token by token {dtype} D={D}")
    b = Batch([(40, 1), (40, 1), (40, 1)], H_q=2, H_kv=2, D=D, dtype=dtype, varlen=False)
    d = b.upload()
    rng = np.random.default_rng(5)
    for t in range(40):
        size = 2.0 ** np.array([rng.integers(-1, 2), rng.integers(-20, 21), rng.integers(-125, 127)])[:, None, None]
        kn, vn = (b.round(np.clip(rng.standard_normal((3, 2, D)), -1.9, 1.9) * size) for _ in range(2))
        b.ctx[:] = t + 1
        d["cl"] = b.cuda(b.ctx)
        b.k, b.v, b.scales = ref = b.written(kn, vn)
        b.append(d, kn, vn, max_context_len=40)
        assert same_bytes(d, ref) == "", f"token {t}"


def test_every_code_rounded_to_every_larger_scale():
    announce("q8 append, every code rounded again")
    D = 128
    for grow in list(range(1, 20)) + [60, 200]:
        b = Batch([(16, 1), (16, 1)], H_q=1, H_kv=1, D=D, varlen=False)
        for which, pool in (("k", b.k), ("v", b.v)):
            codes = np.arange(256, dtype=np.uint8).reshape(2, D)
            for page in range(2):
                pool[b.bt[page, 0], 0, q8.places(which, D)[:15]] = codes[page]
        b.scales[:] = 30
        x = np.full((2, 1, D), 1.5 * 2.0 ** (30 - 127 + 8 + grow))
        kn = vn = b.round(np.minimum(x, 3e38))
        d = b.upload()
        b.append(d, kn, vn)
        assert same_bytes(d, b.written(kn, vn)) == "", f"scale 2^{grow} times the first"


def test_every_value_and_border_quantised():
    """Each e4m3 value, each midpoint and its neighbours in 32 bits."""
    announce("q8 append, values and borders")
    m = q8.VALUES[:127]
    y = np.concatenate([m, (m[:-1] + m[1:]) / 2]).astype(np.float32)
    y = np.concatenate([y, np.nextafter(y, np.float32(1e9)), np.nextafter(y, np.float32(-1e9))])
    y = np.concatenate([y, -y])[:1518]
    y = y[np.abs(y) <= 448]
    x = np.zeros(16 * 128, np.float32)
    x[1:1 + y.size] = y
    x[0] = 448.0
    for e in (0, -100, 60, 119):
        b = Batch([(16, 16)], H_q=1, H_kv=1, D=128, dtype="fp32")
        kn = (x * np.float32(2.0 ** e)).reshape(16, 1, 128) if e < 100 else (x * np.float32(0.5) * np.float32(2.0 ** 120)).reshape(16, 1, 128)
        d = b.upload()
        b.append(d, kn, -kn)
        assert same_bytes(d, b.written(kn, -kn)) == "", f"2^{e}"


def test_read_every_code_and_scale():
    announce("q8 read, every code and scale")
    for dtype in ("bf16", "fp32"):
        b = Batch([(230 * 16, 230 * 16)], H_q=1, H_kv=1, D=128, dtype=dtype, spare=1)
        for which, pool in (("k", b.k), ("v", b.v)):
            pool[:] = np.arange(2048, dtype=np.int64) % 256
        for p in range(230):
            b.scales[b.bt[0, p], 0] = (17 + p, 246 - p)
        got = b.read(b.upload()).astype(np.float64)
        assert np.array_equal(got, q8.read(b.k, b.v, b.scales, b.bt, b.ctx, 128, b.qsl), equal_nan=True)


def test_read_whole_contexts():
    announce("q8 read whole contexts")
    b = Batch([(c, c) for c in (1, 47, 16, 0, 130, 64)], H_q=2, H_kv=2, D=128, spare=1)
    got = b.read(b.upload())
    assert np.array_equal(got.astype(np.float64), q8.read(b.k, b.v, b.scales, b.bt, b.ctx, 128, b.qsl))


def test_rows_outside_the_contract():
    announce("q8 append and read, rows outside the contract")
    b = Batch([(20, 4), (40, 2), (33, 33), (18, 18), (9, 2)], H_q=2, H_kv=2, D=64)
    kn, vn = b.new_rows(1), b.new_rows(2)
    d = b.upload()
    ctx = b.ctx.copy()
    ctx[0] = 3        # a chunk longer than its context
    ctx[1] = 1000     # a context above max_context_len
    d["cl"] = b.cuda(ctx)
    bt = b.bt.copy()
    bt[2, 1], bt[3, 1] = -1, b.num_pages  # pages outside the pool: tokens 16 .. 31, 16, 17
    d["bt"] = b.cuda(bt)
    b.append(d, kn, vn, max_context_len=48)
    keep = np.ones(b.T, bool)
    keep[:6] = False
    keep[6 + 16:6 + 32] = False
    keep[6 + 33 + 16:6 + 33 + 18] = False
    ref = b.written(kn, vn, keep)
    assert same_bytes(d, ref) == ""
    got = b.read(d, max_context_len=48)
    assert np.array_equal(got.astype(np.float64), q8.read(*ref, b.bt, b.ctx, 64, b.qsl, keep), equal_nan=True)


def test_rows_behind_the_last_sequence():
    announce("q8 append and read, rows behind the last sequence")
    b = Batch([(20, 4), (40, 1)], H_q=4, H_kv=2, D=64)
    d = b.upload()
    rows = torch.full((2, b.T + 3, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    b.read(d, rows, num_q_rows=b.T + 3)
    assert (rows[:, b.T:] == 7.0).all() and not (rows[:, :b.T] == 7.0).all(-1).any()
    kn, vn = b.new_rows(1), b.new_rows(2)
    more = [np.concatenate([x, x[:3]]) for x in (kn, vn)]
    b.append(d, *more, num_q_rows=b.T + 3)
    assert same_bytes(d, b.written(kn, vn)) == ""
