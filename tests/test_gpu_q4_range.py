"""The 4-bit cache's attention over the whole range of its values: V up to the largest
that a block holds, queries up to the largest, and every code with every scale byte."""
import numpy as np
import pytest
import torch

from oracle import q4
from q4_util import Batch, bound, check

from parity_util import announce

pytestmark = pytest.mark.gpu

FAR = 1 << 20  # a declared context for which a call's chunks share V's operands (bf16)
KINDS = ["decode", "chunks", "shared"]


def _lens(kind, ctx):
    if kind == "decode":
        return [(c, 1) for c in ctx]
    return [(c, min(c, 1 + 40 * (i % 2) + 9 * i)) for i, c in enumerate(ctx)]


def _attend(b, kind):
    """The call's output on the host, its chunks by the kernel that `kind` names."""
    d = b.upload()
    if kind != "shared":
        return b.attend(d).float().cpu()
    b.widen(d, FAR)
    return b.attend(d, b.dims(d, max_context_len=FAR)).float().cpu()


def _scales(D, tokens=range(16), blocks=None):
    return [q4.scale_byte_of(D, t, j) for t in tokens for j in (range(D // 32) if blocks is None else blocks)]


# --- V up to 6 * 2^125 ---------------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("byte", [191, 192, 200, 240, 248, 252])
def test_large_values(kind, dtype, D, byte):
    """Every V of a size from 2^64 to the largest that there is, or one block's, or one
    token's: a weighted mean is no larger than what it is of."""
    announce(f"q4 {kind} {dtype} D={D}, V of scale byte {byte}")
    ctx = [1, 40, 700, 33, 64, 300, 520]
    b = Batch(_lens(kind, ctx), 8, 2, D, dtype, seed=byte, varlen=kind != "decode")
    pages = [b.bt[i, :-(-c // 16)] for i, c in enumerate(ctx)]
    for i in (0, 1, 2):
        b.v[np.ix_(pages[i], range(2), _scales(D))] = byte
    b.v[np.ix_(pages[3], [1], _scales(D, blocks=[1]))] = byte             # a block of one head
    b.v[np.ix_(pages[4][3:], range(2), _scales(D, tokens=[15]))] = byte   # the last key
    b.v[np.ix_(pages[5][:1], range(2), _scales(D, tokens=[0]))] = byte    # the first key
    b.v[np.ix_(pages[6][12:14], range(2), _scales(D, tokens=[3, 9]))] = byte
    ref = b.expected_gpu()
    assert np.isfinite(ref[0]).all() and np.abs(ref[0]).max() < 2.0 ** 128
    check(_attend(b, kind), ref, 700, dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_means_of_the_largest(kind, dtype):
    """Thousands of keys of one weight, each V the largest there is: their sum is not a
    number of 32 bits, their mean is."""
    announce(f"q4 {kind} {dtype}, means of the largest values")
    b = Batch(_lens(kind, [5000, 3000]), 4, 1, 64, dtype, seed=1, varlen=kind != "decode")
    b.q[:] = 0
    b.v[..., :8 * 64] = 0x77
    b.v[..., 8 * 64:] = 252
    got = _attend(b, kind).double().numpy()
    top = 6 * 2.0 ** 125
    # (the weights are alike, so numerator and denominator carry the sums' errors alone)
    assert (np.abs(got - top) <= (2.0 ** -8 * (dtype == "bf16") + 2 * 5000 * 2.0 ** -24 + 2.0 ** -22) * top).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_values_leave_other_rows_alone(dtype):
    """Rows that do not see the large V keep small ones, to 2^-120."""
    announce(f"q4 chunks {dtype}, large V behind small ones")
    b = Batch([(60, 40), (400, 1)], 4, 2, 64, dtype, seed=4)
    at = _scales(64)
    b.v[:, :, at] = np.clip(b.v[:, :, at].astype(int) - 116, 2, 252)
    b.v[b.bt[0, 3], :, q4.scale_byte_of(64, 2, 0)] = 250  # token 50: rows from 30 on
    out, ref = _attend(b, "chunks"), b.expected_gpu()
    ref = [x[:30] for x in ref]
    assert (np.abs(ref[0]).max(-1) < 2.0 ** -100).all()
    off = np.abs(out[:30].double().numpy() - ref[0])
    tight = bound(*ref, 60, dtype, 64) - 1e-37 + 2.0 ** -133  # (bf16's last step)
    assert (off <= tight).all()


# --- scores --------------------------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_queries_up_to_the_largest(kind, dtype, D):
    """The largest finite queries, on keys small enough that the scores are usual ones."""
    announce(f"q4 {kind} {dtype} D={D}, queries up to the largest")
    b = Batch(_lens(kind, [50, 90, 17]), 8, 2, D, dtype, seed=3, varlen=kind != "decode")
    at = _scales(D)
    b.k[:, :, at] = np.clip(b.k[:, :, at].astype(int) - 127 + 2, 2, 8)
    top = float(np.finfo(np.float32).max) if dtype == "fp32" else float(np.uint32(0x7F7F0000).view(np.float32))
    b.q[:] = b.round(np.clip(b.q, -1, 1) * 1e37)
    b.q[:, 1, 7], b.q[:, 2, 40], b.q[:, 6, 0] = top, -top, top
    b.scale = 0.02
    check(_attend(b, kind), b.expected_gpu(), 90, dtype)


# --- every code and scale byte ---------------------------------------------------

CODES = np.concatenate([q4.MAGS, -q4.MAGS])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_values_of_every_code_and_scale(kind, dtype, D):
    """Contexts of one token return its V: every code with every scale byte (in fp32
    within the normalisation's rounding)."""
    announce(f"q4 {kind} {dtype} D={D}, V of every code and scale byte")
    n = 251
    b = Batch(_lens("decode" if kind == "decode" else "chunks", [1] * n + ([40] if kind != "decode" else [])), 8, 1, D, dtype, seed=7,
              varlen=kind != "decode")
    codes = np.arange(D) % 16
    for i in range(n):
        page = b.bt[i, 0]
        for m in range(D // 2):
            b.v[page, 0, q4.byte_of("v", D, 0, m)] = codes[2 * m] | codes[2 * m + 1] << 4
        b.v[page, 0, _scales(D, tokens=[0])] = 2 + i
    got = _attend(b, kind).double().numpy()
    for i in range(n):
        r = i if kind == "decode" else int(b.qsl[i])
        x = CODES[codes] * 2.0 ** (i + 2 - 127)
        assert (np.abs(got[r] - x) <= (0.0 if dtype == "bf16" else 2.0 ** -22) * np.abs(x)).all(), i + 2
