"""The 4-bit cache's attention over the whole range of its values: V up to the largest
that a block holds, scores up to 2^27 in log2 units, queries up to the largest and ones
that are not finite, and every code with every scale byte."""
import numpy as np
import pytest
import torch

from oracle import q4
from paper_2504_09345_amd import binding as pb
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
@pytest.mark.parametrize("sign", [1, -1])
def test_largest_scores(kind, dtype, D, sign):
    """Keys that all score the same, up to 2^27 in log2 units, weigh alike."""
    announce(f"q4 {kind} {dtype} D={D}, scores of {sign} 2^27")
    ctx = [1, 40, 700]
    b = Batch(_lens(kind, ctx), 8, 2, D, dtype, seed=2, varlen=kind != "decode")
    b.k[..., :8 * D] = 0x77
    b.k[..., 8 * D:] = 127 + 23
    b.q[:] = 0
    for h in range(8):
        b.q[:, h, 5] = sign * 1.75 * 2.0 ** -h
    b.scale = 1.0
    assert 2.0 ** 26 < 6 * 2.0 ** 23 * 1.75 / np.log(2) < 2.0 ** 27
    got = _attend(b, kind).double().numpy()
    for i, C in enumerate(ctx):
        v = q4.dense("v", b.v, b.bt, i, C, D)
        r0, L = (i, 1) if kind == "decode" else (int(b.qsl[i]), b.n_rows[i])
        for r in range(L):
            n = C - L + r + 1
            for h in range(8):
                x = v[h // 4, :n]
                # (equal weights: the output's rounding, and of the sums)
                tol = (2.0 ** -8 * (dtype == "bf16") + 2 * n * 2.0 ** -24 + 2.0 ** -22) * np.abs(x).mean(0)
                assert (np.abs(got[r0 + r, h] - x.mean(0)) <= tol).all(), (C, r, h)


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


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_queries_that_are_not_finite(kind, dtype, D, value):
    """Such a (row, head) is NaN, and the others of its columns keep their values."""
    announce(f"q4 {kind} {dtype} D={D}, a query of {value}")
    b = Batch(_lens(kind, [50, 90, 7]), 8, 2, D, dtype, seed=5, varlen=kind != "decode")
    for r, h, d in ((1, 2, 5), (1, 4, D - 1), (2, 0, 33)):
        b.q[r, h, d] = value
    ref = b.expected_gpu()
    for r, h in ((1, 2), (1, 4), (2, 0)):  # (an infinity times a code of zero, or infinities less each other)
        for x in ref:
            x[r, h] = np.nan
    assert np.isfinite(ref[0][0]).all() and np.isfinite(ref[0][1, [0, 1, 3, 5, 6, 7]]).all()
    check(_attend(b, kind), ref, 90, dtype)


# --- every code and scale byte ---------------------------------------------------

CODES = np.concatenate([q4.MAGS, -q4.MAGS])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_of_every_code_and_scale(kind, dtype, D):
    """16 keys hold the 16 codes, in another order in each dim, and a query of 1 in one
    dim alone makes them scores; each key's V is 1 in a dim of its own, so the outputs
    are the softmax of the codes' values."""
    announce(f"q4 {kind} {dtype} D={D}, scores of every code and scale byte")
    H_q = 8
    rows, extra = (1, 0) if kind == "decode" else (5, 4)  # a chunk's first row sees the 16 keys
    pages = 1 if kind == "decode" else 2
    k, v = (np.zeros((pages, 1, q4.tile_bytes(D)), np.uint8) for _ in range(2))
    v[..., 8 * D:] = 127
    for t in range(16):
        codes = (t + np.arange(D)) % 16
        for m in range(D // 2):
            k[0, 0, q4.byte_of("k", D, t, m)] = codes[2 * m] | codes[2 * m + 1] << 4
        v[0, 0, q4.byte_of("v", D, t, t // 2)] |= 2 << 4 * (t % 2)
    kind_t = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.zeros(D, rows, H_q, D, dtype=kind_t, device="cuda")
    q[torch.arange(D), :, :, torch.arange(D)] = 1
    q = q.view(D * rows, H_q, D)
    far = FAR if kind == "shared" else 32
    bt = torch.full((D, far // 16), -1, dtype=torch.int32, device="cuda")
    bt[:, :pages] = torch.arange(pages, device="cuda")
    cl = torch.full((D,), 16 + extra, dtype=torch.int32, device="cuda")
    qsl = torch.arange(D + 1, dtype=torch.int32, device="cuda") * rows
    dk, dv, out = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), torch.empty_like(q)
    ws = None
    if kind == "decode":
        dims = pb.make_dims_q4(q, dk, bt, far)
    else:
        dims = pb.make_dims_q4(q, dk, bt, far, num_q_rows=D * rows, max_q_len=rows)
    ws = torch.empty(max(1, pb.pa_workspace_size_q4(dims)), dtype=torch.uint8, device="cuda")
    got = []
    for byte in range(2, 253):
        dk[..., 8 * D:] = byte
        scale = 2.0 ** (127 - byte)
        if kind == "decode":
            pb.paged_attn_q4(q, dk, dv, bt, cl, scale, out, dims, workspace=ws)
        else:
            pb.paged_attn_varlen_q4(q, dk, dv, bt, cl, qsl, scale, out, dims, workspace=ws)
        got.append(out.view(D, rows, H_q, D)[:, 0].float().cpu().numpy())
    x = CODES[(np.arange(16)[None, :] + np.arange(D)[:, None]) % 16]
    w = np.exp(x)
    ref = np.zeros((D, H_q, D))
    ref[..., :16] = (w / w.sum(-1, keepdims=True))[:, None]
    mass = (ref > 0).astype(np.float64)
    size, reach = np.full((D, H_q), 6.0), np.full((D, H_q), float(np.abs(CODES).mean() * D))
    most = bound(ref, ref, mass, size, reach, 16, dtype, D)
    for byte, g in zip(range(2, 253), got):
        assert (np.abs(g - ref) <= most).all(), byte


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
