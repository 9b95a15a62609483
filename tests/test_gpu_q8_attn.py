"""Attention over the 8-bit paged KV cache on the GPU against float64, within its
arithmetic's bound (q4_util.bound: the same products and softmax): decode rows, chunks
by each of their kernels, NaN, every size of V, of queries and of scores."""
import numpy as np
import pytest
import torch

from oracle import q8
from paper_2504_09345_amd import binding as pb
from q4_util import bound, check
from q8_util import Batch

from parity_util import announce

pytestmark = pytest.mark.gpu

FAR = 1 << 22  # a declared context for which a call's waves have 32 columns (bf16)
KINDS = ["decode", "chunks", "wide"]
DECODE = [1, 15, 16, 17, 31, 32, 33, 0, 64, 200, 333, 48]


def _lens(kind, ctx):
    if kind == "decode":
        return [(c, 1) for c in ctx]
    return [(c, min(c, 1 + 40 * (i % 2) + 9 * i)) for i, c in enumerate(ctx)]


def _attend(b, kind, d=None):
    """The call's output on the host, its chunks by the kernel that `kind` names."""
    d = b.upload() if d is None else d
    if kind != "wide":
        return b.attend(d).float().cpu()
    b.widen(d, FAR)
    return b.attend(d, b.dims(d, max_context_len=FAR)).float().cpu()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H_q,H_kv", [(8, 8), (4, 2), (4, 1), (18, 3), (64, 8)])
def test_decode(dtype, D, H_q, H_kv):
    announce(f"q8 decode {dtype} D={D} heads={H_q}/{H_kv}")
    b = Batch([(c, 1) for c in DECODE], H_q, H_kv, D, dtype, seed=H_q, varlen=False)
    check(b.attend(b.upload()).float().cpu(), b.expected(), max(DECODE), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H_q,H_kv", [(2, 2), (4, 2), (4, 1), (6, 1), (16, 2)])
@pytest.mark.parametrize("lens", [
    [(1, 1), (40, 2), (33, 1), (0, 0), (18, 3)],                    # few rows each
    [(100, 7), (64, 64), (16, 1), (90, 33), (1, 1), (200, 5)],       # chunks beside decode rows
    [(130, 130), (150, 65)],                                         # chunks alone
], ids=["few", "mixed", "chunks"])
def test_varlen(dtype, D, H_q, H_kv, lens):
    announce(f"q8 varlen {dtype} D={D} heads={H_q}/{H_kv} {lens}")
    b = Batch(lens, H_q, H_kv, D, dtype, seed=len(lens))
    check(b.attend(b.upload()).float().cpu(), b.expected(), max(c for c, _ in lens), dtype)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H_q,H_kv", [(34, 34), (68, 34), (8, 2), (6, 1), (16, 2)])
@pytest.mark.parametrize("lens", [
    [(100, 7), (64, 64), (16, 1), (90, 33), (1, 1), (0, 0), (200, 50)],
    [(130, 130), (150, 65)],
    [(300, 40)],
], ids=["mixed", "chunks", "one"])
def test_wide(D, H_q, H_kv, lens):
    """Waves of 32 columns, chosen by a declared context far above the real ones."""
    announce(f"q8 wide D={D} heads={H_q}/{H_kv} {lens}")
    b = Batch(lens, H_q, H_kv, D, seed=len(lens))
    check(_attend(b, "wide"), b.expected(), max(c for c, _ in lens), "bf16")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H_q,H_kv", [(32, 8), (48, 8), (8, 1)])
@pytest.mark.parametrize("lens", [
    [(1000, 256)] * 9 + [(300, 1), (1, 1)],      # whole items
    [(5000, 100), (4700, 120), (33, 2)],          # items in parts
    [(2600, 2600)],
], ids=["items", "parts", "prompt"])
def test_wide_at_size(D, H_q, H_kv, lens):
    announce(f"q8 wide at size D={D} heads={H_q}/{H_kv} {lens[0]}")
    b = Batch(lens, H_q, H_kv, D, seed=9)
    check(b.attend(b.upload()).float().cpu(), b.expected(), max(c for c, _ in lens), "bf16")


@pytest.mark.parametrize("n,ctx", [(1, 5000), (3, 2500)])
def test_long_contexts_are_cut_and_joined(n, ctx):
    announce(f"q8 decode {n} x {ctx}")
    b = Batch([(ctx - 100 * i, 1) for i in range(n)], 8, 2, 128, varlen=False, seed=n)
    d = b.upload()
    check(b.attend(d).float().cpu(), b.expected(), ctx, "bf16")
    # a declared bound far above the contexts changes the parts, not the result
    b.widen(d, 64000)
    check(b.attend(d, b.dims(d, max_context_len=64000)).float().cpu(), b.expected(), ctx, "bf16")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("dtype,H_q,H_kv,lens", [
    ("fp32", 32, 8, [(600, 600)]),                      # two waves share an item
    ("fp32", 32, 8, [(1500, 1500)]),                    # each its own
    ("fp32", 8, 8, [(31, 31), (32, 32), (33, 33)]),     # one unit and two, four waves for them
    ("bf16", 16, 2, [(100, 1), (64, 3), (7000, 40)]),   # parts in the workspace too
    ("bf16", 6, 1, [(97, 5), (65, 64)]),                # columns left over
    ("fp32", 8, 2, [(4000, 3), (50, 2), (3000, 1)]),
], ids=["two", "one", "short", "parts", "six", "few"])
def test_waves_that_share_an_item(D, dtype, H_q, H_kv, lens):
    announce(f"q8 chunks {dtype} D={D} heads={H_q}/{H_kv} {lens}")
    b = Batch(lens, H_q, H_kv, D, dtype=dtype, seed=len(lens))
    check(b.attend(b.upload()).float().cpu(), b.expected(), max(c for c, _ in lens), dtype)


@pytest.mark.parametrize("H_kv,n,ctx", [(8, 3, 2048), (1, 1, 512), (3, 5, 7), (64, 2, 33), (8, 40, 64), (5, 300, 100), (1, 3, 1500), (4, 40, 700)])
def test_decode_items_and_workgroups(H_kv, n, ctx):
    """Items within a wave, a workgroup, and over several of them; the same bits every
    time, whatever the workspace holds."""
    announce(f"q8 decode ranges {n} x {ctx} H_kv={H_kv}")
    rng = np.random.default_rng(n)
    b = Batch([(int(c), 1) for c in rng.integers(max(1, ctx // 2), ctx + 1, n)], 2 * H_kv, H_kv, 64, seed=n, varlen=False)
    d = b.upload()
    first = b.attend(d)
    check(first.float().cpu(), b.expected(), ctx, "bf16")
    ws = torch.full((pb.pa_workspace_size_q8(b.dims(d)),), 0xA5, dtype=torch.uint8, device="cuda")
    for fill in (0xA5, 0xFF):
        ws.fill_(fill)
        assert torch.equal(b.attend(d, workspace=ws), first)
    for _ in range(3):
        assert torch.equal(b.attend(d, workspace=ws), first)


@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "fp32")])
@pytest.mark.parametrize("lens", [[(0, 0)] * 40 + [(70, 2)] + [(9, 0)] * 30, [(300, 39)] + [(0, 0)] * 200 + [(33, 1)]],
                         ids=["two rows", "a chunk and a row"])
def test_more_sequences_than_rows(D, dtype, lens):
    announce(f"q8 chunks among empty sequences D={D} {dtype}")
    b = Batch(lens, 8, 2, D, dtype=dtype, seed=2)
    check(b.attend(b.upload()).float().cpu(), b.expected(), 300, dtype)


@pytest.mark.parametrize("ctx", [4000, 70000, 1100000])
@pytest.mark.parametrize("H_q", [1, 8])
def test_items_over_many_workgroups(H_q, ctx):
    """One item over 16 to 512 workgroups, each size of the joins' groups.  Queries of
    zeros weigh every key alike, and all sums are exact: the output is the mean of V,
    1 / l and one product from exact (2^-22 of it)."""
    announce(f"q8 one item of {ctx} tokens H_q={H_q}")
    D, pool = 64, 97
    rng = np.random.default_rng(ctx)
    k = rng.integers(0, 127, (pool, 1, 16 * D), dtype=np.uint8)
    v = (0x38 + rng.integers(0, 16, (pool, 1, 16 * D)) + 128 * rng.integers(0, 2, (pool, 1, 16 * D))).astype(np.uint8)  # 1 .. 3.75
    scales = np.full((pool, 1, 2), 127, np.uint8)
    pages = -(-ctx // 16)
    bt = rng.integers(0, pool, (1, pages)).astype(np.int32)
    count = np.bincount(bt[0, :ctx // 16], minlength=pool)
    x = q8.unpack("v", v[:, 0], scales[:, 0, 1], D)  # [page][token][dim]
    total = np.einsum("p,ptd->d", count.astype(np.float64), x)
    if ctx % 16:
        total += x[bt[0, -1], :ctx % 16].sum(0)
    t = [torch.from_numpy(a).cuda() for a in (k, v, scales, bt, np.array([ctx], np.int32))]
    q = torch.zeros(1, H_q, D, device="cuda")
    for dtype, step in ((torch.float32, 2.0 ** -24), (torch.bfloat16, 2.0 ** -8)):
        out = torch.empty(1, H_q, D, dtype=dtype, device="cuda")
        pb.paged_attn_q8(q.to(dtype), *t, 1.0, out, pb.make_dims_q8(out, t[0], t[3], ctx))
        off = np.abs(out[0].double().cpu().numpy() - total / ctx)
        assert (off <= (step + 2.0 ** -22) * np.abs(total / ctx)).all()


@pytest.mark.parametrize("varlen", [False, True])
def test_shortest(varlen):
    """Contexts of one token (its value) and of none."""
    announce(f"q8 shortest contexts varlen={varlen}")
    b = Batch([(1, 1), (0, 0) if varlen else (0, 1), (1, 1), (2, 2) if varlen else (2, 1)], 4, 1, 128, seed=3, varlen=varlen)
    got = b.attend(b.upload()).float().cpu()
    ref = b.expected()
    check(got, ref, 2, "bf16")
    assert np.array_equal(got[0].numpy(), ref[0][0].astype(np.float32))  # (one weight of 1: V itself)


@pytest.mark.parametrize("B,ctx", [(8192, 4224), (9000, 40)])
def test_many_sequences_share_their_pages(B, ctx):
    """More sequences than a launch takes.  All read the same pages, with a few different
    queries."""
    announce(f"q8 decode {B} sequences of {ctx}")
    one = Batch([(ctx, 1)], 1, 1, 64, varlen=False)
    d = one.upload()
    q = one.cuda(one.round(np.random.default_rng(1).standard_normal((8, 1, 64)))).to(torch.bfloat16)
    which = torch.arange(B, device="cuda") * 7 % 8
    d["q"] = q[which].contiguous()
    d["bt"] = d["bt"].expand(B, -1).contiguous()
    d["cl"] = d["cl"].expand(B).contiguous()
    out = one.attend(d)
    for i in range(8):
        one.q = q[i:i + 1].float().cpu().numpy()
        mine = out[which == i].float().cpu()
        check(mine, [np.repeat(r, len(mine), 0) for r in one.expected()], ctx, "bf16")


# --- NaN and what the contract does not allow ----------------------------------

@pytest.mark.parametrize("kind", ["chunks", "wide"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_nan_reaches_the_rows_that_see_it(kind, dtype, D):
    """A NaN of V in a dim of the rows that see its key, one of K in all of them."""
    announce(f"q8 {kind} {dtype} D={D}, NaN in K and V")
    b = Batch([(170, 140), (64, 1), (100, 90), (33, 33)], 8, 2, D, dtype, seed=3)
    for which, seq, token, g, dim, code in (("v", 0, 45, 1, 33, 127), ("v", 0, 46, 0, D - 1, 255), ("v", 0, 150, 1, 0, 127), ("v", 0, 3, 1, 7, 255),
                                            ("k", 2, 20, 0, 11, 127), ("v", 1, 5, 0, 60, 127), ("v", 3, 32, 1, 17, 255)):
        pool = b.k if which == "k" else b.v
        pool[b.bt[seq, token // 16], g, q8.byte_of(which, token % 16, dim)] = code
    ref = b.expected()
    assert np.isnan(ref[0]).any() and not np.isnan(ref[0][:15, :4]).any() and not np.isnan(ref[0][231:241]).any()
    check(_attend(b, kind), ref, 170, dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("D", [64, 128])
def test_rows_outside_the_contract(kind, D):
    announce(f"q8 attention, rows outside the contract {kind} D={D}")
    varlen = kind != "decode"
    b = Batch([(50, 5), (40, 3), (33, 20), (64, 1), (20, 2)], 4, 2, D, varlen=varlen)
    ref = b.expected()
    d = b.upload()
    ctx, bt = b.ctx.copy(), b.bt.copy()
    ctx[0] = 5000 if kind != "wide" else 2 * FAR  # above max_context_len
    bt[2, 1] = b.num_pages + 7    # outside the pool
    bt[3, 0] = -5
    d["cl"], d["bt"] = b.cuda(ctx), b.cuda(bt)
    q0 = list(range(6)) if not varlen else b.qsl
    ref[0][q0[0]:q0[1]] = np.nan
    for r in range(q0[2], q0[3]):
        if int(b.ctx[2]) - (q0[3] - r) >= 16:  # sees page 1
            ref[0][r] = np.nan
    ref[0][q0[3]:q0[4]] = np.nan
    if varlen:  # a chunk longer than its context
        ctx[1] = 2
        d["cl"] = b.cuda(ctx)
        ref[0][q0[1]:q0[2]] = np.nan
    if kind == "wide":
        check(_attend(b, kind, d), ref, 64, "bf16")
    else:
        check(b.attend(d, b.dims(d, max_context_len=64)).float().cpu(), ref, 64, "bf16")


def test_rows_behind_the_last_sequence():
    announce("q8 attention, rows behind the last sequence")
    b = Batch([(20, 4), (40, 1)], 4, 2, 64)
    d = b.upload()
    d["q"] = torch.cat([d["q"], d["q"][:3]])
    out = b.attend(d, b.dims(d, num_q_rows=b.T + 3), torch.full_like(d["q"], 7.0))
    assert (out[b.T:] == 7.0).all()
    check(out[:b.T].float().cpu(), b.expected(), 40, "bf16")


def test_chunks_longer_than_max_q_len():
    announce("q8 varlen, chunks longer than max_q_len")
    b = Batch([(40, 9), (33, 1), (64, 4)], 4, 2, 64)
    d = b.upload()
    for most, nan in ((1, (0, 2)), (4, (0,))):
        ref = b.expected()
        for i in nan:
            ref[0][b.qsl[i]:b.qsl[i + 1]] = np.nan
        check(b.attend(d, b.dims(d, max_q_len=most)).float().cpu(), ref, 64, "bf16")


@pytest.mark.parametrize("kind", KINDS)
def test_no_pages(kind):
    """A pool of none: rows of a context are NaN (every entry lies outside), those of none
    as ever."""
    announce(f"q8 attention, a pool without pages, {kind}")
    b = Batch([(20, 3), (0, 0), (40, 1), (4000, 30)], 40, 40, 64, varlen=kind != "decode")
    d = b.upload()
    if kind == "wide":
        b.widen(d, FAR)
    dims = b.dims(d, max_context_len=FAR if kind == "wide" else None)
    dims.num_pages = 0
    d["k"], d["v"], d["scales"] = d["k"][:1], d["v"][:1], d["scales"][:1]
    out = b.attend(d, dims, torch.zeros_like(d["q"]))
    live = torch.ones(b.T, dtype=torch.bool, device="cuda")
    if kind == "decode":
        live[1] = False
        assert (out[1] == 0).all()
    assert torch.isnan(out[live]).all()


# --- sizes -----------------------------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -25, 2.0 ** -10, 2.0 ** 14, 2.0 ** 60])
@pytest.mark.parametrize("D", [64, 128])
def test_values_of_any_size(kind, dtype, D, size):
    """V far outside fp16's range, in all or some of the pages."""
    announce(f"q8 {kind} {dtype} D={D}, V of size {size}")
    b = Batch(_lens(kind, [100, 90, 33]), 8, 2, D, dtype, seed=1, varlen=kind != "decode")
    for page in b.bt[0, :7:2].tolist() + b.bt[1, :6].tolist():
        b.scales[page, :, 1] = np.clip(b.scales[page, :, 1].astype(int) + int(np.log2(size)), 17, 246)
    check(_attend(b, kind), b.expected(), 100, dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("byte", [182, 183, 200, 240, 246])
def test_large_values(kind, dtype, D, byte):
    """Every V of a size from 2^64 to the largest that there is, or one page's: a weighted
    mean is no larger than what it is of."""
    announce(f"q8 {kind} {dtype} D={D}, V of scale byte {byte}")
    ctx = [1, 40, 700, 33, 64, 300, 520]
    b = Batch(_lens(kind, ctx), 8, 2, D, dtype, seed=byte, varlen=kind != "decode")
    pages = [b.bt[i, :-(-c // 16)] for i, c in enumerate(ctx)]
    for i in (0, 1, 2):
        b.scales[pages[i], :, 1] = byte
    b.scales[pages[3], 1, 1] = byte         # of one head
    b.scales[pages[4][3:], :, 1] = byte     # the last page
    b.scales[pages[5][:1], :, 1] = byte     # the first
    b.scales[pages[6][12:14], :, 1] = byte
    ref = b.expected()
    assert np.isfinite(ref[0]).all() and np.abs(ref[0]).max() < 2.0 ** 128
    check(_attend(b, kind), ref, 700, dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_means_of_the_largest(kind, dtype):
    """Thousands of keys of one weight, each V the largest there is: their sum is not a
    number of 32 bits, their mean is."""
    announce(f"q8 {kind} {dtype}, means of the largest values")
    b = Batch(_lens(kind, [5000, 3000]), 4, 1, 64, dtype, seed=1, varlen=kind != "decode")
    b.q[:] = 0
    b.v[:] = 126
    b.scales[..., 1] = 246
    got = _attend(b, kind).double().numpy()
    top = 448 * 2.0 ** 119
    # (the weights are alike, so numerator and denominator carry the sums' errors alone)
    assert (np.abs(got - top) <= (2.0 ** -8 * (dtype == "bf16") + 2 * 5000 * 2.0 ** -24 + 2.0 ** -22) * top).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sign", [1, -1])
def test_largest_scores(kind, dtype, D, sign):
    """Keys that all score the same, up to 2^27 in log2 units, weigh alike."""
    announce(f"q8 {kind} {dtype} D={D}, scores of {sign} 2^27")
    ctx = [1, 40, 700]
    b = Batch(_lens(kind, ctx), 8, 2, D, dtype, seed=2, varlen=kind != "decode")
    b.k[:] = 126
    b.scales[..., 0] = 127 + 17
    b.q[:] = 0
    for h in range(8):
        b.q[:, h, 5] = sign * 1.5 * 2.0 ** -h
    b.scale = 1.0
    assert 2.0 ** 26 < 448 * 2.0 ** 17 * 1.5 / np.log(2) < 2.0 ** 27
    got = _attend(b, kind).double().numpy()
    for i, C in enumerate(ctx):
        v = q8.dense("v", b.v, b.scales, b.bt, i, C, D)
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
def test_small_products_beside_a_large_one(kind, dtype, D):
    """A channel of K that all keys share, up to 2^17 times its neighbours' products: the
    scores' differences are the neighbours'."""
    announce(f"q8 {kind} {dtype} D={D}, small products beside a large one")
    b = Batch(_lens(kind, [40, 90, 33]), 8, 2, D, dtype, seed=4, varlen=kind != "decode")
    rng = np.random.default_rng(1)
    for i, c in enumerate((40, 90, 33)):
        for p in range(-(-c // 16)):
            x = rng.choice([0, 0, 1, 1.125, -1.875], (2, 16, D)) * (rng.random((2, 16, 1)) < 0.7)
            x[..., 3], x[..., D - 9] = 1.0, -1.0
            b.put("k", b.bt[i, p], x, min(16, c - 16 * p))
    b.q = rng.choice([-1.0, 1.0, 1.25], b.q.shape)
    for h in range(8):
        b.q[:, h, 3] = 2.0 ** (6 + h)
        b.q[:, h, D - 9] = 2.0 ** (17 - 2 * h)
    b.q = b.round(b.q)
    b.scale = 1 / 16
    check(_attend(b, kind), b.expected(), 90, dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_queries_of_any_size(kind, dtype, D):
    """Queries of zeros, small and large ones, and of very different sizes in one row."""
    announce(f"q8 {kind} {dtype} D={D}, queries of any size")
    b = Batch([(100, 1)] * 8 if kind == "decode" else [(100, 5)] * 8, 8, 2, D, dtype, seed=2, varlen=kind != "decode")
    q = b.q.reshape(8, -1, 8, D)
    for i, f in enumerate([0.0, 2.0 ** -130, 2.0 ** -60, 2.0 ** -10, 1.0, 30.0, 1.0, 1.0]):
        q[i] *= f
    q[6] *= np.exp2(-np.arange(D) / 4.0).astype(np.float32)
    q[7, ..., ::2] *= 2.0 ** -20
    b.q = b.round(q.reshape(-1, 8, D))
    check(_attend(b, kind), b.expected(), 100, dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_queries_up_to_the_largest(kind, dtype, D):
    """The largest finite queries, on keys small enough that the scores are usual ones."""
    announce(f"q8 {kind} {dtype} D={D}, queries up to the largest")
    b = Batch(_lens(kind, [50, 90, 17]), 8, 2, D, dtype, seed=3, varlen=kind != "decode")
    for i, c in enumerate((50, 90, 17)):
        b.scales[b.bt[i, :-(-c // 16)], :, 0] = 17
    top = float(np.finfo(np.float32).max) if dtype == "fp32" else float(np.uint32(0x7F7F0000).view(np.float32))
    b.q[:] = b.round(np.clip(b.q, -1, 1) * 1e37)
    b.q[:, 1, 7], b.q[:, 2, 40], b.q[:, 6, 0] = top, -top, top
    b.scale = 2.0 ** -18
    check(_attend(b, kind), b.expected(), 90, dtype)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
def test_queries_that_are_not_finite(kind, dtype, D, value):
    """Such a (row, head) is NaN, and the others of its columns keep their values."""
    announce(f"q8 {kind} {dtype} D={D}, a query of {value}")
    b = Batch(_lens(kind, [50, 90, 7]), 8, 2, D, dtype, seed=5, varlen=kind != "decode")
    for r, h, d in ((1, 2, 5), (1, 4, D - 1), (2, 0, 33)):
        b.q[r, h, d] = value
    ref = b.expected()
    for r, h in ((1, 2), (1, 4), (2, 0)):  # (scores that are infinite, less each other)
        for x in ref:
            x[r, h] = np.nan
    assert np.isfinite(ref[0][0]).all() and np.isfinite(ref[0][1, [0, 1, 3, 5, 6, 7]]).all()
    check(_attend(b, kind), ref, 90, dtype)


# --- waves of 32 columns in small calls ----------------------------------------

def _wide_only(b):
    """Of a batch whose far declared bound does give its waves 32 columns: bf16, and more
    columns in the longest chunk than one such wave has."""
    assert b.dtype == "bf16" and max(b.n_rows) * b.H_q // b.H_kv > 32
    return b


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H_q,H_kv", [(40, 40), (12, 2)])
def test_wide_without_pages(D, H_q, H_kv):
    """A pool of none: rows of a context are NaN (every entry lies outside)."""
    announce(f"q8 wide D={D} heads={H_q}/{H_kv}, a pool without pages")
    b = _wide_only(Batch([(20, 3), (0, 0), (40, 1), (4000, 40)], H_q, H_kv, D))
    d = b.upload()
    b.widen(d, FAR)
    dims = b.dims(d, max_context_len=FAR)
    dims.num_pages = 0
    d["k"], d["v"], d["scales"] = d["k"][:1], d["v"][:1], d["scales"][:1]
    assert torch.isnan(b.attend(d, dims, torch.zeros_like(d["q"]))).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows", [9, 60])
def test_wide_queries_of_any_size(D, rows):
    """Queries of zeros, small and large ones, and of very different sizes in one row."""
    announce(f"q8 wide D={D}, {rows} queries of any size")
    b = _wide_only(Batch([(100, rows)] * 8, 8, 2, D, seed=2))
    q = b.q.reshape(8, rows, 8, D)
    for i, f in enumerate([0.0, 2.0 ** -130, 2.0 ** -60, 2.0 ** -10, 1.0, 30.0, 1.0, 1.0]):
        q[i] *= f
    q[6] *= np.exp2(-np.arange(D) / 4.0).astype(np.float32)
    q[7, ..., ::2] *= 2.0 ** -20
    b.q = b.round(q.reshape(-1, 8, D))
    check(_attend(b, "wide"), b.expected(), 100, "bf16")


@pytest.mark.parametrize("D", [64, 128])
def test_wide_rows_of_no_sequence_and_too_many(D):
    """Rows behind the last sequence stay, those of a chunk longer than max_q_len are NaN."""
    announce(f"q8 wide D={D}, rows of no sequence and of too long a chunk")
    b = _wide_only(Batch([(64, 40), (70, 41), (40, 1), (9, 2)], 4, 2, D))
    d = b.upload()
    b.widen(d, FAR)
    d["q"] = torch.cat([d["q"], d["q"][:3]])
    dims = b.dims(d, max_context_len=FAR, num_q_rows=b.T + 3, max_q_len=40)
    out = b.attend(d, dims, torch.full_like(d["q"], 7.0))
    assert (out[b.T:] == 7.0).all()
    ref = b.expected()
    ref[0][40:81] = np.nan
    check(out[:b.T].float().cpu(), ref, 70, "bf16")


# --- every code and scale byte -----------------------------------------------------

@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_of_every_code_and_scale(kind, dtype, D):
    """16 keys of one head hold codes of their own in each dim, and a query in one dim
    alone makes them scores; each key's V is 1 in a dim of its own, so the outputs are the
    softmax of the codes' values."""
    announce(f"q8 {kind} {dtype} D={D}, scores of every code and scale byte")
    H_q, heads = 8, 1
    rows, extra = (1, 0) if kind == "decode" else (5, 4)  # a chunk's first row sees the 16 keys
    pages = 1 if kind == "decode" else 2
    fine = np.array([c for c in range(256) if c & 127 != 127])
    codes = fine[(np.arange(16)[:, None] + 16 * np.arange(D)[None, :]) % len(fine)].astype(np.uint8)  # [key][dim]
    assert set(codes.ravel()) == set(fine)
    k, v = (np.zeros((pages, heads, 16 * D), np.uint8) for _ in range(2))
    k[0, 0, q8.places("k", D)] = codes
    v[0, 0, q8.places("v", D)[np.arange(16), np.arange(16)]] = 0x38
    kind_t = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.zeros(D, rows, H_q, D, dtype=kind_t, device="cuda")
    q[torch.arange(D), :, :, torch.arange(D)] = 2.0 ** -6
    q = q.view(D * rows, H_q, D)
    far = FAR if kind == "wide" else 32
    bt = torch.full((D, far // 16), -1, dtype=torch.int32, device="cuda")
    bt[:, :pages] = torch.arange(pages, device="cuda")
    cl = torch.full((D,), 16 + extra, dtype=torch.int32, device="cuda")
    qsl = torch.arange(D + 1, dtype=torch.int32, device="cuda") * rows
    dk, dv, out = torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), torch.empty_like(q)
    scales = torch.full((pages, heads, 2), 127, dtype=torch.uint8, device="cuda")
    if kind == "decode":
        dims = pb.make_dims_q8(q, dk, bt, far)
    else:
        dims = pb.make_dims_q8(q, dk, bt, far, num_q_rows=D * rows, max_q_len=rows)
    ws = torch.empty(max(1, pb.pa_workspace_size_q8(dims)), dtype=torch.uint8, device="cuda")
    got = []
    for byte in range(17, 247):
        scales[..., 0] = byte
        scale = 2.0 ** (127 - byte)
        if kind == "decode":
            pb.paged_attn_q8(q, dk, dv, scales, bt, cl, scale, out, dims, workspace=ws)
        else:
            pb.paged_attn_varlen_q8(q, dk, dv, scales, bt, cl, qsl, scale, out, dims, workspace=ws)
        got.append(out.view(D, rows, H_q, D)[:, 0].float().cpu().numpy())
    x = (q8.VALUES[codes] * 2.0 ** -6).T  # [dim][key]
    w = np.exp(x - x.max(-1, keepdims=True))
    ref = np.zeros((D, H_q, D))
    ref[..., :16] = (w / w.sum(-1, keepdims=True))[:, None]
    mass = np.zeros_like(ref)
    mass[..., :16] = 1
    size = np.repeat(np.abs(x).max(-1)[:, None], H_q, 1)
    reach = np.full((D, H_q), np.abs(q8.VALUES[codes]).sum(-1).max() * 2.0 ** -6)
    most = bound(ref, ref, mass, size, reach, 16, dtype, D)
    for byte, g in zip(range(17, 247), got):
        assert (np.abs(g - ref) <= most).all(), byte


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
def test_values_of_every_code_and_scale(kind, dtype, D):
    """Contexts of one token return its V: every code with every scale byte (in fp32
    within the normalisation's rounding)."""
    announce(f"q8 {kind} {dtype} D={D}, V of every code and scale byte")
    n, parts = 230, 256 // D  # (a head for each part of the codes)
    b = Batch(_lens("decode" if kind == "decode" else "chunks", [1] * n + ([40] if kind != "decode" else [])), 2 * parts, parts, D, dtype,
              seed=7, varlen=kind != "decode")
    codes = np.arange(256, dtype=np.uint8).reshape(parts, D)
    for i in range(n):
        b.v[b.bt[i, 0]][:, q8.places("v", D)[0]] = codes
        b.scales[b.bt[i, 0], :, 1] = 17 + i
    got = _attend(b, kind).double().numpy()
    for i in range(n):
        r = i if kind == "decode" else int(b.qsl[i])
        x = np.repeat(q8.VALUES[codes] * 2.0 ** (17 + i - 127), 2, 0)
        assert np.array_equal(np.isnan(got[r]), np.isnan(x))
        off = np.abs(got[r] - x)[~np.isnan(x)]
        assert (off <= (0.0 if dtype == "bf16" else 2.0 ** -22) * np.abs(x[~np.isnan(x)])).all(), 17 + i
